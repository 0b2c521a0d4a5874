// Writing a cache in 4 bits and reading it back (see quant_cache.cuh for the format).  Both are bound by memory: a thread has a word of a row of K and
// the same one of V, 16 bytes of each as bf16, and the threads of a warp follow the rows as they lie there.
#include "quant_cache.cuh"

namespace dsmoe {

namespace {

constexpr int kThreads = 256, kReadRows = 4;      // kReadRows: rows a thread of the reading kernel has under way

// (a scale that is no number makes all of the group's values none)
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight values of a word
__device__ __forceinline__ uint4 values_of(uint32_t word, float scale) {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = (float)((int)(word >> (8 * i) & 15u) - 8), hi = (float)((int)(word >> (8 * i + 4) & 15u) - 8);
        r[i] = bf16_pair(lo * scale, hi * scale);                     // (exact)
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// The word of eight values whose group's other values the three neighbouring lanes have; all lanes of the warp call it
__device__ __forceinline__ uint32_t quantise(const uint4 in, float* scale_out) {
    const uint32_t w[4] = {in.x, in.y, in.z, in.w};
    uint32_t top = 0;                                                 // magnitudes in order, as integers: what is no finite number is above all
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // Up to four significant bits (or a multiple of 2^-129), 2^122 at most (24 s is a number then).  The quotient is rounded to 24 bits first, which
    // moves it over no border: between a bf16 number / 7 and a border lie 2^-10 of it or more, or nothing.
    const uint32_t raw = (__float_as_uint(__fdiv_rn(__uint_as_float(top << 16), 7.f)) + 0xfffffu) & ~0xfffffu;
    const float s = top >= 0x7f80u ? __uint_as_float(0x7fff0000u) : fminf(__uint_as_float(raw), 0x1p122f);
    *scale_out = s;
    if (top == 0u || top >= 0x7f80u) return 0x88888888u;
    // x / s as x * (1 / s): a little off, but halves have to be halves.  With eight and four bits x / s is a half or further than 2^-11 from one, so it
    // is rounded to a multiple of 2^-13 first.  (For scales whose reciprocal may overflow both are multiplied by 2^64.)
    const float up = s < 0x1p-64f ? 0x1p64f : 1.f, inv = __frcp_rn(s * up);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        const float fine = __fsub_rn(__fadd_rn(__fmul_rn(x * up, inv), 0x1.8p10f), 0x1.8p10f);
        const int c = min(max(__float2int_rn(fine), -7), 7);         // (rounds what is too large to the largest integer)
        word |= (uint32_t)(c + 8) << (4 * i);
    }
    return word;
}

__global__ void __launch_bounds__(kThreads) quant_write_kernel(const __grid_constant__ QuantView C, const __grid_constant__ QuantWrite W) {
    chain_wait();
    chain_next();
    const int words = C.d_head / 8, G = C.d_head / kQuantGroup, at_once = kThreads / words;
    // (a group's four lanes are neighbours in a warp: words is a multiple of 4)
    const int x = (int)threadIdx.x % words, r = (int)threadIdx.x / words, g = x / 4, t = x % 4;
    const long long row = (long long)blockIdx.x * at_once + r;
    const bool real = r < at_once && row < (long long)W.T * C.n_head;
    const int token = real ? (int)(row / C.n_head) : 0, head = real ? (int)(row % C.n_head) : 0;
    const int p = W.pos[token], seq = W.tok_seq ? W.tok_seq[token] : 0;
    const uint4 k = *reinterpret_cast<const uint4*>(W.k + token * W.i_t + head * W.i_h + 8 * x);
    const uint4 v = *reinterpret_cast<const uint4*>(W.v + token * W.i_t + head * W.i_h + 8 * x);
    // a token that a later one of the call takes the slot of
    const bool has_later = W.ring > 0 && token + (long long)W.ring < W.T;
    const int p_later = has_later ? W.pos[token + W.ring] : -1, seq_later = has_later && W.tok_seq ? W.tok_seq[token + W.ring] : 0;
    float ks, vs;
    const uint32_t kw = quantise(k, &ks), vw = quantise(v, &vs);
    if (!real || p == -1) return;
    if (seq < 0 || seq >= C.n_seq || p < 0 || (W.ring ? p == 0x7fffffff : p >= C.L)) {
        if (x == 0 && head == 0) report_status(W.dev_status, DSMOE_ERR_INVALID_ARG);
        return;
    }
    if (W.k_back) *reinterpret_cast<uint4*>(W.k_back + token * W.b_t + head * W.b_h + 8 * x) = values_of(kw, ks);
    if (W.v_back) *reinterpret_cast<uint4*>(W.v_back + token * W.b_t + head * W.b_h + 8 * x) = values_of(vw, vs);
    if (has_later && p >= W.sinks && seq_later == seq && p_later == (long long)p + W.ring) return;
    const int slot = !W.ring || p < W.sinks ? p : W.sinks + (p - W.sinks) % W.ring;
    const long long at = seq * C.c_s + head * C.c_h + slot * C.c_p + (t * G + g) * 4, s_at = seq * C.s_s + head * C.s_h + slot * C.s_p + g;
    *reinterpret_cast<uint32_t*>(C.K + at) = kw;
    *reinterpret_cast<uint32_t*>(C.V + at) = vw;
    if (t == 0) {
        C.K_scale[s_at] = __float2bfloat16_rn(ks);                    // (exact)
        C.V_scale[s_at] = __float2bfloat16_rn(vs);
    }
}

// by_slot: the heads of a slot lie side by side in the cache, and are read side by side
__global__ void __launch_bounds__(kThreads) quant_read_kernel(const __grid_constant__ QuantView C, const __grid_constant__ QuantRead R, int by_slot) {
    chain_wait();
    chain_next();
    const int words = C.d_head / 8, G = C.d_head / kQuantGroup, at_once = kThreads / words;
    const int x = (int)threadIdx.x % words, r = (int)threadIdx.x / words, g = x / 4, t = x % 4;
    const unsigned inner = by_slot ? C.n_head : R.rows;
    const long long rows = (long long)R.rows * C.n_head, tile = at_once * kReadRows, per_seq = (rows + tile - 1) / tile, all = per_seq * C.n_seq;
    if (r >= at_once) return;
    for (long long b = blockIdx.x; b < all; b += gridDim.x) {
        const int seq = (int)(b / per_seq);
        const long long base = b % per_seq * tile;
        const int outer0 = (int)(base / inner);
        const unsigned inner0 = (unsigned)(base % inner) + r;         // (below 2^31)
        const int len = R.len ? R.len[seq] : INT_MAX;
        const int4 range = R.range ? R.range[seq] : make_int4(INT_MAX, 0, 0, 0);
        uint32_t kw[kReadRows], vw[kReadRows];
        float ks[kReadRows], vs[kReadRows];
        long long to[kReadRows];
#pragma unroll
        for (int u = 0; u < kReadRows; ++u) {
            const unsigned in = inner0 + u * at_once, over = in / inner;
            const int outer = outer0 + (int)over, rest = (int)(in - over * inner), head = by_slot ? rest : outer, n = by_slot ? outer : rest;
            const long long slot = (long long)R.first + n;
            to[u] = -1;
            if (base + r + u * at_once >= rows || slot >= len || (slot >= range.x && (slot < range.y || slot >= range.z))) continue;
            const long long at = seq * C.c_s + head * C.c_h + slot * C.c_p + (t * G + g) * 4, s_at = seq * C.s_s + head * C.s_h + slot * C.s_p + g;
            kw[u] = *reinterpret_cast<const uint32_t*>(C.K + at);
            vw[u] = *reinterpret_cast<const uint32_t*>(C.V + at);
            ks[u] = __bfloat162float(C.K_scale[s_at]);
            vs[u] = __bfloat162float(C.V_scale[s_at]);
            to[u] = seq * R.o_s + head * R.o_h + n * R.o_p + 8 * x;
        }
#pragma unroll
        for (int u = 0; u < kReadRows; ++u) {
            if (to[u] < 0) continue;
            *reinterpret_cast<uint4*>(R.K + to[u]) = values_of(kw[u], ks[u]);
            *reinterpret_cast<uint4*>(R.V + to[u]) = values_of(vw[u], vs[u]);
        }
    }
}

// A CTA per sequence
__global__ void __launch_bounds__(512) quant_range_kernel(const __grid_constant__ AttnView A, int4* __restrict__ range) {
    chain_wait();
    chain_next();
    __shared__ int low_s, high_s, sinks_s;
    if (threadIdx.x == 0) {
        low_s = INT_MAX;
        high_s = 0;
        sinks_s = 0;
    }
    __syncthreads();
    int low = INT_MAX, high = 0, sinks = 0;
    for (int t = threadIdx.x; t < A.T; t += 512) {
        bool bad = false;
        const Sight s = sight_of(A, t, &bad);
        if (s.seq != (int)blockIdx.x) continue;
        sinks = max(sinks, s.sinks);
        if (s.last < s.first) continue;
        low = min(low, s.first);
        high = max(high, s.last + 1);
    }
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    sinks = __reduce_max_sync(0xffffffffu, sinks);
    if ((threadIdx.x & 31) == 0) {
        atomicMin(&low_s, low);
        atomicMax(&high_s, high);
        atomicMax(&sinks_s, sinks);
    }
    __syncthreads();
    // a ring that has gone round: everything
    if (threadIdx.x == 0) range[blockIdx.x] = A.ring ? make_int4(min(high_s, A.L), 0, 0, 0) : make_int4(sinks_s, low_s, high_s, 0);
}

}  // namespace

dsmoe_status launch_quant_write(const QuantView& C, const QuantWrite& W, cudaStream_t s) {
    const long long at_once = kThreads / (C.d_head / 8), blocks = ((long long)W.T * C.n_head + at_once - 1) / at_once;
    if (blocks > 0x7fffffffll) return DSMOE_ERR_UNSUPPORTED;
    DSMOE_CUDA_TRY(launch_chained(quant_write_kernel, (unsigned)blocks, kThreads, 0, s, C, W));
    return DSMOE_OK;
}

dsmoe_status launch_quant_read(const QuantView& C, const QuantRead& R, cudaStream_t s) {
    const long long tile = kThreads / (C.d_head / 8) * kReadRows, all = ((long long)R.rows * C.n_head + tile - 1) / tile * C.n_seq;
    const long long most = 16ll * sm_count(), grid = all < most ? all : most;
    DSMOE_CUDA_TRY(launch_chained(quant_read_kernel, (unsigned)grid, kThreads, 0, s, C, R, (int)(C.n_head > 1 && C.c_h < C.c_p)));
    return DSMOE_OK;
}

dsmoe_status launch_quant_range(const AttnView& A, int4* range, cudaStream_t s) {
    DSMOE_CUDA_TRY(launch_chained(quant_range_kernel, (unsigned)A.n_seq, 512, 0, s, A, range));
    return DSMOE_OK;
}

}  // namespace dsmoe
