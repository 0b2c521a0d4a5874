// Writing a cache in 4 bits and reading it back (see quant_cache.cuh for the format): a thread has a word of a row of K and the same one of V, 16 bytes of each as
// bf16, and the threads of a warp follow the rows as they lie there.  Reading 32 caches of up to 8192 slots of 4 heads of 128 takes 88 us, 5.9 TB/s, of which three
// quarters are writes.  Writing 4 x 8192 tokens takes 31 us, 5 TB/s, and is bound by instructions (410 a warp of 512 values; issue slots 84 %).
#include "quant_cache.cuh"

namespace dsmoe {

namespace {

// kReadRows: rows that a thread of the reading kernel has under way.  32 caches of up to 8192 slots of 4 heads of 128, us: 88 with 4 of them and 128 threads (5.9 TB/s),
// with 2 99, with 8 95, with 256 threads 102, with 512 112.
constexpr int kThreads = 128, kReadRows = 4;

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// a * b + c, two bf16 numbers at a time
__device__ __forceinline__ uint32_t fma_pair(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Eight values of a word.  4 bits beside the exponent of 16 are 16 + 8 + c, for values i and i + 4 at a time; less 24 they are c, and the product with the scale is
// exact (it is rounded to bf16 where somebody else has left a scale of more than four significant bits).
__device__ __forceinline__ uint4 values_of(uint32_t word, uint32_t scale) {
    const uint32_t s = scale | scale << 16;
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = ((i == 0 ? word << 3 : word >> (4 * i - 3)) & 0x00780078u) | 0x41804180u;
        v[i] = fma_pair(fma_pair(x, 0x3f803f80u, 0xc1c0c1c0u), s, 0x80008000u);
    }
    return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
}

// A word of eight values, their scale and, with BACK, what it stands for; the three neighbouring lanes have the group's other values, and all lanes of the
// warp call it
struct Quantised {
    uint32_t word;
    uint16_t scale;
    uint4 back;
};
template <bool BACK>
__device__ __forceinline__ Quantised quantise(const uint4 in) {
    const uint32_t w[4] = {in.x, in.y, in.z, in.w};
    // magnitudes in order, as integers: what is no finite number is above all
    uint32_t top = max_pair(max_pair(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), max_pair(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
    top = max_pair(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max_pair(top, __shfl_xor_sync(0xffffffffu, top, 2));
    top = max(top & 0xffffu, top >> 16);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    // A seventh of the largest, up to four significant bits (or a multiple of 2^-129).  The product is a little small, by 2^-23 of it at most, so that what is
    // a border does not pass it; between a bf16 number / 7 that is none and a border lie 2^-10 of it.
    float s = __uint_as_float((__float_as_uint(__uint_as_float(top << 16) * 0x1.249248p-3f) + 0xfffffu) & ~0xfffffu), times = s;
    // Groups of the smallest numbers (whose scale has no reciprocal), of the largest (beyond 7 2^122), of zeros, and with what is no number
    if (s < 0x1p-64f || top > 0x7de0u) {
        const bool number = top < 0x7f80u;
        s = number ? fminf(s, 0x1p122f) : 0.f;
        const float up = s < 0x1p-64f ? 0x1p64f : 1.f, most = 7.f * s;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s > 0.f ? fminf(fmaxf(x[i], -most), most) * up : 0.f;
        times = s > 0.f ? s * up : 1.f;
        if (!number) s = __uint_as_float(0x7fff0000u);
    }
    // x / s as x * (1 / s): a little off, but halves have to be halves.  With eight and four bits x / s is a half or further than 2^-11 from one, so it
    // is rounded to a multiple of 2^-13 first (beside 1.5 2^10), then to an integer (beside 1.5 2^23, whose lowest bits it then is).
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(times));
    float n[8];
    uint32_t word = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
        n[i] = __fadd_rn(__fsub_rn(__fmaf_rn(x[i], inv, 0x1.8p10f), 0x1.8p10f), 0x1.8p23f);
        word = word * 16u + __float_as_uint(n[i]);
    }
    Quantised q;
    q.word = word - 0x4b400000u * 0x11111111u + 0x88888888u;          // (modulo 2^32; c + 8)
    q.scale = (uint16_t)(__float_as_uint(s) >> 16);
    if (BACK) {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = bf16_pair(__fsub_rn(n[2 * i], 0x1.8p23f) * s, __fsub_rn(n[2 * i + 1], 0x1.8p23f) * s);       // (exact)
        q.back = make_uint4(v[0], v[1], v[2], v[3]);
    }
    return q;
}

template <bool BACK>
__global__ void __launch_bounds__(kThreads) quant_write_kernel(const __grid_constant__ QuantView C, const __grid_constant__ QuantWrite W) {
    chain_wait();
    chain_next();
    const int words = C.d_head / 8, G = C.d_head / kQuantGroup, at_once = kThreads / words;
    // (a group's four lanes are neighbours in a warp: words is a multiple of 4)
    const int x = (int)threadIdx.x % words, r = (int)threadIdx.x / words, g = x / 4, t = x % 4;
    const uint32_t row = blockIdx.x * (uint32_t)at_once + r;          // (T * n_head is below 2^30)
    const bool real = r < at_once && row < (uint32_t)W.T * C.n_head;
    const int token = real ? (int)(row / (uint32_t)C.n_head) : 0, head = real ? (int)(row - (uint32_t)token * C.n_head) : 0;
    const int p = W.pos[token], seq = W.tok_seq ? W.tok_seq[token] : 0;
    const uint4 k = *reinterpret_cast<const uint4*>(W.k + token * W.i_t + head * W.i_h + 8 * x);
    const uint4 v = *reinterpret_cast<const uint4*>(W.v + token * W.i_t + head * W.i_h + 8 * x);
    // a token that a later one of the call takes the slot of
    const bool has_later = W.ring > 0 && token + (long long)W.ring < W.T;
    const int p_later = has_later ? W.pos[token + W.ring] : -1, seq_later = has_later && W.tok_seq ? W.tok_seq[token + W.ring] : 0;
    const Quantised kq = quantise<BACK>(k), vq = quantise<BACK>(v);
    if (!real || p == -1) return;
    if (seq < 0 || seq >= C.n_seq || p < 0 || (W.ring ? p == 0x7fffffff : p >= C.L)) {
        if (x == 0 && head == 0) report_status(W.dev_status, DSMOE_ERR_INVALID_ARG);
        return;
    }
    if (BACK) {
        const long long to = token * W.b_t + head * W.b_h + 8 * x;
        if (W.k_back) *reinterpret_cast<uint4*>(W.k_back + to) = kq.back;
        if (W.v_back) *reinterpret_cast<uint4*>(W.v_back + to) = vq.back;
    }
    if (has_later && p >= W.sinks && seq_later == seq && p_later == (long long)p + W.ring) return;
    const int slot = !W.ring || p < W.sinks ? p : W.sinks + (p - W.sinks) % W.ring;
    const long long at = seq * C.c_s + head * C.c_h + slot * C.c_p + (t * G + g) * 4;
    *reinterpret_cast<uint32_t*>(C.K + at) = kq.word;
    *reinterpret_cast<uint32_t*>(C.V + at) = vq.word;
    if (t == 0) {
        const long long s_at = seq * C.s_s + head * C.s_h + slot * C.s_p + g;
        reinterpret_cast<uint16_t*>(C.K_scale)[s_at] = kq.scale;
        reinterpret_cast<uint16_t*>(C.V_scale)[s_at] = vq.scale;
    }
}

// by_slot: the heads of a slot lie side by side in the cache, and are read side by side.  What there is to read of each sequence the host does not know, only how many
// slots there are.  COUNTED: the sequences' tiles of rows are counted first, kThreads sequences at a time, and a CTA takes each gridDim.x-th of them.  Otherwise all
// slots' tiles are looked at (see launch_quant_read).
template <bool COUNTED>
__global__ void __launch_bounds__(kThreads, 8) quant_read_kernel(const __grid_constant__ QuantView C, const __grid_constant__ QuantRead R, int by_slot) {
    chain_wait();
    chain_next();
    const int words = C.d_head / 8, G = C.d_head / kQuantGroup, at_once = kThreads / words;
    const int x = (int)threadIdx.x % words, r = (int)threadIdx.x / words, g = x / 4, t = x % 4;
    const int word_at = (t * G + g) * 4;
    const long long tile = at_once * kReadRows;
    // kReadRows times the CTA's rows from the base-th of the sequence's n * n_head on; slot_of_nth(i): where the i-th slot of those n lies from R.first on, or less than 0
    const auto read = [&](int seq, long long base, int n, const auto& slot_of_nth) {
        const long long rows = (long long)n * C.n_head;
        const uint32_t inner = by_slot ? C.n_head : n;
        const int outer0 = (int)divide(base, inner);
        const uint32_t inner0 = (uint32_t)(base - (long long)outer0 * inner) + r;                // (below 2^31)
        const unsigned char *const K = C.K + seq * C.c_s + word_at, *const V = C.V + seq * C.c_s + word_at;
        const uint16_t* const Ks = reinterpret_cast<const uint16_t*>(C.K_scale) + seq * C.s_s + g;
        const uint16_t* const Vs = reinterpret_cast<const uint16_t*>(C.V_scale) + seq * C.s_s + g;
        uint32_t kw[kReadRows], vw[kReadRows], ks[kReadRows], vs[kReadRows];
        long long to[kReadRows];
#pragma unroll
        for (int u = 0; u < kReadRows; ++u) {
            const uint32_t in = inner0 + u * at_once, over = in / inner, rest = in - over * inner;
            const int outer = outer0 + (int)over, head = by_slot ? (int)rest : outer, at_n = slot_of_nth(by_slot ? outer : (int)rest), slot = R.first + at_n;
            to[u] = -1;
            if (base + r + u * at_once >= rows || at_n < 0) continue;
            const long long at = head * C.c_h + slot * C.c_p, s_at = head * C.s_h + slot * C.s_p;
            kw[u] = *reinterpret_cast<const uint32_t*>(K + at);
            vw[u] = *reinterpret_cast<const uint32_t*>(V + at);
            ks[u] = Ks[s_at];
            vs[u] = Vs[s_at];
            to[u] = seq * R.o_s + head * R.o_h + at_n * R.o_p + 8 * x;
        }
#pragma unroll
        for (int u = 0; u < kReadRows; ++u) {
            if (to[u] < 0) continue;
            *reinterpret_cast<uint4*>(R.K + to[u]) = values_of(kw[u], ks[u]);
            *reinterpret_cast<uint4*>(R.V + to[u]) = values_of(vw[u], vs[u]);
        }
    };
    if constexpr (COUNTED) {
        __shared__ long long end_s[kThreads];           // tiles up to this sequence and with it
        __shared__ int3 part_s[kThreads];               // of its slots: .x from the first on, then those from .y on, .z in all
        __shared__ long long warp_sum_s[kThreads / 32];
        const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
        long long b = blockIdx.x, before = 0;           // the next tile of this CTA; tiles of earlier sequences
        for (int seq0 = 0; seq0 < C.n_seq; seq0 += kThreads) {
            const int mine = seq0 + tid;
            int3 part = make_int3(0, 0, 0);
            if (mine < C.n_seq) {
                if (R.range) {
                    const int4 range = R.range[mine];
                    part.x = range.x;
                    part.y = max(range.y, range.x);
                    part.z = range.x + max(range.z - part.y, 0);
                } else {
                    part.x = part.z = R.len ? min(max(R.len[mine], R.first) - R.first, R.rows) : R.rows;
                }
            }
            long long end = ((long long)part.z * C.n_head + tile - 1) / tile;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(0xffffffffu, end, o);
                if (lane >= o) end += up;
            }
            __syncthreads();                            // (everybody is past the tiles of the last ones)
            if (lane == 31) warp_sum_s[warp] = end;
            __syncthreads();
            end += before;
            for (int w = 0; w < warp; ++w) end += warp_sum_s[w];
            end_s[tid] = end;
            part_s[tid] = part;
            __syncthreads();
            const long long last = end_s[kThreads - 1];
            for (; b < last; b += gridDim.x) {
                int i = 0;                              // the sequences that end at or before tile b
#pragma unroll
                for (int k = 0; k < kThreads; k += 32) i += __popc(__ballot_sync(0xffffffffu, end_s[k + lane] <= b));
                if (r >= at_once) continue;
                const int3 p = part_s[i];
                read(seq0 + i, (b - (i > 0 ? end_s[i - 1] : before)) * tile, p.z, [&](int n) { return n < p.x ? n : p.y + (n - p.x); });
            }
            before = last;
        }
    } else {
        const long long per_seq = ((long long)R.rows * C.n_head + tile - 1) / tile, all = per_seq * C.n_seq;
        if (r >= at_once) return;
        for (long long b = blockIdx.x; b < all; b += gridDim.x) {
            const int seq = (int)divide(b, per_seq);
            const int len = R.len ? R.len[seq] : INT_MAX;
            const int4 range = R.range ? R.range[seq] : make_int4(INT_MAX, 0, 0, 0);
            read(seq, (b - seq * per_seq) * tile, R.rows, [&](int n) {
                const int slot = R.first + n;
                return slot >= len || (slot >= range.x && (slot < range.y || slot >= range.z)) ? -1 : n;
            });
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
    DSMOE_CUDA_TRY(launch_chained(W.k_back || W.v_back ? quant_write_kernel<true> : quant_write_kernel<false>, (unsigned)blocks, kThreads, 0, s, C, W));
    return DSMOE_OK;
}

// Counting the sequences' tiles costs 1 us, and 3 for each kThreads sequences more; looking at slots that hold nothing takes far longer where caches are large and hold little.
// So they are counted where all slots are more than four rounds of the grid, and one more for each kThreads sequences.  Counted and not, us: 32 caches of 131072 slots that hold 200 9.7, 596 (and 32 prompts of 16 tokens on
// them, 4 x 5 heads of 128, 43, 628); 32 of 819 to 8192 of 8192, 4 heads of 128 66, 81, full 116, 117 (6.9 rounds); 8 of 400 to 4000, heads of 96 10.8, 11.8, full 17.2, 15.6 (0.7);
// 256 of 500, 2 heads of 64 23.2, 18.5 (0.9); 1000 of 300, one head of 128 63, 37 (2.1).
dsmoe_status launch_quant_read(const QuantView& C, const QuantRead& R, cudaStream_t s) {
    const long long tile = kThreads / (C.d_head / 8) * kReadRows, all = ((long long)R.rows * C.n_head + tile - 1) / tile * C.n_seq;
    const long long most = 32ll * sm_count(), grid = all < most ? all : most;
    DSMOE_CUDA_TRY(launch_chained(all > most * (4 + C.n_seq / kThreads) ? quant_read_kernel<true> : quant_read_kernel<false>, (unsigned)grid, kThreads, 0, s, C, R, (int)(C.n_head > 1 && C.c_h < C.c_p)));
    return DSMOE_OK;
}

dsmoe_status launch_quant_range(const AttnView& A, int4* range, cudaStream_t s) {
    DSMOE_CUDA_TRY(launch_chained(quant_range_kernel, (unsigned)A.n_seq, 512, 0, s, A, range));
    return DSMOE_OK;
}

}  // namespace dsmoe
