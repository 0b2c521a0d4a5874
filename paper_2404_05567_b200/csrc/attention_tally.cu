// The weights that the keys of a cache get from the tokens of a call, added up per key (dsmoe_tally_attention's second half):
//
//     tally_out[s][j][l] = tally_in[s][j][l] + sum over tokens t of sequence s with pos[t] >= l, members g, of 2^(logit(t,j,g,l) - m) / sum
//
// with m and the sum of every row from the attention itself.  Either the attention has left its logits (decoding): tally_add_kernel reads them,
// a thread per four keys.  Or they are computed again.  attention_tally_tile_kernel (prompts): a CTA has 128 keys as the rows of a tcgen05 tile and
// walks the rows that see them as its columns, 128 at a time; a thread owns a key, takes its line of logits out of tensor memory and adds up the
// weights: no sum crosses threads.  Four warps fetch the next rows' queries meanwhile, two CTAs fill an SM, and where there are few keys the rows
// are cut into parts.  attention_tally_kernel (other head widths and strides): a CTA owns 64 keys of a (sequence, head) and walks the rows that see them, in
// order of the tokens, so that every sum is taken in one order and nothing is added in memory.  The logits are computed again, keys as the
// rows and queries as the columns of the MMA tile: a thread keeps two keys' sums in registers.
#include <climits>

#include "cache_attention.cuh"
#include "tensor_maps.cuh"
#include "umma.cuh"

namespace dsmoe {

namespace {

constexpr int kTallyWarps = 4, kTallyKeys = 16 * kTallyWarps, kTallyRows = 32, kTallyList = 1024;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

constexpr int kAddThreads = 256, kAddKeys = 4 * kAddThreads;

// A CTA per 1024 keys of a (sequence, head); A.T up to kListTokens
__global__ void __launch_bounds__(kAddThreads) tally_add_kernel(const __grid_constant__ AttnView A, const float* logits, const long long pitch,
                                                                const float* tally_in, float* tally_out) {
    __shared__ int list_s[kListTokens], last_s[kListTokens], count_s[kAddThreads / 32];
    chain_wait();
    chain_next();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int blocks = (A.L + kAddKeys - 1) / kAddKeys;
    const int kb = (int)(blockIdx.x % blocks), sj = (int)(blockIdx.x / blocks), s = sj / A.n_head, j = sj % A.n_head;
    const int key0 = kb * kAddKeys + 4 * tid;
    int n = 0;                                           // the sequence's tokens that see a key of this block, in order
    for (int c = 0; c < A.T; c += kAddThreads) {
        const int t = c + tid;
        bool bad = false, mine = false;
        int last = -1;
        if (t < A.T) {
            const Sight w = sight_of(A, t, &bad);
            mine = w.seq == s && w.last >= kb * kAddKeys;
            last = w.last;
        }
        const uint32_t votes = __ballot_sync(0xffffffffu, mine);
        if (lane == 0) count_s[warp] = __popc(votes);
        __syncthreads();
        int at = n;
        for (int w = 0; w < kAddThreads / 32; ++w) {
            if (w < warp) at += count_s[w];
            n += count_s[w];
        }
        if (mine) {
            at += __popc(votes & ((1u << lane) - 1u));
            list_s[at] = t;
            last_s[at] = last;
        }
        __syncthreads();
    }
    if (n == 0 && tally_in == tally_out) return;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) {
        const int last = last_s[i];
        if (key0 > last) continue;
        const long long r0 = row_at(A, list_s[i], j, 0);
#pragma unroll 5
        for (int m = 0; m < A.group; ++m) {
            const float4 x = *reinterpret_cast<const float4*>(logits + (r0 + m) * pitch + key0);
            const float2 ml = A.ml[r0 + m];
            // (chosen, not multiplied by zero: behind the token's last key lies anything)
            sum[0] += exp2_fast(x.x - ml.x) * ml.y;
            if (key0 + 1 <= last) sum[1] += exp2_fast(x.y - ml.x) * ml.y;
            if (key0 + 2 <= last) sum[2] += exp2_fast(x.z - ml.x) * ml.y;
            if (key0 + 3 <= last) sum[3] += exp2_fast(x.w - ml.x) * ml.y;
        }
    }
    const size_t at = (size_t)sj * A.L + key0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (key0 + k < A.L) tally_out[at + k] = (tally_in ? tally_in[at + k] : 0.f) + sum[k];
}

template <int DH>
__global__ void __launch_bounds__(32 * kTallyWarps) attention_tally_kernel(const __grid_constant__ AttnView A, const float* tally_in,
                                                                           float* tally_out) {
    constexpr int STRIDE = DH * 2 + 16, KS = DH / 16, CH = DH / 8, THREADS = 32 * kTallyWarps;
    extern __shared__ __align__(16) unsigned char at_smem[];
    unsigned char* const k_s = at_smem;                            // [64][STRIDE]
    unsigned char* const q_s = at_smem + kTallyKeys * STRIDE;      // [32][STRIDE]
    __shared__ int list_s[kTallyList], last_s[kTallyList], count_s[kTallyWarps + 1];
    __shared__ float2 ml_s[kTallyRows];
    __shared__ int row_last_s[kTallyRows];
    chain_wait();
    chain_next();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
    const int blocks = (A.L + kTallyKeys - 1) / kTallyKeys;
    const int kb = (int)(blockIdx.x % blocks), sj = (int)(blockIdx.x / blocks), s = sj / A.n_head, j = sj % A.n_head;
    const int key0 = kb * kTallyKeys;
    const __nv_bfloat16* const K = A.K + s * A.kv_s + j * A.kv_h;
    float sum0 = 0.f, sum1 = 0.f;
    bool have_keys = false;
    uint32_t kf[KS][4];
    for (int t0 = 0; t0 < A.T; t0 += kTallyList) {
        // the tokens of this sequence, among the next 1024, that see a key of this block: in order
        int n = 0;
        __syncthreads();
        for (int c = 0; c < kTallyList && t0 + c < A.T; c += THREADS) {
            const int t = t0 + c + tid;
            bool bad = false, mine = false;
            int last = -1;
            if (t < A.T) {
                const Sight w = sight_of(A, t, &bad);
                mine = w.seq == s && w.last >= key0;
                last = w.last;
            }
            const uint32_t votes = __ballot_sync(0xffffffffu, mine);
            if (lane == 0) count_s[warp] = __popc(votes);
            __syncthreads();
            int at = n;
            for (int w = 0; w < warp; ++w) at += count_s[w];
            if (mine) {
                at += __popc(votes & ((1u << lane) - 1u));
                list_s[at] = t;
                last_s[at] = last;
            }
            for (int w = 0; w < kTallyWarps; ++w) n += count_s[w];
            __syncthreads();
        }
        if (n == 0) continue;
        if (!have_keys) {                               // (the same for the whole CTA)
            for (int idx = tid; idx < kTallyKeys * CH; idx += THREADS) {
                const int row = idx / CH, ch = idx % CH;
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (key0 + row < A.L) v = *reinterpret_cast<const uint4*>(K + (key0 + row) * A.kv_p + ch * 8);
                *reinterpret_cast<uint4*>(k_s + row * STRIDE + ch * 16) = v;
            }
            __syncthreads();
            const uint32_t krow = ptx::smem_u32(k_s) + (uint32_t)((warp * 16 + (lane & 15)) * STRIDE + (lane >> 4) * 16);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) ldsm_x4(kf[ks], krow + (uint32_t)(ks * 32));
            have_keys = true;
        }
        const long long rows = (long long)n * A.group;
        for (long long r0 = 0; r0 < rows; r0 += kTallyRows) {
            __syncthreads();
            for (int idx = tid; idx < kTallyRows * CH; idx += THREADS) {
                const int row = idx / CH, ch = idx % CH;
                const long long r = r0 + row;
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (r < rows) {
                    const int t = list_s[r / A.group], m = (int)(r % A.group);
                    v = *reinterpret_cast<const uint4*>(A.q + t * A.q_t + j * A.q_h + m * A.q_g + ch * 8);
                    if (ch == 0) {
                        ml_s[row] = A.ml[((size_t)t * A.n_head + j) * A.group + m];
                        row_last_s[row] = last_s[r / A.group];
                    }
                } else if (ch == 0) {
                    ml_s[row] = make_float2(0.f, 0.f);
                    row_last_s[row] = -1;
                }
                *reinterpret_cast<uint4*>(q_s + row * STRIDE + ch * 16) = v;
            }
            __syncthreads();
#pragma unroll
            for (int np = 0; np < kTallyRows / 16; ++np) {
                float sc[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
                const uint32_t qa = ptx::smem_u32(q_s) + (uint32_t)((np * 16 + (lane >> 4) * 8 + (lane & 7)) * STRIDE + ((lane >> 3) & 1) * 16);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    uint32_t b[4];
                    ldsm_x4(b, qa + (uint32_t)(ks * 32));
                    mma_16816(sc[0], kf[ks], b[0], b[1]);
                    mma_16816(sc[1], kf[ks], b[2], b[3]);
                }
                const int k0 = key0 + warp * 16 + g, k1 = k0 + 8;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int row = np * 16 + i * 8 + q4 * 2 + c;
                        const float2 ml = ml_s[row];
                        const int last = row_last_s[row];
                        // (chosen, not multiplied by zero: a key that the row does not see may hold anything)
                        if (k0 <= last) sum0 = fmaf(exp2_fast(fmaf(sc[i][c], A.scale_log2, -ml.x)), ml.y, sum0);
                        if (k1 <= last) sum1 = fmaf(exp2_fast(fmaf(sc[i][2 + c], A.scale_log2, -ml.x)), ml.y, sum1);
                    }
            }
        }
    }
    sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1);
    sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1);
    sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2);
    sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
    if (q4 < 2) {
        const int key = key0 + warp * 16 + g + 8 * q4;
        const size_t at = (size_t)sj * A.L + key;
        if (key < A.L && (have_keys || tally_in != tally_out)) tally_out[at] = (tally_in ? tally_in[at] : 0.f) + (q4 == 0 ? sum0 : sum1);
    }
}

// ---------------------------------------------------------------- prompts, on the 5th-generation tensor cores

constexpr int kTtKeys = 128, kTtRows = 128, kTtThreads = 256, kTtAhead = 4;

// The tokens of every sequence, in order, with their last visible keys: sequence s's are list[from[s].x .. + from[s].y - 1].  A CTA per sequence.
// (Each CTA of the next launch looked through all tokens itself at first: 16 rounds of 256 for 4000 tokens, 20 of its 60 us.)
__global__ void __launch_bounds__(1024) tally_list_kernel(const __grid_constant__ AttnView A, int2* list, int2* from) {
    __shared__ int warp_s[2][32];
    chain_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, s = (int)blockIdx.x;
    int before = 0, n = 0;                // tokens of earlier sequences; of this one, so far
    for (int turn = 0; turn < 2; ++turn) {
        n = 0;
        for (int t0 = 0; t0 < A.T; t0 += 1024 * kTtAhead) {
            int last[kTtAhead], less = 0, mine = 0;
#pragma unroll
            for (int i = 0; i < kTtAhead; ++i) {
                const int t = t0 + tid * kTtAhead + i;
                last[i] = -1;
                if (t < A.T) {
                    bool bad = false;
                    const Sight w = sight_of(A, t, &bad);
                    less += w.last >= 0 && w.seq < s;
                    if (w.seq == s) last[i] = w.last;
                    mine += last[i] >= 0;
                }
            }
            if (turn == 0) {
                before += less;           // (this thread's)
                continue;
            }
            int incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            __syncthreads();
            if (lane == 31) warp_s[0][warp] = incl;
            __syncthreads();
            const int w = warp_s[0][lane];
            int at = n + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + incl - mine;
            n += __reduce_add_sync(0xffffffffu, w);
#pragma unroll
            for (int i = 0; i < kTtAhead; ++i)
                if (last[i] >= 0) list[before + at++] = make_int2(t0 + tid * kTtAhead + i, last[i]);
        }
        if (turn == 0) {
            before = __reduce_add_sync(0xffffffffu, before);
            if (lane == 0) warp_s[1][warp] = before;
            __syncthreads();
            before = __reduce_add_sync(0xffffffffu, warp_s[1][lane]);
        }
    }
    if (tid == 0) from[s] = make_int2(before, n);
    chain_next();
}

template <int DH>
struct TallyGeo {
    static constexpr int HALVES = (DH + 63) / 64;
    static constexpr uint32_t PIECE = kTtRows * 128, TILE = HALVES * PIECE;
    static constexpr uint32_t K = 0, Q = TILE, END = 3 * TILE;         // two buffers of queries
    static constexpr int SMEM = (int)END + 1024;
};

struct TallyArgs {
    AttnView A;
    int at_pos, at_head, at_seq;
    int parts;
    const int2 *list, *from;              // the sequences' tokens
    const float* in;                      // parts == 1: the tallies
    float* out;                           // ... or [parts][n_seq * n_head * L]
};

// Whether all of the four fetching warps' threads say so
__device__ __forceinline__ bool fetchers_agree(bool x) {
    uint32_t all;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"((uint32_t)x) : "memory");
    return all != 0;
}

template <int DH>
__global__ void __launch_bounds__(kTtThreads, 2) attention_tally_tile_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ TallyArgs P) {
    using G = TallyGeo<DH>;
    constexpr int CH = DH / 8, KS = DH / 16;
    extern __shared__ unsigned char tt_smem[];
    __shared__ int first_s, last_s;       // the first and the last of the sequence's tokens that see a key of this tile
    __shared__ long long q_s[kTtRows];    // where the rows' queries are
    __shared__ __align__(16) float2 ml_s[2][kTtRows];
    __shared__ __align__(16) int row_last_s[2][kTtRows];
    __shared__ int all_see_s[2];
    __shared__ uint64_t k_full, rows_full[2], s_full[2], s_empty[2];
    __shared__ uint32_t tmem_s;
    __shared__ volatile int abort_flag;
    const AttnView& A = P.A;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = ptx::smem_u32(tt_smem), base = (raw + 1023u) & ~1023u;
    // (sequence, head) by (sequence, head), the first keys, which most rows see, first
    const int part = (int)(blockIdx.x % P.parts);
    const int kt = (int)(blockIdx.x / P.parts / (A.n_seq * A.n_head)), sj = (int)(blockIdx.x / P.parts % (A.n_seq * A.n_head));
    const int s = sj / A.n_head, j = sj % A.n_head, key0 = kt * kTtKeys, tokens = kTtRows / A.group;
    if (tid == 0) {
        ptx::mbar_init(ptx::smem_u32(&k_full), 1);
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(ptx::smem_u32(&rows_full[b]), 128);
            ptx::mbar_init(ptx::smem_u32(&s_full[b]), 1);
            ptx::mbar_init(ptx::smem_u32(&s_empty[b]), kTtKeys);
        }
        abort_flag = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 0) {
        ptx::tmem_alloc(ptx::smem_u32(&tmem_s), 256);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    chain_wait();
    const uint32_t tmem = tmem_s;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    int done = 0;                         // tiles of rows that this CTA has taken
    bool alive = true;
    const int2 from = P.from[s];
    const int2* const list = P.list + from.x;
    if (tid == 0) {
        first_s = 0x7fffffff;
        last_s = -1;
    }
    __syncthreads();
    {
        int first = 0x7fffffff, last = -1;
        for (int i = tid; i < from.y; i += kTtThreads)
            if (list[i].y >= key0) {
                first = min(first, i);
                last = i;
            }
        first = __reduce_min_sync(0xffffffffu, first);
        last = __reduce_max_sync(0xffffffffu, last);
        if (lane == 0 && last >= 0) {
            atomicMin(&first_s, first);
            atomicMax(&last_s, last);
        }
    }
    __syncthreads();
    {
        const int i0 = first_s, n = last_s < 0 ? 0 : last_s + 1 - i0, tiles = (n + tokens - 1) / tokens;
        // a fetching thread's row: its token and sums, asked for a tile ahead.  Places without a row have the tile's first row once more, by a factor of
        // 0: with zeros for a query, a key that holds an infinity would have a logit that is no number, and so would its sum.
        const int at = tid - 128;
        const int of = at / A.group;
        int member = 0;
        bool real = false;
        int2 token = make_int2(0, -1);
        float2 ml = make_float2(0.f, 0.f);
        const auto ask = [&](int i) {
            const int k = i * tokens + of;
            real = of < tokens && k < n;
            member = real ? at % A.group : 0;
            token = list[i0 + (real ? k : i * tokens)];
            ml = A.ml[row_at(A, token.x, j, member)];
            if (!real) ml.y = 0.f;
        };
        if (warp >= 4 && part < tiles) ask(part);
        for (int i = part; i < tiles; i += P.parts) {
            if (!alive) break;
            const int b = done & 1;
            const uint32_t turn = (uint32_t)(done >> 1) & 1u;
            if (warp >= 4) {
                // ---- the rows' queries and sums
                if (done >= 2) alive = ptx::mbar_sleep(ptx::smem_u32(&s_empty[b]), turn ^ 1u, &abort_flag);
                alive = fetchers_agree(alive);          // (they meet below, or none does)
                if (alive) {
                    const bool partial = real && token.y < key0 + kTtKeys - 1;
                    q_s[at] = token.x * A.q_t + j * A.q_h + member * A.q_g;
                    ml_s[b][at] = ml;
                    row_last_s[b][at] = real ? token.y : -1;
                    const bool all = fetchers_agree(!partial);         // (and the rows' places are there)
                    if (at == 0) all_see_s[b] = all;
                    for (int idx = at; idx < kTtRows * CH; idx += 128) {
                        const int rw = idx / CH, ch = idx % CH;
                        const uint32_t dst = base + G::Q + b * G::TILE + (uint32_t)((ch >> 3) * G::PIECE + rw * 128 + (((ch & 7) ^ (rw & 7)) << 4));
                        ptx::cp_async16(dst, A.q + q_s[rw] + ch * 8);
                    }
                    if (i + P.parts < tiles) ask(i + P.parts);
                    ptx::cp_async_commit();
                    ptx::cp_async_wait<0>();
                    ptx::fence_proxy_async();
                    __syncwarp();
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                    ptx::mbar_arrive(ptx::smem_u32(&rows_full[b]));
                }
                if (warp == 4 && alive) {
                    if (ptx::elect_one()) {
                        bool keys = true;
                        if (done == 0) {
                            const uint32_t bar = ptx::smem_u32(&k_full);
                            ptx::mbar_expect_tx(bar, G::TILE);
                            int c[4];
                            c[P.at_pos] = key0, c[P.at_head] = j, c[P.at_seq] = s;
#pragma unroll
                            for (int h = 0; h < G::HALVES; ++h) ptx::tma_load_4d(base + G::K + h * G::PIECE, &mapK, bar, h * 64, c[1], c[2], c[3]);
                            keys = ptx::mbar_sleep(bar, 0, &abort_flag);
                        }
                        ptx::tc_fence_after();
                        const uint32_t q0 = base + G::Q + b * G::TILE, idesc = ptx::make_idesc_bf16(kTtKeys, kTtRows);
#pragma unroll
                        for (int k = 0; k < KS && keys; ++k)
                            ptx::umma_bf16(tmem + b * 128, ptx::make_desc_k_sw128(base + G::K + (k >> 2) * G::PIECE + (k & 3) * 32),
                                           ptx::make_desc_k_sw128(q0 + (k >> 2) * G::PIECE + (k & 3) * 32), idesc, (uint32_t)(k != 0));
                        if (keys) ptx::umma_commit(ptx::smem_u32(&s_full[b]));
                    }
                    __syncwarp();
                }
            } else {
                // ---- a key's weights
                alive = ptx::mbar_sleep(ptx::smem_u32(&rows_full[b]), turn, &abort_flag) && ptx::mbar_sleep(ptx::smem_u32(&s_full[b]), turn, &abort_flag);
                alive = __all_sync(0xffffffffu, alive);
                if (alive) {
                    ptx::tc_fence_after();
                    const uint32_t line = tmem + ((uint32_t)(warp * 32) << 16) + b * 128;
                    const int key = key0 + tid;
                    const bool all_see = all_see_s[b] != 0;
#pragma unroll 1
                    for (int c0 = 0; c0 < kTtRows; c0 += 32) {
                        uint32_t v[32];
                        ptx::tmem_ld32(line + c0, v);
                        ptx::tmem_ld_wait();
                        if (all_see) {
#pragma unroll
                            for (int c = 0; c < 32; c += 2) {
                                const float4 ml = *reinterpret_cast<const float4*>(&ml_s[b][c0 + c]);
                                sum[c & 3] = fmaf(exp2_fast(fmaf(__uint_as_float(v[c]), A.scale_log2, -ml.x)), ml.y, sum[c & 3]);
                                sum[(c + 1) & 3] = fmaf(exp2_fast(fmaf(__uint_as_float(v[c + 1]), A.scale_log2, -ml.z)), ml.w, sum[(c + 1) & 3]);
                            }
                        } else {
                            // (chosen, not multiplied by zero: a key that the row does not see may hold anything)
#pragma unroll
                            for (int c = 0; c < 32; ++c) {
                                const float2 ml = ml_s[b][c0 + c];
                                if (key <= row_last_s[b][c0 + c])
                                    sum[c & 3] = fmaf(exp2_fast(fmaf(__uint_as_float(v[c]), A.scale_log2, -ml.x)), ml.y, sum[c & 3]);
                            }
                        }
                    }
                    ptx::tc_fence_before();
                    ptx::mbar_arrive(ptx::smem_u32(&s_empty[b]));
                }
            }
            ++done;
        }
    }
    chain_next();
    if (!alive && lane == 0) report_status(A.dev_status, DSMOE_ERR_TIMEOUT);
    if (warp < 4 && key0 + tid < A.L) {
        const size_t cells = (size_t)A.n_seq * A.n_head * A.L, at = (size_t)sj * A.L + key0 + tid;
        const float x = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (P.parts > 1) P.out[part * cells + at] = x;
        else P.out[at] = (P.in ? P.in[at] : 0.f) + x;
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 256);
    }
}

// Adds up the parts
__global__ void __launch_bounds__(256) tally_parts_kernel(const float* sums, const int parts, const size_t cells, const float* tally_in, float* tally_out) {
    chain_wait();
    chain_next();
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= cells) return;
    float x = 0.f;
    for (int p = 0; p < parts; ++p) x += sums[p * cells + i];
    tally_out[i] = (tally_in ? tally_in[i] : 0.f) + x;
}

template <int DH>
dsmoe_status launch_tally_tile(const AttnView& A, int parts, float* sums, int2* list, int2* from, const float* tally_in, float* tally_out, cudaStream_t s) {
    using G = TallyGeo<DH>;
    static bool attr[kMaxDeviceSlots] = {};
    int dev = 0;
    DeviceState* st = nullptr;
    DSMOE_TRY(device_state(&st, &dev));
    if (!attr[dev]) {
        DSMOE_CUDA_TRY(cudaFuncSetAttribute(attention_tally_tile_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::SMEM));
        attr[dev] = true;
    }
    CUtensorMap mapK;
    int at[3];
    DSMOE_TRY(make_cache_map(&mapK, A, A.K, at));
    const int key_tiles = ceil_div(A.L, kTtKeys);
    DSMOE_CUDA_TRY(launch_chained(tally_list_kernel, (unsigned)A.n_seq, 1024, 0, s, A, list, from));
    const size_t cells = (size_t)A.n_seq * A.n_head * A.L;
    const long long ctas = (long long)A.n_seq * A.n_head * key_tiles * parts;
    if (ctas > 0x7fffffffll || (cells + 255) / 256 > 0x7fffffffull) return DSMOE_ERR_UNSUPPORTED;
    const TallyArgs P{A, at[0], at[1], at[2], parts, list, from, tally_in, parts > 1 ? sums : tally_out};
    DSMOE_CUDA_TRY(launch_chained(attention_tally_tile_kernel<DH>, (unsigned)ctas, kTtThreads, G::SMEM, s, mapK, P));
    if (parts > 1) DSMOE_CUDA_TRY(launch_chained(tally_parts_kernel, (unsigned)((cells + 255) / 256), 256, 0, s, sums, parts, cells, tally_in, tally_out));
    return DSMOE_OK;
}

template <int DH>
dsmoe_status launch_tally_dh(const AttnView& A, const float* tally_in, float* tally_out, cudaStream_t s) {
    const long long ctas = (long long)A.n_seq * A.n_head * ((A.L + kTallyKeys - 1) / kTallyKeys);
    if (ctas > 0x7fffffffll) return DSMOE_ERR_UNSUPPORTED;
    constexpr size_t smem = (size_t)(kTallyKeys + kTallyRows) * (DH * 2 + 16);
    static bool attr[kMaxDeviceSlots] = {};
    int dev = 0;
    DeviceState* st = nullptr;
    DSMOE_TRY(device_state(&st, &dev));
    if (!attr[dev]) {
        DSMOE_CUDA_TRY(cudaFuncSetAttribute(attention_tally_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        attr[dev] = true;
    }
    DSMOE_CUDA_TRY(launch_chained(attention_tally_kernel<DH>, (unsigned)ctas, 32 * kTallyWarps, smem, s, A, tally_in, tally_out));
    return DSMOE_OK;
}

}  // namespace

dsmoe_status launch_tally_add(const AttnView& A, const float* logits, long long pitch, const float* tally_in, float* tally_out, cudaStream_t s) {
    const long long ctas = (long long)A.n_seq * A.n_head * ((A.L + kAddKeys - 1) / kAddKeys);
    if (A.T > kListTokens || ctas > 0x7fffffffll) return DSMOE_ERR_UNSUPPORTED;
    DSMOE_CUDA_TRY(launch_chained(tally_add_kernel, (unsigned)ctas, kAddThreads, 0, s, A, logits, pitch, tally_in, tally_out));
    return DSMOE_OK;
}

dsmoe_status launch_tally(const AttnView& A, int parts, float* sums, int2* list, int2* from, const float* tally_in, float* tally_out, cudaStream_t s) {
    if (parts > 0) {
        if (A.d_head == 64) return launch_tally_tile<64>(A, parts, sums, list, from, tally_in, tally_out, s);
        if (A.d_head == 96) return launch_tally_tile<96>(A, parts, sums, list, from, tally_in, tally_out, s);
        return launch_tally_tile<128>(A, parts, sums, list, from, tally_in, tally_out, s);
    }
    switch (A.d_head) {
        case 32: return launch_tally_dh<32>(A, tally_in, tally_out, s);
        case 64: return launch_tally_dh<64>(A, tally_in, tally_out, s);
        case 96: return launch_tally_dh<96>(A, tally_in, tally_out, s);
        case 128: return launch_tally_dh<128>(A, tally_in, tally_out, s);
        case 160: return launch_tally_dh<160>(A, tally_in, tally_out, s);
        case 192: return launch_tally_dh<192>(A, tally_in, tally_out, s);
        case 224: return launch_tally_dh<224>(A, tally_in, tally_out, s);
        case 256: return launch_tally_dh<256>(A, tally_in, tally_out, s);
        default: return DSMOE_ERR_UNSUPPORTED;
    }
}

}  // namespace dsmoe
