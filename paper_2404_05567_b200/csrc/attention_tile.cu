// Attention of many rows that share their keys (prompts; a batch's shared prefix) on the 5th-generation tensor cores.
//
// A CTA owns up to 256 rows (neighbouring tokens' query heads of one key/value head) as two tiles of 128, and walks the keys that any of them sees in
// tiles of 128 keys, which both tiles use.  Per tile of rows and keys: S = Q.K^T into tensor memory; a row's two threads take its logits from
// there, its weights 2^(logit - m) go back as bf16 where the logits lay, and O += P.V with P as the operand in tensor memory and V as it lies in
// memory (N-major).  The weights are rounded to bf16 (by 2^-8 of each at most): the tensor pipe takes no wider ones at this rate.  Sums and O are
// fp32.  The running maximum hardly ever moves (kMoves); if it does, the row's threads rescale O in tensor memory.
// Roles: warps 0-7 and 8-15 are the two tiles' rows, two threads a row; warp 16 copies (TMA, a ring of tiles), warp 17 issues the MMAs, warp 18 clears
// the values behind a stretch's last key (0 times what is no number is no number).  While one tile's threads are at their weights the tensor
// pipe works for the other one.
// Bound by the threads' way from logits to weights: a step of 256 rows and 128 keys of 128 numbers takes 3400 cycles, of which the exponentials
// alone take the special-function units 2048 and the MMAs the tensor pipe 2100; with an eighth of the MMAs a call still took four fifths of its time.
// 8192 tokens of 4 x 5 heads with a window of 4096: 274 us, 0.57 of the tensor rate, at the power limit (1.7 GHz).  Tried there, us: a quarter of the
// exponentials by polynomial 289 (276 without), the two row tiles taking turns at their exponentials 312 (311 without).
//
// What a CTA's tokens see: tokens of one sequence that follow one another are a run; a run's keys are at most three stretches of slots (sinks, and
// the window, cut in two where a ring ends).  In blocks of many runs, those too short to be worth a
// pass of a tile's over their keys are left to attention_stream_kernel.
// A value that is not finite reaches all rows of a tile, also those that do not see it: rows that come out as no numbers are done again, one by one.
#include <stddef.h>

#include "cache_attention.cuh"
#include "tensor_maps.cuh"
#include "umma.cuh"

namespace dsmoe {

namespace {

// A block of up to kFewRuns runs (prompts' ends and beginnings) is taken as it is: each costs a pass over its keys
constexpr int kTileRows = 128, kTileKeys = 128, kTileThreads = 608, kLoadWarp = 16, kMmaWarp = 17, kClearWarp = 18, kFewRuns = 4, kMaxRuns = 16, kMaxStretches = 3 * kMaxRuns, kSightWarps = 8;

template <int DH>
struct TileGeo {
    static constexpr int HALVES = (DH + 63) / 64;                      // 128-byte pieces of a row
    static constexpr uint32_t PIECE = kTileRows * 128, TILE = HALVES * PIECE;
    static constexpr int STAGES = HALVES == 1 ? 4 : 2;
    static constexpr uint32_t Q = 0, K = 2 * TILE, V = K + STAGES * TILE, END = V + STAGES * TILE;
    static constexpr int SMEM = (int)END + 1024;
};

struct Stretch {
    int run, seq, slot0, pos0, n, tile0;  // n keys of a run's, from slot0 / position pos0 on; tile0: tiles before
};

struct TileShared {
    // (in one row: a thread each sets them up)
    uint64_t k_full[4], k_empty[4], v_full[4], v_clear[4], v_empty[4], s_full[2], p_full[2][2], o_done[2];
    uint32_t tmem;
    volatile int abort_flag;
    int n_stretches, n_runs, alike;      // (alike: of one sequence)
    int begin, end;                       // this CTA's tiles
    long long q_at[2 * kTileRows];        // where a row's queries are; -1: no row
    int seq[2 * kTileRows], first[2 * kTileRows], last[2 * kTileRows], run[2 * kTileRows];
    int run_len[2 * kTileRows], run_lo[2 * kTileRows], run_hi[2 * kTileRows];
    int redo[2 * kTileRows];              // rows that came out as no numbers
    float tops[2][2][2][kTileRows];       // the largest logit of each half of a tile's, by turn
    float swap[2][2][kTileRows];          // the halves of a row's threads tell each other
    Stretch st[kMaxStretches];
};
constexpr int kTileBars = 28, kFirstPFull = 22;
static_assert(offsetof(TileShared, tmem) == kTileBars * 8 && offsetof(TileShared, p_full) == kFirstPFull * 8, "the barriers in a row");

__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Two fp32 numbers at a time
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void halves_of(uint64_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Operand B = V as it lies in memory, [128 keys][64 columns] in the 128-byte swizzle: N-major.  Eight keys are 1024 bytes, the next 64 columns
// begin 128 rows further on.
__device__ __forceinline__ uint64_t make_desc_values(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFF) >> 4);
    d |= (uint64_t)((kTileKeys * 128) >> 4) << 16;                     // leading byte offset: between 64-column groups
    d |= (uint64_t)(1024 >> 4) << 32;                                  // stride byte offset: between groups of 8 keys
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 columns, waited for.  (A wait of its own needs a fence for each of the 32 registers, and those cost moves.)
__device__ __forceinline__ void tmem_ld32_now(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// The two warps that share rows (64 threads) at their barrier: whether any of them, or all, say so
__device__ __forceinline__ bool pair_any(int id, bool x) {
    uint32_t y;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.or.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(y) : "r"(id), "r"((uint32_t)x) : "memory");
    return y != 0;
}
__device__ __forceinline__ bool pair_all(int id, bool x) {
    uint32_t y;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.and.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(y) : "r"(id), "r"((uint32_t)x) : "memory");
    return y != 0;
}
__device__ __forceinline__ void pair_sync(int id) {
    __syncwarp();
    asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
}

__device__ __forceinline__ void sight_sync() {
    __syncwarp();
    asm volatile("bar.sync 9, %0;" ::"n"(32 * (kSightWarps + 1)) : "memory");
}

struct TileArgs {
    AttnView A;
    int tile_tokens;                      // tokens of a 128-row tile
    int least_run;
    int blocks, splits;
    int at_pos, at_head, at_seq;          // which of the tensor map's dimensions 1 .. 3 are positions, heads, sequences
    float *o, *ml;                        // parts [split][T * n_head * group][DH], [..][2]; nullptr: out and lse are written
    int32_t *count, *list;                // the tokens that are left: block b's count[b], from list[b * span] on; nullptr: none is
    int2* head;                           // the stream kernel's, nullable
};

// Key tile i: the stretch that holds it (the caller's `at` only grows), its first key there
struct Tile {
    int run, seq, slot, pos, n;           // n: keys of the tile, up to 128
};
__device__ __forceinline__ Tile tile_at(const TileShared& S, int i, int& at) {
    while (at + 1 < S.n_stretches && S.st[at + 1].tile0 <= i) ++at;
    const Stretch& s = S.st[at];
    const int k = (i - s.tile0) * kTileKeys;
    return Tile{s.run, s.seq, s.slot0 + k, s.pos0 + k, min(kTileKeys, s.n - k)};
}

template <int DH>
__global__ void __launch_bounds__(kTileThreads, 1)
attention_tile_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ TileArgs P) {
    using G = TileGeo<DH>;
    constexpr int CH = DH / 8, KS = DH / 16, STAGES = G::STAGES;
    extern __shared__ unsigned char tile_smem[];
    __shared__ TileShared S;
    const AttnView& A = P.A;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = ptx::smem_u32(tile_smem), base = (raw + 1023u) & ~1023u;
    unsigned char* const smem = tile_smem + (base - raw);
    // the blocks with the most keys (the last tokens) go first
    const int j = (int)(blockIdx.x % A.n_head), split = (int)(blockIdx.x / A.n_head) % P.splits;
    const int block = P.blocks - 1 - (int)(blockIdx.x / A.n_head / P.splits);
    const int span = 2 * P.tile_tokens, tg0 = block * span, ng = min(A.T - tg0, span);
    const int tiles_of_rows = ng > P.tile_tokens ? 2 : 1;
    if (tid < kTileBars) {
        ptx::mbar_init(ptx::smem_u32(&S.k_full[0]) + 8u * tid, tid >= kFirstPFull && tid < kFirstPFull + 4 ? 2 * kTileRows : 1);
        ptx::fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(ptx::smem_u32(&S.tmem), 512);
        ptx::tmem_relinquish();
    }
    if (tid < 2 * kTileRows) {
        const int r = tid >> 7, at = tid & 127, tl = r * P.tile_tokens + at / A.group;
        S.q_at[tid] = at < P.tile_tokens * A.group && tl < ng ? (tg0 + tl) * A.q_t + j * A.q_h + at % A.group * A.q_g : -1;
        S.redo[tid] = 0;
    }
    if (tid == 0) {
        S.abort_flag = 0;
        S.n_runs = 1;
        S.alike = 1;
        S.run_lo[0] = 0x7fffffff;
        S.run_hi[0] = -1;
    }
    __syncthreads();
    chain_wait();
    int load_at = 0;                      // the stretch of the load warp's next tile
    const auto load = [&](const CUtensorMap* map, uint32_t dst, uint64_t* bar, const Tile& t) {
        const uint32_t b = ptx::smem_u32(bar);
        ptx::mbar_expect_tx(b, G::TILE);
        int c[4];
        c[P.at_pos] = t.slot, c[P.at_head] = j, c[P.at_seq] = t.seq;
#pragma unroll
        for (int h = 0; h < G::HALVES; ++h) ptx::tma_load_4d(dst + h * G::PIECE, map, b, h * 64, c[1], c[2], c[3]);
    };
    if (warp < kSightWarps || warp == kLoadWarp) {
        // ---- what the tokens see, and the runs
        bool bad = false, like = true;
        if (warp * 32 < ng) {
            int lo = 0x7fffffff, hi = -1;
            if (tid < ng) {
                const Sight s = sight_of(A, tg0 + tid, &bad);
                like = s.seq == (A.tok_seq ? min(max(A.tok_seq[tg0], 0), A.n_seq - 1) : 0);
                hi = s.last;
                const int first = hi >= A.window ? hi - A.window + 1 : 0;
                if (hi >= 0) lo = first;
                S.seq[tid] = s.seq;
                S.last[tid] = hi;
                S.first[tid] = first;
            }
            // (of one run: of all tokens)
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (lane == 0) {
                atomicMin(&S.run_lo[0], lo);
                atomicMax(&S.run_hi[0], hi);
            }
            if (bad) report_status(A.dev_status, DSMOE_ERR_INVALID_ARG);
        }
        if (__any_sync(0xffffffffu, !like) && lane == 0) S.alike = 0;
        sight_sync();
        const bool alike = S.alike != 0;
        if (!alike) {
            if (tid < ng) {
                S.run_len[tid] = 0;
                S.run_lo[tid] = 0x7fffffff;
                S.run_hi[tid] = -1;
            }
            if (warp == 0) {                  // a token's run: how many runs begin at or before it, less one
                int before = 0;
                for (int c = 0; c < ng; c += 32) {
                    const int t = c + lane;
                    const bool begins = t < ng && t > 0 && S.seq[t] != S.seq[t - 1];
                    const uint32_t votes = __ballot_sync(0xffffffffu, begins);
                    if (t < ng) S.run[t] = before + __popc(votes & (0xffffffffu >> (31 - lane)));
                    before += __popc(votes);
                }
                if (lane == 0) S.n_runs = before + 1;
            }
            sight_sync();
            if (tid < ng) {
                const int r = S.run[tid];
                atomicAdd(&S.run_len[r], 1);
                if (S.last[tid] >= 0) {
                    atomicMin(&S.run_lo[r], S.first[tid]);
                    atomicMax(&S.run_hi[r], S.last[tid]);
                }
            }
            sight_sync();
        }
        const bool takes_all = alike || !P.count || S.n_runs <= kFewRuns;
        if (split == 0 && P.head && tid < ng)
            for (int i = 0; i < A.row_tiles; ++i) P.head[((long long)(tg0 + tid) * A.n_head + j) * A.row_tiles + i] = make_int2(0, 0);
        if (warp == 1 && split == 0 && j == 0 && P.count) {        // the tokens that are left, in order
            int n = 0;
            for (int c = 0; c < ng && !takes_all; c += 32) {
                const int t = c + lane;
                const bool left = t < ng && S.run_len[S.run[t]] < P.least_run;
                const uint32_t votes = __ballot_sync(0xffffffffu, left);
                if (left) P.list[(long long)block * span + n + __popc(votes & ((1u << lane) - 1u))] = tg0 + t;
                n += __popc(votes);
            }
            if (lane == 0) P.count[block] = n;
        }
        if (warp == kLoadWarp) {
            // ---- the stretches, and the first tiles' copies
            if (ptx::elect_one()) {
                int n = 0, tiles = 0, t = 0;
                const auto put = [&](int run, int seq, int pos0, int count) {
                    while (count > 0) {       // (in a ring, up to its end and then from its beginning)
                        const int slot = slot_of(A, pos0), m = A.ring && pos0 >= A.sinks ? min(count, A.L - slot) : count;
                        S.st[n++] = Stretch{run, seq, slot, pos0, m, tiles};
                        tiles += (m + kTileKeys - 1) / kTileKeys;
                        pos0 += m;
                        count -= m;
                        if (n == kMaxStretches) return;
                    }
                };
                const int n_runs = alike ? 1 : S.n_runs;
                for (int r = 0; r < n_runs; ++r) {
                    const int len = alike ? ng : S.run_len[r], hi = S.run_hi[r];
                    int lo = S.run_lo[r];
                    if (A.ring && hi - max(lo, A.sinks) >= A.ring) {      // more positions than a ring holds: the latest of them, and no more
                        lo = hi - A.ring + 1;
                        report_status(A.dev_status, DSMOE_ERR_INVALID_ARG);
                    }
                    if ((takes_all || len >= P.least_run) && hi >= 0 && n + 3 <= kMaxStretches) {
                        const int sinks = min(A.sinks, hi + 1);
                        if (lo <= sinks) {
                            put(r, S.seq[t], 0, hi + 1);
                        } else {
                            put(r, S.seq[t], 0, sinks);
                            put(r, S.seq[t], lo, hi + 1 - lo);
                        }
                    }
                    t += len;
                }
                S.n_stretches = n;
                const int begin = P.splits == 1 ? 0 : (int)((long long)tiles * split / P.splits);
                const int end = P.splits == 1 ? tiles : (int)((long long)tiles * (split + 1) / P.splits);
                S.begin = begin;
                S.end = end;
                for (int i = 0; i < min(STAGES, end - begin); ++i) {
                    const Tile x = tile_at(S, begin + i, load_at);
                    load(&mapK, base + G::K + i * G::TILE, &S.k_full[i], x);
                    load(&mapV, base + G::V + i * G::TILE, &S.v_full[i], x);
                }
            }
            __syncwarp();
        }
    } else {
        // ---- queries, in the swizzle's order; rows that are none are zeros
        constexpr int QUERY_THREADS = kTileThreads - 32 * (kSightWarps + 1);
        for (int idx = tid - 32 * (warp < kLoadWarp ? kSightWarps : kSightWarps + 1); idx < tiles_of_rows * kTileRows * CH; idx += QUERY_THREADS) {
            const int row = idx / CH, ch = idx % CH, r = row >> 7, at = row & 127;
            const long long from = S.q_at[row];
            const uint32_t dst = base + G::Q + r * G::TILE + (uint32_t)((ch >> 3) * G::PIECE + at * 128 + (((ch & 7) ^ (at & 7)) << 4));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(A.q + (from < 0 ? 0 : from) + ch * 8), "r"(from < 0 ? 0u : 16u) : "memory");
        }
        ptx::cp_async_commit();
    }
    // the rows' threads: two each, with 64 of a tile's 128 logits and half of O's columns
    const int r = warp >> 3, half = (warp >> 2) & 1, at = (warp & 3) * 32 + lane;      // row tile, half, row of the tile = lane of tensor memory
    const int tl = r * P.tile_tokens + at / A.group, m_of = at % A.group;
    const bool real = at < P.tile_tokens * A.group && tl < ng;
    ptx::cp_async_wait<0>();
    ptx::fence_proxy_async();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const bool alike = S.alike != 0, takes_all = alike || !P.count || S.n_runs <= kFewRuns;
    const uint32_t tmem = S.tmem;
    const int begin = S.begin, n = S.end - S.begin;
    bool not_finite = false;              // this thread's row

    if (warp == kLoadWarp) {
        // ---- copies
        if (ptx::elect_one()) {
            int issued = min(STAGES, n);
            for (int i = issued; i < n; ++i) {
                const int s = i % STAGES;
                const uint32_t parity = (uint32_t)((i / STAGES) & 1) ^ 1u;
                const Tile t = tile_at(S, begin + i, load_at);
                if (!ptx::mbar_sleep(ptx::smem_u32(&S.k_empty[s]), parity, &S.abort_flag)) break;
                load(&mapK, base + G::K + s * G::TILE, &S.k_full[s], t);
                if (!ptx::mbar_sleep(ptx::smem_u32(&S.v_empty[s]), parity, &S.abort_flag)) break;
                load(&mapV, base + G::V + s * G::TILE, &S.v_full[s], t);
                issued = i + 1;
            }
            if (S.abort_flag) {           // copies in flight end before the CTA does
                int none = 0;
                for (int i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i) {
                    ptx::mbar_wait(ptx::smem_u32(&S.k_full[i % STAGES]), (uint32_t)((i / STAGES) & 1), &none);
                    ptx::mbar_wait(ptx::smem_u32(&S.v_full[i % STAGES]), (uint32_t)((i / STAGES) & 1), &none);
                }
                if (issued < n) ptx::mbar_wait(ptx::smem_u32(&S.k_full[issued % STAGES]), (uint32_t)((issued / STAGES) & 1), &none);
            }
        }
        __syncwarp();
    } else if (warp == kClearWarp) {
        // ---- values that are no keys': zeros
        int at = 0;
        for (int i = 0; i < n; ++i) {
            const Tile t = tile_at(S, begin + i, at);
            const int s = i % STAGES;
            if (!__all_sync(0xffffffffu, ptx::mbar_sleep(ptx::smem_u32(&S.v_full[s]), (uint32_t)((i / STAGES) & 1), &S.abort_flag))) break;
            if (t.n < kTileKeys) {
                unsigned char* const v = smem + G::V + s * G::TILE;
                for (int idx = lane; idx < (kTileKeys - t.n) * 8 * G::HALVES; idx += 32) {
                    const int piece = idx % (8 * G::HALVES), row = t.n + idx / (8 * G::HALVES);
                    *reinterpret_cast<uint4*>(v + (piece >> 3) * G::PIECE + row * 128 + (piece & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                ptx::fence_proxy_async();
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&S.v_clear[s]));         // (of every tile: the MMAs wait for it alone)
        }
    } else if (warp == kMmaWarp) {
        // ---- MMAs
        if (ptx::elect_one()) {
            const uint32_t idesc_s = ptx::make_idesc_bf16(kTileRows, kTileKeys), idesc_o = ptx::make_idesc_bf16(kTileRows, DH) | (1u << 16);
            const auto logits = [&](int i, int r) {
                const uint32_t q0 = base + G::Q + r * G::TILE, k0 = base + G::K + (i % STAGES) * G::TILE;
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    ptx::umma_bf16(tmem + r * 128, ptx::make_desc_k_sw128(q0 + (k >> 2) * G::PIECE + (k & 3) * 32),
                                   ptx::make_desc_k_sw128(k0 + (k >> 2) * G::PIECE + (k & 3) * 32), idesc_s, (uint32_t)(k != 0));
                ptx::umma_commit(ptx::smem_u32(&S.s_full[r]));
            };
            bool ok = true;
            if (n > 0) {
                ok = ptx::mbar_sleep(ptx::smem_u32(&S.k_full[0]), 0, &S.abort_flag);
                if (ok) {
                    for (int r = 0; r < tiles_of_rows; ++r) logits(0, r);
                    ptx::umma_commit(ptx::smem_u32(&S.k_empty[0]));
                }
            }
            for (int i = 0; ok && i < n; ++i) {
                const int s = i % STAGES;
                ok = ptx::mbar_sleep(ptx::smem_u32(&S.v_clear[s]), (uint32_t)((i / STAGES) & 1), &S.abort_flag);
                if (ok && i + 1 < n)
                    ok = ptx::mbar_sleep(ptx::smem_u32(&S.k_full[(i + 1) % STAGES]), (uint32_t)(((i + 1) / STAGES) & 1), &S.abort_flag);
                for (int r = 0; ok && r < tiles_of_rows; ++r) {
                    const uint32_t v0 = base + G::V + s * G::TILE;
                    // The weights of keys 0 .. 63 lie in the first 32 columns of those keys' logits, and the others' in the first of theirs; each 64
                    // come in two parts, and the first ones' products run while the rows' threads are at the second
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        ok = ok && ptx::mbar_sleep(ptx::smem_u32(&S.p_full[r][part]), (uint32_t)(i & 1), &S.abort_flag);
                        if (!ok) break;
                        ptx::tc_fence_after();
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int k = (q >> 1) * 4 + part * 2 + (q & 1);
                            umma_bf16_ts(tmem + 256 + r * 128, tmem + r * 128 + (k >> 2) * 64 + (k & 3) * 8, make_desc_values(v0 + k * 2048), idesc_o,
                                         (uint32_t)(i != 0 || k != 0));
                        }
                    }
                    if (!ok) break;
                    ptx::umma_commit(ptx::smem_u32(&S.o_done[r]));
                    if (i + 1 < n) logits(i + 1, r);
                }
                if (!ok) break;
                ptx::umma_commit(ptx::smem_u32(&S.v_empty[s]));
                if (i + 1 < n) ptx::umma_commit(ptx::smem_u32(&S.k_empty[(i + 1) % STAGES]));
            }
        }
        __syncwarp();
    } else {
        // ---- rows
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + r * 128, tO = tmem + lanes + 256 + r * 128 + half * (DH / 2);
        const int pair = 1 + r * 4 + (warp & 3);                          // the barrier of the two warps that share rows
        const bool taken = real && (takes_all || S.run_len[S.run[tl]] >= P.least_run);
        const int run = !taken ? -1 : alike ? 0 : S.run[tl], last = taken ? S.last[tl] : -1, first = taken ? S.first[tl] : 0;
        const float sl2 = A.scale_log2;
        float m = taken ? -INFINITY : 0.f, l = 0.f, top = -INFINITY;
        bool alive = true;                // (no tile is left out when a wait runs out, so that the warps of a pair keep meeting)
        int stretch = 0;
        if (r < tiles_of_rows) {
            const uint32_t place = tS + half * 64;
            const uint64_t scale2 = pair_of(sl2, sl2);
            for (int i = 0; i < n; ++i) {
                const Tile t = tile_at(S, begin + i, stretch);
                // keys a .. b of this half of the tile are the row's, and those before c
                // (positions reach 2^31 - 2, so they are compared before anything is added)
                const int off = half * 64;
                const int b = t.run == run ? min(max(last - t.pos, -1), t.n - 1) - off : -1, a = max(first - t.pos, 0) - off, c = max(A.sinks - t.pos, 0) - off;
                // (rows that are nobody's see anything; the same sequence may have two runs in this block)
                const bool full = __all_sync(0xffffffffu, !taken || (b >= 63 && (a <= 0 || c >= 64)));
                uint64_t seen = ~0ull;
                if (!full) {
                    const uint64_t upto = b < 0 ? 0ull : b >= 63 ? ~0ull : (2ull << b) - 1ull;
                    const uint64_t from = a <= 0 ? ~0ull : a >= 64 ? 0ull : ~0ull << a;
                    const uint64_t sinks = c <= 0 ? 0ull : c >= 64 ? ~0ull : (1ull << c) - 1ull;
                    seen = upto & (from | sinks);
                }
                alive = ptx::mbar_sleep(ptx::smem_u32(&S.s_full[r]), (uint32_t)(i & 1), &S.abort_flag) && alive;
                __syncwarp();
                ptx::tc_fence_after();
                // The maximum moves if the tile before asks for it.  (What the other half found there lies ready: these logits come behind both
                // halves' weights.  O is all there too: S of this tile follows the tile before's P.V in the tensor pipe.)
                // So that tile's weights were relative to the maximum before it: up to 2^128, beyond which the row is no number and is done again.
                // The smallest factor is 2^-126 (a smaller one would be flushed, and the tile's sums with it): the rest is within kMoves.
                if (i > 0) {
                    top = fmaxf(top, S.tops[(i - 1) & 1][r][half ^ 1][at]);
                    const bool moves = m != -INFINITY && top > m + kMoves;
                    if (__any_sync(0xffffffffu, moves)) {
                        const float by = moves ? fminf(top - m, 126.f) : 0.f, f = exp2_fast(-by);
                        m += by;
                        l *= f;
#pragma unroll 1
                        for (int q = 0; q < DH / 32; ++q) {
                            uint32_t o[16];
                            ptx::tmem_ld16(tO + q * 16, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_st16(tO + q * 16, o);
                        }
                    }
                }
                const auto logits_of = [&](int part, uint32_t (&x)[32]) {
                    tmem_ld32_now(place + part * 32, x);
                    if (!full) {
                        const uint32_t bits = (uint32_t)(seen >> (32 * part));
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = bits & (1u << k) ? x[k] : 0xff800000u;   // -inf
                    }
                };
                // Rows that have no maximum yet (m is the same in both halves) find one first
                if (__any_sync(0xffffffffu, m == -INFINITY)) {
                    top = -INFINITY;
#pragma unroll 1
                    for (int part = 0; part < 2; ++part) {
                        uint32_t x[32];
                        logits_of(part, x);
#pragma unroll
                        for (int k = 0; k < 32; k += 2) top = max3(top, __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                    }
                    S.swap[r][half][at] = top * sl2;
                    pair_sync(pair);
                    if (m == -INFINITY) m = fmaxf(top * sl2, S.swap[r][half ^ 1][at]);
                }
                const float z = m == -INFINITY ? 0.f : -m;
                const uint64_t z2 = pair_of(z, z);
                uint64_t s2[2] = {pair_of(0.f, 0.f), pair_of(0.f, 0.f)};
                float top2 = -INFINITY;
                top = -INFINITY;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t x[32], w[16];
                    logits_of(part, x);
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        top = max3(top, __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                        top2 = max3(top2, __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
                    }
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float a, b;
                        halves_of(fma2(pair_of(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), scale2, z2), a, b);
                        a = exp2_fast(a);
                        b = exp2_fast(b);
                        s2[k & 1] = add2(s2[k & 1], pair_of(a, b));
                        w[k] = pack2(a, b);
                    }
                    tmem_st16(place + part * 16, w);
                    if (part == 1) {
                        top = fmaxf(top, top2) * sl2;
                        S.tops[i & 1][r][half][at] = top;
                    }
                    tmem_st_wait();
                    ptx::tc_fence_before();
                    ptx::mbar_arrive(ptx::smem_u32(&S.p_full[r][part]));
                }
                float s_a, s_b;
                halves_of(add2(s2[0], s2[1]), s_a, s_b);
                l += s_a + s_b;
            }
            // (one phase to wait for: the last logits came behind the last but one tile's P.V)
            if (n > 0) alive = ptx::mbar_sleep(ptx::smem_u32(&S.o_done[r]), (uint32_t)((n - 1) & 1), &S.abort_flag) && alive;
            __syncwarp();
            alive = pair_all(pair, alive && !S.abort_flag);
            ptx::tc_fence_after();
            if (!alive && lane == 0) report_status(A.dev_status, DSMOE_ERR_TIMEOUT);
        }
        if (alive && r < tiles_of_rows) {
            S.swap[r][half][at] = l;
            pair_sync(pair);
            l = S.swap[r][0][at] + S.swap[r][1][at];
            // Where weights were far above 1, the maximum follows them by a power of two: 1 / l and other parts' factors keep their bits, and parts of
            // large values have a sum
            const bool high = l >= 0x1p16f;                               // (infinite sums are found below)
            const int up = high ? min((int)(__float_as_uint(l) >> 23) - 127, 126) : 0;
            const float down = __uint_as_float((uint32_t)(127 - up) << 23);
            l *= down;
            m += (float)up;
            const long long row = row_at(A, tg0 + tl, j, m_of);
            const float inv = P.o ? 1.f : l == 0.f ? 0.f : 1.f / l;
            constexpr int HC = DH / 2;                                    // a thread's columns
            constexpr int LINE = (int)(G::TILE / kTileRows) / 2;          // its staging: 64 or 128 bytes, through the queries' place (every S is done)
            uint32_t o[HC];
            if (n > 0) {
                ptx::tmem_ld32(tO, *reinterpret_cast<uint32_t(*)[32]>(o));
                if (HC == 64) ptx::tmem_ld32(tO + 32, *reinterpret_cast<uint32_t(*)[32]>(o + HC - 32));
                if (HC == 48) ptx::tmem_ld16(tO + 32, *reinterpret_cast<uint32_t(*)[16]>(o + HC - 16));
                ptx::tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < HC; ++k) asm volatile("" : "+r"(o[k]));
                if (__any_sync(0xffffffffu, high)) {
#pragma unroll
                    for (int k = 0; k < HC; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * down);
                }
            } else {
#pragma unroll
                for (int k = 0; k < HC; ++k) o[k] = 0u;
            }
            float check = l * 0.f;
#pragma unroll
            for (int k = 0; k < HC; ++k) check = fmaf(__uint_as_float(o[k]), 0.f, check);
            unsigned char* const stage = smem + G::Q + r * G::TILE + ((warp & 3) * 2 + half) * 32 * LINE;
            const long long dst = (P.o ? (real ? ((long long)split * A.T * A.n_head * A.group + row) * DH : -1)
                                       : (taken ? (tg0 + tl) * A.o_t + j * A.o_h + m_of * A.o_g : -1));
            if (P.o) {
                constexpr int AT_ONCE = LINE / 4;                         // columns
#pragma unroll
                for (int c0 = 0; c0 < HC; c0 += AT_ONCE) {
                    constexpr int SLOTS = LINE / 16;
                    const int chunks = min(AT_ONCE, HC - c0) / 4;
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < SLOTS; ++k)
                        if (c0 + 4 * k < HC)
                            *reinterpret_cast<uint4*>(stage + lane * LINE + ((k ^ (lane % SLOTS)) << 4)) =
                                make_uint4(o[(c0 + 4 * k) % HC], o[(c0 + 4 * k + 1) % HC], o[(c0 + 4 * k + 2) % HC], o[(c0 + 4 * k + 3) % HC]);
                    __syncwarp();
                    for (int idx = lane; idx < 32 * chunks; idx += 32) {
                        const int rw = idx / chunks, ch = idx % chunks;
                        const long long to = __shfl_sync(0xffffffffu, dst, rw);
                        if (to >= 0)
                            *reinterpret_cast<uint4*>(P.o + to + half * HC + c0 + ch * 4) = *reinterpret_cast<const uint4*>(stage + rw * LINE + ((ch ^ (rw % SLOTS)) << 4));
                    }
                }
            } else {
                constexpr int CHUNKS = HC / 8, SLOTS = LINE / 16;
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = pack2(__uint_as_float(o[8 * k + 2 * e]) * inv, __uint_as_float(o[8 * k + 2 * e + 1]) * inv);
                    *reinterpret_cast<uint4*>(stage + lane * LINE + ((k ^ (lane % SLOTS)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                __syncwarp();
#pragma unroll
                for (int x = 0; x < CHUNKS; ++x) {
                    const int idx = lane + 32 * x, rw = idx / CHUNKS, ch = idx % CHUNKS;
                    const long long to = __shfl_sync(0xffffffffu, dst, rw);
                    if (to >= 0) *reinterpret_cast<uint4*>(A.out + to + half * HC + ch * 8) = *reinterpret_cast<const uint4*>(stage + rw * LINE + ((ch ^ (rw % SLOTS)) << 4));
                }
            }
            not_finite = taken && check != 0.f;
            if (not_finite) S.redo[r * kTileRows + at] = 1;
            if (half == 0) {
                if (P.o) {
                    if (real)
                        *reinterpret_cast<float2*>(P.ml + ((size_t)split * A.T * A.n_head * A.group + row) * 2) =
                            taken && l != 0.f ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
                } else if (taken) {
                    const float z = m == -INFINITY ? 0.f : m;
                    if (A.lse) A.lse[row] = (z + log2f(l)) * 0.6931471805599453f;
                    if (A.ml) A.ml[row] = make_float2(z, inv);
                }
            }
        }
    }
    chain_next();
    ptx::tc_fence_before();
    const bool again = __syncthreads_or(not_finite) != 0;
    if (warp == kMmaWarp) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
    if (!again) return;
    // ---- rows that came out as no numbers: a warp per row, a key at a time, over this CTA's tiles
    for (int rr = warp; rr < 2 * kTileRows; rr += kTileThreads / 32) {
        if (!S.redo[rr]) continue;
        constexpr int PER = DH / 32;
        const int r = rr / kTileRows, at = rr % kTileRows, tl = r * P.tile_tokens + at / A.group, m_of = at % A.group;
        const __nv_bfloat16* const q = A.q + (tg0 + tl) * A.q_t + j * A.q_h + m_of * A.q_g;
        float qv[PER], o[PER], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            qv[e] = __bfloat162float(q[lane + 32 * e]);
            o[e] = 0.f;
        }
        int stretch = 0;
        for (int i = 0; i < n; ++i) {
            const Tile t = tile_at(S, begin + i, stretch);
            if (!alike && t.run != S.run[tl]) continue;
            for (int k = 0; k < t.n; ++k) {
                const int pos = t.pos + k;
                if (pos > S.last[tl] || (pos < S.first[tl] && pos >= A.sinks)) continue;
                const long long src = t.seq * A.kv_s + j * A.kv_h + slot_of(A, pos) * A.kv_p + lane;
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < PER; ++e) dot = fmaf(qv[e], __bfloat162float(A.K[src + 32 * e]), dot);
#pragma unroll
                for (int w = 16; w > 0; w >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, w);
                dot *= A.scale_log2;
                const float top = fmaxf(m, dot), f = m == -INFINITY ? 0.f : exp2_fast(m - top), p = dot == -INFINITY ? 0.f : exp2_fast(dot - top);
                m = top;
                l = fmaf(l, f, p);
#pragma unroll
                for (int e = 0; e < PER; ++e) o[e] = fmaf(o[e], f, p * __bfloat162float(A.V[src + 32 * e]));
            }
        }
        const long long row = ((long long)(tg0 + tl) * A.n_head + j) * A.group + m_of;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (P.o) P.o[((size_t)split * A.T * A.n_head * A.group + row) * DH + lane + 32 * e] = o[e];
            else A.out[(tg0 + tl) * A.o_t + j * A.o_h + m_of * A.o_g + lane + 32 * e] = __float2bfloat16_rn(o[e] * inv);
        }
        if (lane == 0) {
            const float z = m == -INFINITY ? 0.f : m;
            if (P.o) {
                *reinterpret_cast<float2*>(P.ml + ((size_t)split * A.T * A.n_head * A.group + row) * 2) = make_float2(m, l);
            } else {
                if (A.lse) A.lse[row] = (z + log2f(l)) * 0.6931471805599453f;
                if (A.ml) A.ml[row] = make_float2(z, inv);
            }
        }
    }
}

template <int DH>
dsmoe_status launch_tile(const AttnView& A, const TilePlan& plan, cudaStream_t s) {
    using G = TileGeo<DH>;
    static bool attr[kMaxDeviceSlots] = {};
    int dev = 0;
    DeviceState* st = nullptr;
    DSMOE_TRY(device_state(&st, &dev));
    if (!attr[dev]) {
        DSMOE_CUDA_TRY(cudaFuncSetAttribute(attention_tile_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::SMEM));
        attr[dev] = true;
    }
    CUtensorMap mapK, mapV;
    int at[3];
    DSMOE_TRY(make_cache_map(&mapK, A, A.K, at));
    DSMOE_TRY(make_cache_map(&mapV, A, A.V, at));
    TileArgs P{A, kTileRows / A.group, tile_least_run(A.group), tile_blocks(A.T, A.group), plan.splits, at[0], at[1], at[2], plan.o, plan.ml,
               plan.count, plan.list, plan.head};
    const long long ctas = (long long)P.blocks * A.n_head * plan.splits;
    if (ctas > 0x7fffffffll) return DSMOE_ERR_UNSUPPORTED;
    DSMOE_CUDA_TRY(launch_chained(attention_tile_kernel<DH>, (unsigned)ctas, kTileThreads, G::SMEM, s, mapK, mapV, P));
    return DSMOE_OK;
}

}  // namespace

// K or V as a tensor of four dimensions, d_head and then positions, heads and sequences in the order of their strides
dsmoe_status make_cache_map(CUtensorMap* m, const AttnView& A, const void* ptr, int (&at)[3]) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return DSMOE_ERR_CUDA;
    const long long stride[3] = {A.kv_p, A.kv_h, A.kv_s};
    const cuuint64_t size[3] = {(cuuint64_t)A.L, (cuuint64_t)A.n_head, (cuuint64_t)A.n_seq};
    int order[3] = {0, 1, 2};
    for (int a = 0; a < 2; ++a)
        for (int b = 0; b < 2 - a; ++b) {
            // (a dimension of one element has no stride to speak of: last)
            const long long x = size[order[b]] == 1 ? 1ll << 50 : stride[order[b]], y = size[order[b + 1]] == 1 ? 1ll << 50 : stride[order[b + 1]];
            if (x > y) {
                const int t = order[b];
                order[b] = order[b + 1];
                order[b + 1] = t;
            }
        }
    cuuint64_t dims[4] = {(cuuint64_t)A.d_head}, strides[3];
    cuuint32_t box[4] = {64, 1, 1, 1};
    const cuuint32_t es[4] = {1, 1, 1, 1};
    for (int d = 0; d < 3; ++d) {
        const int o = order[d];
        dims[d + 1] = size[o];
        strides[d] = size[o] == 1 ? (d == 0 ? (cuuint64_t)A.d_head * 2 : strides[d - 1] * dims[d]) : (cuuint64_t)stride[o] * 2;
        at[o] = d + 1;
        if (o == 0) box[d + 1] = kTileKeys;
    }
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DSMOE_OK : DSMOE_ERR_CUDA;
}

bool tile_supported(const AttnView& A) {
    if (A.d_head != 64 && A.d_head != 96 && A.d_head != 128) return false;
    if (!(A.scale_log2 > 0.f)) return false;          // (what is hidden is -inf before it is scaled)
    const long long stride[3] = {A.kv_p, A.kv_h, A.kv_s};
    const int size[3] = {A.L, A.n_head, A.n_seq};
    for (int d = 0; d < 3; ++d)
        if (size[d] > 1 && (stride[d] <= 0 || stride[d] >= 1ll << 38)) return false;
    return true;
}

dsmoe_status launch_tile_attention(const AttnView& A, const TilePlan& plan, cudaStream_t s) {
    switch (A.d_head) {
        case 64: return launch_tile<64>(A, plan, s);
        case 96: return launch_tile<96>(A, plan, s);
        case 128: return launch_tile<128>(A, plan, s);
        default: return DSMOE_ERR_UNSUPPORTED;
    }
}

}  // namespace dsmoe
