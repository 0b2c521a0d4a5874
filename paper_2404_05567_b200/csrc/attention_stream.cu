// Attention of single tokens against their caches, on warp-level MMAs: every key and value is read once per (token, head) and nothing is
// shared between tokens (see cache_attention.cuh for what a row sees and what parts are).
//
// The keys of all (token, head, row tile) pairs, in units of 16, are one list, cut into equal runs, one per CTA; the CTA's warps take its units
// in turn, each through a ring of its own (cp.async), and the 16 rows of the MMA tile are the group's query heads.  A unit holds keys
// that its token sees and no others, so that no mask compares positions: the sinks' units come first, then the window's, from its first key on.
// The warps' triples of a pair meet in shared memory; a pair that several runs share leaves a part per run, added up by the next launch.
// Bound by the keys' and values' way out of memory.
#include "cache_attention.cuh"
#include "umma.cuh"

namespace dsmoe {

namespace {

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
__device__ __forceinline__ void ldsm_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float low_part(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high_part(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Where the part of pair p of a group of HB lies that a run leaves: a run has room for the parts of the pairs that began before it and for those
// of the pairs that begin in it
__device__ __forceinline__ long long part_slot(long long run, bool begins, int HB, int p) { return (2 * run + (begins ? 1 : 0)) * HB + p; }
// What is said of a pair's parts beside its first run: their number, and how many runs there are from one to the next
__device__ __forceinline__ int parts_word(int parts, int stride) { return parts == 0 ? 0 : parts | stride << 16; }

// Row `at`'s largest logit z (0 if it sees nothing) and sum, for whoever asks
__device__ __forceinline__ void write_sums(const AttnView& A, size_t at, float z, float den) {
    if (A.lse) A.lse[at] = (z + log2f(den)) * 0.6931471805599453f;
    if (A.ml) A.ml[at] = make_float2(z, den == 0.f ? 0.f : 1.f / den);
}

// BY_WARP: runs that `total` units are cut into, `most` at most.  None is shorter than a kPartsAtMost-th of the longest pair's units, so that no pair lies in
// more than kPartsAtMost + 1 runs.
constexpr int kPartsAtMost = 200;
__host__ __device__ constexpr long long warp_runs(long long total, long long longest, long long most) {
    const long long least = (longest + kPartsAtMost - 1) / kPartsAtMost, runs = total / least;
    return runs < 1 ? 1 : runs < most ? runs : most;
}
// (runs are of total / runs units and more: 250 units beside 159 and 1183 pairs of one)
static_assert(250 <= (kPartsAtMost - 1) * (409 / warp_runs(409, 250, 1184)) + 1 && 250 <= (kPartsAtMost - 1) * (1433 / warp_runs(1433, 250, 1184)) + 1);
static_assert(warp_runs(1, 1, 1184) == 1 && warp_runs(100000, 400, 1184) == 1184 && warp_runs(800, 800, 1184) == 200);

template <int DH>
struct StreamGeo {
    static constexpr int WARPS = stream_warps(DH);
    static constexpr int STRIDE = DH * 2 + 16;                     // bytes per key row in shared memory: 16 of padding, no bank conflicts
    static constexpr int UNIT = 2 * kUnit * STRIDE;                // K and V; also holds a warp's 16 x (DH + 8) accumulators
    static constexpr int FIT = 208 * 1024 / (WARPS * UNIT);
    static constexpr int BUFS = FIT > 6 ? 6 : FIT;
    static constexpr int SMEM = WARPS * BUFS * UNIT;
    static_assert(BUFS >= 2 && 16 * (DH + 8) * 4 <= UNIT, "accumulators take a unit's place");
};

// HB: heads that a CTA takes at a time.  A unit of the list is 16 keys of HB neighbouring (head, row tile)s; warp w's is the (w % HB)-th, and of the
// units it takes every (WARPS / HB)-th.  Heads that lie side by side in memory (a cache stored by position) are so read side by side: 62 tokens of
// 4 heads that see 2052 keys, stored by position, 68 us with one head at a time, 60 with two, 62 with four; by head 53, 53, 60 (cold caches); with fewer
// keys than warps, a pair's parts are more the more heads share a CTA: 4 tokens behind 1500 keys 15, 23, 34.
//
// A run is a CTA's, whose warps share its units and meet at the end of each pair; or, where there are as many pairs as warps, BY_WARP, a warp's (of each of
// the HB heads), which takes its units one after the other and owes the others nothing.  256 tokens of 8 heads with 384 keys each, behind a
// prefix, us: a CTA's 275, a warp's 260; 32 tokens of 4 heads with 3000 keys, with sums and tallies, 56, 61.
template <int DH, int HB, bool BY_WARP>
__global__ void __launch_bounds__(32 * StreamGeo<DH>::WARPS, 1)
attention_stream_kernel(const __grid_constant__ AttnView A, const __grid_constant__ StreamPlan P) {
    using G = StreamGeo<DH>;
    constexpr int STRIDE = G::STRIDE, KS = DH / 16, DT = DH / 8, CH = DH / 8, LDO = DH + 8, BUFS = G::BUFS, WARPS = G::WARPS;
    constexpr int THREADS = 32 * WARPS, PER = kListTokens / THREADS, KW = WARPS / HB, QN = (HB * 16 * CH + THREADS - 1) / THREADS;
    extern __shared__ __align__(16) unsigned char as_smem[];
    __shared__ long long base_s[kListTokens + 2];       // units before entry e's: the shared keys (in the first pass), then tokens
    __shared__ int token_s[kListTokens];                // left tokens: their numbers
    __shared__ long long warp_sum_s[WARPS];
    __shared__ int longest_s[WARPS];
    __shared__ float ms[WARPS][16], ls[WARPS][16];
    __shared__ uint32_t at_s[WARPS];                    // where each warp's accumulators of the pair are
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
    const int hb = warp % HB, kw = warp / HB;
    __shared__ __align__(16) unsigned char q_s[BY_WARP ? 16 : HB * 16 * STRIDE];
    const int own_heads = A.n_head * A.row_tiles, shared_heads = A.n_head * P.shared.row_tiles;
    chain_wait();
    if (P.run_head)
        for (int i = tid; i < P.passes * KW; i += THREADS) P.run_head[(long long)(i / KW) * P.ctas * KW + blockIdx.x * KW + i % KW] = make_int2(0, 0);

    // Sum over the CTA's threads of what lies before this one's x; *all: of all
    const auto scan = [&](long long x, long long* all) {
        long long incl = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        __syncthreads();
        if (lane == 31) warp_sum_s[warp] = incl;
        __syncthreads();
        long long before = incl - x, sum = 0;
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) before += warp_sum_s[w];
            sum += warp_sum_s[w];
        }
        *all = sum;
        return before;
    };

    for (int pass = 0; pass < P.passes; ++pass) {
    // ---- the pass's entries and their units
    const int first = pass == 0 && P.shared.P > 0 ? 1 : 0;          // the first token's entry
    const int n0 = pass * kListTokens;
    int n = P.own ? min(kListTokens, A.T - n0) : 0;
    __syncthreads();
    if (P.own && P.count) {
        long long so_far = 0;
        for (int b0 = 0; b0 < P.blocks; b0 += THREADS) {
            const int b = b0 + tid, c = b < P.blocks ? P.count[b] : 0;
            long long sum;
            const long long at = so_far + scan(c, &sum) - n0;
            for (int i = 0; i < c; ++i)
                if (at + i >= 0 && at + i < kListTokens) token_s[at + i] = P.list[(long long)b * P.span + i];
            so_far += sum;
        }
        n = (int)max(0ll, min((long long)kListTokens, so_far - n0));
        __syncthreads();
    }
    const auto token_of = [&](int e) { return P.count ? token_s[e - first] : n0 + e - first; };
    if (n + first == 0) break;
    {
        long long mine[PER], sum = 0, total;
        int longest = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = tid * PER + i;
            mine[i] = 0;
            if (e < n) {
                bool bad = false;
                const int units = sight_of(A, token_of(e + first), &bad).units();
                longest = max(longest, units);
                mine[i] = (long long)units * (own_heads / HB);
                if (bad && blockIdx.x == 0) report_status(A.dev_status, DSMOE_ERR_INVALID_ARG);
            }
            sum += mine[i];
        }
        const long long shared_units = first ? (long long)((P.shared.P + kUnit - 1) / kUnit) * (shared_heads / HB) : 0;
        longest = __reduce_max_sync(0xffffffffu, longest);
        if (lane == 0) longest_s[warp] = longest;
        long long before = scan(sum, &total) + shared_units;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = tid * PER + i;
            if (e < n) base_s[first + e] = before;
            before += mine[i];
        }
        if (tid == 0) {
            base_s[0] = 0;
            base_s[first + n] = total + shared_units;
        }
        __syncthreads();
    }
    // Equal runs, of at least a unit for each warp
    const int entries = n + first;
    const long long total = base_s[entries];
    long long wanted = min((long long)gridDim.x, (total + KW - 1) / KW);
    if (BY_WARP) {
        int longest = first ? (P.shared.P + kUnit - 1) / kUnit : 1;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) longest = max(longest, longest_s[w]);
        wanted = warp_runs(total, longest, (long long)gridDim.x * KW);
    }
    const int pairs_each = own_heads / HB;              // pairs (of HB heads) of a token
    if (P.whole) wanted = (long long)n * pairs_each;
    const int n_runs = (int)wanted, stride = BY_WARP ? 1 : KW, run_no = BY_WARP ? (int)blockIdx.x * KW + kw : (int)blockIdx.x;
    if (run_no >= n_runs) {
        __syncwarp();
        continue;
    }
    const long long share = total / n_runs, extra = total - share * n_runs;
    const auto run_start = [&](long long c) { return c * share + (c < extra ? c : extra); };
    const auto run_of = [&](long long u) {              // the run that holds unit u
        const long long cut = extra * (share + 1);
        return u < cut ? u / (share + 1) : extra + (u - cut) / share;
    };
    long long u0, u1;
    if (P.whole) {
        const int e = run_no / pairs_each;
        const long long units = (base_s[e + 1] - base_s[e]) / pairs_each;
        u0 = base_s[e] + run_no % pairs_each * units;
        u1 = u0 + units;
    } else {
        u0 = run_start(run_no);
        u1 = run_start(run_no + 1);
    }
    // where a run's parts lie, and the next run's after it
    const long long run = (long long)pass * P.ctas * KW + (long long)run_no * stride;

    // Where a unit lies: entry, its first (head, row tile), key block of it
    struct Cursor {
        int e, h, k, units;
        Sight s;
    };
    const auto is_shared = [&](int e) { return e < first; };
    const auto look = [&](Cursor& c) {
        bool bad = false;
        if (c.e >= entries) return;
        if (is_shared(c.e)) c.s = Sight{0, 0, 0, P.shared.P - 1};
        else c.s = sight_of(A, token_of(c.e), &bad);
        c.units = c.s.units();
    };
    const auto settle = [&](Cursor& c) {                // k past the pair's units: on to the pair that holds it
        while (c.e < entries && c.k >= c.units) {
            c.k -= c.units;
            c.h += HB;
            if (c.h == (is_shared(c.e) ? shared_heads : own_heads)) {
                c.h = 0;
                ++c.e;
                look(c);
            }
        }
    };
    Cursor seg;
    {
        int lo = 0, hi = entries - 1;                   // the last entry whose units begin at or before u0
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (base_s[mid] <= u0) lo = mid;
            else hi = mid - 1;
        }
        seg.e = lo;
        look(seg);
        const long long in = u0 - base_s[lo];
        seg.h = (int)(in / seg.units) * HB;
        seg.k = (int)(in % seg.units);
    }
    Cursor ahead = seg;                                 // the next unit to fetch
    const int hop = BY_WARP ? 1 : KW, begin = BY_WARP ? 0 : kw;
    long long u_ahead = u0 + begin;
    if (u_ahead < u1) {
        ahead.k += begin;
        settle(ahead);
    }
    unsigned char* const ring = as_smem + (size_t)warp * BUFS * G::UNIT;
    const uint32_t ring0 = ptx::smem_u32(ring);
    const auto fetch = [&](int buf) {
        if (u_ahead < u1) {
            const Sight& s = ahead.s;
            const bool sh = is_shared(ahead.e);
            const int su = s.sink_units();
            const int key0 = ahead.k < su ? ahead.k * kUnit : s.first + (ahead.k - su) * kUnit;
            const int nk = ahead.k < su ? s.sinks - key0 : s.last + 1 - key0;       // keys of the unit, if fewer than kUnit
            const int slot0 = sh ? key0 : slot_of(A, key0);
            const int j = (ahead.h + hb) / (sh ? P.shared.row_tiles : A.row_tiles);
            const long long head = sh ? j * P.shared.kv_h : (long long)s.seq * A.kv_s + j * A.kv_h, step = sh ? P.shared.kv_p : A.kv_p;
            const __nv_bfloat16 *const K = (sh ? P.shared.K : A.K) + head, *const V = (sh ? P.shared.V : A.V) + head;
            const uint32_t kd = ring0 + (uint32_t)(buf * G::UNIT), vd = kd + (uint32_t)(kUnit * STRIDE);
            // a unit of neighbouring slots that is full: no piece needs a look at its row (with that for every piece the kernel issued half as
            // many instructions again, and they, not the keys, were what it waited for)
            const bool plain = (CH & (CH - 1)) == 0 && nk >= kUnit && (sh || !A.ring || slot0 + kUnit <= A.L);
            if (plain) {
                constexpr int LANES = CH < 32 ? CH : 32, ROWS = 32 / LANES;          // lanes of a row, rows at a time
                const long long from = (slot0 + lane / LANES) * step + lane % LANES * 8, down = ROWS * step;
                const __nv_bfloat16 *k = K + from, *v = V + from;
                const uint32_t to = (uint32_t)(lane / LANES * STRIDE + lane % LANES * 16);
#pragma unroll
                for (int i = 0; i < kUnit / ROWS; ++i) {
                    ptx::cp_async16(kd + to + i * ROWS * STRIDE, k);
                    ptx::cp_async16(vd + to + i * ROWS * STRIDE, v);
                    k += down;
                    v += down;
                }
            } else {
#pragma unroll 1
                for (int i = 0; i < CH * kUnit / 32; ++i) {
                    const int idx = lane + 32 * i, row = idx / CH, ch = idx % CH;
                    int slot = slot0 + (row < nk ? row : 0);
                    if (A.ring && !sh && slot >= A.L) slot -= A.ring;  // in a unit across the end of the ring the slots are not neighbours
                    const long long src = slot * step + ch * 8;
                    const uint32_t nbytes = row < nk ? 16u : 0u, dst = (uint32_t)(row * STRIDE + ch * 16);      // past the last key: zeros
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(kd + dst), "l"(K + src), "r"(nbytes) : "memory");
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vd + dst), "l"(V + src), "r"(nbytes) : "memory");
                }
            }
            u_ahead += hop;
            if (u_ahead < u1) {                         // (settling may wait for a token's sequence and position)
                ahead.k += hop;
                settle(ahead);
            }
        }
        ptx::cp_async_commit();
    };
    for (int b = 0; b < BUFS - 1; ++b) fetch(b);

    const uint32_t kfrag = (uint32_t)(((lane >> 4) * 8 + (lane & 7)) * STRIDE + ((lane >> 3) & 1) * 16);
    const uint32_t vfrag = (uint32_t)((((lane >> 3) & 1) * 8 + (lane & 7)) * STRIDE + (lane >> 4) * 16);
    int buf = 0;
    long long mine = u0 + begin;                        // this warp's next unit
    uint4 next_q[QN];                                   // a thread's pieces of the next pairs' queries; rows that are none are zeros
    const auto ask_queries = [&](const Cursor& c) {
        const bool sh = is_shared(c.e);
        const int tiles = sh ? P.shared.row_tiles : A.row_tiles, t0 = sh ? 0 : token_of(c.e);
        const long long all = sh ? (long long)A.T * A.group : A.group;
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int idx = tid + i * THREADS, x = idx / CH, h = c.h + x / 16, row = h % tiles * 16 + x % 16;
            next_q[i] = make_uint4(0u, 0u, 0u, 0u);
            if (idx < HB * 16 * CH && row < all)
                next_q[i] = *reinterpret_cast<const uint4*>(A.q + (t0 + row / A.group) * A.q_t + h / tiles * A.q_h + row % A.group * A.q_g + idx % CH * 8);
        }
    };
    if (!BY_WARP) ask_queries(seg);
    for (long long at = u0; at < u1;) {
        const bool sh = is_shared(seg.e);
        const int tiles = sh ? P.shared.row_tiles : A.row_tiles, t = sh ? 0 : token_of(seg.e);
        const int units = seg.units;
        const long long end = min(u1, at + units - seg.k), all_rows = sh ? (long long)A.T * A.group : A.group;
        const int first_k = seg.k;
        const Sight& s = seg.s;
        const int su = s.sink_units();
        // this warp's pair
        const int j = (seg.h + hb) / tiles, row0 = (seg.h + hb) % tiles * 16, rows = (int)min(16ll, all_rows - row0);
        uint32_t qf[KS][4];                             // its queries (the MMAs' A operand); rows that are none are zeros
        if (BY_WARP) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int row = row0 + g + 8 * half;
                const bool real = row < all_rows;
                const __nv_bfloat16* const q = A.q + (t + (real ? row / A.group : 0)) * A.q_t + j * A.q_h + (real ? row % A.group : 0) * A.q_g + q4 * 2;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qf[ks][half] = real ? *reinterpret_cast<const uint32_t*>(q + ks * 16) : 0u;
                    qf[ks][2 + half] = real ? *reinterpret_cast<const uint32_t*>(q + ks * 16 + 8) : 0u;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < QN; ++i) {
                const int idx = tid + i * THREADS;
                if (idx < HB * 16 * CH) *reinterpret_cast<uint4*>(q_s + (idx / CH) * STRIDE + idx % CH * 16) = next_q[i];
            }
            __syncthreads();
            const uint32_t qrow = ptx::smem_u32(q_s) + (uint32_t)((hb * 16 + (lane & 15)) * STRIDE + (lane >> 4) * 16);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) ldsm_x4(qf[ks], qrow + (uint32_t)(ks * 32));
        }
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[DT][4];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        for (; mine < end; mine += hop) {
            __syncwarp();                               // every lane is past its reads of the buffer that is filled again now
            fetch((buf + BUFS - 1) % BUFS);
            ptx::cp_async_wait<BUFS - 1>();
            __syncwarp();
            const uint32_t kb = ring0 + (uint32_t)(buf * G::UNIT) + kfrag, vb = ring0 + (uint32_t)(buf * G::UNIT + kUnit * STRIDE) + vfrag;
            float sc[2][4], sd[2][4];                   // two chains each, even and odd steps of the reduction
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) sc[i][c] = sd[i][c] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t b[4];
                ldsm_x4(b, kb + (uint32_t)(ks * 32));
                mma_16816(ks & 1 ? sd[0] : sc[0], qf[ks], b[0], b[1]);
                mma_16816(ks & 1 ? sd[1] : sc[1], qf[ks], b[2], b[3]);
            }
            // to base 2; what is no key is hidden
            const int k = first_k + (int)(mine - at);
            const int nk = (k < su ? s.sinks - k * kUnit : s.last + 1 - s.first - (k - su) * kUnit) - q4 * 2;
            float b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const bool seen = i * 8 + (c & 1) < nk;
                    sc[i][c] = seen ? (sc[i][c] + sd[i][c]) * A.scale_log2 : -INFINITY;
                    if (c < 2) b0 = fmaxf(b0, sc[i][c]);
                    else b1 = fmaxf(b1, sc[i][c]);
                }
            if (P.logits && !sh) {
                const int col = k * kUnit + q4 * 2;
                float* const to = P.logits + row_at(A, t, j, row0) * P.logit_pitch + col;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (g < rows) *reinterpret_cast<float2*>(to + g * P.logit_pitch + i * 8) = make_float2(sc[i][0], sc[i][1]);
                    if (g + 8 < rows) *reinterpret_cast<float2*>(to + (g + 8) * P.logit_pitch + i * 8) = make_float2(sc[i][2], sc[i][3]);
                }
            }
            // (see kStreamMoves)
            if (__any_sync(0xffffffffu, b0 > m0 + kStreamMoves || b1 > m1 + kStreamMoves || (m0 == -INFINITY && b0 > m0) || (m1 == -INFINITY && b1 > m1))) {
                b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 1));
                b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 1));
                b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 2));
                b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 2));
                const float n0 = fmaxf(m0, b0), n1 = fmaxf(m1, b1);
                const float c0 = n0 == -INFINITY ? 1.f : exp2_fast(m0 - n0), c1 = n1 == -INFINITY ? 1.f : exp2_fast(m1 - n1);
                m0 = n0;
                m1 = n1;
                l0 *= c0;
                l1 *= c1;
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    o[i][0] *= c0;
                    o[i][1] *= c0;
                    o[i][2] *= c1;
                    o[i][3] *= c1;
                }
            }
            const float z0 = m0 == -INFINITY ? 0.f : m0, z1 = m1 == -INFINITY ? 0.f : m1;
            // the weights as two bf16 numbers each, the second the first's rounding error: the tensor pipe has the time
            uint32_t pf[4], pr[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float p0 = exp2_fast(sc[i][0] - z0), p1 = exp2_fast(sc[i][1] - z0);
                const float p2 = exp2_fast(sc[i][2] - z1), p3 = exp2_fast(sc[i][3] - z1);
                l0 += p0 + p1;
                l1 += p2 + p3;
                pf[2 * i] = pack2(p0, p1);
                pf[2 * i + 1] = pack2(p2, p3);
                pr[2 * i] = pack2(p0 - low_part(pf[2 * i]), p1 - high_part(pf[2 * i]));
                pr[2 * i + 1] = pack2(p2 - low_part(pf[2 * i + 1]), p3 - high_part(pf[2 * i + 1]));
            }
#pragma unroll
            for (int dp = 0; dp < DT / 2; ++dp) {
                uint32_t v[4];
                ldsm_x4_trans(v, vb + (uint32_t)(dp * 32));
                mma_16816(o[2 * dp], pf, v[0], v[1]);
                mma_16816(o[2 * dp + 1], pf, v[2], v[3]);
                mma_16816(o[2 * dp], pr, v[0], v[1]);
                mma_16816(o[2 * dp + 1], pr, v[2], v[3]);
            }
            buf = buf + 1 == BUFS ? 0 : buf + 1;
        }
        Cursor next = seg;
        if (end < u1) {
            next.k += (int)(end - at);
            settle(next);
            if (!BY_WARP) ask_queries(next);            // (on their way while the triples meet)
        } else if (pass + 1 == P.passes) {
            chain_next();
        }
        const bool whole = end - at == units, begins = first_k == 0;
        if (begins && (BY_WARP ? lane == 0 : tid < HB)) {
            const int p = BY_WARP ? hb : tid, parts = whole ? 0 : parts_word((int)(run_of(at + units - 1) - run_no + 1), stride);
            if (P.keep) P.head[sh ? seg.h + p : shared_heads + (long long)t * own_heads + seg.h + p] = make_int2((int)run, parts);
            else if (!whole && p == 0) P.run_head[run] = make_int2(t * own_heads + seg.h, parts);
        }
        // ---- the warps' triples of the pair, through the buffer that each has just finished (the next fetch would fill it)
        l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
        const uint32_t free_at = (uint32_t)((warp * BUFS + (buf + BUFS - 1) % BUFS) * G::UNIT);
        __syncwarp();
        if (q4 == 0) {
            ms[warp][g] = m0;
            ms[warp][g + 8] = m1;
            ls[warp][g] = l0;
            ls[warp][g + 8] = l1;
            if (g == 0) at_s[warp] = free_at;
        }
        float* const acc = reinterpret_cast<float*>(as_smem + free_at);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            *reinterpret_cast<float2*>(acc + g * LDO + dt * 8 + q4 * 2) = make_float2(o[dt][0], o[dt][1]);
            if (rows > 8) *reinterpret_cast<float2*>(acc + (g + 8) * LDO + dt * 8 + q4 * 2) = make_float2(o[dt][2], o[dt][3]);
        }
        if (BY_WARP) __syncwarp();
        else __syncthreads();
        float* const row_o = sh ? P.shared_rows.o : P.own_rows.o;
        float* const row_ml = sh ? P.shared_rows.ml : P.own_rows.ml;
        // where two columns of a row go, and beside the first ones the row's sums
        const auto put = [&](int p, int row, int col, float nx, float ny, float M, float den) {
            const int head = (seg.h + p) / tiles, first_row = (seg.h + p) % tiles * 16;
            const int member = (first_row + row) % A.group, tok = t + (first_row + row) / A.group;
            const long long r = row_at(A, tok, head, member);
            if (!whole) {
                float* const slot = P.slots + part_slot(run, begins, HB, p) * 16 * (DH + 2);
                *reinterpret_cast<float2*>(slot + row * DH + col) = make_float2(nx, ny);
                if (col == 0) *reinterpret_cast<float2*>(slot + 16 * DH + row * 2) = make_float2(M, den);
                // (the row's whole part: none)
                if (col == 0 && P.keep && begins) *reinterpret_cast<float2*>(row_ml + r * 2) = make_float2(-INFINITY, 0.f);
            } else if (P.keep) {
                *reinterpret_cast<float2*>(row_o + r * DH + col) = make_float2(nx, ny);
                if (col == 0) *reinterpret_cast<float2*>(row_ml + r * 2) = make_float2(M, den);
            } else {
                const float inv = den == 0.f ? 0.f : 1.f / den;           // no key: zeros
                *reinterpret_cast<uint32_t*>(A.out + tok * A.o_t + head * A.o_h + member * A.o_g + col) = pack2(nx * inv, ny * inv);
                if (col == 0) write_sums(A, r, M == -INFINITY ? 0.f : M, den);
            }
        };
        if (BY_WARP) {
            for (int idx = lane; idx < rows * (DH / 2); idx += 32) {
                const int row = idx / (DH / 2), col = idx % (DH / 2) * 2;
                const float2 v = *reinterpret_cast<const float2*>(acc + row * LDO + col);
                put(hb, row, col, v.x, v.y, ms[warp][row], ls[warp][row]);
            }
            __syncwarp();                               // ... read before the next fetch overwrites them
            seg = next;
            at = end;
            continue;
        }
        // the group's pairs side by side, 16 rows each
        for (int idx = tid; idx < HB * 16 * (DH / 2); idx += THREADS) {
            const int x = idx / (DH / 2), col = idx % (DH / 2) * 2, p = x / 16, row = x % 16;
            if (row >= all_rows - (seg.h + p) % tiles * 16) continue;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < KW; ++w) M = fmaxf(M, ms[w * HB + p][row]);
            const float z = M == -INFINITY ? 0.f : M;
            float nx = 0.f, ny = 0.f, den = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float wgt = exp2_fast(ms[w * HB + p][row] - z);     // 0 for a warp that saw no key
                const float2 v = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(as_smem + at_s[w * HB + p]) + row * LDO + col);
                nx = fmaf(wgt, v.x, nx);
                ny = fmaf(wgt, v.y, ny);
                den = fmaf(wgt, ls[w * HB + p][row], den);
            }
            put(p, row, col, nx, ny, M, den);
        }
        __syncthreads();                                // the warps' triples are read before the next fetch overwrites them
        seg = next;
        at = end;
    }
    ptx::cp_async_wait<0>();
    }
}

// Adds up the parts of a pair's rows, in order: parts of whole rows, those of the shared keys, then those of the token's own.  A CTA per pair, or
// (no `keep`) per run of the stream kernel's, for the pair that begins there and goes on.  First the weights of all parts, a warp per
// row, then the sums, a thread per four columns, with sixteen loads under way.
// Parts at most: the prefix's and the own caches' parts of whole rows, and of the shared keys' pair and the own one a part a CTA, or a run of warp_runs
constexpr int kSumParts = 544;
static_assert(kSumParts >= 2 * kMaxSplits + 2 * (kMostStreamCtas > kPartsAtMost + 1 ? kMostStreamCtas : kPartsAtMost + 1), "a place for each part");

// ROWS: rows at a time, a warp each: four for groups of up to four, so that twice as many CTAs fit an SM: 2048 pairs of 4 rows and 5 parts, 11.6 us, with
// eight 19.7.
template <int DH, int ROWS>
__global__ void __launch_bounds__(32 * ROWS) attention_sum_kernel(const __grid_constant__ AttnView A, const __grid_constant__ StreamPlan P,
                                                                    const __grid_constant__ RowParts M) {
    __shared__ float wgt_s[ROWS][kSumParts];
    __shared__ uint32_t from_s[ROWS][kSumParts];     // where a part's values begin, in float4s from the slots on (all parts lie behind those)
    __shared__ float inv_s[ROWS];
    __shared__ int n_s[ROWS];
    chain_wait();
    chain_next();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int heads = A.n_head * A.row_tiles, shared_heads = A.n_head * P.shared.row_tiles;
    long long pair = blockIdx.x;
    int2 own = make_int2(0, 0);                          // first run, number of parts
    if (P.keep) {
        if (P.own) own = P.head[shared_heads + pair];
    } else {
        const int run = (int)blockIdx.x / P.heads_at_once * (P.by_warp ? 1 : stream_warps(DH) / P.heads_at_once);
        own = make_int2(run, P.run_head[run].y);
        if (own.y == 0) return;
        pair = P.run_head[run].x + (int)blockIdx.x % P.heads_at_once;
    }
    const int t = (int)(pair / heads), h = (int)(pair % heads), j = h / A.row_tiles, row0 = h % A.row_tiles * 16;
    constexpr long long SLOT = 16 * (DH + 2);
    for (int c0 = row0; c0 < min(row0 + 16, A.group); c0 += ROWS) {
    const int rows = min(min(ROWS, row0 + 16 - c0), A.group - c0);
    __syncthreads();
    for (int row = warp; row < rows; row += ROWS) {
        const long long r = row_at(A, t, j, c0 + row), folded = (long long)t * A.group + c0 + row;
        int2 sh = make_int2(0, 0);
        int sh_pair = 0;
        if (P.keep && P.shared.P > 0) {
            sh_pair = j * P.shared.row_tiles + (int)(folded / 16);
            sh = P.head[sh_pair];
            sh_pair %= P.heads_at_once;
        }
        const int sh_n = sh.y & 0xffff, n = M.n + sh_n + (own.y & 0xffff);
        float top = -INFINITY, den = 0.f;
        for (int i = lane; i < n; i += 32) {
            const float *o, *ml;
            if (i < M.n) {
                o = M.o + (i * M.rows + r) * DH;
                ml = M.ml + (i * M.rows + r) * 2;
            } else {
                const bool s = i < M.n + sh_n;
                const int k = i - M.n - (s ? 0 : sh_n), at = s ? (int)(folded % 16) : c0 - row0 + row;
                const int2 head = s ? sh : own;
                const float* const slot = P.slots + part_slot(head.x + (long long)k * (head.y >> 16), k == 0, P.heads_at_once, s ? sh_pair : h % P.heads_at_once) * SLOT;
                o = slot + at * DH;
                ml = slot + 16 * DH + at * 2;
            }
            const float2 x = *reinterpret_cast<const float2*>(ml);
            wgt_s[row][i] = x.x;
            from_s[row][i] = (uint32_t)((o - P.slots) >> 2);
            const float up = fmaxf(top, x.x);            // (this lane's parts' sum, relative to their maximum)
            // (a part without a maximum has seen no key, or none whose logit is a number: then its sum is none either, and the row's is none)
            den = den * (up == -INFINITY ? 1.f : exp2_fast(top - up)) + (x.x == -INFINITY ? x.y : x.y * exp2_fast(x.x - up));
            top = up;
        }
        float all = top;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
        const float z = all == -INFINITY ? 0.f : all;
        den = top == -INFINITY ? den : den * exp2_fast(top - z);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
        for (int i = lane; i < n; i += 32) wgt_s[row][i] = exp2_fast(wgt_s[row][i] - z);
        if (lane == 0) {
            inv_s[row] = den == 0.f ? 0.f : 1.f / den;
            n_s[row] = n;
            write_sums(A, r, z, den);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < rows * (DH / 4); idx += (32 * ROWS)) {
        const int row = idx / (DH / 4), col = idx % (DH / 4), n = n_s[row];
        const float4* const from = reinterpret_cast<const float4*>(P.slots) + col;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i0 = 0; i0 < n; i0 += 16) {
            float4 v[16];
            float w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                w[k] = i0 + k < n ? wgt_s[row][i0 + k] : 0.f;
                // (a part of no weight is not looked at: it may hold anything)
                v[k] = w[k] != 0.f ? from[from_s[row][i0 + k]] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                sum.x = fmaf(w[k], v[k].x, sum.x);
                sum.y = fmaf(w[k], v[k].y, sum.y);
                sum.z = fmaf(w[k], v[k].z, sum.z);
                sum.w = fmaf(w[k], v[k].w, sum.w);
            }
        }
        const float inv = inv_s[row];
        *reinterpret_cast<uint2*>(A.out + t * A.o_t + j * A.o_h + (c0 + row) * A.o_g + col * 4) =
            make_uint2(pack2(sum.x * inv, sum.y * inv), pack2(sum.z * inv, sum.w * inv));
    }
    }
}

template <int DH, int HB, bool BY_WARP>
dsmoe_status launch_stream_heads(const AttnView& A, const StreamPlan& plan, cudaStream_t s) {
    auto* kernel = attention_stream_kernel<DH, HB, BY_WARP>;
    static bool attr[kMaxDeviceSlots] = {};
    int dev = 0;
    DeviceState* st = nullptr;
    DSMOE_TRY(device_state(&st, &dev));
    if (!attr[dev]) {
        DSMOE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamGeo<DH>::SMEM));
        attr[dev] = true;
    }
    DSMOE_CUDA_TRY(launch_chained(kernel, (unsigned)plan.ctas, 32 * StreamGeo<DH>::WARPS, StreamGeo<DH>::SMEM, s, A, plan));
    return DSMOE_OK;
}

template <int DH>
dsmoe_status launch_stream(const AttnView& A, const StreamPlan& plan, cudaStream_t s) {
    const bool by_warp = plan.by_warp;
    if (plan.heads_at_once == 2) return by_warp ? launch_stream_heads<DH, 2, true>(A, plan, s) : launch_stream_heads<DH, 2, false>(A, plan, s);
    return by_warp ? launch_stream_heads<DH, 1, true>(A, plan, s) : launch_stream_heads<DH, 1, false>(A, plan, s);
}

template <int DH>
dsmoe_status launch_sum(const AttnView& A, const StreamPlan& plan, const RowParts& rows, cudaStream_t s) {
    const long long ctas = plan.keep ? (long long)A.T * A.n_head * A.row_tiles : (long long)plan.passes * plan.ctas * (plan.by_warp ? stream_warps(A.d_head) : plan.heads_at_once);
    if (A.group <= 4) DSMOE_CUDA_TRY(launch_chained(attention_sum_kernel<DH, 4>, (unsigned)ctas, 128, 0, s, A, plan, rows));
    else DSMOE_CUDA_TRY(launch_chained(attention_sum_kernel<DH, 8>, (unsigned)ctas, 256, 0, s, A, plan, rows));
    return DSMOE_OK;
}

}  // namespace

#define DSMOE_BY_HEAD(DH, CALL)               \
    switch (DH) {                             \
        case 32: return CALL(32);             \
        case 64: return CALL(64);             \
        case 96: return CALL(96);             \
        case 128: return CALL(128);           \
        case 160: return CALL(160);           \
        case 192: return CALL(192);           \
        case 224: return CALL(224);           \
        case 256: return CALL(256);           \
        default: return DSMOE_ERR_UNSUPPORTED; \
    }

// Two where neighbouring heads are nearer than neighbouring positions (see the kernel)
int stream_heads_at_once(const AttnView& A) { return A.n_head % 2 == 0 && A.kv_h < A.kv_p ? 2 : 1; }

// Whether a CTA takes all of a pair's keys, so that no part is left to add up: the second launch and the parts' way through memory cost as much as three
// rounds of a unit a warp, so where the CTAs that stay idle would save fewer.  One launch, and two, us: a token of 4 heads and 256 keys 7.5,
// 9.4, 384 8.8, 9.4, 512 10.3, 9.6; 16 such tokens with 512 keys 11.0, 13.9, 1024 16.0, 16.4; 32 with 2048 28.7, 33.2.
bool stream_whole(const AttnView& A, const StreamPlan& plan) {
    const long long seen = A.window < A.L ? (long long)A.window + A.sinks : A.L, pairs = (long long)A.T * A.n_head * A.row_tiles;
    return !plan.keep && !plan.list && pairs <= sm_count() && seen * (sm_count() - pairs) <= 3ll * kUnit * stream_warps(A.d_head) * sm_count();
}

// As many pairs as warps (those of a list of tokens are not known here: few)
bool stream_by_warp(const AttnView& A, const StreamPlan& plan) {
    const long long pairs = plan.list ? 0 : (plan.own ? (long long)A.T * A.n_head * A.row_tiles : 0) + (long long)A.n_head * plan.shared.row_tiles;
    return pairs >= (long long)plan.ctas * stream_warps(A.d_head);
}

// One CTA per SM, as far as each has a unit per warp in the longest case
int stream_ctas(const AttnView& A, const SharedKeys& shared, bool own) {
    const long long seen = A.window < A.L ? (long long)A.window + A.sinks : A.L, warps = stream_warps(A.d_head);
    long long units = own ? ((seen + kUnit - 1) / kUnit + 1) * ((long long)A.T * A.n_head * A.row_tiles) : 0;
    units += (long long)((shared.P + kUnit - 1) / kUnit) * A.n_head * shared.row_tiles;
    const long long wanted = (units + warps - 1) / warps, most = sm_count() < kMostStreamCtas ? sm_count() : kMostStreamCtas;
    return (int)(wanted < most ? wanted : most);
}

dsmoe_status launch_stream_attention(const AttnView& A, const StreamPlan& plan, cudaStream_t s) {
#define DSMOE_CALL(DH) launch_stream<DH>(A, plan, s)
    DSMOE_BY_HEAD(A.d_head, DSMOE_CALL)
#undef DSMOE_CALL
}

dsmoe_status launch_attention_sum(const AttnView& A, const StreamPlan& plan, const RowParts& rows, cudaStream_t s) {
#define DSMOE_CALL(DH) launch_sum<DH>(A, plan, rows, s)
    DSMOE_BY_HEAD(A.d_head, DSMOE_CALL)
#undef DSMOE_CALL
}

}  // namespace dsmoe
