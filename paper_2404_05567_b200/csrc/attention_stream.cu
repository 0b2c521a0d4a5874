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

// Row `at`'s largest logit z (0 if it sees nothing) and sum, for whoever asks
__device__ __forceinline__ void write_sums(const AttnView& A, size_t at, float z, float den) {
    if (A.lse) A.lse[at] = (z + log2f(den)) * 0.6931471805599453f;
    if (A.ml) A.ml[at] = make_float2(z, den == 0.f ? 0.f : 1.f / den);
}

template <int DH>
struct StreamGeo {
    static constexpr int WARPS = DH <= 128 ? 8 : 4;
    static constexpr int STRIDE = DH * 2 + 16;                     // bytes per key row in shared memory: 16 of padding, no bank conflicts
    static constexpr int UNIT = 2 * kUnit * STRIDE;                // K and V; also holds a warp's 16 x (DH + 8) accumulators
    static constexpr int FIT = 208 * 1024 / (WARPS * UNIT);
    static constexpr int BUFS = FIT > 6 ? 6 : FIT;
    static constexpr int SMEM = WARPS * BUFS * UNIT;
    static_assert(BUFS >= 2 && 16 * (DH + 8) * 4 <= UNIT, "accumulators take a unit's place");
};

template <int DH>
__global__ void __launch_bounds__(32 * StreamGeo<DH>::WARPS, 1)
attention_stream_kernel(const __grid_constant__ AttnView A, const __grid_constant__ PartPlan P) {
    using G = StreamGeo<DH>;
    constexpr int STRIDE = G::STRIDE, KS = DH / 16, DT = DH / 8, CH = DH / 8, LDO = DH + 8, BUFS = G::BUFS, WARPS = G::WARPS;
    constexpr int THREADS = 32 * WARPS, QN = (16 * CH + THREADS - 1) / THREADS, PER = kListTokens / THREADS;
    extern __shared__ __align__(16) unsigned char as_smem[];
    __shared__ long long base_s[kListTokens + 1];       // units before token t's
    __shared__ long long warp_sum_s[WARPS];
    __shared__ float ms[WARPS][16], ls[WARPS][16];
    __shared__ uint32_t at_s[WARPS];                    // where each warp's accumulators of the pair are
    __shared__ __align__(16) unsigned char q_s[16 * STRIDE];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
    const int T = A.T, heads = A.n_head * A.row_tiles;
    chain_wait();
    {
        long long mine[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int t = tid * PER + i;
            mine[i] = 0;
            if (t < T) {
                bool bad = false;
                if (is_streams(A, t)) mine[i] = (long long)sight_of(A, t, &bad).units() * heads;
                else if (blockIdx.x == 0)
                    for (int h = 0; h < heads; ++h) P.head[(long long)t * heads + h] = make_int2(0, 0);
                if (bad && blockIdx.x == 0) report_status(A.dev_status, DSMOE_ERR_INVALID_ARG);
            }
            sum += mine[i];
        }
        long long incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) warp_sum_s[warp] = incl;
        __syncthreads();
        long long before = incl - sum;
        for (int w = 0; w < warp; ++w) before += warp_sum_s[w];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int t = tid * PER + i;
            if (t < T) base_s[t] = before;
            before += mine[i];
            if (t == T - 1) base_s[T] = before;
        }
        __syncthreads();
    }
    // Equal runs; no CTA without a unit per warp, as far as there are so many
    const long long total = base_s[T];
    if (total == 0) return;
    const long long wanted = (total + WARPS - 1) / WARPS;
    const int n_cta = (int)(wanted < (long long)gridDim.x ? wanted : (long long)gridDim.x);
    if ((int)blockIdx.x >= n_cta) return;
    const long long share = total / n_cta, extra = total - share * n_cta;
    const auto run_start = [&](long long c) { return c * share + (c < extra ? c : extra); };
    const auto run_of = [&](long long u) {              // the CTA whose run holds unit u
        const long long cut = extra * (share + 1);
        return u < cut ? u / (share + 1) : extra + (u - cut) / share;
    };
    const long long u0 = run_start(blockIdx.x), u1 = run_start(blockIdx.x + 1);

    // Where a unit lies: token, its (head, row tile), key block of it
    struct Cursor {
        int t, h, k, units;
        Sight s;
    };
    const auto look = [&](Cursor& c) {                  // (tokens without units are passed over)
        bool bad = false;
        while (c.t < T && base_s[c.t + 1] == base_s[c.t]) ++c.t;
        if (c.t < T) {
            c.s = sight_of(A, c.t, &bad);
            c.units = c.s.units();
        }
    };
    const auto settle = [&](Cursor& c) {                // k past the pair's units: on to the pair that holds it
        while (c.t < T && c.k >= c.units) {
            c.k -= c.units;
            if (++c.h == heads) {
                c.h = 0;
                ++c.t;
                look(c);
            }
        }
    };
    Cursor seg;
    {
        int lo = 0, hi = T - 1;                         // the last token whose units begin at or before u0
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (base_s[mid] <= u0) lo = mid;
            else hi = mid - 1;
        }
        seg.t = lo;
        look(seg);
        const long long in = u0 - base_s[lo];
        seg.h = (int)(in / seg.units);
        seg.k = (int)(in - (long long)seg.h * seg.units);
    }
    Cursor ahead = seg;                                 // the next unit to fetch
    ahead.k += warp;
    settle(ahead);
    long long u_ahead = u0 + warp;
    unsigned char* const ring = as_smem + (size_t)warp * BUFS * G::UNIT;
    const uint32_t ring0 = ptx::smem_u32(ring);
    const auto fetch = [&](int buf) {
        if (u_ahead < u1) {
            const Sight& s = ahead.s;
            const int su = s.sink_units();
            const int key0 = ahead.k < su ? ahead.k * kUnit : s.first + (ahead.k - su) * kUnit;
            const int nk = ahead.k < su ? s.sinks - key0 : s.last + 1 - key0;       // keys of the unit, if fewer than kUnit
            const int slot0 = slot_of(A, key0 < 0 ? 0 : key0);
            const long long head = (long long)s.seq * A.kv_s + (long long)(ahead.h / A.row_tiles) * A.kv_h;
            const uint32_t kd = ring0 + (uint32_t)(buf * G::UNIT), vd = kd + (uint32_t)(kUnit * STRIDE);
#pragma unroll
            for (int i = 0; i < CH * kUnit / 32; ++i) {
                const int idx = lane + 32 * i, row = idx / CH, ch = idx % CH;
                int slot = slot0 + (row < nk ? row : 0);
                // in a unit across the end of the sinks, or of the ring, the slots are not neighbours
                if (A.ring && slot >= A.L) slot -= A.ring;
                const long long src = head + (long long)slot * A.kv_p + ch * 8;
                const uint32_t nbytes = row < nk ? 16u : 0u, dst = (uint32_t)(row * STRIDE + ch * 16);      // past the last key: zeros
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(kd + dst), "l"(A.K + src), "r"(nbytes) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vd + dst), "l"(A.V + src), "r"(nbytes) : "memory");
            }
            ahead.k += WARPS;
            settle(ahead);
            u_ahead += WARPS;
        }
        ptx::cp_async_commit();
    };
    for (int b = 0; b < BUFS - 1; ++b) fetch(b);

    const uint32_t kfrag = (uint32_t)(((lane >> 4) * 8 + (lane & 7)) * STRIDE + ((lane >> 3) & 1) * 16);
    const uint32_t vfrag = (uint32_t)((((lane >> 3) & 1) * 8 + (lane & 7)) * STRIDE + (lane >> 4) * 16);
    int buf = 0;
    long long mine = u0 + warp;                         // this warp's next unit
    uint4 next_q[QN];                                   // a thread's pieces of the next pair's queries; rows that are none are zeros
    const auto ask_queries = [&](const Cursor& c) {
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int idx = tid + i * THREADS, row = (c.h % A.row_tiles) * 16 + idx / CH;
            next_q[i] = make_uint4(0u, 0u, 0u, 0u);
            if (idx < 16 * CH && row < A.group * A.fold) {
                const int t = c.t + row / A.group;
                next_q[i] = *reinterpret_cast<const uint4*>(A.q + t * A.q_t + (c.h / A.row_tiles) * A.q_h + row % A.group * A.q_g + idx % CH * 8);
            }
        }
    };
    ask_queries(seg);
    for (long long at = u0; at < u1;) {
        const int units = seg.units, t = seg.t, j = seg.h / A.row_tiles, row0 = seg.h % A.row_tiles * 16;
        const long long end = min(u1, at + units - seg.k);
        const int rows = min(16, A.group * A.fold - row0), first_k = seg.k;
        const Sight& s = seg.s;
        const int su = s.sink_units();
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int idx = tid + i * THREADS;
            if (idx < 16 * CH) *reinterpret_cast<uint4*>(q_s + (idx / CH) * STRIDE + idx % CH * 16) = next_q[i];
        }
        __syncthreads();
        const uint32_t qrow = ptx::smem_u32(q_s) + (uint32_t)((lane & 15) * STRIDE + (lane >> 4) * 16);
        uint32_t qf[KS][4];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) ldsm_x4(qf[ks], qrow + (uint32_t)(ks * 32));
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[DT][4];
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        for (; mine < end; mine += WARPS) {
            __syncwarp();                               // every lane is past its reads of the buffer that is filled again now
            fetch((buf + BUFS - 1) % BUFS);
            ptx::cp_async_wait<BUFS - 1>();
            __syncwarp();
            const uint32_t kb = ring0 + (uint32_t)(buf * G::UNIT) + kfrag, vb = ring0 + (uint32_t)(buf * G::UNIT + kUnit * STRIDE) + vfrag;
            float sc[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t b[4];
                ldsm_x4(b, kb + (uint32_t)(ks * 32));
                mma_16816(sc[0], qf[ks], b[0], b[1]);
                mma_16816(sc[1], qf[ks], b[2], b[3]);
            }
            // to base 2; what is no key is hidden
            const int k = first_k + (int)(mine - at);
            const int nk = (k < su ? s.sinks - k * kUnit : s.last + 1 - s.first - (k - su) * kUnit) - q4 * 2;
            float b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const bool seen = i * 8 + c < nk;
                    sc[i][c] = seen ? sc[i][c] * A.scale_log2 : -INFINITY;
                    sc[i][2 + c] = seen ? sc[i][2 + c] * A.scale_log2 : -INFINITY;
                    b0 = fmaxf(b0, sc[i][c]);
                    b1 = fmaxf(b1, sc[i][2 + c]);
                }
            b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 1));
            b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 1));
            b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 2));
            b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 2));
            if (__any_sync(0xffffffffu, b0 > m0 || b1 > m1)) {
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
            // the weights as two bf16 numbers each, the second the first's rounding error: the tensor pipe is idle anyway
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
        next.k += (int)(end - at);
        settle(next);
        if (end < u1) ask_queries(next);
        else chain_next();
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
        __syncthreads();
        const bool whole = end - at == units, keep = P.keep_parts;
        const long long pair = (long long)t * heads + seg.h;
        // a pair that begins in this run leaves its first part in the run's second slot, one that began before in the first
        const long long slot_at = whole ? 2ll * P.ctas + pair : 2ll * blockIdx.x + (first_k == 0 ? 1 : 0);
        float* const slot = P.slots + slot_at * 16 * (DH + 2);
        if (tid == 0 && first_k == 0) {
            const long long through = run_of(base_s[t] + (long long)(seg.h + 1) * units - 1);
            P.head[pair] = make_int2((int)slot_at, whole ? (keep ? 1 : 0) : (int)(through - blockIdx.x + 1));
        }
        for (int idx = tid; idx < rows * (DH / 2); idx += THREADS) {
            const int row = idx / (DH / 2), col = idx % (DH / 2) * 2;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ms[w][row]);
            const float z = M == -INFINITY ? 0.f : M;
            float nx = 0.f, ny = 0.f, den = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float wgt = exp2_fast(ms[w][row] - z);              // 0 for a warp that saw no key
                const float2 v = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(as_smem + at_s[w]) + row * LDO + col);
                nx = fmaf(wgt, v.x, nx);
                ny = fmaf(wgt, v.y, ny);
                den = fmaf(wgt, ls[w][row], den);
            }
            if (whole && !keep) {
                const float inv = den == 0.f ? 0.f : 1.f / den;           // no key: zeros
                *reinterpret_cast<uint32_t*>(A.out + t * A.o_t + j * A.o_h + (row0 + row) * A.o_g + col) = pack2(nx * inv, ny * inv);
                if (col == 0) write_sums(A, ((size_t)t * A.n_head + j) * A.group + row0 + row, z, den);
            } else {
                *reinterpret_cast<float2*>(slot + row * DH + col) = make_float2(nx, ny);
                if (col == 0) *reinterpret_cast<float2*>(slot + 16 * DH + row * 2) = make_float2(M, den);
            }
        }
        __syncthreads();                                // the warps' triples are read before the next fetch overwrites them
        seg = next;
        at = end;
    }
}

// A pair's parts: where they are.  The first lies in its first run's second slot, the others in their runs' first ones (a whole one by itself)
template <int DH>
struct Parts {
    const float* slots;
    int2 head;
    __device__ __forceinline__ const float* at(int i) const {
        return slots + (size_t)(i == 0 ? head.x : (head.x & ~1) + 2 * i) * (16 * (DH + 2));
    }
    __device__ __forceinline__ float2 sums(int i, int row) const { return *reinterpret_cast<const float2*>(at(i) + 16 * DH + row * 2); }
    __device__ __forceinline__ float2 values(int i, int row, int col) const { return *reinterpret_cast<const float2*>(at(i) + row * DH + col); }
};

// Adds up a pair's parts, in order: the 128-row kernel's, then those of the folded tokens, then the token's own.  A CTA per pair.
template <int DH>
__global__ void __launch_bounds__(128) attention_sum_kernel(const __grid_constant__ AttnView A, const __grid_constant__ PartPlan P,
                                                            const __grid_constant__ PartPlan F, const int folded_tiles, const int token0,
                                                            const __grid_constant__ TileParts M) {
    chain_wait();
    chain_next();
    const int heads = A.n_head * A.row_tiles;
    const long long pair = blockIdx.x;
    const int t = (int)(pair / heads), h = (int)(pair % heads), j = h / A.row_tiles, row0 = h % A.row_tiles * 16;
    const Parts<DH> own{P.slots, P.slots ? P.head[pair] : make_int2(0, 0)};
    if (own.head.y == 0 && M.n == 0 && !F.slots) return;
    const int rows = min(16, A.group - row0);
    for (int idx = threadIdx.x; idx < rows * (DH / 2); idx += blockDim.x) {
        const int row = idx / (DH / 2), col = idx % (DH / 2) * 2;
        const long long at = ((long long)t * A.n_head + j) * A.group + row0 + row, folded = (long long)(token0 + t) * A.group + row0 + row;
        const int frow = (int)(folded % 16);
        const Parts<DH> shared{F.slots, F.slots ? F.head[j * folded_tiles + folded / 16] : make_int2(0, 0)};
        float top = -INFINITY;
        for (int i = 0; i < M.n; ++i) top = fmaxf(top, M.ml[(i * M.rows + at) * 2]);
        for (int i = 0; i < shared.head.y; ++i) top = fmaxf(top, shared.sums(i, frow).x);
        for (int i = 0; i < own.head.y; ++i) top = fmaxf(top, own.sums(i, row).x);
        const float z = top == -INFINITY ? 0.f : top;
        float nx = 0.f, ny = 0.f, den = 0.f;
        const auto add = [&](const float2 ml, const float2 v) {
            const float wgt = exp2_fast(ml.x - z);
            const bool any = ml.x != -INFINITY;         // (a part without keys may hold anything else)
            nx = fmaf(wgt, any ? v.x : 0.f, nx);
            ny = fmaf(wgt, any ? v.y : 0.f, ny);
            den = fmaf(wgt, ml.y, den);
        };
#pragma unroll 4
        for (int i = 0; i < M.n; ++i) {
            const size_t r = i * M.rows + at;
            add(*reinterpret_cast<const float2*>(M.ml + r * 2), *reinterpret_cast<const float2*>(M.o + r * DH + col));
        }
#pragma unroll 4
        for (int i = 0; i < shared.head.y; ++i) add(shared.sums(i, frow), shared.values(i, frow, col));
#pragma unroll 4
        for (int i = 0; i < own.head.y; ++i) add(own.sums(i, row), own.values(i, row, col));
        const float inv = den == 0.f ? 0.f : 1.f / den;
        *reinterpret_cast<uint32_t*>(A.out + t * A.o_t + j * A.o_h + (row0 + row) * A.o_g + col) = pack2(nx * inv, ny * inv);
        if (col == 0) write_sums(A, at, z, den);
    }
}

template <int DH>
dsmoe_status launch_stream(const AttnView& A, const PartPlan& parts, cudaStream_t s) {
    static bool attr[kMaxDeviceSlots] = {};
    int dev = 0;
    DeviceState* st = nullptr;
    DSMOE_TRY(device_state(&st, &dev));
    if (!attr[dev]) {
        DSMOE_CUDA_TRY(cudaFuncSetAttribute(attention_stream_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamGeo<DH>::SMEM));
        attr[dev] = true;
    }
    DSMOE_CUDA_TRY(launch_chained(attention_stream_kernel<DH>, (unsigned)parts.ctas, 32 * StreamGeo<DH>::WARPS, StreamGeo<DH>::SMEM, s, A, parts));
    return DSMOE_OK;
}

template <int DH>
dsmoe_status launch_sum(const AttnView& A, const PartPlan& parts, const PartPlan& folded, int folded_tiles, int token0, const TileParts& more,
                        cudaStream_t s) {
    const long long pairs = (long long)A.T * A.n_head * A.row_tiles;
    DSMOE_CUDA_TRY(launch_chained(attention_sum_kernel<DH>, (unsigned)pairs, 128, 0, s, A, parts, folded, folded_tiles, token0, more));
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

// One CTA per SM, as far as each has a unit per warp in the longest case
int stream_ctas(const AttnView& A) {
    const long long seen = A.window < A.L ? (long long)A.window + A.sinks : A.L;
    const long long units = (seen + kUnit - 1) / kUnit + 1, warps = A.d_head <= 128 ? 8 : 4;
    const long long pairs = (long long)(A.T < kListTokens ? A.T : kListTokens) * A.n_head * A.row_tiles, most = sm_count();
    const long long wanted = (pairs * units + warps - 1) / warps;
    return (int)(wanted < most ? wanted : most);
}

dsmoe_status launch_stream_attention(const AttnView& A, const PartPlan& parts, cudaStream_t s) {
#define DSMOE_CALL(DH) launch_stream<DH>(A, parts, s)
    DSMOE_BY_HEAD(A.d_head, DSMOE_CALL)
#undef DSMOE_CALL
}

dsmoe_status launch_attention_sum(const AttnView& A, const PartPlan& parts, const PartPlan& folded, int folded_tiles, int token0,
                                  const TileParts& more, cudaStream_t s) {
#define DSMOE_CALL(DH) launch_sum<DH>(A, parts, folded, folded_tiles, token0, more, s)
    DSMOE_BY_HEAD(A.d_head, DSMOE_CALL)
#undef DSMOE_CALL
}

}  // namespace dsmoe
