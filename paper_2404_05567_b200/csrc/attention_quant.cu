// Attention of single tokens against their caches in 4 bits (see quant_cache.cuh for the format, cache_attention.cuh for what a row sees and what parts are).
//
// The keys of all (token, head, row tile) pairs, in units of 32, are one list, cut into equal runs of the CTAs and those into equal runs of their warps; a pair that
// several CTAs share leaves a part per CTA, added up by the next launch.
//
// A warp brings its units' codes and scales into a ring of its own (cp.async), and takes 16 keys at a time to its tensor instructions with the keys, not the rows, as
// the 16-row operand: S^T = K q^T and O^T += V^T P^T.  Codes become operands in registers, once for all of the pair's rows, of which 8 are the
// narrow side of an instruction (two of those for groups of more than 8).
//   K: a code's 4 bits at the lower end of a half word are an fp16 number as they are, (8 + c) 2^-24, and 16 times that four bits further up: half a word of
//      codes is an operand of masks alone.  A row's queries are multiplied by the power of two that makes the largest 2^14 to 2^15 (and 1 / 16 in the
//      second kind of place) and so are fp16 numbers exactly, down to 2^-28 of the largest.  A group's sum begins with -8 times the sum of the row's queries
//      there, and its scale multiplies it into the logit.  (With e4m3 operands, for which whole words of codes would do, the tensor instructions cost twice
//      as much and others beside: 62 tokens with up to 8192 keys 77.9 us instead of 70.6 with bf16 operands.)
//   V: operands of masks too, less 8 2^-24, or 16 times that.  The scales multiply the weights instead, as fp16 numbers, a weight and group at a time (rounded to
//      11 bits).  The scales are relative to a power of two near the largest that the warp has met, 1/2 to 2 times it, which moves as the maximum of the logits does.
//      A product is a multiple of 2^-34 of that (2^-24, and kRaise): it has 11 bits where the weight is 2^-23 of the row's largest or more beside scales like the
//      largest, 2^-17 beside the smallest, 2^-7; it is nothing below 2^-35 and 2^-28.  So once the warp has met scales of a pair that are further apart (2^6 to
//      2^8), or no numbers, it goes another way: values are bf16 numbers s * c and weights two bf16 numbers each (62 tokens with up to 8192 keys, of which the first
//      four have values 2^-9 as large: 69 us instead of 66).
// The logits' layout holds two rows of a key side by side, the weights' two keys of a row: movmatrix.
// What bounds it: 62 tokens with up to 8192 keys, 4 x 5 heads of 128 by position, take 66 us (their 4.5 bits a value at 6.45 TB/s 34): the copies alone 50, of which 35
// at 6.3 TB/s and the rest before the first key and behind the last one; a unit's chain of scales, products, maximum, exponentials, transposition and products,
// with three warps a scheduler to cover it, 16 more (ALU 52 %, tensor pipe 20 %, issue slots 56 % of the cycles).  2 tokens with 131072 keys, 8 x 4 heads: 74 (44).
#include <cuda_fp16.h>

#include <algorithm>

#include "quant_cache.cuh"
#include "umma.cuh"

namespace dsmoe {

namespace {

constexpr int kQuantUnit = 32;            // keys that a warp takes at a time
// The maximum that weights are relative to moves when a logit passes it by more than kQuantMoves.  Weights of up to 2^(kQuantMoves + kRaise), times scales
// below 2, are fp16 numbers; each of the 14 that the moves do not take keeps products of small weights and small scales one bit longer.  With moves of 8, 4, 2 and 1,
// us: 62 tokens with up to 8192 keys 65.8, 65.6, 65.8, 66.6; 48 tokens of 4 x 16 heads of 96, window 4090 55.6, 56.1, 57.7, 59.3; 62 of 4 x 16 of 256, 4096 keys 252, 262, 279, 294.
constexpr float kQuantMoves = 4.f, kRaise = 10.f;

__device__ __forceinline__ void mma_half_first(float (&d)[4], const uint32_t (&a)[4], uint2 b, float c0, float c1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %10, %11};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void mma_half(float (&d)[4], const uint32_t (&a)[4], uint2 b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ void mma_next(float (&d)[4], const uint32_t (&a)[4], uint2 b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
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
__device__ __forceinline__ uint32_t pack2_half(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// a * b + c, two bf16 numbers at a time
__device__ __forceinline__ uint32_t fma_pair(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// The larger ones of two numbers of 16 bits each
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul_half_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t add_half_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }        // -126 <= e <= 127
// (x & mask) | bits
__device__ __forceinline__ uint32_t masked(uint32_t x, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "r"(mask), "r"(bits));
    return r;
}

// N words from shared memory, at a multiple of N words
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&r)[N], uint32_t addr) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]) : "r"(addr + 4 * i));
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r[i]), "=r"(r[i + 1]) : "r"(addr + 4 * i));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[i]) : "r"(addr + 4 * i));
    }
}
template <int N>
__device__ __forceinline__ void store_words(uint32_t addr, const uint32_t (&r)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("st.shared.v4.b32 [%4], {%0, %1, %2, %3};" ::"r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(addr + 4 * i) : "memory");
    } else if constexpr (N == 2) {
        asm volatile("st.shared.v2.b32 [%2], {%0, %1};" ::"r"(r[0]), "r"(r[1]), "r"(addr) : "memory");
    } else {
        static_assert(N == 1, "a word, two, or fours");
        asm volatile("st.shared.b32 [%1], %0;" ::"r"(r[0]), "r"(addr) : "memory");
    }
}
// BYTES (4, 8, 16), or zeros
template <int BYTES>
__device__ __forceinline__ void copy_piece(uint32_t dst, const void* src, bool real) {
    const uint32_t n = real ? BYTES : 0;
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
}

__host__ __device__ static inline int quant_units(const Sight& s) {
    const int n = (s.sinks + kQuantUnit - 1) / kQuantUnit + (s.last >= s.first ? (s.last - s.first) / kQuantUnit + 1 : 0);
    return n > 0 ? n : 1;                 // a token that sees nothing has one unit without keys, so that somebody writes its row
}

// Warps of a CTA: as many as their registers and rings allow.  With 12 and with 8, us: 62 tokens with up to 8192 keys 66, 74; 2 with 131072 75, 87; 256 with up to 500
// 17.6, 18.9; one token with 512 10.5, 10.1.
__host__ __device__ static constexpr int quant_warps(int d_head, int nt) { return d_head <= 128 ? nt == 1 ? 12 : 8 : nt == 1 ? 6 : 4; }

// The first unit of run c of n equal ones (the first ones a unit longer), and the run that holds unit u
__device__ __forceinline__ long long run_start(long long total, int n, int c) {
    const long long share = divide(total, n);
    return c * share + min((long long)c, total - share * n);
}
__device__ __forceinline__ int run_of(long long total, int n, long long u) {
    const long long share = divide(total, n), extra = total - share * n, cut = extra * (share + 1);
    return (int)(u < cut ? u / (share + 1) : extra + (u - cut) / share);
}

// The natural logarithm of a row's sum
__device__ __forceinline__ float row_lse(float M, float den) { return ((M == -INFINITY ? 0.f : M) + log2f(den)) * 0.6931471805599453f; }

// NT: tiles of 8 rows that a pair has
template <int DH, int NT>
struct QuantGeo {
    static constexpr int G = DH / kQuantGroup, ROW = 16 * G, SC = 2 * quant_scales(DH);
    // bytes from one key's codes to the next in shared memory, with which neither the keys' nor the values' reads meet in a bank
    static constexpr int KROW = ROW + (G == 8 ? 16 : 0), VROW = ROW + (G % 2 == 0 ? 16 : 0);
    static constexpr int V = kQuantUnit * KROW, KS = V + kQuantUnit * VROW, VS = KS + kQuantUnit * 2 * SC, UNIT = VS + kQuantUnit * SC;
    static constexpr int WARPS = quant_warps(DH, NT);
    static constexpr int LDO = DH + 4;    // floats from one row of a warp's sums to the next, where they meet
    static constexpr int SUMS = 8 * NT * LDO * 4;
    static constexpr int FIT = (216 * 1024 / WARPS - SUMS) / UNIT, BUFS = FIT > 4 ? 4 : FIT;
    static constexpr int OWN = BUFS * UNIT + SUMS, SMEM = WARPS * OWN;       // a warp's: its ring, and the sums of the pair that began before its run
    static_assert(BUFS >= 2 && SUMS <= BUFS * UNIT && UNIT % 16 == 0, "rings of two units and more, in which a warp's last sums find a place");
    static_assert(SMEM + 20 * 1024 <= 227 * 1024, "and the lists");
};

// What a warp leaves of a pair that is not its alone: rows' largest logits and sums beside the values' sums
template <int ROWS>
struct Piece {
    int there, begins, ends;              // whether there is one; begins or ends with the pair
    int e, h, units;                      // the pair: token, (head, row tile), units
    uint32_t sums;                        // where they lie
    float m[ROWS], l[ROWS];
};

// HB: neighbouring pairs that a CTA takes at a time, a warp each.  Where the heads of a position lie side by side they are so read side by side, and rows of
// one head beyond 16 read its keys out of L2 or nearer.  62 tokens with up to 8192 keys, 4 heads side by side: 66 us with 4 at a time, 69 with 2, 83 with 1.
//
// A CTA's run of the list is cut into equal runs of its warps (of each of the HB pairs), which take their units one after the other and owe the others
// nothing until the end.  What a warp has of a pair that began before its run or goes on behind it is a piece; the CTA's pieces of a pair are added up once all
// are there, and a pair that several CTAs share leaves a part per CTA.
template <int DH, int NT, int HB>
__global__ void __launch_bounds__(32 * QuantGeo<DH, NT>::WARPS, 1)
attention_quant_kernel(const __grid_constant__ AttnView A, const __grid_constant__ QuantView C, const __grid_constant__ QuantPlan P) {
    using Geo = QuantGeo<DH, NT>;
    constexpr int G = Geo::G, BUFS = Geo::BUFS, WARPS = Geo::WARPS, THREADS = 32 * WARPS, PER = (kListTokens + THREADS - 1) / THREADS, LDO = Geo::LDO;
    constexpr int SW = quant_scales(DH) / 2;            // words of a key's scales
    constexpr int KW = WARPS / HB;                      // runs of a CTA
    extern __shared__ __align__(16) unsigned char aq_smem[];
    __shared__ long long base_s[kListTokens + 1];       // units before token e's
    __shared__ Sight sight_s[kListTokens];
    __shared__ long long warp_sum_s[WARPS];
    __shared__ Piece<8 * NT> piece_s[HB][2 * KW];       // of each run: what began before it, what goes on behind it
    __shared__ int head_s[WARPS][2 * KW + 1];           // first pieces of pairs
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, q4 = lane & 3;
    const int hb = warp % HB, kw = warp / HB;
    const int groups = A.n_head * A.row_tiles / HB;     // of a token, HB pairs each
    chain_wait();
    // (runs beyond the grid's are the last CTA's)
    for (int i = tid; i < P.passes * P.runs; i += THREADS)
        if (min(i % P.runs, (int)gridDim.x - 1) == (int)blockIdx.x) P.run_head[i] = make_int2(0, 0);

    for (int pass = 0; pass < P.passes; ++pass) {
    // ---- the pass's tokens and their units
    const int n0 = pass * kListTokens, n = min(kListTokens, A.T - n0);
    __syncthreads();
    {
        long long mine[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = tid * PER + i;
            mine[i] = 0;
            if (e < n) {
                bool bad = false;
                const Sight s = sight_of(A, n0 + e, &bad);
                sight_s[e] = s;
                mine[i] = (long long)quant_units(s) * groups;
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
        if (lane < 2) piece_s[hb][2 * kw + lane].there = 0;
        __syncthreads();
        long long before = incl - sum;
        for (int w = 0; w < warp; ++w) before += warp_sum_s[w];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = tid * PER + i;
            if (e < n && e < kListTokens) base_s[e] = before;
            before += mine[i];
        }
        if (tid == THREADS - 1) base_s[n] = before;
        __syncthreads();
    }
    // Equal runs of the CTAs, of at least a unit for each warp
    const int n_runs = P.whole ? n * groups : (int)min((long long)gridDim.x, divide(base_s[n] + KW - 1, KW));
    if ((int)blockIdx.x >= n_runs) continue;
    long long u0, left;                                 // the first unit of this warp's run, and the number of those that are still to be taken
    {
        long long first, units;
        if (P.whole) {
            const int e = (int)blockIdx.x / groups;
            units = quant_units(sight_s[e]);
            first = base_s[e] + (int)blockIdx.x % groups * units;
        } else {
            first = run_start(base_s[n], n_runs, blockIdx.x);
            units = run_start(base_s[n], n_runs, blockIdx.x + 1) - first;
        }
        const long long a = divide(units * kw, KW), b = divide(units * (kw + 1), KW);
        u0 = first + a;
        left = b - a;
    }

    // Where a unit lies: token, its group of pairs, key block of it
    struct Cursor {
        int e, h, k, units;
        Sight s;
    };
    const auto look = [&](Cursor& c) {
        if (c.e >= n) return;
        c.s = sight_s[c.e];
        c.units = quant_units(c.s);
    };
    const auto settle = [&](Cursor& c) {                // k past the pair's units: on to the pair that holds it
        if (c.k < c.units) return false;
        c.k = 0;
        if (++c.h == groups) {
            c.h = 0;
            ++c.e;
            look(c);
        }
        return true;
    };
    Cursor seg;
    {
        // the last token whose units begin at or before u0: its 16, then which of them
        static_assert(kListTokens <= 32 * 16, "two looks of a warp");
        int lo = 16 * (__popc(__ballot_sync(0xffffffffu, 16 * lane < n && base_s[min(16 * lane, n)] <= u0)) - 1);
        lo += __popc(__ballot_sync(0xffffffffu, lane < 16 && lo + lane < n && base_s[min(lo + lane, n)] <= u0)) - 1;
        seg.e = lo;
        look(seg);
        const long long in = u0 - base_s[lo];
        seg.h = (int)divide(in, seg.units);
        seg.k = (int)(in - (long long)seg.h * seg.units);
    }
    Cursor ahead = seg;                                 // the next unit to fetch
    long long to_fetch = left, code = 0, scales = 0;    // ... where its pair's codes and scales begin
    const auto aim = [&]() {
        const int j = (ahead.h * HB + hb) / A.row_tiles;
        code = ahead.s.seq * C.c_s + j * C.c_h;
        scales = ahead.s.seq * C.s_s + j * C.s_h;
    };
    aim();
    const uint32_t ring0 = ptx::smem_u32(aq_smem) + (uint32_t)(warp * Geo::OWN);
    const auto fetch = [&](int buf) {
        if (to_fetch > 0) {
            const Sight& s = ahead.s;
            const int su = (s.sinks + kQuantUnit - 1) / kQuantUnit;
            const int key0 = ahead.k < su ? ahead.k * kQuantUnit : s.first + (ahead.k - su) * kQuantUnit;
            const int nk = ahead.k < su ? s.sinks - key0 : s.last + 1 - key0;       // keys of the unit, if fewer than kQuantUnit
            const int slot0 = slot_of(A, key0);
            const uint32_t to = ring0 + (uint32_t)(buf * Geo::UNIT);
            {                                           // a lane's key's scales
                int slot = slot0 + (lane < nk ? lane : 0);
                if (A.ring && slot >= A.L) slot -= A.ring;                           // in a unit across the end of the ring the slots are not neighbours
                copy_piece<Geo::SC>(to + Geo::KS + lane * 2 * Geo::SC, C.K_scale + scales + slot * C.s_p, lane < nk);
                copy_piece<Geo::SC>(to + Geo::VS + lane * Geo::SC, C.V_scale + scales + slot * C.s_p, lane < nk);
            }
            // a unit of neighbouring slots that is full: no piece needs a look at its row
            if ((G & (G - 1)) == 0 && nk >= kQuantUnit && (!A.ring || slot0 + kQuantUnit <= A.L)) {
                constexpr int ROWS = 32 / G;                                         // rows at a time
                const long long from = code + (slot0 + lane / G) * C.c_p + lane % G * 16, down = ROWS * C.c_p;
                const unsigned char *k = C.K + from, *v = C.V + from;
                const uint32_t kd = to + lane / G * Geo::KROW + lane % G * 16, vd = to + Geo::V + lane / G * Geo::VROW + lane % G * 16;
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    ptx::cp_async16(kd + i * ROWS * Geo::KROW, k);
                    ptx::cp_async16(vd + i * ROWS * Geo::VROW, v);
                    k += down;
                    v += down;
                }
            } else {
#pragma unroll 1
                for (int i = 0; i < G; ++i) {
                    const int idx = lane + 32 * i, row = idx / G, ch = idx % G;
                    int slot = slot0 + (row < nk ? row : 0);
                    if (A.ring && slot >= A.L) slot -= A.ring;
                    const long long src = code + slot * C.c_p + ch * 16;
                    copy_piece<16>(to + row * Geo::KROW + ch * 16, C.K + src, row < nk);    // past the last key: zeros
                    copy_piece<16>(to + Geo::V + row * Geo::VROW + ch * 16, C.V + src, row < nk);
                }
            }
            ++ahead.k;
            if (--to_fetch > 0 && settle(ahead)) aim();
        }
        ptx::cp_async_commit();
    };

    const uint32_t kfrag = (uint32_t)(g8 * Geo::KROW + q4 * 4 * G), vfrag = (uint32_t)(Geo::V + 2 * q4 * Geo::VROW + (g8 >> 1) * 4 * G);
    const uint32_t half = g8 & 1 ? 0x7632u : 0x5410u;   // which half of a word of the values' is this lane's
    int buf = 0, fetched = 0;                           // (the first unit is preceded by BUFS - 1 of them)
    while (left > 0) {
        const int t = n0 + seg.e, units = seg.units, first_k = seg.k, end_k = (int)min((long long)units, first_k + left);
        const Sight& s = seg.s;
        const int su = (s.sinks + kQuantUnit - 1) / kQuantUnit;
        const int pair = seg.h * HB + hb, j = pair / A.row_tiles, row0 = pair % A.row_tiles * 16, rows = min(8 * NT, A.group - row0);
        // queries as the narrow operand, in the order in which codes leave their words; what a group's sum begins with; and what makes a row's sums logits in
        // base 2
        uint2 qf[NT][2 * G];
        float init[NT][G][2], to_logit[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool real = nt * 8 + g8 < rows;
            const __nv_bfloat16* const q = A.q + t * A.q_t + j * A.q_h + (real ? row0 + nt * 8 + g8 : 0) * A.q_g + q4 * 8;
            uint4 in[G];
            uint32_t top = 0;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                in[g] = *reinterpret_cast<const uint4*>(q + g * kQuantGroup);
                if (!real) in[g] = make_uint4(0u, 0u, 0u, 0u);
                const uint32_t w[4] = {in[g].x, in[g].y, in[g].z, in[g].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // the power of two (2^126 at most), and the inverse of 2^-24 times it
            const int exponent = min(max((int)(top >> 7), 15), 254);
            const float up = copysignf(power_of_two(141 - exponent), A.scale_log2);       // (a negative scale: the queries' signs)
            float down = power_of_two(exponent - 141) * (0x1p24f * fabsf(A.scale_log2));
            if (top >= 0x7f80u) down = __uint_as_float(0x7fffffffu);              // a query that is no number: the row is none
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t w[4] = {in[g].x, in[g].y, in[g].z, in[g].w};
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (i & 1 ? high_part(w[i / 2]) : low_part(w[i / 2])) * up;
                qf[nt][2 * g] = make_uint2(pack2_half(x[0], x[4]), pack2_half(x[1] * 0.0625f, x[5] * 0.0625f));
                qf[nt][2 * g + 1] = make_uint2(pack2_half(x[2], x[6]), pack2_half(x[3] * 0.0625f, x[7] * 0.0625f));
                float sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                init[nt][g][0] = -0x1p-21f * __shfl_sync(0xffffffffu, sum, q4 * 8);
                init[nt][g][1] = -0x1p-21f * __shfl_sync(0xffffffffu, sum, q4 * 8 + 4);
            }
            to_logit[nt][0] = __shfl_sync(0xffffffffu, down, q4 * 8);
            to_logit[nt][1] = __shfl_sync(0xffffffffu, down, q4 * 8 + 4);
        }
        // Rows 2 q4 and 2 q4 + 1 of each tile.  The largest sum m so far, as it was when it last moved, and the sum beyond which it moves; weights are
        // 2^(to_logit x - z), 2^kRaise times those relative to the largest logit, so that small ones are fp16 numbers.
        float m[NT][2], limit[NT][2], z[NT][2], l[NT][2];
        // Sums of values in units of 2^(base - 88), each second one 16 times as large
        float o[2 * G][NT][4];
        int base = 0, first_base = 0;                   // the exponent (of a bf16) whose scales' exponent as an fp16 is 0; what it was at first
        bool plain = true;                              // so far all scales are near one another
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = limit[nt][0] = limit[nt][1] = -INFINITY;
            z[nt][0] = z[nt][1] = l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * G; ++i) o[i][nt][0] = o[i][nt][1] = o[i][nt][2] = o[i][nt][3] = 0.f;
        }
        for (int k = first_k; k < end_k; ++k) {
            __syncwarp();                               // every lane is past its reads of the buffer that is filled again now
#pragma unroll 1
            for (;; ++fetched) {
                const int to = buf + fetched;
                fetch(to < BUFS ? to : to - BUFS);
                if (fetched == BUFS - 1) break;
            }
            ptx::cp_async_wait<BUFS - 1>();
            const uint32_t unit = ring0 + (uint32_t)(buf * Geo::UNIT);
            // ---- a lane's key's scales (it has copied them itself): K's to fp32; V's to fp16, relative to base, with two keys' side by side
            {
                const uint32_t k_at = unit + (uint32_t)(Geo::KS + lane * 2 * Geo::SC), v_at = unit + (uint32_t)(Geo::VS + lane * Geo::SC);
                uint32_t ks[SW], wide[2 * SW], vs[SW], top = 0, low = 0xffffffffu;
                bool bad = false;
                load_words<SW>(ks, k_at);
                load_words<SW>(vs, v_at);
#pragma unroll
                for (int i = 0; i < SW; ++i) {
                    wide[2 * i] = ks[i] << 16;
                    wide[2 * i + 1] = ks[i] & 0xffff0000u;
                }
                store_words<2 * SW>(k_at, wide);
#pragma unroll
                for (int g = 0; g < G; ++g) {           // (places behind the last group may hold anything)
                    const uint32_t v = g & 1 ? vs[g / 2] >> 16 : vs[g / 2] & 0xffffu, size = v & 0x7fffu;
                    if (size < 0x7f80u) top = max(top, size);
                    low = min(low, v - 1u);             // (zeros: the largest)
                    bad = bad || v >= 0x7f80u;          // (also what is below zero)
                }
                // Plain: scales of a bf16's exponents base + 8 to base + 15, and zeros; base does not rise far.  Otherwise they may reach to base + 95, and so may values
                // of all kinds be bf16 numbers.
                const auto near = [&](int b) { return !bad && top < (uint32_t)(b + 16) << 7 && low >= ((uint32_t)(b + 8) << 7) - 1u; };
                if (!plain || __any_sync(0xffffffffu, !near(base))) {
                    int next = base;
                    if (__any_sync(0xffffffffu, top >= (uint32_t)(base + (plain ? 16 : 96)) << 7)) {
                        next = max((int)(__reduce_max_sync(0xffffffffu, top) >> 7) - (plain ? 14 : 94), 0);
                        if (base == 0) first_base = next;
                    }
                    if (plain && (next > first_base + 6 || __any_sync(0xffffffffu, !near(next)))) {
                        plain = false;
                        next = max(next - 80, 0);
                    }
                    const float f = exp2_fast((float)(base - next));
                    base = next;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int i = 0; i < 2 * G; ++i) o[i][nt][c] *= f;
                }
                if (plain) {
                    const uint32_t none = (uint32_t)base << 7 | (uint32_t)base << 23;
                    uint32_t pairs[SW];
#pragma unroll
                    for (int i = 0; i < SW; ++i) vs[i] = max_pair(vs[i], none) * 8u - none * 8u;      // (mantissas of 7 and 10 bits)
                    // of keys 2 i and 2 i + 1: one group's of both in a word; the even key's lane writes the first half of the groups
                    if constexpr (SW == 1) {
                        const uint32_t other = __shfl_xor_sync(0xffffffffu, vs[0], 1);
                        pairs[0] = lane & 1 ? __byte_perm(other, vs[0], 0x7632) : __byte_perm(vs[0], other, 0x5410);
                    } else {
#pragma unroll
                        for (int i = 0; i < SW / 2; ++i) {
                            const uint32_t mine = lane & 1 ? vs[SW / 2 + i] : vs[i];
                            const uint32_t other = __shfl_xor_sync(0xffffffffu, lane & 1 ? vs[i] : vs[SW / 2 + i], 1);
                            const uint32_t even = lane & 1 ? other : mine, odd = lane & 1 ? mine : other;
                            pairs[2 * i] = __byte_perm(even, odd, 0x5410);
                            pairs[2 * i + 1] = __byte_perm(even, odd, 0x7632);
                        }
                    }
                    store_words<SW>(v_at, pairs);
                }
            }
            __syncwarp();
            // ---- sums of keys g8 and g8 + 8 of each half of the unit
            float x[2][NT][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w0[G], w1[G], s0[2 * SW], s1[2 * SW];
                load_words<G>(w0, unit + kfrag + (uint32_t)(16 * h * Geo::KROW));
                load_words<G>(w1, unit + kfrag + (uint32_t)((16 * h + 8) * Geo::KROW));
                load_words<2 * SW>(s0, unit + (uint32_t)(Geo::KS + (16 * h + g8) * 2 * Geo::SC));
                load_words<2 * SW>(s1, unit + (uint32_t)(Geo::KS + (16 * h + 8 + g8) * 2 * Geo::SC));
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint32_t v0 = w0[g] >> 8, v1 = w1[g] >> 8;
                    const uint32_t a[4] = {w0[g] & 0x000f000fu, w1[g] & 0x000f000fu, w0[g] & 0x00f000f0u, w1[g] & 0x00f000f0u};
                    const uint32_t b[4] = {v0 & 0x000f000fu, v1 & 0x000f000fu, v0 & 0x00f000f0u, v1 & 0x00f000f0u};
                    const float sa = __uint_as_float(s0[g]), sb = __uint_as_float(s1[g]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float c[4];
                        mma_half_first(c, a, qf[nt][2 * g], init[nt][g][0], init[nt][g][1]);
                        mma_half(c, b, qf[nt][2 * g + 1]);
                        x[h][nt][0] = g == 0 ? sa * c[0] : fmaf(sa, c[0], x[h][nt][0]);
                        x[h][nt][1] = g == 0 ? sa * c[1] : fmaf(sa, c[1], x[h][nt][1]);
                        x[h][nt][2] = g == 0 ? sb * c[2] : fmaf(sb, c[2], x[h][nt][2]);
                        x[h][nt][3] = g == 0 ? sb * c[3] : fmaf(sb, c[3], x[h][nt][3]);
                    }
                }
            }
            // what is no key is hidden
            const int nk = k < su ? s.sinks - k * kQuantUnit : s.last + 1 - s.first - (k - su) * kQuantUnit;
            if (nk < kQuantUnit) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (16 * h + (c >> 1) * 8 + g8 >= nk) x[h][nt][c] = -INFINITY;
            }
            float top[NT][2];
            bool moves = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    top[nt][r] = max3(fmaxf(x[0][nt][r], x[0][nt][2 + r]), x[1][nt][r], x[1][nt][2 + r]);
                    moves = moves || top[nt][r] > limit[nt][r];
                }
            // (see kQuantMoves)
            if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float b = top[nt][r];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, d));
                        if (!(b > m[nt][r])) continue;  // (the row's lanes agree)
                        const float before = z[nt][r];
                        z[nt][r] = fmaf(b, to_logit[nt][r], -kRaise);
                        limit[nt][r] = b + kQuantMoves / to_logit[nt][r];
                        const float f = m[nt][r] == -INFINITY ? 1.f : exp2_fast(before - z[nt][r]);
                        m[nt][r] = b;
                        l[nt][r] *= f;
#pragma unroll
                        for (int i = 0; i < 2 * G; ++i) {
                            o[i][nt][r] *= f;
                            o[i][nt][2 + r] *= f;
                        }
                    }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[h][nt][c] = exp2_fast(fmaf(x[h][nt][c], to_logit[nt][c & 1], -z[nt][c & 1]));
            if (nk < kQuantUnit) {                      // (a scale of 0 makes hidden logits no numbers)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (16 * h + (c >> 1) * 8 + g8 >= nk) x[h][nt][c] = 0.f;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) l[nt][r] += (x[0][nt][r] + x[0][nt][2 + r]) + (x[1][nt][r] + x[1][nt][2 + r]);
            // ---- values of keys 2 q4, 2 q4 + 1 and the same + 8 of each half
            if (plain) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t v0[G], v1[G], v2[G], v3[G], s0[2 * SW], s1[2 * SW];
                    load_words<G>(v0, unit + vfrag + (uint32_t)(16 * h * Geo::VROW));
                    load_words<G>(v1, unit + vfrag + (uint32_t)((16 * h + 1) * Geo::VROW));
                    load_words<G>(v2, unit + vfrag + (uint32_t)((16 * h + 8) * Geo::VROW));
                    load_words<G>(v3, unit + vfrag + (uint32_t)((16 * h + 9) * Geo::VROW));
                    load_words<2 * SW>(s0, unit + (uint32_t)(Geo::VS + (16 * h + 2 * q4) * Geo::SC));
                    load_words<2 * SW>(s1, unit + (uint32_t)(Geo::VS + (16 * h + 8 + 2 * q4) * Geo::SC));
                    uint2 pf[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        pf[nt] = make_uint2(transpose8(pack2_half(x[h][nt][0], x[h][nt][1])), transpose8(pack2_half(x[h][nt][2], x[h][nt][3])));
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const uint32_t w0 = __byte_perm(v0[g], v1[g], half), w1 = __byte_perm(v2[g], v3[g], half), u0 = w0 >> 8, u1 = w1 >> 8;
                        // (0x8008: -8 2^-24)
                        const uint32_t a[4] = {add_half_pair(w0 & 0x000f000fu, 0x80088008u), add_half_pair(w0 & 0x00f000f0u, 0x80808080u),
                                               add_half_pair(w1 & 0x000f000fu, 0x80088008u), add_half_pair(w1 & 0x00f000f0u, 0x80808080u)};
                        const uint32_t b[4] = {add_half_pair(u0 & 0x000f000fu, 0x80088008u), add_half_pair(u0 & 0x00f000f0u, 0x80808080u),
                                               add_half_pair(u1 & 0x000f000fu, 0x80088008u), add_half_pair(u1 & 0x00f000f0u, 0x80808080u)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint2 w = make_uint2(mul_half_pair(pf[nt].x, s0[g]), mul_half_pair(pf[nt].y, s1[g]));
                            mma_half(o[2 * g][nt], a, w);
                            mma_half(o[2 * g + 1][nt], b, w);
                        }
                    }
                }
            } else {
                // the scales in the sums' units
                const int e = 88 - base;
                const uint32_t f0 = pack2(power_of_two(e / 2), power_of_two(e / 2)), f1 = pack2(power_of_two(e - e / 2), power_of_two(e - e / 2));
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint2 pf[NT], pr[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float p[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) p[c] = h == 0 ? x[0][nt][c] : x[1][nt][c];
                        const uint32_t w0 = pack2(p[0], p[1]), w1 = pack2(p[2], p[3]);
                        pf[nt] = make_uint2(transpose8(w0), transpose8(w1));
                        pr[nt] = make_uint2(transpose8(pack2(p[0] - low_part(w0), p[1] - high_part(w0))), transpose8(pack2(p[2] - low_part(w1), p[3] - high_part(w1))));
                    }
                    const uint32_t at = unit + vfrag + (uint32_t)(16 * h * Geo::VROW), s_at = unit + (uint32_t)(Geo::VS + (16 * h + 2 * q4) * Geo::SC);
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        uint32_t v0[1], v1[1], v2[1], v3[1], s0[1], s1[1], s2[1], s3[1];
                        load_words<1>(v0, at + 4 * g);
                        load_words<1>(v1, at + 4 * g + Geo::VROW);
                        load_words<1>(v2, at + 4 * g + 8 * Geo::VROW);
                        load_words<1>(v3, at + 4 * g + 9 * Geo::VROW);
                        load_words<1>(s0, s_at + g / 2 * 4);
                        load_words<1>(s1, s_at + g / 2 * 4 + Geo::SC);
                        load_words<1>(s2, s_at + g / 2 * 4 + 8 * Geo::SC);
                        load_words<1>(s3, s_at + g / 2 * 4 + 9 * Geo::SC);
                        const uint32_t w0 = __byte_perm(v0[0], v1[0], half), w1 = __byte_perm(v2[0], v3[0], half), side = g & 1 ? 0x7632 : 0x5410;
                        const uint32_t sa = fma_pair(fma_pair(__byte_perm(s0[0], s1[0], side), f0, 0x80008000u), f1, 0x80008000u);
                        const uint32_t sb = fma_pair(fma_pair(__byte_perm(s2[0], s3[0], side), f0, 0x80008000u), f1, 0x80008000u);
                        const uint32_t sa16 = fma_pair(sa, 0x41804180u, 0x80008000u), sb16 = fma_pair(sb, 0x41804180u, 0x80008000u);
                        const auto value = [](uint32_t x, uint32_t s) {            // 4 bits beside the exponent of 16 are 24 + c
                            return fma_pair(fma_pair(masked(x, 0x00780078u, 0x41804180u), 0x3f803f80u, 0xc1c0c1c0u), s, 0x80008000u);
                        };
                        const uint32_t a[4] = {value(w0 << 3, sa), value(w0 >> 1, sa16), value(w1 << 3, sb), value(w1 >> 1, sb16)};
                        const uint32_t b[4] = {value(w0 >> 5, sa), value(w0 >> 9, sa16), value(w1 >> 5, sb), value(w1 >> 9, sb16)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma_next(o[2 * g][nt], a, pf[nt]);
                            mma_next(o[2 * g + 1][nt], b, pf[nt]);
                            mma_next(o[2 * g][nt], a, pr[nt]);
                            mma_next(o[2 * g + 1][nt], b, pr[nt]);
                        }
                    }
                }
            }
            buf = buf + 1 == BUFS ? 0 : buf + 1;
        }
        // ---- the sums as numbers, relative to the largest logit
        {
            const int e = base - 88 - (int)kRaise;
            const float f0 = power_of_two(e / 2), f1 = power_of_two(e - e / 2);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    l[nt][r] *= exp2_fast(-kRaise);
                    m[nt][r] = m[nt][r] == -INFINITY ? -INFINITY : m[nt][r] * to_logit[nt][r];
#pragma unroll
                    for (int i = 0; i < 2 * G; ++i) {
                        o[i][nt][r] = o[i][nt][r] * f0 * f1;
                        o[i][nt][2 + r] = o[i][nt][2 + r] * (f0 * 0.0625f) * f1;
                    }
                }
        }
        // ---- sums over the keys that the lanes of a row had
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nt][r] += __shfl_xor_sync(0xffffffffu, l[nt][r], d);
        if (end_k - first_k == units) {                        // the pair is this warp's
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int member = row0 + nt * 8 + 2 * q4 + r;
                    if (nt * 8 + 2 * q4 + r >= rows) continue;
                    const float den = l[nt][r], inv = den == 0.f ? 0.f : 1.f / den;       // no key: zeros
                    __nv_bfloat16* const out = A.out + t * A.o_t + j * A.o_h + member * A.o_g + g8 * 4;
#pragma unroll
                    for (int g = 0; g < G; ++g)
                        *reinterpret_cast<uint2*>(out + g * kQuantGroup) = make_uint2(pack2(o[2 * g][nt][r] * inv, o[2 * g][nt][2 + r] * inv),
                                                                                      pack2(o[2 * g + 1][nt][r] * inv, o[2 * g + 1][nt][2 + r] * inv));
                    if (g8 == 0 && A.lse) A.lse[row_at(A, t, j, member)] = row_lse(m[nt][r], den);
                }
        } else {
            // what goes on behind the run lies where the ring was, as nothing is fetched any more
            const bool begins = first_k == 0;
            Piece<8 * NT>& piece = piece_s[hb][2 * kw + (begins ? 1 : 0)];
            const uint32_t sums = (uint32_t)(warp * Geo::OWN + (begins ? 0 : BUFS * Geo::UNIT));
            if (begins) ptx::cp_async_wait<0>();
            __syncwarp();
            if (lane == 0) {
                piece.there = 1;
                piece.begins = begins;
                piece.ends = end_k == units;
                piece.e = seg.e, piece.h = pair, piece.units = units;
                piece.sums = sums;
            }
            float* const to = reinterpret_cast<float*>(aq_smem + sums);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = nt * 8 + 2 * q4 + r;
                    if (g8 == 0) {
                        piece.m[row] = m[nt][r];
                        piece.l[row] = l[nt][r];
                    }
#pragma unroll
                    for (int g = 0; g < G; ++g)
                        *reinterpret_cast<float4*>(to + row * LDO + g * kQuantGroup + g8 * 4) =
                            make_float4(o[2 * g][nt][r], o[2 * g][nt][2 + r], o[2 * g + 1][nt][r], o[2 * g + 1][nt][2 + r]);
                }
        }
        left -= end_k - first_k;
        seg.k = end_k;
        if (left > 0) settle(seg);
    }
    ptx::cp_async_wait<0>();
    if (pass + 1 == P.passes) chain_next();
    __syncthreads();

    // ---- the CTA's pieces of a pair follow one another, a chain: what goes on behind a run, and what began before the next ones, up to its end.  A chain may
    // also begin before the CTA's first run, or go on behind its last.  The threads of a pair of the HB share out its rows and columns.
    {
        const Piece<8 * NT>* const pieces = piece_s[hb];
        static_assert(2 * KW <= 32, "a lane for each piece");
        const bool there = lane < 2 * KW && pieces[lane].there;
        const uint32_t all = __ballot_sync(0xffffffffu, there), ends = __ballot_sync(0xffffffffu, there && pieces[lane].ends);
        // (if the first one does not begin its pair, an earlier CTA does)
        const uint32_t heads = __ballot_sync(0xffffffffu, there && pieces[lane].begins) | (all & (0u - all));
        const int chains = __popc(heads);
        if (heads >> lane & 1u) head_s[warp][__popc(heads & ((1u << lane) - 1u))] = lane;
        if (lane == 0) head_s[warp][chains] = 2 * KW;
        __syncwarp();
        const long long run = (long long)pass * P.runs + blockIdx.x;
        if (hb == 0 && kw == 0 && lane == 0 && chains > 0) {
            // the last chain may go on: the run that holds its pair's last unit
            const int head = head_s[warp][chains - 1];
            const Piece<8 * NT>& f = pieces[head];
            if (f.begins && (ends >> head) == 0)
                P.run_head[run] = make_int2((n0 + f.e) * A.n_head * A.row_tiles + f.h,
                                            parts_word(run_of(base_s[n], n_runs, base_s[f.e] + (long long)(f.h / HB + 1) * f.units - 1) - (int)blockIdx.x + 1, 1));
        }
        const int most = min(8 * NT, A.group) * (DH / 4);
        for (int item = kw * 32 + lane; item < chains * most; item += KW * 32) {
            const int c = item / most, idx = item - c * most, row = idx / (DH / 4), col = idx % (DH / 4) * 4;
            const int head = head_s[warp][c], next = head_s[warp][c + 1];
            const Piece<8 * NT>& f = pieces[head];
            const int t = n0 + f.e, j = f.h / A.row_tiles, row0 = f.h % A.row_tiles * 16, member = row0 + row;
            if (member >= A.group) continue;
            const uint32_t chain = all & (next == 32 ? ~0u : (1u << next) - 1u) & (~0u << head);
            const bool begins = f.begins, whole = begins && (ends & chain) != 0;
            float* const slot = P.slots + part_slot(run, begins, HB, hb) * 16 * (DH + 2);
            {
                float M = -INFINITY;
#pragma unroll 4
                for (int i = head; i < next; ++i) M = fmaxf(M, chain >> i & 1u ? pieces[i].m[row] : -INFINITY);
                const float z = M == -INFINITY ? 0.f : M;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                float den = 0.f;
#pragma unroll 4
                for (int i = head; i < next; ++i) {
                    if (!(chain >> i & 1u)) continue;
                    const float w = exp2_fast(pieces[i].m[row] - z);      // 0 for a piece that saw no key
                    const float4 v = *reinterpret_cast<const float4*>(aq_smem + pieces[i].sums + row * LDO * 4 + col * 4);
                    sum.x = fmaf(w, v.x, sum.x);
                    sum.y = fmaf(w, v.y, sum.y);
                    sum.z = fmaf(w, v.z, sum.z);
                    sum.w = fmaf(w, v.w, sum.w);
                    den = fmaf(w, pieces[i].l[row], den);
                }
                if (whole) {
                    const float inv = den == 0.f ? 0.f : 1.f / den;
                    *reinterpret_cast<uint2*>(A.out + t * A.o_t + j * A.o_h + member * A.o_g + col) =
                        make_uint2(pack2(sum.x * inv, sum.y * inv), pack2(sum.z * inv, sum.w * inv));
                    if (col == 0 && A.lse) A.lse[row_at(A, t, j, member)] = row_lse(M, den);
                } else {
                    float2* const to = reinterpret_cast<float2*>(slot + row * DH + col);          // (multiples of 8 bytes)
                    to[0] = make_float2(sum.x, sum.y);
                    to[1] = make_float2(sum.z, sum.w);
                    if (col == 0) *reinterpret_cast<float2*>(slot + 16 * DH + row * 2) = make_float2(M, den);
                }
            }
        }
    }
    }
}

template <int DH, int NT>
struct QuantLaunch {
    using Geo = QuantGeo<DH, NT>;
    template <int HB>
    static dsmoe_status heads(const AttnView& A, const QuantView& C, const QuantPlan& P, int ctas, cudaStream_t s) {
        auto* kernel = attention_quant_kernel<DH, NT, HB>;
        static bool attr[kMaxDeviceSlots] = {};
        int dev = 0;
        DeviceState* st = nullptr;
        DSMOE_TRY(device_state(&st, &dev));
        if (!attr[dev]) {
            DSMOE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo::SMEM));
            attr[dev] = true;
        }
        DSMOE_CUDA_TRY(launch_chained(kernel, (unsigned)ctas, 32 * Geo::WARPS, Geo::SMEM, s, A, C, P));
        return DSMOE_OK;
    }
    static dsmoe_status go(const AttnView& A, const QuantView& C, const QuantPlan& P, int hb, int ctas, cudaStream_t s) {
        if constexpr (Geo::WARPS % 4 == 0)
            if (hb == 4) return heads<4>(A, C, P, ctas, s);
        return hb == 2 ? heads<2>(A, C, P, ctas, s) : heads<1>(A, C, P, ctas, s);
    }
};

int quant_warps_of(const AttnView& A) { return quant_warps(A.d_head, A.group <= 8 ? 1 : 2); }

// Keys that a token sees at most
long long quant_seen(const AttnView& A) { return A.window < A.L ? std::min((long long)A.window + A.sinks, (long long)A.L) : A.L; }

constexpr int kWholeUnits = 6;            // of a warp, at most, where a CTA takes all of a pair's keys

// CTAs: one an SM, as far as each has a unit per warp in the longest case
int quant_ctas(const AttnView& A) {
    const long long units = ((quant_seen(A) + kQuantUnit - 1) / kQuantUnit + 1) * A.T * A.n_head * A.row_tiles, warps = quant_warps_of(A);
    return (int)std::min((units + warps - 1) / warps, (long long)std::min(sm_count(), kMostStreamCtas));
}

constexpr int kMostHeadsAtOnce = 4;

}  // namespace

// Whether a CTA takes all of a pair's keys, `seen` at most, so that no part is left to add up: where the CTAs that stay idle would save less than the second launch
// costs, as long as one pair of all keys beside others of few holds up the call by no more than that launch.  One launch and two, us, with 4 x 5 heads of 128:
//   one token    512 keys 10.1, 12.6; 1024 12.4, 13.1; 1536 14.6, 13.1; 2048 17.2, 13.1 (two from 1185 on)
//   32 tokens    512 keys 10.8, 16.1; 1024 13.1, 18.7; 2048 18.6, 22.3; 4096 28.0, 31.8; 8192 46.2, 47.3
//   the same, but a tenth of the keys to all of them: 512 11.2, 14.0; 1024 13.2, 17.1; 2048 18.4, 18.8; 4096 26.9, 24.5; 8192 44.3, 34.0
//   the same, by position: 1024 13.5, 18.0; 2048 18.7, 20.6; 4096 27.5, 25.9; 8192 45.1, 36.7 (neighbouring heads are read side by side in runs alone)
//   37 tokens, one of 131072 keys and the others of 200: 560, 42.4
// 4 x 16 heads of 96, 32 tokens, a tenth to all: 1024 keys 15.1, 24.4; 2048 21.2, 27.4; 4096 33.3, 33.6; 8192 58.6, 46.1.
bool quant_whole(long long pairs, long long seen, int warps, int sms) {
    return pairs <= sms && seen <= (long long)kWholeUnits * kQuantUnit * warps && seen * (sms - pairs) <= 3ll * kQuantUnit * warps * sms;
}
bool quant_whole(const AttnView& A) {
    return quant_whole((long long)A.T * A.n_head * A.row_tiles, quant_seen(A), quant_warps_of(A), std::min(sm_count(), kMostStreamCtas));
}

// The runs are numbered as attention_sum_kernel takes those of single warps, of which stream_warps are a CTA's there
void quant_plan_size(const AttnView& A, QuantPlan* plan, size_t* slots, size_t* run_head) {
    plan->passes = ceil_div(A.T, kListTokens);
    plan->runs = (int)align_up(std::min((long long)A.T * A.n_head * A.row_tiles + quant_ctas(A), (long long)std::min(sm_count(), kMostStreamCtas)), 8);
    *run_head = (size_t)plan->passes * plan->runs * sizeof(int2);
    *slots = 2 * (size_t)plan->passes * plan->runs * kMostHeadsAtOnce * part_bytes(A.d_head);
}

dsmoe_status launch_quant_attention(const AttnView& A, const QuantView& C, const QuantPlan& plan, cudaStream_t s) {
    QuantPlan P = plan;
    const long long pairs = (long long)A.T * A.n_head * A.row_tiles;
    const int warps = quant_warps_of(A), each = A.n_head * A.row_tiles;
    P.whole = quant_whole(A);
    const bool side_by_side = A.row_tiles > 1 || (A.n_head > 1 && C.c_h < C.c_p);
    const int hb = P.whole || !side_by_side ? 1 : each % 4 == 0 && warps % 4 == 0 ? 4 : each % 2 == 0 ? 2 : 1;
    const int ctas = P.whole ? (int)pairs : quant_ctas(A);
#define DSMOE_CALL(DH) (A.group <= 8 ? QuantLaunch<DH, 1>::go(A, C, P, hb, ctas, s) : QuantLaunch<DH, 2>::go(A, C, P, hb, ctas, s))
    switch (A.d_head) {
        case 32: DSMOE_TRY(DSMOE_CALL(32)); break;
        case 64: DSMOE_TRY(DSMOE_CALL(64)); break;
        case 96: DSMOE_TRY(DSMOE_CALL(96)); break;
        case 128: DSMOE_TRY(DSMOE_CALL(128)); break;
        case 160: DSMOE_TRY(DSMOE_CALL(160)); break;
        case 192: DSMOE_TRY(DSMOE_CALL(192)); break;
        case 224: DSMOE_TRY(DSMOE_CALL(224)); break;
        case 256: DSMOE_TRY(DSMOE_CALL(256)); break;
        default: return DSMOE_ERR_UNSUPPORTED;
    }
#undef DSMOE_CALL
    if (P.whole) return DSMOE_OK;
    StreamPlan sum{};
    sum.passes = P.passes;
    sum.ctas = P.runs * hb / stream_warps(A.d_head);
    sum.by_warp = true;
    sum.heads_at_once = hb;
    sum.slots = P.slots;
    sum.run_head = P.run_head;
    return launch_attention_sum(A, sum, RowParts{}, s);
}

}  // namespace dsmoe
