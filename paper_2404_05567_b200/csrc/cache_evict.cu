// Eviction from a key/value cache by accumulated attention weight (dsmoe_cache_evict).
//
// Of the n keys of a (sequence, head) that holds more than `keep`, the first `sinks`, the last `recent` and those of the others with the
// largest tally stay, in their order.  A CTA per (sequence, head) finds the smallest tally that stays, and how many of the candidates with exactly
// that tally do (the first ones); a pass in order of the keys writes the indices and the tallies that stay.  evict_move_kernel closes up the rows.
//
// The bound is found by the bits of numbers in the tallies' order, eight at a time: a histogram of the candidates that share the bits found so
// far, then the bin in which the wanted rank falls, until all of a bin stay.  evict_select_kernel (up to 32768 positions) reads the tallies once
// and has them in registers; evict_select_long_kernel reads them again for every eight bits.
// 14 caches of 5001 positions, us: a bit at a time by counting what reaches it, without a histogram, 18; two bits 20; so 14.
#include "cache_attention.cuh"

namespace dsmoe {

namespace {

constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32, kMoveThreads = 256;
// 16-byte pieces that a thread of evict_move_kernel has under way, and CTAs of an SM: 128 caches of 16384 positions, 2000 of which stay, us: 1 and 8
// 94, 2 and 8 76, 3 and 8 71, 4 and 8 70, 4 and 6 75, 8 and 4 78, 16 and 2 105.  In place a CTA has a whole cache to move, and more under way:
// 4 caches of 32768, half of which stays, 618 us, into other caches 49; 128 of 16384, an eighth of which stays, 116 and 69.
__host__ __device__ constexpr int move_pieces(bool in_place) { return in_place ? 8 : 4; }

// Tallies in the order of unsigned numbers: -0 and 0 are alike, what is no number comes before all others
__device__ __forceinline__ uint32_t rank_bits(float v) {
    if (v != v) return 0u;
    const uint32_t u = __float_as_uint(v + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Keys of sequence s, clamped into the cache
__device__ __forceinline__ int length_of(const EvictView& E, int s) {
    const int n = E.len[s];
    if ((n < 0 || n > E.L) && threadIdx.x == 0) report_status(E.dev_status, DSMOE_ERR_INVALID_ARG);
    return min(max(n, 0), E.L);
}

// a[0 .. n - 1] (n up to 1024): each becomes the sum of those before it; returns the sum of all
__device__ __forceinline__ int scan_counts(int* a, int n, int* warp_s) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __syncthreads();
    const int x = tid < n ? a[tid] : 0;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == 31) warp_s[warp] = incl;
    __syncthreads();
    const int w = warp_s[lane];
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0), all = __reduce_add_sync(0xffffffffu, w);
    if (tid < n) a[tid] = before + incl - x;
    __syncthreads();
    return all;
}

// PER: tallies of a thread, tid, tid + 1024 ..
template <int PER>
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ EvictView E) {
    __shared__ int counts_s[PER * kSelWarps], scan_s[kSelWarps];
    __shared__ __align__(16) int hist_s[4][256];         // of the bits from the top, eight at a time; the largest first
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    hist_s[tid >> 8][tid & 255] = 0;
    chain_wait();
    const long long pair = blockIdx.x;
    const int n = length_of(E, (int)(pair / E.n_head));
    const float* const tally = E.tally + pair * E.L;
    const bool all = n <= E.keep;
    const int a = E.sinks, b = n - E.recent;            // candidates: a .. b - 1 (where not all stay)
    const int want = E.keep - E.sinks - E.recent;       // of the candidates
    uint32_t bound = 0u;
    int ties = 0;                                       // candidates with exactly the bound that stay
    uint32_t stays = 0u;                                // bit i: tally tid + 1024 i
    __syncthreads();
    if (all) {
#pragma unroll
        for (int i = 0; i < PER; ++i) stays |= (uint32_t)(i * kSelThreads + tid < n) << i;
    } else {
        uint32_t u[PER];                                // 0: no candidate (or a tally that is no number)
        {
            // (every thread asks for PER numbers at once, for the first one where it has no candidate: behind branches they came one by one, 14 of
            // the 35 thousand cycles with 16)
            float v[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int k = i * kSelThreads + tid;
                v[i] = tally[k >= a && k < b ? k : 0];
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int k = i * kSelThreads + tid;
                u[i] = k >= a && k < b ? rank_bits(v[i]) : 0u;
            }
        }
        bool tied = true;                               // more have exactly the bound than stay
        if (want > 0) {
            int left = want;                            // to find among those that share the bits found so far
#pragma unroll 1
            for (int pass = 0; pass < 4 && tied; ++pass) {
                const int shift = 24 - 8 * pass;
                int* const hist = hist_s[pass];
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int k = i * kSelThreads + tid;
                    if (k >= a && k < b && (pass == 0 || (u[i] ^ bound) >> (shift + 8) == 0u)) atomicAdd(hist + (255u - ((u[i] >> shift) & 255u)), 1);
                }
                __syncthreads();
                // the bin in which the left-th largest lies: a lane looks at eight, every warp for itself
                const int4 x = *reinterpret_cast<const int4*>(hist + 8 * lane), y = *reinterpret_cast<const int4*>(hist + 8 * lane + 4);
                const int mine[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                int incl = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) incl += mine[i];
                const int sum = incl;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += up;
                }
                const int holder = __ffs(__ballot_sync(0xffffffffu, incl >= left)) - 1;
                int before = incl - sum, bin = 0, rest = 0, count = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (before < left && left <= before + mine[i]) {
                        bin = 255 - 8 * lane - i;
                        rest = left - before;
                        count = mine[i];
                    }
                    before += mine[i];
                }
                bound |= (uint32_t)__shfl_sync(0xffffffffu, bin, holder) << shift;
                left = __shfl_sync(0xffffffffu, rest, holder);
                tied = __shfl_sync(0xffffffffu, count, holder) != left;       // otherwise all that share these bits stay
            }
            ties = left;
        } else {
            bound = 0xffffffffu;
        }
        uint32_t tie = 0u;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = i * kSelThreads + tid;
            const bool middle = k >= a && k < b;
            const bool is_tie = middle && tied && u[i] == bound;
            tie |= (uint32_t)is_tie << i;
            stays |= (uint32_t)(k < n && (!middle || (tied ? u[i] > bound : u[i] >= bound))) << i;
        }
        if (tied && ties > 0) {                         // (the same for the whole CTA) the first of them
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t votes = __ballot_sync(0xffffffffu, (tie >> i) & 1u);
                if (lane == 0) counts_s[i * kSelWarps + warp] = __popc(votes);
            }
            scan_counts(counts_s, PER * kSelWarps, scan_s);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t votes = __ballot_sync(0xffffffffu, (tie >> i) & 1u);
                const int rank = counts_s[i * kSelWarps + warp] + __popc(votes & ((1u << lane) - 1u));
                if (((tie >> i) & 1u) && rank < ties) stays |= 1u << i;
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t votes = __ballot_sync(0xffffffffu, (stays >> i) & 1u);
        if (lane == 0) counts_s[i * kSelWarps + warp] = __popc(votes);
    }
    const int n_kept = scan_counts(counts_s, PER * kSelWarps, scan_s);
    chain_next();
    int32_t* const kept = E.kept + pair * E.keep;
    float* const to = E.tally_out + pair * E.tally_pitch;
    const bool in_place = E.tally_out == E.tally;
    constexpr int BATCH = PER < 8 ? PER : 8;
#pragma unroll
    for (int i0 = 0; i0 < PER; i0 += BATCH) {
        float v[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) v[i] = tally[(stays >> (i0 + i)) & 1u ? (i0 + i) * kSelThreads + tid : 0];
        // (in place a tally moves to where one of this batch or an earlier one was: all of it is read)
        if (in_place) __syncthreads();
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const bool stay = (stays >> (i0 + i)) & 1u;
            const uint32_t votes = __ballot_sync(0xffffffffu, stay);
            if (stay) {
                const int at = counts_s[(i0 + i) * kSelWarps + warp] + __popc(votes & ((1u << lane) - 1u));
                kept[at] = (i0 + i) * kSelThreads + tid;
                to[at] = v[i];
            }
        }
    }
    for (int i = n_kept + tid; i < E.keep; i += kSelThreads) kept[i] = -1;
    if (tid == 0) E.count[pair] = n_kept;
}

__global__ void __launch_bounds__(kSelThreads) evict_select_long_kernel(const __grid_constant__ EvictView E) {
    __shared__ int hist[256];
    __shared__ uint32_t prefix_s;
    __shared__ int want_s;
    __shared__ int ties_s[kSelThreads / 32], kept_s[kSelThreads / 32];
    chain_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long pair = blockIdx.x;
    const int s = (int)(pair / E.n_head);
    const int n = length_of(E, s);
    const float* const tally = E.tally + pair * E.L;
    const bool all = n <= E.keep;
    const int a = E.sinks, b = n - E.recent;            // candidates: a .. b - 1 (where not all stay)
    if (tid == 0) {
        prefix_s = 0u;
        want_s = E.keep - E.sinks - E.recent;           // of the candidates
    }
    if (!all) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            const uint32_t prefix = prefix_s;
            for (int i = a + tid; i < b; i += kSelThreads) {
                const uint32_t u = rank_bits(tally[i]);
                if (shift == 24 || (u >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(u >> shift) & 255u], 1);
            }
            __syncthreads();
            if (warp == 0) {                            // the bin in which the want-th largest lies: lane l looks at bins 255 - 8 l and below
                int mine[8], sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    mine[i] = hist[255 - 8 * lane - i];
                    sum += mine[i];
                }
                int incl = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += up;
                }
                int before = incl - sum;
                const int want = want_s;
                __syncwarp();
                if (before < want && want <= incl) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (before < want && want <= before + mine[i]) {
                            prefix_s = prefix | ((uint32_t)(255 - 8 * lane - i) << shift);
                            want_s = want - before;     // ... among those with these bits
                        }
                        before += mine[i];
                    }
                }
            }
            __syncthreads();
        }
    } else {
        __syncthreads();
    }
    // with nothing wanted of the candidates no bin was found: none is above the bound, and no tie stays
    const bool none = !all && E.keep == E.sinks + E.recent;
    const uint32_t bound = none ? 0xffffffffu : prefix_s;
    const int ties = none ? 0 : want_s;
    int32_t* const kept = E.kept + pair * E.keep;
    float* const to = E.tally_out + pair * E.tally_pitch;
    int n_ties = 0, n_kept = 0;
    // four neighbours a thread: a call on 32 caches of 131072 positions 141 us, with one 422
    constexpr int NEXT = 4;
    // x of this thread's and what the threads before it have, on top of *so_far, which grows by all of it
    const auto place = [&](int x, int* warps, int* so_far) {
        int incl = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) warps[warp] = incl;
        __syncthreads();
        const int w = warps[lane];
        const int at = *so_far + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + incl - x;
        *so_far += __reduce_add_sync(0xffffffffu, w);
        return at;
    };
    for (int i0 = 0; i0 < n; i0 += NEXT * kSelThreads) {
        const int first = i0 + NEXT * tid;
        float v[NEXT];
#pragma unroll
        for (int k = 0; k < NEXT; ++k) v[k] = tally[first + k < n ? first + k : 0];
        uint32_t ties_here = 0u, stays = 0u;
#pragma unroll
        for (int k = 0; k < NEXT; ++k) {
            const int i = first + k;
            const uint32_t u = rank_bits(v[k]);
            const bool middle = !all && i >= a && i < b;
            ties_here |= (uint32_t)(i < n && middle && u == bound) << k;
            stays |= (uint32_t)(i < n && (!middle || u > bound)) << k;
        }
        int rank = place(__popc(ties_here), ties_s, &n_ties);
#pragma unroll
        for (int k = 0; k < NEXT; ++k)
            if ((ties_here >> k) & 1u) stays |= (uint32_t)(rank++ < ties) << k;
        int at = place(__popc(stays), kept_s, &n_kept);        // (its wait: every thread has read its tallies, so they may be written over)
#pragma unroll
        for (int k = 0; k < NEXT; ++k)
            if ((stays >> k) & 1u) {
                kept[at] = first + k;
                to[at++] = v[k];
            }
    }
    for (int i = n_kept + tid; i < E.keep; i += kSelThreads) kept[i] = -1;
    if (tid == 0) E.count[pair] = n_kept;
    chain_next();
}

// A CTA per (sequence, head), keys or values, and stretch of rows.  A row moves towards the front of its cache, to a place that no later row comes
// from: where source and destination are one buffer, one CTA takes all rows in order, and a batch is read before any of it is written.
// Otherwise a CTA takes one batch.
template <bool IN_PLACE>
__global__ void __launch_bounds__(kMoveThreads, IN_PLACE ? 4 : 8) evict_move_kernel(const __grid_constant__ EvictView E, const int stretches) {
    constexpr int PIECES = move_pieces(IN_PLACE);
    chain_wait();
    chain_next();
    const unsigned tid = threadIdx.x, CH = (unsigned)E.d_head / 8;
    const int stretch = (int)(blockIdx.x % stretches), which = (int)(blockIdx.x / stretches) & 1;
    const long long pair = blockIdx.x / stretches / 2;
    const int s = (int)(pair / E.n_head), j = (int)(pair % E.n_head);
    const int count = E.count[pair];
    if (j == 0 && which == 0 && stretch == 0 && tid == 0) E.len_out[s] = count;
    const __nv_bfloat16* const from = (which ? E.V : E.K) + s * E.kv_s + j * E.kv_h;
    __nv_bfloat16* const to = (which ? E.V_out : E.K_out) + s * E.o_s + j * E.o_h;
    const int32_t* const kept = E.kept + pair * E.keep;
    constexpr unsigned BATCH = PIECES * kMoveThreads;
    const unsigned per = IN_PLACE ? (unsigned)count : BATCH / CH, r0 = stretch * per;
    if (r0 >= (unsigned)count) return;
    const unsigned long long pieces = (unsigned long long)(min((unsigned)count, r0 + per) - r0) * CH;
    for (unsigned long long p0 = 0; p0 < pieces; p0 += BATCH) {
        uint4 v[PIECES];
        const unsigned n = (unsigned)min((unsigned long long)BATCH, pieces - p0), row0 = (unsigned)(p0 / CH), ch0 = (unsigned)(p0 % CH);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const unsigned p = i * kMoveThreads + tid, at = ch0 + p;
            if (p < n) v[i] = *reinterpret_cast<const uint4*>(from + kept[r0 + row0 + at / CH] * E.kv_p + at % CH * 8);
        }
        if (IN_PLACE) __syncthreads();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const unsigned p = i * kMoveThreads + tid, at = ch0 + p;
            if (p < n) *reinterpret_cast<uint4*>(to + (r0 + row0 + at / CH) * E.o_p + at % CH * 8) = v[i];
        }
    }
}

template <int PER>
cudaError_t launch_select(const EvictView& E, unsigned pairs, cudaStream_t s) {
    return launch_chained(evict_select_kernel<PER>, pairs, kSelThreads, 0, s, E);
}

}  // namespace

dsmoe_status launch_evict(const EvictView& E, cudaStream_t s) {
    const long long pairs = (long long)E.n_seq * E.n_head;
    const int rows = move_pieces(false) * kMoveThreads / (E.d_head / 8), stretches = E.in_place ? 1 : ceil_div(E.keep, rows);
    if (pairs * 2 * stretches > 0x7fffffffll) return DSMOE_ERR_UNSUPPORTED;
    const unsigned n = (unsigned)pairs;
    if (E.L <= 2 * kSelThreads) DSMOE_CUDA_TRY(launch_select<2>(E, n, s));
    else if (E.L <= 8 * kSelThreads) DSMOE_CUDA_TRY(launch_select<8>(E, n, s));
    else if (E.L <= 16 * kSelThreads) DSMOE_CUDA_TRY(launch_select<16>(E, n, s));
    else if (E.L <= 32 * kSelThreads) DSMOE_CUDA_TRY(launch_select<32>(E, n, s));
    else DSMOE_CUDA_TRY(launch_chained(evict_select_long_kernel, n, kSelThreads, 0, s, E));
    DSMOE_CUDA_TRY(launch_chained(E.in_place ? evict_move_kernel<true> : evict_move_kernel<false>, (unsigned)(pairs * 2 * stretches), kMoveThreads,
                                  0, s, E, stretches));
    return DSMOE_OK;
}

}  // namespace dsmoe
