// Eviction from a key/value cache by accumulated attention weight (dsmoe_cache_evict).
//
// Of the n keys of a (sequence, head) that holds more than `keep`, the first `sinks`, the last `recent` and those of the others with the
// largest tally stay, in their order.  evict_select_kernel finds the smallest tally that stays by its bits, eight at a time (a histogram
// of the candidates that share the bits found so far, then the bin in which the wanted rank falls), and how many of the candidates with exactly
// that tally stay (the first ones); a last pass in order of the keys writes the indices and the tallies that stay.  evict_move_kernel
// closes up the rows.
#include "cache_attention.cuh"

namespace dsmoe {

namespace {

constexpr int kSelThreads = 1024, kMoveThreads = 256, kMoveRows = 64;

// Tallies in the order of unsigned numbers: -0 and 0 are alike, what is no number comes before all others
__device__ __forceinline__ uint32_t rank_bits(float v) {
    if (v != v) return 0u;
    const uint32_t u = __float_as_uint(v + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ EvictView E) {
    __shared__ int hist[256];
    __shared__ uint32_t prefix_s;
    __shared__ int want_s;
    __shared__ int ties_s[kSelThreads / 32], kept_s[kSelThreads / 32];
    chain_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long pair = blockIdx.x;
    const int s = (int)(pair / E.n_head);
    int n = E.len[s];
    if (n < 0 || n > E.L) {
        if (tid == 0) report_status(E.dev_status, DSMOE_ERR_INVALID_ARG);
        n = min(max(n, 0), E.L);
    }
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
    for (int i0 = 0; i0 < n; i0 += kSelThreads) {
        const int i = i0 + tid;
        const float v = i < n ? tally[i] : 0.f;
        const uint32_t u = rank_bits(v);
        const bool middle = !all && i >= a && i < b, tie = i < n && middle && u == bound;
        const uint32_t tie_votes = __ballot_sync(0xffffffffu, tie);
        if (lane == 0) ties_s[warp] = __popc(tie_votes);
        __syncthreads();
        int rank = n_ties + __popc(tie_votes & ((1u << lane) - 1u));
        for (int w = 0; w < kSelThreads / 32; ++w) {
            const int c = ties_s[w];
            if (w < warp) rank += c;
            n_ties += c;
        }
        const bool stays = i < n && (!middle || u > bound || (tie && rank < ties));
        const uint32_t votes = __ballot_sync(0xffffffffu, stays);
        if (lane == 0) kept_s[warp] = __popc(votes);
        __syncthreads();                                // (and every thread has read its tally: it may be written over now)
        int at = n_kept + __popc(votes & ((1u << lane) - 1u));
        for (int w = 0; w < kSelThreads / 32; ++w) {
            const int c = kept_s[w];
            if (w < warp) at += c;
            n_kept += c;
        }
        if (stays) {
            kept[at] = i;
            to[at] = v;
        }
    }
    for (int i = n_kept + tid; i < E.keep; i += kSelThreads) kept[i] = -1;
    if (tid == 0) E.count[pair] = n_kept;
    chain_next();
}

// A CTA per (sequence, head), keys or values, and stretch of rows.  A row moves towards the front of its cache, to a place that no later row comes
// from: where source and destination are one buffer, one CTA takes all rows in order, and a batch is read before any of it is written.
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictView E, const int stretches) {
    chain_wait();
    chain_next();
    const int tid = threadIdx.x, CH = E.d_head / 8;
    const int stretch = (int)(blockIdx.x % stretches), which = (int)(blockIdx.x / stretches) & 1;
    const long long pair = blockIdx.x / stretches / 2;
    const int s = (int)(pair / E.n_head), j = (int)(pair % E.n_head);
    const int count = E.count[pair];
    if (j == 0 && which == 0 && stretch == 0 && tid == 0) E.len_out[s] = count;
    const __nv_bfloat16* const from = (which ? E.V : E.K) + s * E.kv_s + j * E.kv_h;
    __nv_bfloat16* const to = (which ? E.V_out : E.K_out) + s * E.o_s + j * E.o_h;
    const int32_t* const kept = E.kept + pair * E.keep;
    const int per = (count + stretches - 1) / stretches, r0 = stretch * per, r1 = min(count, r0 + per);
    constexpr int PER = 8;
    const long long pieces = (long long)(r1 - r0) * CH;
    for (long long p0 = 0; p0 < pieces; p0 += PER * kMoveThreads) {
        uint4 v[PER];
        int row[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long long p = p0 + i * kMoveThreads + tid;
            row[i] = -1;
            if (p < pieces) {
                row[i] = r0 + (int)(p / CH);
                v[i] = *reinterpret_cast<const uint4*>(from + kept[row[i]] * E.kv_p + (p % CH) * 8);
            }
        }
        if (E.in_place) __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long long p = p0 + i * kMoveThreads + tid;
            if (row[i] >= 0) *reinterpret_cast<uint4*>(to + row[i] * E.o_p + (p % CH) * 8) = v[i];
        }
    }
}

}  // namespace

dsmoe_status launch_evict(const EvictView& E, cudaStream_t s) {
    const long long pairs = (long long)E.n_seq * E.n_head;
    int stretches = 1;
    if (!E.in_place) {
        const long long wanted = 4ll * sm_count() / (2 * pairs) + 1, most = (E.keep + kMoveRows - 1) / kMoveRows;
        stretches = (int)(wanted < most ? wanted : most);
    }
    if (pairs * 2 * stretches > 0x7fffffffll) return DSMOE_ERR_UNSUPPORTED;
    DSMOE_CUDA_TRY(launch_chained(evict_select_kernel, (unsigned)pairs, kSelThreads, 0, s, E));
    DSMOE_CUDA_TRY(launch_chained(evict_move_kernel, (unsigned)(pairs * 2 * stretches), kMoveThreads, 0, s, E, stretches));
    return DSMOE_OK;
}

}  // namespace dsmoe
