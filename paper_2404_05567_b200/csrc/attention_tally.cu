// The weights that the keys of a cache get from the tokens of a call, added up per key (dsmoe_tally_attention's second half):
//
//     tally_out[s][j][l] = tally_in[s][j][l] + sum over tokens t of sequence s with pos[t] >= l, members g, of 2^(logit(t,j,g,l) - m) / sum
//
// with m and the sum of every row from the attention itself.  Either the attention has left its logits (decoding): tally_add_kernel reads them,
// a thread per four keys.  Or they are computed again (attention_tally_kernel): a CTA owns 64 keys of a (sequence, head) and walks the rows that see them, in
// order of the tokens, so that every sum is taken in one order and nothing is added in memory.  The logits are computed again, keys as the
// rows and queries as the columns of the MMA tile: a thread keeps two keys' sums in registers.
#include <climits>

#include "cache_attention.cuh"
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

dsmoe_status launch_tally(const AttnView& A, const float* tally_in, float* tally_out, cudaStream_t s) {
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
