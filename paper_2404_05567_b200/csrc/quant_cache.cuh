// A key/value cache in 4 bits (dsmoe_quant_cache_write, dsmoe_quant_cache_read, dsmoe_quant_attention): the format, and what the kernels and their
// launchers share.
//
// A row (sequence, head, position) of d_head values is G = d_head / 32 groups of 32 neighbours, each with a scale s; value x is s * c, c an integer of
// -7 .. 7 that is held as c + 8.  The 32-bit word t * G + g of a row (t < 4) holds values 32 g + 8 t .. 32 g + 8 t + 7, the first in the lowest bits:
//   a quarter t of a warp's four lanes of a key then reads G neighbouring words and has eight values of each group, so that a step of the MMAs'
//   reduction stays within a group, whose scale multiplies its sum;
//   (w >> 4 i) & 0x000f000f are values i and i + 4 of a word, or, of two keys' halves of words side by side, value i of both keys.
// Scales have four significant bits: with the codes' four at most, s * c has eight, those of a bf16, so that reading back is exact, whatever reads.
#pragma once

#include "cache_attention.cuh"

namespace dsmoe {

constexpr int kQuantGroup = 32;
// Places for scales in a row: as many as one load takes
__host__ __device__ static constexpr int quant_scales(int d_head) { return d_head <= 64 ? 2 : d_head <= 128 ? 4 : 8; }

// a / b of numbers that are not negative, which nearly always are small
__device__ __forceinline__ long long divide(long long a, long long b) { return (a | b) >> 32 == 0 ? (uint32_t)a / (uint32_t)b : a / b; }

struct QuantView {
    int n_seq, n_head, L, d_head;
    unsigned char *K, *V;                 // codes
    __nv_bfloat16 *K_scale, *V_scale;
    long long c_s, c_h, c_p;              // bytes between sequences, heads, positions
    long long s_s, s_h, s_p;              // elements between those of the scales
};

struct QuantWrite {
    int T, sinks, ring;                   // ring: as in AttnView
    const __nv_bfloat16 *k, *v;
    long long i_t, i_h;
    const int32_t *tok_seq, *pos;
    __nv_bfloat16 *k_back, *v_back;       // nullable, one by one
    long long b_t, b_h;
    int32_t* dev_status;
};
dsmoe_status launch_quant_write(const QuantView& C, const QuantWrite& W, cudaStream_t s);

struct QuantRead {
    int first, rows;                      // slots first .. first + rows - 1
    const int32_t* len;                   // nullable: slots below len[sequence] alone
    const int4* range;                    // nullable (first 0, no len): of each sequence, slots below .x and those from .y to .z - 1 alone
    __nv_bfloat16 *K, *V;
    long long o_s, o_h, o_p;
};
dsmoe_status launch_quant_read(const QuantView& C, const QuantRead& R, cudaStream_t s);

// range[s]: the slots that the tokens of sequence s see (QuantRead)
dsmoe_status launch_quant_range(const AttnView& A, int4* range, cudaStream_t s);

// Attention of all tokens (A.K, A.V and kv_ unused)
struct QuantPlan {
    int runs, passes;                     // places for runs of each pass, a multiple of 8
    bool whole;                           // each CTA's run is a pair's units: no parts
    float* slots;                         // [passes][runs][2][up to 4 pairs][16][d_head + 2]
    int2* run_head;                       // [passes][runs]
};
// The most runs that any window needs (A has none), and the bytes of `slots` and `run_head`
void quant_plan_size(const AttnView& A, QuantPlan* plan, size_t* slots, size_t* run_head);
// Whether it takes one launch, a CTA for each of the pairs (token, head, 16 rows) that see `seen` keys at most, with so many warps a CTA, on so many SMs
bool quant_whole(long long pairs, long long seen, int warps, int sms);
bool quant_whole(const AttnView& A);
dsmoe_status launch_quant_attention(const AttnView& A, const QuantView& C, const QuantPlan& plan, cudaStream_t s);

}  // namespace dsmoe
