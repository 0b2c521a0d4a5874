// Attention over a key/value cache as a step of its own (dsmoe_window_attention, dsmoe_prefix_attention, dsmoe_tally_attention): what the
// kernels and their launchers share.
//
// Token t, key/value head j, member g (one of the `group` query heads of that key/value head) is a row.  Position l of the cache is visible to
// token t at position p = pos[t] iff 0 <= l <= p and (p - l < window or l < sinks).  A row's result over any part of its keys is a triple:
// the largest logit m, the sum l of 2^(logit - m), and the sum o of 2^(logit - m) V (logits in base 2: scale * log2 e * <q, k>).  Triples of
// disjoint parts add up after scaling to the larger m, which is how work is split over CTAs, caches and kernels.
#pragma once

#include "common.cuh"

namespace dsmoe {

struct AttnView {
    int T, n_head, group;
    // Tokens that see the same keys (a shared prefix) can be taken as one: row r of head j is then member r % group of token r / group, and T is 1
    int fold;                             // tokens taken as one (1: none)
    int row_tiles;                        // 16-row tiles of the fold * group rows of a (token, head)
    int d_head, n_seq, L;
    int window, sinks, ring;              // ring: slots of the rolling part, 0 if position l lies in slot l
    float scale_log2;
    const __nv_bfloat16* q;
    long long q_t, q_h, q_g;
    const __nv_bfloat16 *K, *V;
    long long kv_s, kv_h, kv_p;
    const int32_t *tok_seq, *pos;         // pos nullptr: every token sees all L keys of sequence 0
    __nv_bfloat16* out;
    long long o_t, o_h, o_g;
    float* lse;                           // nullable
    float2* ml;                           // nullable: (largest logit, 1 / sum) of every row, [T][n_head][group]
    int32_t* dev_status;
    // The stream kernel beside the 128-row kernel: it attends the tokens that the latter leaves alone.  The call has all_T tokens, of which these
    // begin at token0 (all_T 0: it attends all tokens).
    int token0, all_T;
};

constexpr int kUnit = 16;                 // keys that a warp takes at a time
constexpr int kListTokens = 1024;         // tokens whose keys one launch cuts into runs

// The keys that a token sees: 0 .. sinks - 1 and first .. last (nothing: last < first and sinks == 0).
struct Sight {
    int seq, sinks, first, last;
    __host__ __device__ int sink_units() const { return (sinks + kUnit - 1) / kUnit; }
    // a token that sees nothing has one unit without keys, so that somebody writes its row
    __host__ __device__ int units() const {
        const int n = sink_units() + (last >= first ? (last - first) / kUnit + 1 : 0);
        return n > 0 ? n : 1;
    }
};

// A token's sequence and position, clamped into the cache; *bad: they were not in it
__device__ __forceinline__ Sight sight_of(const AttnView& A, int t, bool* bad) {
    int sq = A.tok_seq ? A.tok_seq[t] : 0, p = A.pos ? A.pos[t] : A.L - 1;
    if (sq < 0 || sq >= A.n_seq || p < -1 || (!A.ring && p >= A.L)) {
        *bad = true;
        sq = min(max(sq, 0), A.n_seq - 1);
        p = max(p, -1);
        if (!A.ring) p = min(p, A.L - 1);
    }
    Sight s;
    s.seq = sq;
    s.last = p;
    s.first = p >= A.window ? p - A.window + 1 : 0;
    s.sinks = min(A.sinks, p + 1);
    if (s.first <= s.sinks) {             // one stretch
        s.first = 0;
        s.sinks = 0;
    }
    return s;
}
// The 128-row kernel's blocks of tokens: two tiles of as many tokens as have their rows in 128.  Tokens of one sequence that follow one another
// there are a run; runs that fill less than a quarter of a tile, unless the block is one, are left to the stream kernel.
__host__ __device__ static inline int tile_span(int group) { return 2 * (128 / group); }
__host__ __device__ static inline int tile_least_run(int group) { return (32 + group - 1) / group; }
__host__ __device__ static inline int tile_blocks(int T, int group) { return (T + tile_span(group) - 1) / tile_span(group); }
__device__ __forceinline__ int seq_of_token(const AttnView& A, int t) { return A.tok_seq ? min(max(A.tok_seq[t], 0), A.n_seq - 1) : 0; }
// Whether the stream kernel attends token t (numbered from A.token0)
__device__ __forceinline__ bool is_streams(const AttnView& A, int t) {
    if (A.all_T == 0) return true;
    const int span = tile_span(A.group), least = tile_least_run(A.group), at = A.token0 + t;
    const int b0 = at / span * span, b1 = min(A.all_T, b0 + span), seq = seq_of_token(A, t);
    int lo = at, hi = at + 1;
    while (lo > b0 && hi - lo < least && seq_of_token(A, lo - 1 - A.token0) == seq) --lo;
    while (hi < b1 && hi - lo < least && seq_of_token(A, hi - A.token0) == seq) ++hi;
    return hi - lo < least && (lo > b0 || hi < b1);
}
// The slot of the cache that holds position l
__device__ __forceinline__ int slot_of(const AttnView& A, int l) { return !A.ring || l < A.sinks ? l : A.sinks + (l - A.sinks) % A.ring; }

// Where the parts of a launch lie in the workspace.  Rows of 16 to a (token, head, row tile) = pair.
struct PartPlan {
    float* slots;                         // [2 * ctas (+ pairs, keep_parts)][16][d_head + 2]
    int2* head;                           // [pairs]: first slot, number of parts; 0 parts: the row is written
    int ctas;                             // CTAs that the slots have room for
    bool keep_parts;                      // whole pairs leave a part too (something else is still to be added)
};
static inline size_t part_bytes(int d_head) { return (size_t)16 * (d_head + 2) * 4; }

// Parts of whole rows from the 128-row kernel: n of them, [n][rows][d_head] and [n][rows][2], a row for each token, head and member
struct TileParts {
    int n;
    size_t rows;
    const float* o;
    const float* ml;
};

// The 128-row kernel: heads of 64, 96 and 128, caches that a tensor map describes.  Its rows' keys are cut into `splits`; o, ml: where their parts
// go (TileParts), or nullptr with one split: out and lse are written.
struct TilePlan {
    int splits;
    float *o, *ml;
};
bool tile_supported(const AttnView& A);
dsmoe_status launch_tile_attention(const AttnView& A, const TilePlan& plan, cudaStream_t s);

int stream_ctas(const AttnView& A);       // CTAs of launch_stream_attention at most
dsmoe_status launch_stream_attention(const AttnView& A, const PartPlan& parts, cudaStream_t s);
// Adds up, into out and lse, what launch_stream_attention left of these tokens in `parts`; of all tokens folded into one in `folded` (slots
// nullptr: none), the first of these tokens being number `token0` there; and `more`
dsmoe_status launch_attention_sum(const AttnView& A, const PartPlan& parts, const PartPlan& folded, int folded_tiles, int token0,
                                  const TileParts& more, cudaStream_t s);

// tally_out[s][j][l] = tally_in[s][j][l] (nullptr: 0) + the sum of the softmax weights that the tokens of sequence s gave key l, from A.ml.
// Causal alone: no window, no ring.
dsmoe_status launch_tally(const AttnView& A, const float* tally_in, float* tally_out, cudaStream_t s);

struct EvictView {
    int n_seq, n_head, L, d_head;
    int keep, sinks, recent;
    const int32_t* len;
    const float* tally;
    const __nv_bfloat16 *K, *V;
    long long kv_s, kv_h, kv_p;
    int32_t *kept, *len_out;
    float* tally_out;
    long long tally_pitch;
    __nv_bfloat16 *K_out, *V_out;
    long long o_s, o_h, o_p;
    bool in_place;
    int32_t* count;                       // [n_seq * n_head] (workspace)
    int32_t* dev_status;
};
dsmoe_status launch_evict(const EvictView& E, cudaStream_t s);

}  // namespace dsmoe
