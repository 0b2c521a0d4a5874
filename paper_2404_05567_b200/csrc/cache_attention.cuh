// Attention over a key/value cache as a step of its own (dsmoe_window_attention, dsmoe_prefix_attention, dsmoe_tally_attention): what the
// kernels and their launchers share.
//
// Token t, key/value head j, member g (one of the `group` query heads of that key/value head) is a row.  Position l of the cache is visible to
// token t at position p = pos[t] iff 0 <= l <= p and (p - l < window or l < sinks).  A row's result over any part of its keys is a triple:
// the largest logit m, the sum l of 2^(logit - m), and the sum o of 2^(logit - m) V (logits in base 2: scale * log2 e * <q, k>).  Triples of
// disjoint parts add up after scaling to the larger m, which is how work is split over CTAs, caches and kernels.
#pragma once

#include <cuda.h>
#include <limits.h>

#include "common.cuh"

namespace dsmoe {

struct AttnView {
    int T, n_head, group;
    int row_tiles;                        // 16-row tiles of the group rows of a (token, head)
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
};

// The maximum that weights are relative to moves only when a logit passes it by more than kMoves: until then the weights are at most 2^kMoves, fp32 sums
// and bf16 weights (which have fp32's exponents) lose nothing, and nothing is rescaled.  The 128-row kernel moves it behind the tile that asks for it,
// so a single tile's weights may be larger there.  With 8, a row whose first keys happened to have small
// logits (four sinks) moved now and then, and one such row held up its tile: a prompt of 8192 tokens 359 us, 311 with 32.
constexpr float kMoves = 32.f;
// In the streaming kernel, which has no second way for rows whose sums overflow: with large values (2^96) 2^32 of them do, where 2^8 do not.  Its times are the same.
constexpr float kStreamMoves = 8.f;

constexpr int kUnit = 16;                 // keys that a warp takes at a time
constexpr int kMaxSplits = 64;            // parts that the 128-row kernel's keys are cut into
constexpr int kMostStreamCtas = 160;      // CTAs of the streaming kernel, one an SM
constexpr int kListTokens = 512;         // tokens whose keys are cut into runs at a time

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
    const int most = A.ring ? INT_MAX - 1 : A.L - 1;      // (one more than a position is still a number)
    if (sq < 0 || sq >= A.n_seq || p < -1 || p > most) {
        *bad = true;
        sq = min(max(sq, 0), A.n_seq - 1);
        p = min(max(p, -1), most);
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
// there are a run; in a block of many runs, those that fill less than a quarter of a tile are left to the stream kernel.
__host__ __device__ static inline int tile_span(int group) { return 2 * (128 / group); }
__host__ __device__ static inline int tile_least_run(int group) { return (32 + group - 1) / group; }
__host__ __device__ static inline int tile_blocks(int T, int group) { return (T + tile_span(group) - 1) / tile_span(group); }
// The slot of the cache that holds position l
__device__ __forceinline__ int slot_of(const AttnView& A, int l) { return !A.ring || l < A.sinks ? l : A.sinks + (l - A.sinks) % A.ring; }

// Row (token t, head j, member m) of the calls' row arrays: lse, ml, whole rows' parts
__host__ __device__ static inline long long row_at(const AttnView& A, int t, int j, int m) { return ((long long)t * A.n_head + j) * A.group + m; }

// Parts of whole rows: n of them, [n][rows][d_head] and [n][rows][2] (m, l), a row for each token, head and member
struct RowParts {
    int n;
    size_t rows;
    float *o, *ml;
};

// The keys that all tokens of a call share: they are taken as one token, whose rows are all tokens' members
struct SharedKeys {
    int P;                                // 0: none
    int row_tiles;                        // 16-row tiles of the T * group rows of a head
    const __nv_bfloat16 *K, *V;
    long long kv_h, kv_p;
};

// What launch_stream_attention does: attends all tokens (list nullptr), or those that the 128-row kernel left: count[b] of block b's, list[b * span + i];
// and, `shared`, the shared keys.  Rows of 16 to a (token, head, row tile) = pair; the shared keys' pairs come first.
struct StreamPlan {
    SharedKeys shared;
    const int32_t *count, *list;
    int blocks, span;
    int ctas, passes;                     // passes of kListTokens tokens at most; the shared keys are the first one's
    bool own;                             // attends tokens at all
    // A pair that several CTAs share leaves a part per CTA; one that lies in one CTA's keys is written to out and lse, or (keep) its rows to `own_rows`
    // and `shared_rows`: something else is still to be added
    bool keep;
    bool by_warp;                         // runs are warps', not CTAs'
    bool whole;                           // each CTA's run is a pair's units: no parts (not with shared keys, a list or more than a pass)
    int heads_at_once;                    // neighbouring pairs of a token that a CTA takes together
    float* slots;                         // [passes][runs][2][heads_at_once][16][d_head + 2], runs = ctas * stream_warps / heads_at_once
    int2* head;                           // keep: [pairs]: first run, parts_word
    int2* run_head;                       // otherwise: [passes][runs]: the first of the pairs that begin in that run and go on, parts_word; or 0 parts
    RowParts own_rows, shared_rows;       // n = 1
    float* logits;                        // nullable: the tokens' logits in base 2, row r's from r * logit_pitch on (no window, no ring)
    long long logit_pitch;                // a multiple of 16
};
__host__ __device__ static constexpr int stream_warps(int d_head) { return d_head <= 128 ? 8 : 4; }       // of a CTA
static inline size_t part_bytes(int d_head) { return (size_t)16 * (d_head + 2) * 4; }

// Where the part of pair p of a group of HB lies that a run leaves: a run has room for the parts of the pairs that began before it and for those
// of the pairs that begin in it
__device__ static __forceinline__ long long part_slot(long long run, bool begins, int HB, int p) { return (2 * run + (begins ? 1 : 0)) * HB + p; }
// What is said of a pair's parts beside its first run: their number, and how many runs there are from one to the next
__device__ static __forceinline__ int parts_word(int parts, int stride) { return parts == 0 ? 0 : parts | stride << 16; }

// Runs of single warps that `total` units are cut into, `most` at most.  None is shorter than a kPartsAtMost-th of the longest pair's units, so that no pair lies in
// more than kPartsAtMost + 1 runs.
constexpr int kPartsAtMost = 200;
__host__ __device__ static constexpr long long warp_runs(long long total, long long longest, long long most) {
    const long long least = (longest + kPartsAtMost - 1) / kPartsAtMost, runs = total / least;
    return runs < 1 ? 1 : runs < most ? runs : most;
}
// (runs are of total / runs units and more: 250 units beside 159 and 1183 pairs of one)
static_assert(250 <= (kPartsAtMost - 1) * (409 / warp_runs(409, 250, 1184)) + 1 && 250 <= (kPartsAtMost - 1) * (1433 / warp_runs(1433, 250, 1184)) + 1);
static_assert(warp_runs(1, 1, 1184) == 1 && warp_runs(100000, 400, 1184) == 1184 && warp_runs(800, 800, 1184) == 200);

// The 128-row kernel: heads of 64, 96 and 128, caches that a tensor map describes.  Its rows' keys are cut into `splits`; o, ml: where their parts
// go (TileParts), or nullptr with one split: out and lse are written.
struct TilePlan {
    int splits;
    float *o, *ml;
    // own caches of several sequences: the tokens that it leaves are listed here (see StreamPlan), all heads' parts marked as none (or nullptr)
    int32_t *count, *list;
    int2* head;
};
bool tile_supported(const AttnView& A);
// K or V in boxes of 128 positions and 64 columns, 128-byte swizzle; at[0 .. 2]: the map's dimensions (1 .. 3) of positions, heads, sequences
dsmoe_status make_cache_map(CUtensorMap* m, const AttnView& A, const void* ptr, int (&at)[3]);
dsmoe_status launch_tile_attention(const AttnView& A, const TilePlan& plan, cudaStream_t s);

int stream_heads_at_once(const AttnView& A);
bool stream_whole(const AttnView& A, const StreamPlan& plan);
bool stream_by_warp(const AttnView& A, const StreamPlan& plan);
int stream_ctas(const AttnView& A, const SharedKeys& shared, bool own);       // CTAs of launch_stream_attention at most
dsmoe_status launch_stream_attention(const AttnView& A, const StreamPlan& plan, cudaStream_t s);
// Adds up what launch_stream_attention left in parts, into out and lse: without `keep` the pairs that several CTAs share; with it all rows, whose
// parts `rows` are there too
dsmoe_status launch_attention_sum(const AttnView& A, const StreamPlan& plan, const RowParts& rows, cudaStream_t s);

// tally_out[s][j][l] = tally_in[s][j][l] (nullptr: 0) + the sum of the softmax weights that the tokens of sequence s gave key l, from A.ml.
// Causal alone: no window, no ring.  parts > 0 (tile_supported): on the 5th-generation tensor cores, the rows cut into so many parts, whose sums go to
// `sums`, [parts][n_seq * n_head * L], with more than one; list [T] and from [n_seq]: scratch.
dsmoe_status launch_tally(const AttnView& A, int parts, float* sums, int2* list, int2* from, const float* tally_in, float* tally_out, cudaStream_t s);

// The same from the logits that launch_stream_attention left of every token (StreamPlan); up to kListTokens tokens
dsmoe_status launch_tally_add(const AttnView& A, const float* logits, long long pitch, const float* tally_in, float* tally_out, cudaStream_t s);

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
