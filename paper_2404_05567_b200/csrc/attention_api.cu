// C entry points of the attention steps on a key/value cache: argument checks, workspace, and which kernels a call takes.
#include <math.h>

#include <algorithm>
#include <climits>

#include "quant_cache.cuh"

namespace dsmoe {

namespace {

bool strides_ok(const int64_t* s, int n) {
    for (int i = 0; i < n; ++i)
        if (s[i] < 0 || (s[i] & 7)) return false;
    return true;
}

// Whether the last of rows at these strides begins within 2^50 elements of the first, further than addresses go.  (Beyond it are strides and sizes that
// are allowed one by one, and offsets that no longer fit 64 bits.)
bool within_reach(const int64_t* stride, const int64_t* n, int count) {
    int64_t left = 1ll << 50;
    for (int i = 0; i < count; ++i) {
        if (n[i] <= 1) continue;
        if (stride[i] > left / (n[i] - 1)) return false;
        left -= stride[i] * (n[i] - 1);
    }
    return true;
}

// Whether rows of `row` elements at these strides (within_reach) are apart from one another: each stride, in their order, spans what lies within it
bool rows_apart(const int64_t* stride, const int64_t* n, int64_t row) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
    int64_t span = row;
    for (int i : order) {
        if (n[i] <= 1) continue;
        if (stride[i] < span) return false;
        span += stride[i] * (n[i] - 1);
    }
    return true;
}

// Whether any two rows at these strides (rows_apart), one behind the first address and one behind the second, `apart` elements further on, share an element.
// What lies within a stride spans no more than it, so of each dimension only the two steps on either side of the distance come near enough.
bool rows_meet(int64_t apart, const int64_t* stride, const int64_t* n, int64_t row) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] > stride[b]; });
    for (int ways = 0; ways < 8; ++ways) {
        int64_t left = apart;
        bool there = true;
        for (int k = 0; k < 3; ++k) {
            const int i = order[k];
            if (n[i] <= 1) continue;
            const int64_t steps = left / stride[i] - (left % stride[i] < 0) + (ways >> k & 1);
            there = there && steps < n[i] && steps > -n[i];
            left -= steps * stride[i];
        }
        if (there && left < row && left > -row) return true;
    }
    return false;
}

// The bytes that rows at these strides (within_reach) lie in
struct Extent {
    uintptr_t begin, end;
    bool meets(const Extent& o) const { return begin < o.end && o.begin < end; }
};
Extent extent(const void* p, const int64_t* stride, const int64_t* n, int64_t row, int64_t size) {
    int64_t last = row;
    for (int i = 0; i < 3; ++i) last += stride[i] * (n[i] - 1);
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return Extent{a, a + (uintptr_t)(last * size)};
}

dsmoe_status check_cache(const dsmoe_attention_desc* d) {
    if (!d) return DSMOE_ERR_INVALID_ARG;
    if (d->n_head <= 0 || d->d_head <= 0 || d->n_seq <= 0 || d->L <= 0) return DSMOE_ERR_INVALID_ARG;
    if (!strides_ok(d->kv_stride, 3)) return DSMOE_ERR_INVALID_ARG;
    if (d->d_head % 32 || d->d_head > 256) return DSMOE_ERR_UNSUPPORTED;
    if (d->L > 1 << 30 || (long long)d->n_seq * d->n_head > INT_MAX / 4) return DSMOE_ERR_UNSUPPORTED;
    for (int i = 0; i < 3; ++i)
        if (d->kv_stride[i] > (1ll << 40)) return DSMOE_ERR_UNSUPPORTED;
    const int64_t n[3] = {d->n_seq, d->n_head, d->L};
    return within_reach(d->kv_stride, n, 3) ? DSMOE_OK : DSMOE_ERR_UNSUPPORTED;
}

dsmoe_status check_attention(const dsmoe_attention_desc* d) {
    DSMOE_TRY(check_cache(d));
    if (d->T < 0 || d->group <= 0 || !isfinite(d->scale)) return DSMOE_ERR_INVALID_ARG;
    if (!strides_ok(d->q_stride, 3) || !strides_ok(d->o_stride, 3)) return DSMOE_ERR_INVALID_ARG;
    if (d->group > 64) return DSMOE_ERR_UNSUPPORTED;
    if ((double)d->T * d->n_head * d->group > (double)INT_MAX / 2) return DSMOE_ERR_UNSUPPORTED;
    for (int i = 0; i < 3; ++i)
        if (d->q_stride[i] > (1ll << 40) || d->o_stride[i] > (1ll << 40)) return DSMOE_ERR_UNSUPPORTED;
    const int64_t n[3] = {d->T, d->n_head, d->group};
    if (!within_reach(d->q_stride, n, 3) || !within_reach(d->o_stride, n, 3)) return DSMOE_ERR_UNSUPPORTED;
    if (!rows_apart(d->o_stride, n, d->d_head)) return DSMOE_ERR_INVALID_ARG;
    return DSMOE_OK;
}

dsmoe_status check_attention_call(const dsmoe_attention_desc* d, const void* q, const void* K, const void* V, const int32_t* pos, const void* out) {
    if (!q || !K || !V || !pos || !out) return DSMOE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(out)) return DSMOE_ERR_INVALID_ARG;
    const int64_t n[3] = {d->T, d->n_head, d->group}, c[3] = {d->n_seq, d->n_head, d->L};
    const Extent o = extent(out, d->o_stride, n, d->d_head, 2);
    if (o.meets(extent(q, d->q_stride, n, d->d_head, 2)) || o.meets(extent(K, d->kv_stride, c, d->d_head, 2)) ||
        o.meets(extent(V, d->kv_stride, c, d->d_head, 2)))
        return DSMOE_ERR_INVALID_ARG;
    return DSMOE_OK;
}

AttnView view_of(const dsmoe_attention_desc& d, const void* q, const void* K, const void* V, const int32_t* tok_seq, const int32_t* pos, void* out,
                 float* lse, int32_t* dev_status) {
    AttnView A{};
    A.T = d.T;
    A.n_head = d.n_head;
    A.group = d.group;
    A.row_tiles = ceil_div(d.group, 16);
    A.d_head = d.d_head;
    A.n_seq = d.n_seq;
    A.L = d.L;
    A.window = INT_MAX;
    A.scale_log2 = d.scale * 1.4426950408889634f;
    A.q = static_cast<const __nv_bfloat16*>(q);
    A.q_t = d.q_stride[0], A.q_h = d.q_stride[1], A.q_g = d.q_stride[2];
    A.K = static_cast<const __nv_bfloat16*>(K);
    A.V = static_cast<const __nv_bfloat16*>(V);
    A.kv_s = d.kv_stride[0], A.kv_h = d.kv_stride[1], A.kv_p = d.kv_stride[2];
    A.tok_seq = tok_seq;
    A.pos = pos;
    A.out = static_cast<__nv_bfloat16*>(out);
    A.o_t = d.o_stride[0], A.o_h = d.o_stride[1], A.o_g = d.o_stride[2];
    A.lse = lse;
    A.dev_status = dev_status;
    return A;
}

// Which kernels a call takes, and its workspace.
//
// The prefix: on the 128-row kernel from 33 rows on (two 16-row tiles of the stream kernel read it twice; with more rows the stream kernel is bound by
// its MMAs), its keys cut so that all SMs have some; with fewer rows on the stream kernel, in one launch with the own caches.  The own caches:
// where there are more tokens than sequences, on the 128-row kernel, which leaves tokens that have too few neighbours of their sequence; otherwise,
// and for those, on the stream kernel.
constexpr int kPrefixStreamRows = 32, kOwnTileRows = 64;
constexpr int kMaxTallyParts = 16;
constexpr size_t kMostLogits = (size_t)512 << 20;

struct AttnPlan {
    size_t slots, head, run_head, count, list, ml, logits, sums, tokens, row_o, row_ml, total;
    int tally_parts;                      // tally on the 128-row tiles: parts of the rows; 0: not there
    long long logit_pitch;                // tally: 0 if the logits are not kept
    int ctas, passes;                     // of the stream kernel, at most
    int prefix_splits;                    // 0: the prefix is not the 128-row kernel's
    int own_splits;                       // ... the own caches
    int row_parts;                        // parts of whole rows
    bool fits;                            // a workspace of that size is supported
};

// Parts into which the 128-row kernel's keys are cut: as many as fill the SMs, two tiles of keys or more in each
int tile_splits(const AttnView& A, long long keys) {
    const long long ctas = (long long)tile_blocks(A.T, A.group) * A.n_head, tiles = (keys + 127) / 128;
    return (int)std::max(1ll, std::min({(long long)sm_count() / ctas, tiles / 2, (long long)kMaxSplits}));
}

bool own_on_tiles(const AttnView& A) {
    return tile_supported(A) && (A.tok_seq ? A.T > A.n_seq : A.T > 1) && (long long)A.T * A.group >= kOwnTileRows;
}

SharedKeys shared_keys(const AttnView& A, const dsmoe_prefix& p) {
    return SharedKeys{p.P, (int)(((long long)A.T * A.group + 15) / 16), static_cast<const __nv_bfloat16*>(p.Kp),
                      static_cast<const __nv_bfloat16*>(p.Vp), p.stride[0], p.stride[1]};
}
// The shared keys as a cache of one sequence
AttnView shared_view(const AttnView& A, const SharedKeys& S) {
    AttnView N = A;
    N.n_seq = 1;
    N.L = S.P;
    N.K = S.K, N.V = S.V;
    N.kv_s = 0, N.kv_h = S.kv_h, N.kv_p = S.kv_p;
    N.tok_seq = N.pos = nullptr;
    return N;
}

// may_tile: the prefix's strides allow it
AttnPlan attention_plan(const AttnView& A, const SharedKeys& S, bool may_tile, bool wants_ml) {
    AttnPlan w{};
    size_t off = 0;
    const auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    const size_t rows = (size_t)A.T * A.n_head * A.group, blocks = (size_t)tile_blocks(A.T, A.group);
    // The stream kernel has no token to attend where the 128-row kernel takes all: then it has the shared keys, or is not launched
    const bool tiles = own_on_tiles(A), streams_own = !tiles || A.n_seq > 1;
    w.ctas = stream_ctas(A, S, streams_own);
    w.passes = streams_own ? ceil_div(A.T, kListTokens) : S.P > 0 ? 1 : 0;
    const size_t warps = (size_t)w.passes * w.ctas * stream_warps(A.d_head);
    w.slots = take(2 * warps * part_bytes(A.d_head));
    w.run_head = take(warps * sizeof(int2));
    w.head = take((size_t)A.n_head * ((streams_own ? (size_t)A.T * A.row_tiles : 0) + (S.P > 0 ? S.row_tiles : 0)) * sizeof(int2));
    if (wants_ml) {
        w.ml = take(rows * sizeof(float2));
        // Decoding: the logits are written and read again (8 bytes a key and row), not the keys read and multiplied again
        const size_t pitch = align_up(A.L, 16);
        if (!tiles && A.T <= kListTokens && rows * pitch * 4 <= kMostLogits) {
            w.logit_pitch = (long long)pitch;
            w.logits = take(rows * pitch * 4);
        }
        if (tiles) {
            // parts of the rows until four CTAs come to an SM (two fit; the keys at the end of a sequence are seen by few rows)
            const size_t cells = (size_t)A.n_seq * A.n_head * A.L;
            const long long ctas = (long long)A.n_seq * A.n_head * ((A.L + 127) / 128);
            w.tally_parts = (int)std::max(1ll, std::min(4ll * sm_count() / ctas, (long long)kMaxTallyParts));
            w.tokens = take(((size_t)A.T + A.n_seq) * sizeof(int2));
            if (w.tally_parts > 1) w.sums = take(w.tally_parts * cells * 4);
        }
    }
    if (tiles) {
        w.own_splits = tile_splits(A, A.L);
        if (streams_own) {
            w.count = take(blocks * 4);
            w.list = take(blocks * tile_span(A.group) * 4);
        }
    }
    if (S.P > 0 && may_tile && (long long)A.T * A.group > kPrefixStreamRows) w.prefix_splits = tile_splits(A, S.P);
    if (S.P > 0 || w.own_splits > 1) w.row_parts = (S.P > 0 ? std::max(1, w.prefix_splits) : 0) + std::max(1, w.own_splits);
    w.row_ml = take((size_t)w.row_parts * rows * 2 * 4);
    w.row_o = take((size_t)w.row_parts * rows * A.d_head * 4);
    w.total = std::max(off, (size_t)256); // (so that there is an address to pass)
    w.fits = off < (size_t)1 << 36;       // (attention_sum_kernel finds parts by their number of 16 bytes, in 32 bits)
    return w;
}

// Attention of all tokens: the prefix, the own caches, the sum
dsmoe_status attend(const AttnView& A, const SharedKeys& S, const AttnPlan& w, char* ws, cudaStream_t s) {
    const size_t rows = (size_t)A.T * A.n_head * A.group;
    const bool one_sequence = !A.tok_seq || A.n_seq == 1;
    RowParts parts{0, rows, reinterpret_cast<float*>(ws + w.row_o), reinterpret_cast<float*>(ws + w.row_ml)};
    const auto next_parts = [&](int n) {                // the next n parts of whole rows
        const RowParts p{n, rows, parts.o + parts.n * rows * A.d_head, parts.ml + parts.n * rows * 2};
        parts.n += n;
        return p;
    };
    StreamPlan plan{};
    plan.passes = w.passes;
    plan.heads_at_once = stream_heads_at_once(A);
    plan.slots = reinterpret_cast<float*>(ws + w.slots);
    plan.own = true;
    int2* const head = reinterpret_cast<int2*>(ws + w.head);
    if (w.prefix_splits) {
        const RowParts p = next_parts(w.prefix_splits);
        DSMOE_TRY(launch_tile_attention(shared_view(A, S), TilePlan{w.prefix_splits, p.o, p.ml, nullptr, nullptr, nullptr}, s));
    } else if (S.P > 0) {
        plan.shared = S;
        plan.shared_rows = next_parts(1);
    }
    plan.keep = S.P > 0;
    if (w.logit_pitch) {
        plan.logits = reinterpret_cast<float*>(ws + w.logits);
        plan.logit_pitch = w.logit_pitch;
    }
    if (w.own_splits) {
        // a narrow window needs fewer parts than the workspace has room for
        const long long keys = A.window < A.L ? (long long)A.window + A.sinks + tile_span(A.group) : A.L;
        const int splits = std::min(w.own_splits, tile_splits(A, keys));
        plan.keep = plan.keep || splits > 1;
        TilePlan tile{splits, nullptr, nullptr, nullptr, nullptr, nullptr};
        if (plan.keep) {
            plan.own_rows = next_parts(splits);
            tile.o = plan.own_rows.o, tile.ml = plan.own_rows.ml;
        }
        if (!one_sequence) {
            if (plan.keep) tile.head = head + (size_t)A.n_head * plan.shared.row_tiles;
            plan.count = tile.count = reinterpret_cast<int32_t*>(ws + w.count);
            plan.list = tile.list = reinterpret_cast<int32_t*>(ws + w.list);
            plan.blocks = tile_blocks(A.T, A.group);
            plan.span = tile_span(A.group);
        } else {
            plan.own = false;
        }
        DSMOE_TRY(launch_tile_attention(A, tile, s));
    } else if (plan.keep) {
        plan.own_rows = next_parts(1);
    }
    if (plan.own && stream_whole(A, plan)) {
        plan.whole = true;
        plan.heads_at_once = 1;
        plan.ctas = A.T * A.n_head * A.row_tiles;
        return launch_stream_attention(A, plan, s);
    }
    plan.ctas = std::min(w.ctas, stream_ctas(A, plan.shared, plan.own));
    plan.by_warp = stream_by_warp(A, plan);
    if (plan.keep) plan.head = head;
    else plan.run_head = reinterpret_cast<int2*>(ws + w.run_head);
    if (plan.own || plan.shared.P > 0) DSMOE_TRY(launch_stream_attention(A, plan, s));
    else if (!plan.keep) return DSMOE_OK;
    return launch_attention_sum(A, plan, parts, s);
}

dsmoe_status check_window(const dsmoe_attention_desc* d, int window, int sinks, int rolling) {
    if (window < 1 || sinks < 0 || (rolling != 0 && rolling != 1)) return DSMOE_ERR_INVALID_ARG;
    if (rolling && (sinks >= d->L || window > d->L - sinks)) return DSMOE_ERR_INVALID_ARG;
    return DSMOE_OK;
}

dsmoe_status check_prefix(const dsmoe_attention_desc* d, const dsmoe_prefix* p, const void* out) {
    if (!p || p->P < 0) return DSMOE_ERR_INVALID_ARG;
    if (p->P == 0) return DSMOE_OK;
    if (!p->Kp || !p->Vp || !aligned16(p->Kp) || !aligned16(p->Vp) || !strides_ok(p->stride, 2)) return DSMOE_ERR_INVALID_ARG;
    if (p->P > 1 << 30 || p->stride[0] > (1ll << 40) || p->stride[1] > (1ll << 40)) return DSMOE_ERR_UNSUPPORTED;
    const int64_t n[3] = {d->T, d->n_head, d->group}, c[3] = {1, d->n_head, p->P}, st[3] = {0, p->stride[0], p->stride[1]};
    if (!within_reach(st, c, 3)) return DSMOE_ERR_UNSUPPORTED;
    const Extent o = extent(out, d->o_stride, n, d->d_head, 2);
    if (o.meets(extent(p->Kp, st, c, d->d_head, 2)) || o.meets(extent(p->Vp, st, c, d->d_head, 2))) return DSMOE_ERR_INVALID_ARG;
    return DSMOE_OK;
}

// ---- caches in 4 bits

// Rows of `row` bytes or elements at strides that are multiples of `unit`
dsmoe_status check_rows(const int64_t* stride, const int64_t* n, int count, int64_t unit) {
    for (int i = 0; i < count; ++i)
        if (stride[i] < 0 || stride[i] % unit) return DSMOE_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i)
        if (stride[i] > (1ll << 40)) return DSMOE_ERR_UNSUPPORTED;
    return within_reach(stride, n, count) ? DSMOE_OK : DSMOE_ERR_UNSUPPORTED;
}

dsmoe_status check_quant_cache(const dsmoe_quant_cache* c) {
    if (!c) return DSMOE_ERR_INVALID_ARG;
    if (c->n_seq <= 0 || c->n_head <= 0 || c->L <= 0 || c->d_head <= 0) return DSMOE_ERR_INVALID_ARG;
    if (c->d_head % 32 || c->d_head > 256) return DSMOE_ERR_UNSUPPORTED;
    if (c->L > 1 << 30 || (long long)c->n_seq * c->n_head > INT_MAX / 4) return DSMOE_ERR_UNSUPPORTED;
    if (!c->K || !c->V || !c->K_scale || !c->V_scale) return DSMOE_ERR_INVALID_ARG;
    if (!aligned16(c->K) || !aligned16(c->V)) return DSMOE_ERR_INVALID_ARG;
    const uintptr_t row = 2 * quant_scales(c->d_head);        // (a row of scales is one load)
    if ((uintptr_t)c->K_scale % row || (uintptr_t)c->V_scale % row) return DSMOE_ERR_INVALID_ARG;
    const int64_t n[3] = {c->n_seq, c->n_head, c->L};
    DSMOE_TRY(check_rows(c->code_stride, n, 3, 16));
    return check_rows(c->scale_stride, n, 3, quant_scales(c->d_head));
}

// The memory of a cache's four parts
struct QuantExtents {
    Extent e[4];
    bool meets(const Extent& o) const { return e[0].meets(o) || e[1].meets(o) || e[2].meets(o) || e[3].meets(o); }
};
QuantExtents quant_extents(const dsmoe_quant_cache& c) {
    const int64_t n[3] = {c.n_seq, c.n_head, c.L};
    const int sc = quant_scales(c.d_head);
    return QuantExtents{{extent(c.K, c.code_stride, n, c.d_head / 2, 1), extent(c.V, c.code_stride, n, c.d_head / 2, 1),
                         extent(c.K_scale, c.scale_stride, n, sc, 2), extent(c.V_scale, c.scale_stride, n, sc, 2)}};
}

QuantView quant_view(const dsmoe_quant_cache& c) {
    QuantView v{};
    v.n_seq = c.n_seq, v.n_head = c.n_head, v.L = c.L, v.d_head = c.d_head;
    v.K = static_cast<unsigned char*>(c.K);
    v.V = static_cast<unsigned char*>(c.V);
    v.K_scale = static_cast<__nv_bfloat16*>(c.K_scale);
    v.V_scale = static_cast<__nv_bfloat16*>(c.V_scale);
    v.c_s = c.code_stride[0], v.c_h = c.code_stride[1], v.c_p = c.code_stride[2];
    v.s_s = c.scale_stride[0], v.s_h = c.scale_stride[1], v.s_p = c.scale_stride[2];
    return v;
}

// Prompts are attended to from bf16 copies of what their tokens see, which are exact, on the 128-row kernel.  Reading back and reading that again moves 8 times the
// bytes that a token's own pass over the 4 bits does, so from eight tokens a sequence on; and finding out what is to be read, reading it and that kernel's own
// launches take longer than single tokens do where there is little to do.  us of single tokens and of prompts, 4 x 5 heads of 128: 16 tokens of one cache of 4000
// 23, 27 (8064 units); 64 of 1000 23, 20 (8192); 128 of 1000 31, 22; 32 of each of 4 of 1000 31, 36 (16384), of 2000 46, 39 (32256).  Groups of more than 8, whose
// units cost twice as much and fill tiles better: 16 heads on one, 200 of 350 26, 16 (2200 units).  What single tokens do in one launch they do in less than prompts
// take: 16 heads on one, 64 of 1000 18, 21 (2048), of 1200 19.5, 20.6; 4 x 16 heads, 32 of 1000 18, 21 (4096).
// Where the copies are larger than a workspace may be, single tokens it is.  A sequence's rows have to fill half of a tile, or a quarter with 16 tokens and more: what fills less is left to the streaming kernel, which reads the copies once
// a token.  32 caches of 4000: 4 x 1 heads of 64, 8 tokens 92, 240, 24 255, 616, 32 332, 124; 4 x 2 of 64, 12 131, 327, 16 170, 118; 4 x 5 of 128, 8 132, 192, 12 190, 197,
// 16 248, 189; 4 x 16, 8 216, 167.
bool quant_on_tiles(const AttnView& A) {
    const double units = (double)A.T * A.n_head * A.row_tiles * (A.L / 32 + 1) * (A.group <= 8 ? 1 : 4);
    const long long rows = (long long)A.T * A.group, n_seq = A.n_seq;
    const double copy = (double)A.n_seq * A.n_head * A.L * A.d_head * 2;                  // bytes (beyond 64 bits, with strides of 0)
    return copy < 0x1p40 && own_on_tiles(A) && !quant_whole(A) && A.T >= 8 * n_seq && (rows >= 64 * n_seq || (A.T >= 16 * n_seq && rows >= 32 * n_seq)) &&
           units >= (n_seq == 1 || A.T >= 48 * n_seq ? 8192 : 32768);
}
// The copies as the cache of a view
AttnView quant_copy_view(const AttnView& A, char* ws, size_t bytes) {
    AttnView B = A;
    B.K = reinterpret_cast<const __nv_bfloat16*>(ws);
    B.V = reinterpret_cast<const __nv_bfloat16*>(ws + bytes);
    B.kv_p = A.d_head;
    B.kv_h = (long long)A.L * A.d_head;
    B.kv_s = B.kv_h * A.n_head;
    return B;
}
struct QuantAttnPlan {
    bool tiles;
    size_t copy, range, rest, total;      // tiles: bytes of a copy (K's and V's are first), where the ranges lie, where attend's workspace begins
    size_t run_head;                      // otherwise: (the slots are first)
    QuantPlan plan;
    AttnPlan attn;
    bool fits;
};
QuantAttnPlan quant_attention_plan(const AttnView& A) {
    QuantAttnPlan w{};
    w.tiles = quant_on_tiles(quant_copy_view(A, nullptr, 0));
    if (w.tiles) {
        w.copy = align_up((size_t)A.n_seq * A.n_head * A.L * A.d_head * 2, 256);
        w.range = 2 * w.copy;
        w.rest = w.range + align_up((size_t)A.n_seq * sizeof(int4), 256);
        w.attn = attention_plan(quant_copy_view(A, nullptr, w.copy), SharedKeys{}, false, false);
        w.total = w.rest + w.attn.total;
        w.fits = w.attn.fits;
        if (w.fits) return w;
        w = QuantAttnPlan{};
    }
    size_t slots, heads;
    quant_plan_size(A, &w.plan, &slots, &heads);
    w.run_head = align_up(slots, 256);
    w.total = w.run_head + align_up(heads, 256);
    w.fits = w.total < (size_t)1 << 36;
    return w;
}

dsmoe_attention_desc quant_desc(const dsmoe_attention_desc& d) {         // (the strides of a cache in 16 bits are not looked at)
    dsmoe_attention_desc q = d;
    q.kv_stride[0] = q.kv_stride[1] = q.kv_stride[2] = 0;
    return q;
}

}  // namespace

}  // namespace dsmoe

using namespace dsmoe;

extern "C" {

dsmoe_status dsmoe_attention_workspace_size(const dsmoe_attention_desc* desc, int kind, int prefix_len, size_t* bytes) {
    DSMOE_TRY(check_attention(desc));
    if (!bytes || kind < DSMOE_ATTENTION_WINDOW || kind > DSMOE_ATTENTION_TALLY) return DSMOE_ERR_INVALID_ARG;
    if (kind == DSMOE_ATTENTION_PREFIX && prefix_len < 0) return DSMOE_ERR_INVALID_ARG;
    if (kind == DSMOE_ATTENTION_PREFIX && prefix_len > 1 << 30) return DSMOE_ERR_UNSUPPORTED;
    const AttnView A = view_of(*desc, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr);
    if (desc->T == 0) {
        *bytes = 0;
    } else {
        // (with and without sequence numbers, and whatever the prefix's strides turn out to be)
        dsmoe_prefix p{};
        if (kind == DSMOE_ATTENTION_PREFIX) p.P = prefix_len;
        const bool tiles = A.d_head == 64 || A.d_head == 96 || A.d_head == 128;
        const AttnPlan w = attention_plan(A, shared_keys(A, p), tiles, kind == DSMOE_ATTENTION_TALLY);
        if (!w.fits) return DSMOE_ERR_UNSUPPORTED;
        *bytes = w.total;
        if (kind == DSMOE_ATTENTION_TALLY) {            // (with sequence numbers, as many as there may be, the logits may be kept)
            AttnView several = A;
            several.tok_seq = &desc->n_seq;
            *bytes = std::max(*bytes, attention_plan(several, SharedKeys{}, false, true).total);
        }
    }
    return DSMOE_OK;
}

dsmoe_status dsmoe_window_attention(const dsmoe_attention_desc* desc, int window, int sinks, int rolling, const void* q, const void* K,
                                    const void* V, const int32_t* tok_seq, const int32_t* pos, void* out, float* lse, void* workspace,
                                    size_t ws_bytes, int32_t* dev_status, dsmoe_stream stream) {
    DSMOE_TRY(check_attention(desc));
    DSMOE_TRY(check_window(desc, window, sinks, rolling));
    if (desc->T == 0) return DSMOE_OK;
    DSMOE_TRY(check_attention_call(desc, q, K, V, pos, out));
    AttnView A = view_of(*desc, q, K, V, tok_seq, pos, out, lse, dev_status);
    // (the workspace is that of a window as wide as the cache: the most CTAs that any window can have)
    const AttnPlan w = attention_plan(A, SharedKeys{}, false, false);
    if (!w.fits) return DSMOE_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || ws_bytes < w.total) return DSMOE_ERR_WORKSPACE;
    A.window = window;
    A.sinks = sinks;
    A.ring = rolling ? desc->L - sinks : 0;
    return attend(A, SharedKeys{}, w, static_cast<char*>(workspace), (cudaStream_t)stream);
}

dsmoe_status dsmoe_prefix_attention(const dsmoe_attention_desc* desc, const dsmoe_prefix* prefix, const void* q, const void* K, const void* V,
                                    const int32_t* tok_seq, const int32_t* pos, void* out, float* lse, void* workspace, size_t ws_bytes,
                                    int32_t* dev_status, dsmoe_stream stream) {
    DSMOE_TRY(check_attention(desc));
    if (!prefix || prefix->P < 0) return DSMOE_ERR_INVALID_ARG;
    if (desc->T == 0) return DSMOE_OK;
    DSMOE_TRY(check_attention_call(desc, q, K, V, pos, out));
    DSMOE_TRY(check_prefix(desc, prefix, out));
    const AttnView A = view_of(*desc, q, K, V, tok_seq, pos, out, lse, dev_status);
    const SharedKeys S = prefix->P > 0 ? shared_keys(A, *prefix) : SharedKeys{};
    const AttnPlan w = attention_plan(A, S, S.P > 0 && tile_supported(shared_view(A, S)), false);
    if (!w.fits) return DSMOE_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || ws_bytes < w.total) return DSMOE_ERR_WORKSPACE;
    return attend(A, S, w, static_cast<char*>(workspace), (cudaStream_t)stream);
}

dsmoe_status dsmoe_tally_attention(const dsmoe_attention_desc* desc, const void* q, const void* K, const void* V, const int32_t* tok_seq,
                                   const int32_t* pos, void* out, float* lse, const float* tally_in, float* tally_out, void* workspace,
                                   size_t ws_bytes, int32_t* dev_status, dsmoe_stream stream) {
    DSMOE_TRY(check_attention(desc));
    if (!tally_out) return DSMOE_ERR_INVALID_ARG;
    const size_t cells = (size_t)desc->n_seq * desc->n_head * desc->L;
    if (tally_in && tally_in != tally_out && tally_in < tally_out + cells && tally_out < tally_in + cells) return DSMOE_ERR_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)stream;
    if (desc->T > 0) {
        DSMOE_TRY(check_attention_call(desc, q, K, V, pos, out));
    } else {                                            // no token: the tallies are handed on
        if (tally_in == tally_out) return DSMOE_OK;
        if (tally_in) DSMOE_CUDA_TRY(cudaMemcpyAsync(tally_out, tally_in, cells * 4, cudaMemcpyDeviceToDevice, s));
        else DSMOE_CUDA_TRY(cudaMemsetAsync(tally_out, 0, cells * 4, s));
        return DSMOE_OK;
    }
    AttnView A = view_of(*desc, q, K, V, tok_seq, pos, out, lse, dev_status);
    const AttnPlan w = attention_plan(A, SharedKeys{}, false, true);
    if (!w.fits) return DSMOE_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || ws_bytes < w.total) return DSMOE_ERR_WORKSPACE;
    A.ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + w.ml);
    DSMOE_TRY(attend(A, SharedKeys{}, w, static_cast<char*>(workspace), s));
    if (w.logit_pitch)
        return launch_tally_add(A, reinterpret_cast<const float*>(static_cast<char*>(workspace) + w.logits), w.logit_pitch, tally_in, tally_out, s);
    int2* const tokens = reinterpret_cast<int2*>(static_cast<char*>(workspace) + w.tokens);
    return launch_tally(A, w.tally_parts, reinterpret_cast<float*>(static_cast<char*>(workspace) + w.sums), tokens, tokens + A.T, tally_in, tally_out, s);
}

dsmoe_status dsmoe_evict_workspace_size(const dsmoe_attention_desc* desc, size_t* bytes) {
    DSMOE_TRY(check_cache(desc));
    if (!bytes) return DSMOE_ERR_INVALID_ARG;
    *bytes = align_up((size_t)desc->n_seq * desc->n_head * 4, 256);
    return DSMOE_OK;
}

dsmoe_status dsmoe_cache_evict(const dsmoe_attention_desc* desc, const dsmoe_evict_args* args, const int32_t* len, const float* tally,
                               const void* K, const void* V, int32_t* kept, int32_t* len_out, float* tally_out, void* K_out, void* V_out,
                               void* workspace, size_t ws_bytes, int32_t* dev_status, dsmoe_stream stream) {
    DSMOE_TRY(check_cache(desc));
    if (!args || !len || !tally || !K || !V || !kept || !len_out || !tally_out || !K_out || !V_out) return DSMOE_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V) || !aligned16(K_out) || !aligned16(V_out)) return DSMOE_ERR_INVALID_ARG;
    const dsmoe_evict_args& a = *args;
    if (a.keep < 1 || a.keep > desc->L || a.sinks < 0 || a.recent < 0 || (long long)a.sinks + a.recent > a.keep) return DSMOE_ERR_INVALID_ARG;
    if (!strides_ok(a.out_stride, 3) || a.tally_pitch < a.keep) return DSMOE_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (a.out_stride[i] > (1ll << 40)) return DSMOE_ERR_UNSUPPORTED;
    if (a.tally_pitch > (1ll << 40)) return DSMOE_ERR_UNSUPPORTED;
    const int64_t n[3] = {desc->n_seq, desc->n_head, desc->L}, m[3] = {desc->n_seq, desc->n_head, a.keep};
    const int64_t pairs = (int64_t)desc->n_seq * desc->n_head;
    if (!within_reach(a.out_stride, m, 3) || !within_reach(&a.tally_pitch, &pairs, 1)) return DSMOE_ERR_UNSUPPORTED;
    const bool in_place = K_out == K;
    if (in_place != (V_out == V)) return DSMOE_ERR_INVALID_ARG;
    if (!rows_apart(a.out_stride, m, desc->d_head)) return DSMOE_ERR_INVALID_ARG;
    // (in place the whole caches move, not the first `keep` positions alone)
    const int64_t between = ((intptr_t)V_out - (intptr_t)K_out) / 2;
    const Extent ek = extent(K, desc->kv_stride, n, desc->d_head, 2), ev = extent(V, desc->kv_stride, n, desc->d_head, 2);
    const Extent ok = extent(K_out, a.out_stride, m, desc->d_head, 2), ov = extent(V_out, a.out_stride, m, desc->d_head, 2);
    if (in_place) {
        for (int i = 0; i < 3; ++i)
            if (a.out_stride[i] != desc->kv_stride[i]) return DSMOE_ERR_INVALID_ARG;
        if (!rows_apart(desc->kv_stride, n, desc->d_head) || rows_meet(between, desc->kv_stride, n, desc->d_head)) return DSMOE_ERR_INVALID_ARG;
    } else if (ok.meets(ek) || ok.meets(ev) || ov.meets(ek) || ov.meets(ev) || rows_meet(between, a.out_stride, m, desc->d_head)) {
        return DSMOE_ERR_INVALID_ARG;
    }
    if (tally_out == tally) {
        if (a.tally_pitch != desc->L) return DSMOE_ERR_INVALID_ARG;
    } else if (tally < tally_out + (pairs - 1) * a.tally_pitch + a.keep && tally_out < tally + pairs * desc->L) {
        return DSMOE_ERR_INVALID_ARG;
    }
    if (!workspace || !aligned16(workspace) || ws_bytes < (size_t)pairs * 4) return DSMOE_ERR_WORKSPACE;
    EvictView E{};
    E.n_seq = desc->n_seq, E.n_head = desc->n_head, E.L = desc->L, E.d_head = desc->d_head;
    E.keep = a.keep, E.sinks = a.sinks, E.recent = a.recent;
    E.len = len;
    E.tally = tally;
    E.K = static_cast<const __nv_bfloat16*>(K);
    E.V = static_cast<const __nv_bfloat16*>(V);
    E.kv_s = desc->kv_stride[0], E.kv_h = desc->kv_stride[1], E.kv_p = desc->kv_stride[2];
    E.kept = kept;
    E.len_out = len_out;
    E.tally_out = tally_out;
    E.tally_pitch = a.tally_pitch;
    E.K_out = static_cast<__nv_bfloat16*>(K_out);
    E.V_out = static_cast<__nv_bfloat16*>(V_out);
    E.o_s = a.out_stride[0], E.o_h = a.out_stride[1], E.o_p = a.out_stride[2];
    E.in_place = in_place;
    E.count = static_cast<int32_t*>(workspace);
    E.dev_status = dev_status;
    return launch_evict(E, (cudaStream_t)stream);
}

dsmoe_status dsmoe_quant_cache_write(const dsmoe_quant_cache* cache, const dsmoe_quant_write_args* args, const void* k, const void* v,
                                     const int32_t* tok_seq, const int32_t* pos, void* k_back, void* v_back, int32_t* dev_status, dsmoe_stream stream) {
    DSMOE_TRY(check_quant_cache(cache));
    if (!args) return DSMOE_ERR_INVALID_ARG;
    const dsmoe_quant_write_args& a = *args;
    const dsmoe_quant_cache& c = *cache;
    if (a.T < 0 || a.sinks < 0 || (a.rolling != 0 && a.rolling != 1) || (a.rolling && a.sinks >= c.L)) return DSMOE_ERR_INVALID_ARG;
    const int64_t in[3] = {a.in_stride[0], a.in_stride[1], 0}, back[3] = {a.back_stride[0], a.back_stride[1], 0}, n[3] = {a.T, c.n_head, 1};
    DSMOE_TRY(check_rows(in, n, 2, 8));
    if (k_back || v_back) DSMOE_TRY(check_rows(back, n, 2, 8));
    if ((double)a.T * c.n_head > (double)INT_MAX / 2) return DSMOE_ERR_UNSUPPORTED;
    // Each row of the cache is its own (slots that no token of the call goes to keep what they hold)
    const int64_t places[3] = {c.n_seq, c.n_head, c.L};
    const int64_t code = (intptr_t)c.V - (intptr_t)c.K, scale = ((intptr_t)c.V_scale - (intptr_t)c.K_scale) / 2;
    const int sc = quant_scales(c.d_head);
    if (!rows_apart(c.code_stride, places, c.d_head / 2) || rows_meet(code, c.code_stride, places, c.d_head / 2) ||
        !rows_apart(c.scale_stride, places, sc) || rows_meet(scale, c.scale_stride, places, sc))
        return DSMOE_ERR_INVALID_ARG;
    const QuantExtents held = quant_extents(c);
    if (held.e[0].meets(held.e[2]) || held.e[0].meets(held.e[3]) || held.e[1].meets(held.e[2]) || held.e[1].meets(held.e[3])) return DSMOE_ERR_INVALID_ARG;
    if (a.T == 0) return DSMOE_OK;
    if (!k || !v || !pos || !aligned16(k) || !aligned16(v) || !aligned16(k_back) || !aligned16(v_back)) return DSMOE_ERR_INVALID_ARG;
    const Extent ek = extent(k, in, n, c.d_head, 2), ev = extent(v, in, n, c.d_head, 2);
    if (held.meets(ek) || held.meets(ev)) return DSMOE_ERR_INVALID_ARG;
    if (k_back || v_back) {
        if (!rows_apart(back, n, c.d_head)) return DSMOE_ERR_INVALID_ARG;
        for (const void* b : {k_back, v_back}) {
            if (!b) continue;
            const Extent eb = extent(b, back, n, c.d_head, 2);
            if (held.meets(eb) || eb.meets(ek) || eb.meets(ev)) return DSMOE_ERR_INVALID_ARG;
        }
        if (k_back && v_back && rows_meet(((intptr_t)v_back - (intptr_t)k_back) / 2, back, n, c.d_head)) return DSMOE_ERR_INVALID_ARG;
    }
    QuantWrite W{};
    W.T = a.T, W.sinks = a.sinks, W.ring = a.rolling ? c.L - a.sinks : 0;
    W.k = static_cast<const __nv_bfloat16*>(k);
    W.v = static_cast<const __nv_bfloat16*>(v);
    W.i_t = in[0], W.i_h = in[1];
    W.tok_seq = tok_seq;
    W.pos = pos;
    W.k_back = static_cast<__nv_bfloat16*>(k_back);
    W.v_back = static_cast<__nv_bfloat16*>(v_back);
    W.b_t = back[0], W.b_h = back[1];
    W.dev_status = dev_status;
    return launch_quant_write(quant_view(c), W, (cudaStream_t)stream);
}

dsmoe_status dsmoe_quant_cache_read(const dsmoe_quant_cache* cache, const dsmoe_quant_read_args* args, const int32_t* len, void* K_out, void* V_out,
                                    dsmoe_stream stream) {
    DSMOE_TRY(check_quant_cache(cache));
    if (!args) return DSMOE_ERR_INVALID_ARG;
    const dsmoe_quant_read_args& a = *args;
    const dsmoe_quant_cache& c = *cache;
    if (a.first < 0 || a.rows < 0 || (long long)a.first + a.rows > c.L) return DSMOE_ERR_INVALID_ARG;
    const int64_t n[3] = {c.n_seq, c.n_head, a.rows};
    DSMOE_TRY(check_rows(a.out_stride, n, 3, 8));
    if (a.rows == 0) return DSMOE_OK;
    if (!K_out || !V_out || !aligned16(K_out) || !aligned16(V_out)) return DSMOE_ERR_INVALID_ARG;
    if (!rows_apart(a.out_stride, n, c.d_head) || rows_meet(((intptr_t)V_out - (intptr_t)K_out) / 2, a.out_stride, n, c.d_head)) return DSMOE_ERR_INVALID_ARG;
    const QuantExtents held = quant_extents(c);
    if (held.meets(extent(K_out, a.out_stride, n, c.d_head, 2)) || held.meets(extent(V_out, a.out_stride, n, c.d_head, 2))) return DSMOE_ERR_INVALID_ARG;
    QuantRead R{};
    R.first = a.first, R.rows = a.rows;
    R.len = len;
    R.K = static_cast<__nv_bfloat16*>(K_out);
    R.V = static_cast<__nv_bfloat16*>(V_out);
    R.o_s = a.out_stride[0], R.o_h = a.out_stride[1], R.o_p = a.out_stride[2];
    return launch_quant_read(quant_view(c), R, (cudaStream_t)stream);
}

dsmoe_status dsmoe_quant_attention_workspace_size(const dsmoe_attention_desc* desc, size_t* bytes) {
    if (!desc || !bytes) return DSMOE_ERR_INVALID_ARG;
    const dsmoe_attention_desc d = quant_desc(*desc);
    DSMOE_TRY(check_attention(&d));
    *bytes = 0;
    if (d.T == 0) return DSMOE_OK;
    // (with and without sequence numbers)
    const QuantAttnPlan w = quant_attention_plan(view_of(d, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr));
    if (!w.fits) return DSMOE_ERR_UNSUPPORTED;
    *bytes = w.total;
    return DSMOE_OK;
}

dsmoe_status dsmoe_quant_attention(const dsmoe_attention_desc* desc, const dsmoe_quant_cache* cache, int window, int sinks, int rolling, const void* q,
                                   const int32_t* tok_seq, const int32_t* pos, void* out, float* lse, void* workspace, size_t ws_bytes,
                                   int32_t* dev_status, dsmoe_stream stream) {
    if (!desc) return DSMOE_ERR_INVALID_ARG;
    const dsmoe_attention_desc d = quant_desc(*desc);
    DSMOE_TRY(check_attention(&d));
    DSMOE_TRY(check_quant_cache(cache));
    const dsmoe_quant_cache& c = *cache;
    if (c.n_seq != d.n_seq || c.n_head != d.n_head || c.L != d.L || c.d_head != d.d_head) return DSMOE_ERR_INVALID_ARG;
    DSMOE_TRY(check_window(&d, window, sinks, rolling));
    if (d.T == 0) return DSMOE_OK;
    if (!q || !pos || !out || !aligned16(q) || !aligned16(out)) return DSMOE_ERR_INVALID_ARG;
    const int64_t n[3] = {d.T, d.n_head, d.group};
    const Extent o = extent(out, d.o_stride, n, d.d_head, 2);
    if (o.meets(extent(q, d.q_stride, n, d.d_head, 2)) || quant_extents(c).meets(o)) return DSMOE_ERR_INVALID_ARG;
    AttnView A = view_of(d, q, nullptr, nullptr, tok_seq, pos, out, lse, dev_status);
    // (the workspace is that of a window as wide as the cache)
    QuantAttnPlan w = quant_attention_plan(A);
    if (!w.fits) return DSMOE_ERR_UNSUPPORTED;
    if (!workspace || !aligned16(workspace) || ws_bytes < w.total) return DSMOE_ERR_WORKSPACE;
    A.window = window;
    A.sinks = sinks;
    A.ring = rolling ? d.L - sinks : 0;
    char* const ws = static_cast<char*>(workspace);
    cudaStream_t s = (cudaStream_t)stream;
    if (w.tiles) {
        const AttnView B = quant_copy_view(A, ws, w.copy);
        int4* const range = reinterpret_cast<int4*>(ws + w.range);
        DSMOE_TRY(launch_quant_range(A, range, s));
        QuantRead R{};
        R.rows = A.L;
        R.range = range;
        R.K = const_cast<__nv_bfloat16*>(B.K);
        R.V = const_cast<__nv_bfloat16*>(B.V);
        R.o_s = B.kv_s, R.o_h = B.kv_h, R.o_p = B.kv_p;
        DSMOE_TRY(launch_quant_read(quant_view(c), R, s));
        return attend(B, SharedKeys{}, w.attn, ws + w.rest, s);
    }
    w.plan.slots = reinterpret_cast<float*>(ws);
    w.plan.run_head = reinterpret_cast<int2*>(ws + w.run_head);
    return launch_quant_attention(A, quant_view(c), w.plan, s);
}

}  // extern "C"
