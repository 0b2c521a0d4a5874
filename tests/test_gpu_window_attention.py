"""dsmoe_window_attention against a plain form in 64 bits (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import Case, visible

pytestmark = pytest.mark.gpu


def call(c, window, sinks=0, rolling=False, desc=None, stream=None):
    desc = desc or c.desc()
    ws = torch.empty(dm.dsmoe_attention_workspace_size(desc, dm.ATTENTION_WINDOW), dtype=torch.uint8, device="cuda")
    dm.dsmoe_window_attention(desc, window, sinks, rolling, c.q, c.K, c.V, c.tok_seq, c.pos, c.out, c.lse, ws, c.status, stream=stream)
    torch.cuda.synchronize()


def run(c, window, sinks=0, rolling=False):
    call(c, window, sinks, rolling)
    c.check(c.expected(window, sinks, rolling))
    assert c.status.item() == 0


def unseen(tokens, window, sinks):
    """Whether no token of the call sees a slot of a cache of all positions."""
    seen = {(s, l) for s, p in tokens for l in visible(p, window, sinks)}
    return lambda s, l: (s, l) not in seen


@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("group", [1, 5, 8, 17])
def test_head_widths_and_groups(d, group):
    tokens = [(0, 0), (1, 99), (2, 37), (1, 16), (0, 15)]
    run(Case(tokens, 3, group, d, 3, 100, seed=d + group, hide=unseen(tokens, 30, 2)), 30, 2)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (1, 4), (2, 0), (15, 0), (16, 1), (17, 16), (64, 17), (333, 4), (334, 4), (1000, 0),
                                          (2 ** 31 - 1, 0), (5, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(window, sinks):
    """Windows that end inside units, that touch the sinks, that are as long as the cache and longer; sinks beyond the position."""
    tokens = [(0, p) for p in (0, 1, 3, 4, 5, 15, 16, 17, 63, 336, 337, 338, 339)] + [(1, 200), (1, 18)]
    run(Case(tokens, 2, 5, 64, 2, 340, seed=window % 1000 + sinks % 1000, hide=unseen(tokens, window, sinks)), window, sinks)


@pytest.mark.parametrize("window,sinks,L", [(8, 0, 8), (8, 4, 12), (8, 4, 13), (16, 1, 33), (30, 5, 77), (1, 0, 1), (1, 3, 4)])
def test_rolling_caches(window, sinks, L):
    """Positions far beyond the cache, at its first wrap, before it; a token per sequence."""
    room = L - sinks
    tokens = [(i, p) for i, p in enumerate([0, 1, window - 1, L - 1, L, L + 1, sinks + room * 3 - 1, sinks + room * 3, 1000, 2 ** 31 - 2])]
    c = Case(tokens, 2, 6, 96, len(tokens), L, seed=L)
    # (the reference lists positions: it is given the ones near the end)
    def seen(p, w, k):
        return sorted(set(range(max(0, p - w + 1), p + 1)) | set(range(min(k, p + 1))))
    import cache_attention_reference as ref
    plain, ref.visible = ref.visible, seen
    try:
        want = c.expected(window, sinks, True)
    finally:
        ref.visible = plain
    call(c, window, sinks, True)
    c.check(want)
    assert c.status.item() == 0


def test_several_tokens_of_a_rolling_cache():
    tokens = [(s, p) for s, last in ((0, 90), (1, 12), (2, 500)) for p in range(max(0, last - 6), last + 1)]
    run(Case(tokens, 4, 5, 128, 3, 40 + 3 + 6, seed=5), 40, 3, True)


def test_prompts():
    """Neighbouring tokens of prompts, one that continues a context."""
    tokens = [(0, p) for p in range(150)] + [(1, p) for p in range(70, 130)] + [(2, 0)]
    run(Case(tokens, 2, 5, 128, 3, 160, seed=9, hide=unseen(tokens, 50, 3)), 50, 3)


def test_rows_that_see_nothing():
    tokens = [(0, -1), (1, 40), (0, -1), (1, -1)]
    run(Case(tokens, 2, 3, 64, 2, 41, seed=3, hide=unseen(tokens, 1000, 0)), 1000)
    tokens = [(0, -1)] * 3
    run(Case(tokens, 2, 3, 64, 2, 41, seed=3, hide=lambda s, l: True), 7, 2)


def test_one_sequence_without_its_numbers():
    c = Case([(0, p) for p in (3, 17, 40)], 2, 5, 64, 1, 41, seed=4)
    c.tok_seq = None
    run(c, 20, 1)


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("members_first", [False, True])
def test_orders_in_memory(by_token, members_first):
    tokens = [(0, 55), (1, 30), (1, 31)]
    run(Case(tokens, 4, 5, 128, 2, 64, seed=6, by_token=by_token, members_first=members_first), 25, 2)


def test_caches_by_position_with_many_runs():
    """Two heads at a time: parts of both, groups of more than one tile, a prefix's tests beside it."""
    tokens = [(0, 1999), (1, 700), (2, -1), (1, 33)]
    for group in (5, 20):
        run(Case(tokens, 4, group, 128, 3, 2000, seed=16, by_token=True, hide=unseen(tokens, 1500, 4)), 1500, 4)
    run(Case([(s, 300 + s) for s in range(50)], 6, 5, 64, 50, 350, seed=17, by_token=True), 2 ** 31 - 1)


@pytest.mark.parametrize("by_token", [False, True])
def test_many_short_pairs(by_token):
    """As many pairs as warps and more: runs of single warps, some of which cut pairs in two; whole ones beside them; padding."""
    rng = np.random.default_rng(18)
    tokens = [(s, int(p)) for s, p in enumerate(rng.integers(-1, 400, 320))]
    run(Case(tokens, 4, 3, 64, 320, 400, seed=18, by_token=by_token), 2 ** 31 - 1)
    tokens = [(s % 40, 3000 - 7 * (s % 40)) for s in range(200)]
    run(Case(tokens, 8, 17, 32, 40, 3001, seed=19, by_token=by_token), 100, 4)


def test_parts_of_larger_tensors():
    """A slice of a larger cache, queries that are a slice and broadcast over the members, outputs with gaps that are left as they were."""
    c = Case([(0, 20), (1, 44)], 2, 4, 64, 2, 45, seed=7)
    K, V = (torch.full((3, 4, 60, 72), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[1:, 1:3, 5:50, 8:72], V[1:, 1:3, 5:50, 8:72] = c.K, c.V
    c.K, c.V = K[1:, 1:3, 5:50, 8:72], V[1:, 1:3, 5:50, 8:72]
    c.q_np[:] = c.q_np[:, :, :1]
    c.q = c.q[:, :, :1].contiguous().expand(2, 2, 4, 64)
    whole = torch.full((2, 2, 5, 96), 5.0, dtype=torch.bfloat16, device="cuda")
    c.out = whole[:, :, :4, 16:80]
    run(c, 18, 3)
    rest = whole.clone()
    rest[:, :, :4, 16:80] = 5.0
    assert (rest == 5.0).all()


def test_extreme_logits():
    """One key far above the others, all far below zero, scales of zero and below."""
    c = Case([(0, 63)], 1, 2, 64, 1, 64, seed=8, gain=200.0)
    run(c, 50, 2)
    for scale in (0.0, -0.3):
        run(Case([(0, 63), (0, 5)], 2, 2, 64, 1, 64, seed=8, scale=scale), 50, 2)


def test_many_tokens_and_long_runs():
    """More tokens than one launch lists, and keys of one token that are cut into many runs."""
    rng = np.random.default_rng(1)
    tokens = [(int(s), int(p)) for s, p in zip(rng.integers(0, 40, 1500), rng.integers(0, 60, 1500))]
    run(Case(tokens, 1, 2, 32, 40, 60, seed=10), 20, 1)
    run(Case([(0, 4095), (1, 77)], 1, 16, 64, 2, 4096, seed=11), 4000, 4)


def test_offsets_beyond_32_bits():
    """The last keys of a cache of more than 2^32 elements."""
    L, d = 17_000_000, 128
    K = torch.empty((2, 1, L, d), dtype=torch.bfloat16, device="cuda")
    V = torch.empty((2, 1, L, d), dtype=torch.bfloat16, device="cuda")
    c = Case([(1, 63), (0, 40)], 1, 5, d, 2, 64, seed=12)
    K[:, :, -64:], V[:, :, -64:] = c.K, c.V
    K[:, :, :4], V[:, :, :4] = c.K[:, :, :4], c.V[:, :, :4]
    want = c.expected(30, 0)
    far = c.pos + (L - 64)
    c.K, c.V, c.pos = K, V, far.to(torch.int32)
    run_desc = c.desc()
    call(c, 30, 0, desc=run_desc)
    c.check(want)


def test_positions_outside_the_cache_are_reported():
    for bad in ((0, 64), (0, -2), (2, 5), (-1, 5)):
        c = Case([(0, 10), bad], 2, 3, 64, 2, 64, seed=13)
        call(c, 20, 2)
        assert c.status.item() == 1
        first = Case([(0, 10)], 2, 3, 64, 2, 64, seed=13)
        assert np.isfinite(c.out.float().cpu().numpy()).all()
        c.out, c.lse, c.tokens, c.q_np = c.out[:1], c.lse[:1], c.tokens[:1], c.q_np[:1]
        c.check(c.expected(20, 2))
        del first


def test_the_same_bits_every_time_on_any_stream_and_in_a_graph():
    tokens = [(s, 300 + 20 * s) for s in range(8)] + [(7, 441 + i) for i in range(5)]
    c = Case(tokens, 4, 5, 128, 8, 500, seed=14)
    desc = c.desc()
    ws = torch.empty(dm.dsmoe_attention_workspace_size(desc, dm.ATTENTION_WINDOW), dtype=torch.uint8, device="cuda")

    def once(out, lse, q=c.q):
        dm.dsmoe_window_attention(desc, 200, 4, False, q, c.K, c.V, c.tok_seq, c.pos, out, lse, ws, c.status)
    once(c.out, c.lse)
    torch.cuda.synchronize()
    first, first_lse = c.out.clone(), c.lse.clone()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        once(c.out.fill_(0), c.lse)
    other.synchronize()
    assert torch.equal(c.out, first) and torch.equal(c.lse, first_lse)
    # two captured calls that share the workspace, replayed in turn
    graphs, outs = [], []
    flipped = c.q.flip(0).contiguous()
    for q in (c.q, flipped):
        out, lse = torch.zeros_like(c.out), torch.zeros_like(c.lse)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            once(out, lse, q)
        graphs.append(g)
        outs.append(out)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first)
    once(c.out, c.lse, flipped)
    torch.cuda.synchronize()
    assert torch.equal(outs[1], c.out)


@pytest.mark.parametrize("d", [64, 128, 160])
@pytest.mark.parametrize("T,keys", [(1, 1), (1, 192), (1, 193), (1, 210), (1, 384), (1, 394), (1, 410), (1, 2500), (7, 420), (7, 460), (20, 500),
                                    (20, 560), (40, 700), (73, 900), (75, 230), (80, 1000)])
def test_pairs_of_one_cta_and_pairs_cut_into_parts(T, keys, d):
    """Few pairs of few keys are a CTA's each; with more keys, or more pairs than SMs, they leave parts.  Tokens of one key and of none among them."""
    tokens = [(t, keys - 1 - 3 * t if t % 5 != 3 else [0, -1][t % 2]) for t in range(T)]
    run(Case(tokens, 2, 5, d, T, keys + 3, seed=T + keys, hide=unseen(tokens, 2 ** 31 - 1, 0)), 2 ** 31 - 1)
    run(Case(tokens, 2, 5, d, T, keys + 3, seed=T + keys, hide=unseen(tokens, keys // 2 + 1, 4), by_token=True), keys // 2 + 1, 4)


@pytest.mark.parametrize("d,group", [(64, 5), (128, 2), (32, 5)])
def test_the_last_positions_of_a_rolling_cache(d, group, monkeypatch):
    """A prompt that ends at the last position there is, on the 128-row tiles and on the streaming kernel; padding and a young token beside it."""
    import cache_attention_reference as ref
    monkeypatch.setattr(ref, "visible", lambda p, w, k: sorted(set(range(max(0, p - w + 1), p + 1)) | set(range(min(k, p + 1)))))
    last, window, sinks = 2 ** 31 - 2, 200, 3
    tokens = [(0, p) for p in range(last - 79, last + 1)] + [(0, -1), (1, -1), (1, 5), (2, last)]
    run(Case(tokens, 1, group, d, 3, window + 79 + sinks, seed=d), window, sinks, True)


def test_tokens_too_far_apart_for_a_rolling_cache(monkeypatch):
    """A young and an old token of one sequence, whose keys cannot all be in its ring: the call ends, reports it, and others have their results."""
    import cache_attention_reference as ref
    monkeypatch.setattr(ref, "visible", lambda p, w, k: sorted(set(range(max(0, p - w + 1), p + 1)) | set(range(min(k, p + 1)))))
    last, window, sinks = 2 ** 31 - 2, 60, 3
    tokens = [(0, p) for p in range(200, 240)] + [(1, 5), (1, last)] + [(2, p) for p in range(40)]
    c = Case(tokens, 1, 3, 64, 3, 110, seed=1)
    call(c, window, sinks, True)
    assert c.status.item() == 1
    want = c.expected(window, sinks, True)
    out, lse = torch.from_numpy(want[0]).bfloat16(), torch.from_numpy(want[1]).float()
    c.out[40:42], c.lse[40:42] = out[40:42].cuda(), lse[40:42].cuda()
    c.check(want)


def test_positions_that_are_none_are_reported():
    """Beyond the last one, and of a sequence that there is not: taken as the nearest, and reported."""
    c = Case([(0, 2 ** 31 - 1), (1, -2), (1, 7)], 2, 5, 64, 2, 40, seed=1)
    c.tok_seq[2] = 2
    call(c, 20, 3, True)
    assert c.status.item() == 1
    c.check(nearest(c))


def nearest(c):
    import cache_attention_reference as ref
    c.tokens = [(0, 2 ** 31 - 2), (1, -1), (1, 7)]
    plain, ref.visible = ref.visible, lambda p, w, k: sorted(set(range(max(0, p - w + 1), p + 1)) | set(range(min(k, p + 1))))
    try:
        return c.expected(20, 3, True)
    finally:
        ref.visible = plain
