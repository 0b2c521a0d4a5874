"""The attention steps on many rows that share their keys (the 128-row kernel): several tiles of rows and keys, parts, runs of several sequences,
values that are no numbers (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import Case, visible
from test_gpu_tally_attention import run as run_tally
from test_gpu_prefix_attention import run as run_prefix
from test_gpu_window_attention import call, run, unseen

pytestmark = pytest.mark.gpu


def prompt(s, last, n):
    return [(s, p) for p in range(last - n + 1, last + 1)]


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (128, 4), (200, 0), (31, 130), (1, 1)])
def test_prompts_of_several_tiles(d, window, sinks):
    """No context, a context before, and a window that begins and ends inside tiles of keys."""
    tokens = prompt(0, 299, 300)
    run(Case(tokens, 2, 5, d, 1, 300, seed=d, hide=unseen(tokens, window, sinks)), window, sinks)
    tokens = prompt(1, 700, 60)
    run(Case(tokens, 1, 5, d, 2, 701, seed=d + 1, hide=unseen(tokens, window, sinks)), window, sinks)


@pytest.mark.parametrize("group", [1, 2, 3, 7, 16, 17, 33, 64])
def test_groups_that_do_not_divide_a_tile(group):
    n = 2 * (256 // group) + 3
    run(Case(prompt(0, n + 40, n), 2, group, 64, 1, n + 41, seed=group), 50, 2)


def test_one_block_in_parts():
    """Few rows and many keys: every SM takes some of them; a window that leaves some parts without keys."""
    tokens = prompt(0, 4500, 40)
    run(Case(tokens, 1, 5, 128, 1, 4501, seed=1), 2 ** 31 - 1)
    run(Case(tokens, 1, 5, 128, 1, 4501, seed=2, hide=unseen(tokens, 300, 4)), 300, 4)


def test_runs_of_several_sequences():
    """Prompts beside decoding tokens, one sequence twice in a block, sequences that end in the middle of tiles, padding among them."""
    tokens = ([(s, 50 + s) for s in range(3)] + prompt(3, 99, 90) + [(4, 7)] + prompt(3, 60, 20) + [(0, -1)] * 5 + prompt(5, 30, 31)
              + [(s, 40) for s in range(6)] + prompt(1, 99, 9))
    for window, sinks in ((2 ** 31 - 1, 0), (20, 3)):
        run(Case(tokens, 2, 5, 128, 6, 100, seed=3, hide=unseen(tokens, window, sinks)), window, sinks)
    run_tally(Case(tokens, 2, 5, 64, 6, 100, seed=4))
    run_prefix(Case(tokens, 2, 5, 96, 6, 100, P=333, seed=5))


def test_runs_in_parts():
    """The tokens left to the other kernel and the keys cut into parts at once."""
    tokens = prompt(0, 2000, 20) + [(1, 1500)] + prompt(1, 1800, 12)
    run(Case(tokens, 1, 5, 64, 2, 2001, seed=6), 1500, 4)


def test_positions_in_no_order():
    rng = np.random.default_rng(7)
    tokens = [(0, int(p)) for p in rng.integers(-1, 400, 130)]
    run(Case(tokens, 2, 5, 64, 1, 400, seed=7), 60, 2)
    run(Case([(0, -1)] * 70, 1, 5, 64, 1, 40, seed=7, hide=lambda s, l: True), 60, 2)


@pytest.mark.parametrize("L", [1100, 1111, 1024 + 103])
def test_rolling_caches_with_prompts(L):
    """A ring that ends inside the window: the first tile, the last one, a stretch of a few keys."""
    for last in (1000, 1104, 1500, 3333, L + 60, L + 99):
        tokens = prompt(0, last, 100)
        window, sinks = 1000, 4
        if window + 99 > L - sinks:
            window = L - sinks - 99
        run(Case(tokens, 1, 5, 64, 1, L, seed=last), window, sinks, True)


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("members_first", [False, True])
def test_orders_in_memory(by_token, members_first):
    tokens = prompt(1, 150, 140)
    run(Case(tokens, 4, 5, 128, 2, 160, seed=8, by_token=by_token, members_first=members_first, hide=unseen(tokens, 99, 2)), 99, 2)


def test_strides_that_no_tensor_map_takes():
    """One head's cache for all heads, one sequence's for all."""
    c = Case(prompt(0, 99, 60), 3, 5, 64, 2, 100, seed=9)
    c.K_np[:], c.V_np[:] = c.K_np[:1, :1].copy(), c.V_np[:1, :1].copy()
    c.K, c.V = (x[:1, :1].contiguous().expand(2, 3, 100, 64) for x in (c.K, c.V))
    run(c, 40, 2)


def test_maxima_that_move():
    """Logits that grow with the position by far more than the sums' room, and fall."""
    for falls in (False, True):
        c = Case(prompt(0, 999, 60), 1, 5, 64, 1, 1000, seed=10, gain=1.0)
        ramp = torch.linspace(0.1, 30.0, 1000).view(1, 1, 1000, 1)
        ramp = ramp.flip(2) if falls else ramp
        c.K = (c.K.cpu().float() * ramp).to(torch.bfloat16).cuda()
        c.K_np = c.K.float().cpu().numpy()
        run(c, 2 ** 31 - 1)


@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_scales_that_are_not_positive(scale):
    run(Case(prompt(0, 300, 60), 1, 5, 64, 1, 301, seed=11, scale=scale), 250, 2)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 64])
def test_values_that_some_tokens_see_are_no_numbers(window):
    """A key and a value that only later tokens see: earlier ones are as if they were not there."""
    tokens = prompt(0, 399, 200)
    c = Case(tokens, 1, 5, 64, 1, 400, seed=12)
    want = c.expected(window, 1)
    c.V[0, 0, 333, 5] = float("inf")
    c.K[0, 0, 350, 7] = float("nan")
    call(c, window, 1)
    blind = np.array([333 not in visible(p, window, 1) and 350 not in visible(p, window, 1) for _, p in tokens])
    assert blind.sum() >= 133
    assert (~np.isfinite(c.out.float().cpu().numpy()[~blind])).any(axis=(1, 2, 3)).all()
    at = torch.from_numpy(np.flatnonzero(blind)).cuda()
    c.out, c.lse = c.out[at], c.lse[at]
    c.check([x[blind] for x in want[:4]])


def test_infinite_values_of_a_prefix_in_parts():
    """An infinite value behind weights of exactly zero."""
    c = Case([(s, 3) for s in range(40)], 1, 5, 64, 40, 8, P=3000, seed=13)
    run_prefix(c)


def test_long_prompts_against_the_other_kernel():
    """A large prompt at once, and its tokens a few at a time."""
    L = 2048
    c = Case(prompt(0, L - 1, L), 2, 5, 128, 1, L, seed=14)
    call(c, 700, 4)
    out, lse = c.out.clone(), c.lse.clone()
    for a in (0, 1, 700, 1500, L - 12):
        part = Case([(0, 0)], 2, 5, 128, 1, L, seed=14)
        part.K, part.V = c.K, c.V
        part.q, part.pos, part.tok_seq = c.q[a:a + 12].contiguous(), c.pos[a:a + 12].contiguous(), None
        part.out, part.lse = torch.zeros_like(part.q), torch.zeros((12, 2, 5), device="cuda")
        call(part, 700, 4)
        # two roundings to bf16 of values that differ by the weights' rounding
        assert torch.allclose(part.out.float(), out[a:a + 12].float(), rtol=2 ** -7, atol=0.03)
        assert torch.allclose(part.lse, lse[a:a + 12], rtol=0, atol=1e-4)


def test_the_same_bits_every_time_and_in_a_graph():
    tokens = prompt(0, 899, 200) + [(1, 20)] + prompt(2, 500, 130)
    c = Case(tokens, 4, 5, 128, 3, 900, seed=15)
    desc = c.desc()
    ws = torch.empty(dm.dsmoe_attention_workspace_size(desc, dm.ATTENTION_WINDOW), dtype=torch.uint8, device="cuda")

    def once(q, out, lse):
        dm.dsmoe_window_attention(desc, 300, 4, False, q, c.K, c.V, c.tok_seq, c.pos, out, lse, ws, c.status)
    once(c.q, c.out, c.lse)
    torch.cuda.synchronize()
    first, first_lse = c.out.clone(), c.lse.clone()
    flipped = c.q.flip(0).contiguous()
    outs = [torch.zeros_like(c.out) for _ in range(4)]
    for i, o in enumerate(outs):                       # without a wait between them
        once(flipped if i % 2 else c.q, o, c.lse)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[2], first) and torch.equal(outs[1], outs[3])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        once(c.q, c.out, c.lse)
        once(flipped, outs[0], c.lse)
    c.out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.out, first) and torch.equal(outs[0], outs[1])
    assert c.status.item() == 0


def test_offsets_beyond_32_bits():
    """Prompts at the end of a cache of more than 2^32 elements."""
    L, d = 17_000_000, 128
    K, V = (torch.empty((2, 1, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Case(prompt(1, 199, 60) + prompt(0, 150, 50), 1, 5, d, 2, 200, seed=16)
    K[:, :, -200:], V[:, :, -200:] = c.K, c.V
    want = c.expected(90, 0)
    c.K, c.V, c.pos = K, V, (c.pos + (L - 200)).to(torch.int32)
    call(c, 90, 0)
    c.check(want)
    assert c.status.item() == 0
