"""dsmoe_prefix_attention against a plain form in 64 bits (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import Case

pytestmark = pytest.mark.gpu


def call(c):
    desc = c.desc()
    ws = torch.empty(dm.dsmoe_attention_workspace_size(desc, dm.ATTENTION_PREFIX, c.P), dtype=torch.uint8, device="cuda")
    Kp, Vp = (c.Kp, c.Vp) if c.P else (c.K[0, :, :0], c.V[0, :, :0])
    dm.dsmoe_prefix_attention(desc, Kp, Vp, c.q, c.K, c.V, c.tok_seq, c.pos, c.out, c.lse, ws, c.status)
    torch.cuda.synchronize()


def run(c):
    call(c)
    c.check(c.expected())
    assert c.status.item() == 0


def beyond(tokens):
    last = {}
    for s, p in tokens:
        last[s] = max(last.get(s, -1), p)
    return lambda s, l: l > last.get(s, -1)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("group", [1, 5, 20])
def test_head_widths_and_groups(d, group):
    tokens = [(0, 0), (1, 33), (2, -1), (1, 34), (0, 15)]
    run(Case(tokens, 2, group, d, 3, 40, P=77, seed=d + group, hide=beyond(tokens)))


@pytest.mark.parametrize("P", [0, 1, 15, 16, 17, 64, 127, 128, 129, 1000, 4097])
@pytest.mark.parametrize("T", [1, 3, 26, 60])
def test_lengths(P, T):
    rng = np.random.default_rng(P + T)
    tokens = [(s, int(p)) for s, p in enumerate(rng.integers(-1, 90, T))]
    run(Case(tokens, 2, 5, 64, T, 90, P=P, seed=P + T, hide=beyond(tokens)))


def test_the_prefix_alone_and_the_own_cache_alone():
    run(Case([(0, -1), (0, -1)], 2, 5, 128, 1, 8, P=300, seed=1, hide=lambda s, l: True))
    run(Case([(0, 5), (0, -1)], 2, 5, 128, 1, 8, P=0, seed=1, hide=lambda s, l: l > 5))


def test_many_rows():
    """Several tiles of rows, tokens of one sequence among them, tokens that one launch does not list."""
    tokens = [(i // 3, 20 + i % 3) for i in range(300)]
    run(Case(tokens, 2, 5, 128, 100, 30, P=333, seed=2))
    run(Case([(i % 7, i % 40) for i in range(1200)], 1, 2, 64, 7, 40, P=100, seed=3))


def test_many_short_caches():
    """Runs of single warps that leave parts and whole rows, and the prefix's parts."""
    rng = np.random.default_rng(8)
    for n_head, P in ((8, 777), (16, 20)):
        tokens = [(s, int(p)) for s, p in enumerate(rng.integers(-1, 300, 160))]
        run(Case(tokens, n_head, 4, 64, 160, 300, P=P, seed=P))


def test_prompts_behind_a_prefix():
    tokens = [(0, p) for p in range(120)] + [(1, p) for p in range(40, 90)]
    run(Case(tokens, 2, 5, 128, 2, 128, P=200, seed=4, hide=beyond(tokens)))


def test_orders_in_memory():
    c = Case([(0, 9), (1, 3)], 4, 5, 96, 2, 10, P=50, seed=5, by_token=True, members_first=True)
    c.Kp, c.Vp = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.Kp, c.Vp))
    run(c)


def test_heavy_prefix_and_heavy_own_cache():
    """The larger maximum lies in the prefix, or in the own cache, by far."""
    for heavy in ("Kp", "K"):
        c = Case([(0, 30), (1, 12)], 2, 3, 64, 2, 31, P=40, seed=6)
        x, n = getattr(c, heavy), getattr(c, heavy + "_np")
        x *= 16
        n *= 16
        run(c)


def test_the_same_bits_every_time():
    c = Case([(s, 10 + s) for s in range(40)], 4, 5, 128, 40, 60, P=2000, seed=7)
    call(c)
    first, lse = c.out.clone(), c.lse.clone()
    for _ in range(3):
        c.out.zero_()
        call(c)
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
