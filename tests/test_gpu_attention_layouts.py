"""The attention steps on caches, queries and outputs in other orders and as parts of larger tensors, on each of their kernels; and infinite values that some rows
do not see, in caches and prefixes whose keys lie in parts (GPU required)."""
import numpy as np
import pytest
import torch

from cache_attention_reference import Case
from test_gpu_attention_tiles import prompt
from test_gpu_prefix_attention import call as call_prefix, run as run_prefix
from test_gpu_tally_attention import beyond, run as run_tally
from test_gpu_window_attention import call as call_window, run as run_window

pytestmark = pytest.mark.gpu

DECODING = [(0, 70), (1, 33), (2, -1), (3, 64)]
PROMPTS = prompt(0, 149, 60) + [(2, -1)] * 3 + prompt(3, 90, 41) + [(1, 5)]
BATCHES = {"decoding": DECODING, "prompts": PROMPTS, "one prompt": prompt(0, 140, 90)}


def spread(c):
    """Caches, queries and outputs as parts of larger tensors with gaps between rows, heads and tokens."""
    def part(x):
        whole = torch.full([n + 2 for n in x.shape[:-1]] + [x.shape[-1] + 16], 9.0, dtype=x.dtype, device=x.device)
        inner = whole[tuple([slice(1, -1)] * (x.dim() - 1) + [slice(8, -8)])]
        inner.copy_(x)
        return inner
    for name in ("K", "V", "q", "out"):
        setattr(c, name, part(getattr(c, name)))
    if c.P:
        c.Kp, c.Vp = part(c.Kp), part(c.Vp)
    return c


def batch(name, d, **kw):
    tokens = BATCHES[name]
    return Case(tokens, 4, 5, d, max(s for s, _ in tokens) + 1, 150, hide=None if kw.get("P") else beyond(tokens), **kw)


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("d", [64, 128, 160])
@pytest.mark.parametrize("order", ["by position", "members first", "both", "parts"])
def test_tallies(name, d, order):
    c = batch(name, d, seed=d, by_token=order in ("by position", "both"), members_first=order in ("members first", "both"))
    run_tally(spread(c) if order == "parts" else c)


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("d", [64, 96, 32])
@pytest.mark.parametrize("order", ["by position", "parts", "one head's for all", "one position's for all"])
def test_prefixes_behind_many_rows(name, d, order):
    """More than 32 rows; strides of 0 are no tensor map's, so that the prefix goes with the streaming kernel whatever the own caches' is."""
    c = batch(name, d, seed=d, P=300, by_token=order == "by position")
    if order == "by position":
        c.Kp, c.Vp = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.Kp, c.Vp))
    elif order == "parts":
        spread(c)
    else:
        one = (slice(0, 1), slice(None)) if order == "one head's for all" else (slice(None), slice(0, 1))
        c.Kp_np[:], c.Vp_np[:] = c.Kp_np[one].copy(), c.Vp_np[one].copy()
        c.Kp, c.Vp = (x[one].contiguous().expand(4, 300, d) for x in (c.Kp, c.Vp))
    run_prefix(c)


@pytest.mark.parametrize("order", ["by position", "parts"])
@pytest.mark.parametrize("n,d", [(1, 64), (3, 160), (60, 128), (60, 64)])
def test_rolling_caches(order, n, d):
    """Single tokens, a few and prompts, whose windows lie across the ring's end."""
    L, sinks = 190, 4
    tokens = [(s, p) for s, last in ((0, 185), (1, 340), (2, 1000)) for p in range(last - n + 1, last + 1)]
    c = Case(tokens, 2, 5, d, 3, L, seed=n + d, by_token=order == "by position")
    run_window(spread(c) if order == "parts" else c, L - sinks - n + 1, sinks, True)


@pytest.mark.parametrize("name", BATCHES)
def test_queries_that_all_members_share(name):
    c = batch(name, 64, seed=5)
    c.q_np[:] = c.q_np[:, :, :1].copy()
    c.q = c.q[:, :, :1].contiguous().expand(c.q.shape)
    run_tally(c)
    run_window(c, 40, 2)


def test_infinite_values_that_some_rows_of_split_keys_do_not_see():
    """A prompt whose keys lie in parts: rows that do not see the values are as without them, the others are no numbers in those columns alone."""
    tokens = prompt(0, 1099, 60)
    c = Case(tokens, 1, 5, 64, 1, 1100, seed=12)
    want = c.expected()
    c.V[0, 0, 1090, 5], c.V[0, 0, 1070, 9] = float("inf"), float("nan")
    call_window(c, 2 ** 31 - 1)
    got = c.out.float().cpu().numpy()
    bad = np.zeros(got.shape, dtype=bool)
    for t, (_, p) in enumerate(tokens):
        bad[t, ..., 5], bad[t, ..., 9] = p >= 1090, p >= 1070
    assert 0 < bad[..., 9].sum() < bad[..., 9].size and (~np.isfinite(got[bad])).all()
    c.out[torch.from_numpy(bad).cuda()] = torch.from_numpy(want[0][bad]).bfloat16().cuda()
    c.check(want)
    assert c.status.item() == 0


@pytest.mark.parametrize("n,P", [(40, 3000), (40, 100), (4, 3000)])
def test_infinite_values_of_a_prefix(n, P):
    """All rows see them: those columns are no numbers, the others are as without them."""
    c = Case([(s, s % 8 - 1) for s in range(n)], 2, 5, 64, n, 8, P=P, seed=13)
    want = c.expected()
    c.Vp[:, P - 3, 5], c.Vp[1, 7, 9] = float("inf"), float("-inf")
    call_prefix(c)
    got = c.out.float().cpu().numpy()
    bad = np.zeros(got.shape, dtype=bool)
    bad[..., 5], bad[:, 1, :, 9] = True, True
    assert (~np.isfinite(got[bad])).all()
    c.out[torch.from_numpy(bad).cuda()] = torch.from_numpy(want[0][bad]).bfloat16().cuda()
    c.check(want)
    assert c.status.item() == 0
