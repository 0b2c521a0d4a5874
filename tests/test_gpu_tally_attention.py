"""dsmoe_tally_attention against a plain form in 64 bits (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import Case, tally_tolerance

pytestmark = pytest.mark.gpu


def call(c, tally_in, tally_out):
    desc = c.desc()
    ws = torch.empty(dm.dsmoe_attention_workspace_size(desc, dm.ATTENTION_TALLY), dtype=torch.uint8, device="cuda")
    dm.dsmoe_tally_attention(desc, c.q, c.K, c.V, c.tok_seq, c.pos, c.out, c.lse, tally_in, tally_out, ws, c.status)
    torch.cuda.synchronize()


def run(c, how="apart", seed=0):
    shape = (c.n_seq, c.n_head, c.L)
    before = torch.rand(shape, generator=torch.Generator().manual_seed(seed)).cuda() * 3
    if how == "apart":
        tally_in, tally_out = before, torch.full(shape, 7.0, device="cuda")
    elif how == "same":
        tally_in = tally_out = before.clone()
    else:
        tally_in, tally_out, before = None, torch.full(shape, 7.0, device="cuda"), torch.zeros(shape, device="cuda")
    call(c, tally_in, tally_out)
    want = c.expected()
    c.check(want)
    b, added, error = before.cpu().numpy().astype(np.float64), want[4], want[5]
    rows = len(c.tokens) * c.group
    off = np.abs(tally_out.cpu().numpy() - (b + added)) - tally_tolerance(b, added, error, rows)
    assert off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    untouched = added == 0
    assert np.array_equal(tally_out.cpu().numpy()[untouched], before.cpu().numpy()[untouched])
    assert c.status.item() == 0
    return tally_out


def beyond(tokens):
    last = {}
    for s, p in tokens:
        last[s] = max(last.get(s, -1), p)
    return lambda s, l: l > last.get(s, -1)


@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("group", [1, 5, 17])
def test_head_widths_and_groups(d, group):
    tokens = [(0, 0), (1, 99), (2, -1), (1, 16), (0, 63)]
    run(Case(tokens, 2, group, d, 4, 100, seed=d + group, hide=beyond(tokens)))


@pytest.mark.parametrize("how", ["apart", "same", "none"])
@pytest.mark.parametrize("L", [1, 2, 16, 63, 64, 65, 200])
def test_lengths_and_places(how, L):
    tokens = [(s, p) for s, p in enumerate(sorted({0, L // 2, L - 1}))]
    run(Case(tokens, 2, 3, 64, 4, L, seed=L, hide=beyond(tokens)), how)


def test_prompts():
    tokens = [(0, p) for p in range(150)] + [(2, p) for p in range(30, 100)]
    run(Case(tokens, 2, 5, 128, 3, 150, seed=1, hide=beyond(tokens)))


def test_tokens_in_no_order():
    rng = np.random.default_rng(2)
    tokens = [(int(s), int(p)) for s, p in zip(rng.integers(0, 5, 1300), rng.integers(-1, 70, 1300))]
    run(Case(tokens, 1, 2, 32, 5, 70, seed=2))


@pytest.mark.parametrize("d", [64, 96, 128])
def test_long_prompts_and_several_sequences(d):
    """Parts of the rows, more tokens than are listed at a time, keys that the last tile's rows see in part."""
    run(Case([(0, p) for p in range(5, 305)], 1, 5, d, 1, 310, seed=d, hide=lambda s, l: l > 304))
    rng = np.random.default_rng(d)
    tokens = [(int(s), int(p)) for s, p in zip(rng.integers(0, 3, 1300), rng.integers(-1, 200, 1300))]
    run(Case(tokens, 2, 2, d, 4, 200, seed=d), "same")
    run(Case([(2, p) for p in range(1100)], 1, 1, d, 3, 1100, seed=d))
    run(Case([(s, p) for s in (1, 0) for p in range(100)], 2, 33, d, 2, 129, seed=d), "none")


def test_every_weight_is_counted_once():
    """Each row's weights add up to 1."""
    tokens = [(s, 1000 + 37 * s) for s in range(6)]
    c = Case(tokens, 4, 5, 128, 6, 1300, seed=3)
    got = run(c, "none").double().sum(-1)
    assert torch.allclose(got, torch.full_like(got, 5.0), rtol=0, atol=5 * 1e-5)


def test_no_token_hands_the_tallies_on():
    c = Case([(0, 3)], 2, 3, 64, 2, 30, seed=4)
    c.q, c.out, c.lse, c.tok_seq, c.pos = c.q[:0], c.out[:0], c.lse[:0], c.tok_seq[:0], c.pos[:0]
    before = torch.rand((2, 2, 30), device="cuda")
    after = torch.zeros_like(before)
    call(c, before, after)
    assert torch.equal(before, after)
    call(c, None, after)
    assert (after == 0).all()


def test_the_same_bits_every_time():
    c = Case([(s, 400 + s) for s in range(20)], 4, 5, 128, 20, 512, seed=5)
    a = run(c)
    b = run(c)
    assert torch.equal(a, b)
