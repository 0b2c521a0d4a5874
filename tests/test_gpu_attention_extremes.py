"""The attention steps where a row's logits jump far, and where queries, keys or values are no numbers: each row's result is its own formula's, whatever the
rows, tiles and parts beside it hold (GPU required)."""
import numpy as np
import pytest
import torch

import cache_attention_reference as ref
from cache_attention_reference import Case
from test_gpu_attention_tiles import prompt
from test_gpu_prefix_attention import call as call_prefix, run as run_prefix
from test_gpu_tally_attention import run as run_tally
from test_gpu_window_attention import call as call_window, run

pytestmark = pytest.mark.gpu

LN2 = float(np.float32(np.log(2)))


def with_logits(c, base, peaks):
    """Logits of `base` and at the keys `peaks` of theirs, in base 2, give or take what the other columns add; values far below 1."""
    q, K = c.q.float().cpu(), c.K.float().cpu()
    q[..., 1:] *= 2.0 ** -5
    q[..., 0], K[..., 0] = 1.0, base
    for l, x in peaks.items():
        K[:, :, l, 0] = x
    c.q, c.K, c.V = q.to(torch.bfloat16).cuda(), K.to(torch.bfloat16).cuda(), c.V * 2.0 ** -10
    c.q_np, c.K_np, c.V_np = (x.float().cpu().numpy() for x in (c.q, c.K, c.V))
    return c


@pytest.mark.parametrize("jump", [40.0, 100.0, 125.5, 126.5, 127.5, 140.0])
@pytest.mark.parametrize("at", [50, 140, 200, 300])
def test_logits_that_jump_within_a_tile(jump, at):
    """In the first, the middle and the last tile of keys, and a second key of half the weight in the tile after it."""
    peaks = {at: jump, min(at + 130, 320): jump - 1}
    run(with_logits(Case(prompt(0, 383, 60), 1, 5, 64, 1, 384, seed=at, scale=LN2), 0.0, peaks), 2 ** 31 - 1)


@pytest.mark.parametrize("jump", [40.0, 100.0, 125.5, 126.5, 127.5, 140.0])
@pytest.mark.parametrize("at", [140, 200, 900])
def test_logits_that_jump_within_a_part(jump, at):
    """Keys in four parts, and another part whose largest logit was there from its first tile on."""
    c = Case(prompt(0, 1023, 60), 1, 5, 128, 1, 1024, seed=at, scale=LN2)
    run(with_logits(c, -100.0, {at: jump - 100, 600: jump - 97}), 2 ** 31 - 1)


def rows_of(c, call, want, bad):
    """Runs the call: rows that `bad` [T, n_head, group] marks are no numbers, and neither is their lse; the others are what is wanted."""
    call(c)
    got, lse = c.out.float().cpu().numpy(), c.lse.cpu().numpy()
    assert np.isnan(got[bad]).all() and np.isnan(lse[bad]).all()
    c.out[torch.from_numpy(bad).cuda()] = torch.from_numpy(want[0][bad]).bfloat16().cuda()
    c.lse[torch.from_numpy(bad).cuda()] = torch.from_numpy(want[1][bad]).float().cuda()
    c.check(want)
    assert c.status.item() == 0


# (a CTA's keys; a pair cut into parts; keys of a prompt in parts; beside a prefix on either kernel)
@pytest.mark.parametrize("tokens,L,P", [([(0, 150)], 160, 0), ([(0, 4000), (1, 300)], 4001, 0), (prompt(0, 1099, 60), 1100, 0),
                                        ([(0, 40), (1, 20)], 50, 300), ([(s, 40) for s in range(20)], 50, 1000)])
def test_queries_that_are_no_numbers(tokens, L, P):
    c = Case(tokens, 2, 5, 64, max(s for s, _ in tokens) + 1, L, P=P, seed=L + P)
    want = c.expected()
    bad = np.zeros((len(tokens), 2, 5), dtype=bool)
    bad[0, 1, 3] = bad[-1, 0, 0] = True
    for t, j, g in np.argwhere(bad):
        c.q[t, j, g, 7] = float("nan")
    rows_of(c, call_prefix if P else lambda c: call_window(c, 2 ** 31 - 1), want, bad)


@pytest.mark.parametrize("n,L", [(1, 6), (60, 6), (1, 700)])
def test_keys_that_are_no_numbers_beside_a_prefix(n, L):
    """All that a token sees of its own cache: its result is no number, although the prefix alone has one."""
    c = Case([(s, L - 1) for s in range(n)] + [(n, 2)], 1, 5, 64, n + 1, L, P=300, seed=n + L)
    want = c.expected()
    c.K[0, 0] = float("nan")
    bad = np.zeros((n + 1, 1, 5), dtype=bool)
    bad[0] = True
    rows_of(c, call_prefix, want, bad)


def test_keys_of_a_part_that_are_no_numbers():
    """A prompt whose keys lie in parts, all of one part's no numbers."""
    tokens = prompt(0, 1099, 60)
    c = Case(tokens, 1, 5, 64, 1, 1100, seed=3)
    want = c.expected()
    c.K[0, 0, :512] = float("nan")
    rows_of(c, lambda c: call_window(c, 2 ** 31 - 1), want, np.ones((60, 1, 5), dtype=bool))


@pytest.mark.parametrize("L", [384, 1024])
def test_keys_of_no_weight_before_values_that_are_no_numbers(L, monkeypatch):
    """Rows that are done again for a value that they do not see: their first keys have logits of -inf."""
    monkeypatch.setattr(ref, "visible", lambda p, w, k: [l for l in range(p + 1) if l % 128])
    tokens = prompt(0, L - 1, 50)
    c = Case(tokens, 1, 5, 64, 1, L, seed=L)
    c.q[..., 0] = c.q[..., 0].abs() + 1
    c.q_np = c.q.float().cpu().numpy()
    want = c.expected()
    c.K[0, 0, ::128, 0] = -float("inf")
    c.V[0, 0, L - 20, 5] = float("inf")
    call_window(c, 2 ** 31 - 1)
    sees = np.array([p >= L - 20 for _, p in tokens])
    assert (~np.isfinite(c.out.float().cpu().numpy()[sees][..., 5])).all()
    c.out[torch.from_numpy(sees).cuda(), :, :, 5] = torch.from_numpy(want[0][sees][..., 5]).bfloat16().cuda()
    c.check(want)
    assert c.status.item() == 0


@pytest.mark.parametrize("group", [1, 5, 33])
def test_tallies_of_keys_of_no_weight(group, monkeypatch):
    """Keys whose logits are -inf for all rows get nothing, in tiles that the rows do not fill too."""
    monkeypatch.setattr(ref, "visible", lambda p, w=None, k=0: [l for l in range(p + 1) if l not in (7, 130)])
    c = Case(prompt(0, 399, 100), 1, group, 64, 1, 400, seed=group)
    c.q[..., 0] = c.q[..., 0].abs() + 1
    c.q_np = c.q.float().cpu().numpy()
    c.K[0, 0, [7, 130], 0] = -float("inf")
    run_tally(c)
    want = c.expected()[4]
    assert (want[0, 0, [7, 130]] == 0).all()


# (a CTA's keys; a pair cut into parts; runs of warps; a prompt; keys of a prompt in parts; prefixes on either kernel)
@pytest.mark.parametrize("tokens,n_seq,L,P", [([(0, 150)], 1, 160, 0), ([(0, 4000), (1, 300)], 2, 4001, 0), ([(s % 2, 200) for s in range(1300)], 1300, 201, 0),
                                              (prompt(0, 383, 60), 1, 384, 0), (prompt(0, 1099, 60), 1, 1100, 0), ([(0, 40), (1, 20)], 2, 50, 700),
                                              ([(s, 40) for s in range(20)], 20, 50, 1000)])
@pytest.mark.parametrize("jump", [7.0, 31.0, 60.0, 120.0])
def test_values_far_above_1(tokens, n_seq, L, P, jump):
    """Values of about 2^100, whose weighted mean is a number of 32 bits, behind logits that grow by `jump`."""
    n_head = 1 if len(tokens) > 1000 else 2
    c = with_logits(Case(tokens, n_head, 2, 64, n_seq, L, P=P, seed=L, scale=LN2), 0.0, {l: jump * l / (L - 1) for l in range(0, L, 3)})
    c.V = (c.V.float() * 2.0 ** 110).to(torch.bfloat16)
    c.V_np = c.V.float().cpu().numpy()
    if P:
        c.Kp[..., 0] = torch.linspace(0, jump, P, device="cuda").bfloat16()
        c.Vp = (c.Vp.float() * 2.0 ** 100).to(torch.bfloat16)
        c.Kp_np, c.Vp_np = (x.float().cpu().numpy() for x in (c.Kp, c.Vp))
    run_prefix(c) if P else run(c, 2 ** 31 - 1)
