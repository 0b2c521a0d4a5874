"""dsmoe_quant_attention against a plain form in 64 bits (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import visible
from quant_cache_reference import QuantCase

pytestmark = pytest.mark.gpu

ALL = 2 ** 31 - 1


def call(c, window=ALL, sinks=0, rolling=False, stream=None, ws=None):
    cache = c.cache()
    desc = dm.make_quant_attention_desc(c.q, cache, c.scale, c.out)
    size = dm.dsmoe_quant_attention_workspace_size(desc)
    if ws is None:
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    dm.dsmoe_quant_attention(desc, cache, window, sinks, rolling, c.q, c.tok_seq, c.pos, c.out, c.lse, ws, c.status, stream=stream)
    torch.cuda.synchronize()


def run(c, window=ALL, sinks=0, rolling=False, prompt=False, seen_at=visible):
    """`prompt`: how the call is meant to be taken."""
    assert c.prompts() == prompt
    call(c, window, sinks, rolling)
    c.check(c.expected(window, sinks, rolling, seen_at))
    assert c.status.item() == 0


def unseen(tokens, window, sinks):
    """Whether no token of the call sees a slot of a cache of all positions."""
    seen = {(s, l) for s, p in tokens for l in visible(p, window, sinks)}
    return lambda s, l: (s, l) not in seen


@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("group", [1, 5, 8, 9, 16, 17, 64])
def test_head_widths_and_groups(d, group):
    tokens = [(0, 0), (1, 99), (2, 37), (1, 16), (0, 15)]
    run(QuantCase(tokens, 3, group, d, 3, 100, seed=d + group, hide=unseen(tokens, 40, 2)), 40, 2)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (1, 4), (2, 0), (31, 0), (32, 1), (33, 32), (64, 33), (333, 4), (334, 4), (1000, 0),
                                          (ALL, 0), (5, ALL), (ALL, ALL)])
def test_windows_and_sinks(window, sinks):
    """Windows that end inside units, that touch the sinks, that are as long as the cache and longer; sinks beyond the position."""
    tokens = [(0, p) for p in (0, 1, 3, 4, 5, 31, 32, 33, 63, 336, 337, 338, 339)] + [(1, 200), (1, 34)]
    run(QuantCase(tokens, 2, 5, 64, 2, 340, seed=window % 1000 + sinks % 1000, hide=unseen(tokens, window, sinks)), window, sinks)


@pytest.mark.parametrize("window,sinks,L", [(8, 0, 8), (8, 4, 12), (8, 4, 13), (32, 1, 65), (60, 5, 77), (1, 0, 1), (1, 3, 4), (100, 2, 111)])
def test_rolling_caches(window, sinks, L):
    """Positions far beyond the cache, at its first wrap, before it; a token per sequence."""
    room = L - sinks
    tokens = [(i, p) for i, p in enumerate([0, 1, window - 1, L - 1, L, L + 1, sinks + room * 3 - 1, sinks + room * 3, 1000, 2 ** 31 - 2])]

    def seen_at(p, w, k):                          # (positions near the end)
        return sorted(set(range(max(0, p - w + 1), p + 1)) | set(range(min(k, p + 1))))
    run(QuantCase(tokens, 2, 6, 96, len(tokens), L, seed=L), window, sinks, True, seen_at=seen_at)


@pytest.mark.parametrize("d,group", [(64, 6), (96, 6), (128, 5), (160, 3), (128, 16)])
@pytest.mark.parametrize("by_token", [False, True])
def test_prompts(d, group, by_token):
    """Neighbouring tokens of prompts, one that continues a context, two of few tokens; what none of them sees is anything."""
    tokens = [(0, p) for p in range(150)] + [(1, p) for p in range(70, 130)] + [(2, 0), (3, 158), (3, 159), (2, -1)]
    prompt = d <= 128                              # (wider heads are taken as single tokens)
    run(QuantCase(tokens, 8, group, d, 4, 160, seed=9, by_token=by_token, hide=unseen(tokens, 50, 3)), 50, 3, prompt=prompt)
    one = [(0, p) for p in range(300)]
    c = QuantCase(one, 4, group, d, 1, 310, seed=10, by_token=by_token, hide=unseen(one, ALL, 0))
    c.tok_seq = None
    run(c, prompt=prompt)


def test_prompts_of_rolling_caches():
    def seen_at(p, w, k):
        return sorted(set(range(max(0, p - w + 1), p + 1)) | set(range(min(k, p + 1))))
    tokens = [(s, p) for s, last in ((0, 190), (1, 62), (2, 2 ** 31 - 2)) for p in range(max(0, last - 59), last + 1)]
    run(QuantCase(tokens, 15, 5, 128, 3, 40 + 3 + 60, seed=5), 40, 3, True, prompt=True, seen_at=seen_at)
    few = [(s, p) for s, last in ((0, 90), (1, 12), (2, 500), (3, 2 ** 31 - 2)) for p in range(max(0, last - 30), last + 1)]
    run(QuantCase(few, 4, 5, 128, 4, 40 + 3 + 31, seed=6), 40, 3, True, seen_at=seen_at)


def test_rows_that_see_nothing():
    tokens = [(0, -1), (1, 40), (0, -1), (1, -1)]
    run(QuantCase(tokens, 2, 3, 64, 2, 41, seed=3, hide=unseen(tokens, 1000, 0)), 1000)
    run(QuantCase([(0, -1)] * 3, 2, 3, 64, 2, 41, seed=3, hide=lambda s, l: True), 7, 2)
    run(QuantCase([(0, -1)] * 40, 2, 3, 64, 2, 41, seed=3, hide=lambda s, l: True), 7, 2)
    run(QuantCase([(0, -1)] * 100, 42, 3, 64, 2, 41, seed=3, hide=lambda s, l: True), 7, 2, prompt=True)


def test_one_sequence_without_its_numbers():
    c = QuantCase([(0, p) for p in (3, 17, 40)], 2, 5, 64, 1, 41, seed=4)
    c.tok_seq = None
    run(c, 20, 1)


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("members_first", [False, True])
def test_orders_in_memory(by_token, members_first):
    tokens = [(0, 55), (1, 30), (1, 31)]
    run(QuantCase(tokens, 4, 5, 128, 2, 64, seed=6, by_token=by_token, members_first=members_first), 45, 2)


@pytest.mark.parametrize("d,group", [(128, 5), (64, 20), (96, 12), (256, 3)])
def test_long_caches_of_ragged_lengths(d, group):
    """Pairs that several CTAs share, pairs of one, padding."""
    tokens = [(0, 2999), (1, 700), (2, -1), (1, 33), (2, 1500)]
    run(QuantCase(tokens, 4, group, d, 3, 3000, seed=16, by_token=True, hide=unseen(tokens, 2500, 4)), 2500, 4)


@pytest.mark.parametrize("by_token", [False, True])
def test_many_short_pairs(by_token):
    """As many pairs as warps and more: runs of single warps, some of which cut pairs in two; whole ones beside them; padding; more tokens than a pass."""
    rng = np.random.default_rng(18)
    tokens = [(s, int(p)) for s, p in enumerate(rng.integers(-1, 400, 600))]
    run(QuantCase(tokens, 4, 3, 64, 600, 400, seed=18, by_token=by_token))
    tokens = [(s % 40, 3000 - 7 * (s % 40)) for s in range(300)]
    run(QuantCase(tokens, 8, 17, 32, 40, 3001, seed=19, by_token=by_token), 100, 4)


def test_one_long_pair_beside_many_short_ones():
    """600 tokens of two sequences: with heads of 64 taken as prompts, with heads of 32 as single tokens."""
    tokens = [(0, 20000)] + [(1, i % 5) for i in range(1, 600)]
    run(QuantCase(tokens, 2, 2, 64, 2, 20001, seed=20), prompt=True)
    run(QuantCase(tokens, 2, 2, 32, 2, 20001, seed=20))


def test_parts_of_larger_tensors():
    """Rows of a larger cache, queries that are broadcast over the members, outputs with gaps that are left as they were."""
    c = QuantCase([(0, 20), (1, 44)], 2, 4, 64, 2, 45, seed=7)
    held = []
    for x in (c.K, c.V, c.K_scale, c.V_scale):
        big = torch.full((3, 4, 60, 2 * x.shape[3]), 9, dtype=x.dtype, device="cuda")
        part = big[1:, 1:3, 5:50, x.shape[3]:]
        part.copy_(x)
        held.append(part)
    c.K, c.V, c.K_scale, c.V_scale = held
    q = c.q[:, :, :1].contiguous()
    c.q, c.q_np = q.expand(2, 2, 4, 64), np.repeat(c.q_np[:, :, :1], 4, 2)
    out = torch.full((2, 2, 4, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    c.out = out[..., 16:]
    run(c, 30, 1)
    assert bool((out[..., :16] == 7.0).all())


@pytest.mark.parametrize("gain,value_gain,scale", [(0.0, 1.0, None), (2.0, 1.0, 0.0), (2.0, 1.0, -0.3), (300.0, 1.0, None), (2.0, 2.0 ** 96, None), (2.0, 2.0 ** -120, None),
                                                   (2.0 ** 60, 1.0, 2.0 ** -60), (2.0 ** -60, 1.0, 2.0 ** 60)])
def test_magnitudes(gain, value_gain, scale):
    """Equal logits, negative scales, logits that let one key win, values and queries far from 1."""
    tokens = [(0, 400), (1, 77)]
    c = QuantCase(tokens, 2, 5, 128, 2, 401, seed=8, gain=gain, value_gain=value_gain, scale=scale)
    run(c)


def test_keys_and_values_that_are_no_numbers():
    """A row that sees one is none; others are as they were."""
    for name in ("K_scale", "V_scale"):
        c = QuantCase([(0, 100), (0, 40), (1, 90)], 2, 5, 128, 2, 101, seed=11)
        want = c.expected()
        getattr(c, name)[0, 1, 70, 2] = float("nan")
        call(c)
        assert bool(c.out[0, 1].isnan().all()) if name == "K_scale" else bool(c.out[0, 1, :, 64:96].isnan().all())
        keep = torch.ones_like(c.out, dtype=torch.bool)
        keep[0, 1] = False
        ok = np.abs(c.out.double().cpu().numpy() - want[0]) <= want[2]
        assert ok[keep.cpu().numpy()].all()
    c = QuantCase([(0, 100), (0, 40)], 2, 5, 128, 2, 101, seed=12)
    want = c.expected()
    c.q[0, 1, 3, 7] = float("nan")
    call(c)
    assert bool(c.out[0, 1, 3].isnan().all())
    got = np.abs(c.out.double().cpu().numpy() - want[0]) <= want[2]
    got[0, 1, 3] = True
    assert got.all()


def test_out_of_range():
    """Clamped and reported, as by the other attention steps."""
    for n, n_head in ((1, 2), (30, 2), (150, 30)):
        tokens = [(0, 30)] * n + [(5, 20), (-1, 3), (1, 100), (0, -7)]
        c = QuantCase([(0, 30)] * n + [(1, 20), (0, 3), (1, 40), (0, -1)], n_head, 5, 64, 2, 41, seed=13)
        assert c.prompts() == (n == 150)
        c.tok_seq = torch.tensor([s for s, _ in tokens], dtype=torch.int32, device="cuda")
        c.pos = torch.tensor([p for _, p in tokens], dtype=torch.int32, device="cuda")
        call(c)
        c.check(c.expected())
        assert c.status.item() == 1


def test_same_results_every_time_and_on_another_stream():
    for tokens in ([(s, 1000 + 77 * s) for s in range(9)], [(0, p) for p in range(200)] + [(1, p) for p in range(300, 500)]):
        c = QuantCase(tokens, 4, 5, 128, 9, 2000, seed=14)
        assert c.prompts() == (len(tokens) > 9)
        call(c, 900, 4)
        first, lse = c.out.clone(), c.lse.clone()
        for i in range(3):
            c.out.fill_(7.0)
            c.lse.fill_(7.0)
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            call(c, 900, 4, stream=stream)
            assert torch.equal(c.out, first) and torch.equal(c.lse, lse)


def test_without_lse_and_status():
    c = QuantCase([(0, 50), (1, 20)], 2, 5, 128, 2, 64, seed=15)
    want = c.expected()
    cache = c.cache()
    desc = dm.make_quant_attention_desc(c.q, cache, c.scale)
    ws = torch.empty(dm.dsmoe_quant_attention_workspace_size(desc), dtype=torch.uint8, device="cuda")
    dm.dsmoe_quant_attention(desc, cache, ALL, 0, False, c.q, c.tok_seq, c.pos, c.out, None, ws)
    assert (np.abs(c.out.double().cpu().numpy() - want[0]) <= want[2]).all()


@pytest.mark.parametrize("far", [2.0 ** 96, 2.0 ** 12, 2.0 ** -12, 2.0 ** -96])
def test_values_of_magnitudes_far_apart(far):
    """Keys whose values are far larger than others', with weights so small that both count; or far smaller, with weights so large."""
    from cache_attention_reference import attention
    from quant_cache_reference import quant_logit_error, quant_out_tolerance, quantise, tensors, values
    rng = np.random.default_rng(21)
    n, d, L = 500, 128, 777
    c = QuantCase([(0, n - 1)], 1, 3, d, 1, L, seed=21)
    c.q_np[:, :, :] = c.q_np[:, :, :1]                                   # members alike, so that a key's weight is as small for all
    c.q = torch.from_numpy(c.q_np).to(torch.bfloat16).cuda()
    q = c.q_np[0, 0, 0]
    K, V = rng.standard_normal((1, 1, L, d)), rng.standard_normal((1, 1, L, d))
    at = [5, 40, 41, 100, 333] + list(range(400, 440))
    rare = np.zeros(L, dtype=bool)
    rare[at] = True
    K[0, 0, rare] = q * -np.log(far) / (c.scale * (q @ q))
    kc, ks = quantise(K)
    # by what the keys have become: values in the opposite proportion of the weights
    logit = c.scale * (values(kc, ks)[0, 0] @ q)
    V[0, 0, rare] *= np.exp(np.log(np.exp(logit[:n][~rare[:n]]).sum()) - logit[rare] - 3.0)[:, None]
    V = torch.from_numpy(V).to(torch.bfloat16).double().numpy()
    vc, vs = quantise(V)
    (c.K, c.K_scale), (c.V, c.V_scale) = tensors(kc, ks), tensors(vc, vs)
    K, V = values(kc, ks)[0, 0, :n], values(vc, vs)[0, 0, :n]
    want, lse, weight, absolute, spread = attention(c.q_np[0, 0], K, V, c.scale, np.arange(n))
    rare = rare[:n]
    error = quant_logit_error(c.q_np[0, 0], c.scale, ks[0, 0, :n], spread, d)
    # (what products of less than 2^-14 lose is beside the weights of the keys of one kind, in units of their own scales)
    tol = quant_out_tolerance(want, absolute, error, False, 0, 0.0)
    tol += sum(n * 2.0 ** -31 * 14 * vs[0, 0, :n][kind].max() * weight[:, kind].max() for kind in (rare, ~rare))
    part = V.copy()
    part[~rare] = 0.0
    part = attention(c.q_np[0, 0], K, part, c.scale, np.arange(n))[0]
    assert (np.abs(part).max(-1) > 0.1 * np.abs(want).max(-1)).all() and (np.abs(want - part).max(-1) > 0.1 * np.abs(want).max(-1)).all()
    call(c)
    got = c.out.double().cpu().numpy()[0, 0]
    assert (np.abs(want) > 10 * tol).mean() > 0.5                        # (the tolerance says something)
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    assert (np.abs(c.lse.double().cpu().numpy()[0, 0] - lse) <= error + 1e-4).all()


def test_scales_that_a_writer_never_leaves():
    """Zero bytes, scales below zero, of eight significant bits, of the smallest numbers: values as they read back."""
    from cache_attention_reference import attention
    rng = np.random.default_rng(22)
    n, d = 300, 96
    c = QuantCase([(0, n - 1), (1, n - 1)], 2, 4, d, 2, n, seed=22)
    c.V[0, :, 40:60], c.V_scale[0, :, 40:60] = 0, 0
    c.V_scale[0, :, 100:140, 1] *= -1
    c.V_scale[1] *= torch.from_numpy(rng.uniform(1, 1.9, c.V_scale[1].shape)).cuda().to(torch.bfloat16)
    c.V_scale[1, :, 200:] *= 2.0 ** -100
    cache = c.cache()
    V = torch.empty((2, 2, n, d), dtype=torch.bfloat16, device="cuda")
    dm.dsmoe_quant_cache_read(cache, None, torch.empty_like(V), V)
    call(c)
    V = V.double().cpu().numpy()
    for t in range(2):
        for j in range(2):
            o, _, _, absolute, _ = attention(c.q_np[t, j], c.values_np[0][t, j], V[t, j], c.scale, np.arange(n))
            # (scales of eight bits: the values that are read back are rounded once more, by 2^-8)
            assert (np.abs(c.out.double().cpu().numpy()[t, j] - o) <= 2.0 ** -8 * 1.01 * np.abs(o) + absolute * (2.0 ** -8 + 2.0 ** -8)).all()


@pytest.mark.parametrize("T,L,prompt", [(3, 400, False), (90, 1500, True)])
def test_offsets_beyond_32_bits(T, L, prompt):
    """The same keys at the end of a cache whose codes, and whose copies in 16 bits, reach beyond 2^32 bytes: as at that of a short one."""
    n_seq, n_head, d, room = 3, 8, 128, 2_900_000
    tokens = [(t % n_seq, L - 1 - t // n_seq) if not prompt else (t // 30, L - 30 + t % 30) for t in range(T)]
    c = QuantCase(tokens, n_head, 5, d, n_seq, L, seed=23)
    want = c.expected(200, 0)
    assert c.prompts() == prompt and n_seq * n_head * room * d // 2 > 2 ** 32
    for name in ("K", "V", "K_scale", "V_scale"):
        x = getattr(c, name)
        wide = torch.full((n_seq, n_head, room, x.shape[3]), 0 if x.dtype == torch.uint8 else float("nan"), dtype=x.dtype, device="cuda")
        wide[:, :, room - L:] = x
        setattr(c, name, wide)
    c.pos += room - L
    c.L = room
    assert c.prompts() == prompt
    call(c, 200, 0)
    c.check(want)
    assert c.status.item() == 0
