"""dsmoe_cache_evict against a plain form (GPU required): what stays is exact, value by value."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import evict

pytestmark = pytest.mark.gpu


def tallies(kind, shape, rng):
    if kind == "spread":
        return rng.exponential(1.0, shape).astype(np.float32)
    if kind == "ties":                                   # a few values, zeros of both signs
        return rng.choice(np.array([0.0, -0.0, 0.5, 0.5, 2.0], dtype=np.float32), shape)
    if kind == "equal":
        return np.full(shape, 0.25, dtype=np.float32)
    t = rng.standard_normal(shape).astype(np.float32)    # anything: negative, not numbers, infinite, tiny
    flat = t.reshape(-1)
    for i, v in enumerate((np.nan, np.inf, -np.inf, 1e-42, -1e-42, 3.4e38)):
        flat[i::11] = v
    return t


def run(n_seq, n_head, L, d, keep, sinks, recent, lengths, kind="spread", how="apart", seed=0, by_token=False):
    rng = np.random.default_rng(seed)
    t_np = tallies(kind, (n_seq, n_head, L), rng)
    tally = torch.from_numpy(t_np).cuda()
    K, V = (torch.from_numpy(rng.standard_normal((n_seq, n_head, L, d)).astype(np.float32)).to(torch.bfloat16).cuda() for _ in range(2))
    if by_token:
        K, V = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (K, V))
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kept = torch.full((n_seq, n_head, keep), 77, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    K0, V0, t0 = K.clone(), V.clone(), tally.clone()
    if how == "apart":
        K_out, V_out = (torch.full((n_seq, n_head, keep + 3, d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        tally_out = torch.full((n_seq, n_head, keep + 2), 5.0, device="cuda")
        len_out = torch.full((n_seq,), 9, dtype=torch.int32, device="cuda")
    else:
        K_out, V_out, tally_out, len_out = K, V, tally, length
    before = [x.clone() for x in (K_out, V_out, tally_out)]
    desc = dm.make_attention_desc(None, K)
    ws = torch.empty(dm.dsmoe_evict_workspace_size(desc), dtype=torch.uint8, device="cuda")
    dm.dsmoe_cache_evict(desc, keep, sinks, recent, length, tally, K, V, kept, len_out, tally_out, K_out, V_out, ws, status)
    torch.cuda.synchronize()
    for s in range(n_seq):
        n = min(max(lengths[s], 0), L)
        for j in range(n_head):
            stay = evict(t_np[s, j], n, keep, sinks, recent)
            m = len(stay)
            assert kept[s, j].tolist() == stay + [-1] * (keep - m), (s, j)
            at = torch.tensor(stay, dtype=torch.long, device="cuda")
            for got, source, was in ((K_out, K0, before[0]), (V_out, V0, before[1]), (tally_out, t0, before[2])):
                assert torch.equal(got[s, j, :m].view(torch.int32 if got.dtype == torch.float32 else torch.int16),
                                   source[s, j][at].view(torch.int32 if got.dtype == torch.float32 else torch.int16)), (s, j)
                # rows behind the last that stays are as they were
                assert torch.equal(got[s, j, m:].contiguous().view(torch.int8), was[s, j, m:].contiguous().view(torch.int8)), (s, j)
        assert len_out[s].item() == min(n, keep)
    assert status.item() == (1 if any(not 0 <= n <= L for n in lengths) else 0)


@pytest.mark.parametrize("how", ["apart", "in place"])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "anything"])
@pytest.mark.parametrize("L,keep,sinks,recent", [(1, 1, 0, 0), (2, 1, 0, 1), (2, 1, 1, 0), (40, 17, 3, 5), (1000, 999, 0, 0), (1024, 512, 4, 100),
                                                 (1025, 300, 0, 0), (3000, 1500, 1, 1499), (3000, 2049, 700, 700), (2500, 1, 0, 0)])
def test_what_stays(how, kind, L, keep, sinks, recent):
    lengths = [L, max(0, L - 1), keep, min(L, keep + 1), 0]
    run(5, 2, L, 64, keep, sinks, recent, lengths, kind, how, seed=L + keep)


@pytest.mark.parametrize("how", ["apart", "in place"])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "anything"])
@pytest.mark.parametrize("L", [2048, 2049, 8192, 8193, 16384, 16385, 32768, 32769])
def test_lengths_at_which_the_kernel_changes(how, kind, L):
    run(2, 1, L, 32, L // 3, 3, 500, [L, L - 7], kind, how, seed=L)


@pytest.mark.parametrize("how", ["apart", "in place"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_widths(how, d):
    run(2, 3, 700, d, 345, 2, 40, [700, 513], "spread", how, seed=d)


@pytest.mark.parametrize("how", ["apart", "in place"])
def test_caches_by_position_and_long_ones(how):
    run(3, 4, 555, 128, 222, 4, 33, [555, 222, 400], "ties", how, by_token=True)
    run(2, 1, 70001, 32, 40000, 4, 256, [70001, 65536], "spread", how)


@pytest.mark.parametrize("how", ["apart", "in place"])
def test_lengths_outside_the_cache_are_reported(how):
    run(3, 2, 50, 64, 20, 1, 2, [51, -1, 50], "spread", how)


def test_in_a_graph_and_again():
    """Twice in place: the second call thins out what the first one left."""
    n_seq, n_head, L, d = 2, 2, 600, 64
    rng = np.random.default_rng(3)
    t = torch.from_numpy(tallies("spread", (n_seq, n_head, L), rng)).cuda()
    K, V = (torch.randn((n_seq, n_head, L, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    length = torch.tensor([600, 600], dtype=torch.int32, device="cuda")
    desc = dm.make_attention_desc(None, K)
    ws = torch.empty(dm.dsmoe_evict_workspace_size(desc), dtype=torch.uint8, device="cuda")
    saved = [x.clone() for x in (t, K, V, length)]
    kept = [torch.zeros((n_seq, n_head, keep), dtype=torch.int32, device="cuda") for keep in (400, 100)]

    def both():
        for k in kept:
            dm.dsmoe_cache_evict(desc, k.shape[2], 4, 50, length, t, K, V, k, length, t, K, V, ws)
    both()
    torch.cuda.synchronize()
    want = [x.clone() for x in (t[..., :100], K[:, :, :100], V[:, :, :100], length, *kept)]
    for x, y in zip((t, K, V, length), saved):
        x.copy_(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    g.replay()
    torch.cuda.synchronize()
    for x, y in zip((t[..., :100], K[:, :, :100], V[:, :, :100], length, *kept), want):
        assert torch.equal(x, y)
    assert length.tolist() == [100, 100]
    # the kept of the kept: indices into the first call's result
    first = kept[0][0, 0].long()
    for m in (0, 50, 99):
        assert torch.equal(K[0, 0, m], saved[1][0, 0, first[kept[1][0, 0, m]]])


@pytest.mark.parametrize("how", ["apart", "in place"])
def test_offsets_beyond_32_bits(how):
    """A cache of more than 2^32 elements: what stays lies at its end and at its beginning."""
    L, d, keep, recent = 17_000_000, 128, 40, 25
    K, V = (torch.zeros((2, 1, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tally = torch.zeros((2, 1, L), device="cuda")
    stay = [0, 5, 4000, 8_400_000, 8_500_000, 12_000_000, L - 40_000, L - 300] + list(range(L - 32, L))
    at = torch.tensor(stay, device="cuda")
    K[:, 0, at], V[:, 0, at] = (torch.randn((2, keep, d), device="cuda").bfloat16() for _ in range(2))
    want_K, want_V = K[:, 0, at].clone(), V[:, 0, at].clone()
    tally[:, :, at] = torch.rand((2, 1, keep), device="cuda") + 1
    want_tally = tally[:, :, at].clone()
    length = torch.tensor([L, L], dtype=torch.int32, device="cuda")
    kept = torch.zeros((2, 1, keep), dtype=torch.int32, device="cuda")
    K_out, V_out, tally_out = (K, V, tally) if how == "in place" else (torch.zeros_like(K[:, :, :keep]), torch.zeros_like(V[:, :, :keep]),
                                                                       torch.zeros((2, 1, keep), device="cuda"))
    desc = dm.make_attention_desc(None, K)
    ws = torch.empty(dm.dsmoe_evict_workspace_size(desc), dtype=torch.uint8, device="cuda")
    dm.dsmoe_cache_evict(desc, keep, 0, recent, length, tally, K, V, kept, length, tally_out, K_out, V_out, ws)
    torch.cuda.synchronize()
    assert kept[0, 0].tolist() == stay == kept[1, 0].tolist() and length.tolist() == [keep, keep]
    assert torch.equal(K_out[:, 0, :keep], want_K) and torch.equal(V_out[:, 0, :keep], want_V) and torch.equal(tally_out[..., :keep], want_tally)
