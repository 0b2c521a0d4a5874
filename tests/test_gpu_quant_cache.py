"""dsmoe_quant_cache_write and dsmoe_quant_cache_read against plain forms (GPU required).  Both are exact: codes, scales and values are equal."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from quant_cache_reference import GROUP, pack, quantise, scales_of, slot_of, tensors, unpack, values

pytestmark = pytest.mark.gpu


def empty(n_seq, n_head, L, d, by_token=False):
    """A cache whose bytes are all 0x5a, and its four tensors."""
    def make(last, dtype):
        shape = (n_seq, L, n_head, last) if by_token else (n_seq, n_head, L, last)
        x = torch.full((*shape[:-1], last * dtype.itemsize), 0x5a, dtype=torch.uint8, device="cuda").view(dtype)
        return x.transpose(1, 2) if by_token else x
    held = [make(d // 2, torch.uint8), make(d // 2, torch.uint8), make(scales_of(d), torch.bfloat16), make(scales_of(d), torch.bfloat16)]
    return dm.make_quant_cache(*held), held


def bf16(rng, *shape, by=1.0):
    x = torch.from_numpy((rng.standard_normal(shape) * by).astype(np.float32)).to(torch.bfloat16)
    return x.cuda(), x.double().numpy()


def same(a, b):
    """Equal bit for bit, but for the kind of a NaN."""
    a, b = np.asarray(a, dtype=np.float64), np.asarray(b, dtype=np.float64)
    return np.array_equal(a, b, equal_nan=True)


def written(held, rows, d):
    """Codes and scales of rows (sequence, slot) of K and V: [rows, n_head, d] and [rows, n_head, d / 32]."""
    got = []
    for codes, scales in ((held[0], held[2]), (held[1], held[3])):
        at = [torch.tensor(x, device="cuda") for x in zip(*rows)]
        got.append((unpack(codes[at[0], :, at[1]].cpu().numpy()), scales[at[0], :, at[1], : d // GROUP].double().cpu().numpy()))
    return got


def untouched(held, rows, d):
    for x, dtype in zip(held, (torch.uint8, torch.uint8, torch.bfloat16, torch.bfloat16)):
        x = x.clone()
        groups = d // GROUP if dtype is torch.bfloat16 else x.shape[3]
        for s, l in rows:
            x[s, :, l, :groups] = torch.full((groups * dtype.itemsize,), 0x5a, dtype=torch.uint8, device="cuda").view(dtype)
        if not bool((x.contiguous().view(torch.uint8) == 0x5a).all()):
            return False
    return True


def check(held, k_np, v_np, rows, live, d):
    for (code, scale), x in zip(written(held, [rows[t] for t in live], d), (k_np, v_np)):
        want, s = quantise(x[live])
        assert np.array_equal(code, want) and same(scale, s)
    assert untouched(held, [rows[t] for t in live], d)


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_tokens_are_written_and_come_back(d, by_token):
    rng = np.random.default_rng(d)
    n_seq, n_head, L, T = 3, 5, 37, 23
    cache, held = empty(n_seq, n_head, L, d, by_token)
    k, k_np = bf16(rng, T, n_head, d)
    v, v_np = bf16(rng, T, n_head, d, by=100.0)
    rows = [(int(i) % n_seq, int(i) // n_seq) for i in rng.permutation(n_seq * L)[:T]]
    seq, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*rows))
    back = [torch.full_like(k, 3.0) for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dm.dsmoe_quant_cache_write(cache, k, v, seq, pos, k_back=back[0], v_back=back[1], dev_status=status)
    check(held, k_np, v_np, rows, range(T), d)
    for b, x in zip(back, (k_np, v_np)):
        assert same(b.double().cpu().numpy(), values(*quantise(x)))
    # the same rows by reading, pieces of them, and what is not there
    out = [torch.full((n_seq, n_head, L, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dm.dsmoe_quant_cache_read(cache, None, *out)
    for t, (s, l) in enumerate(rows):
        assert torch.equal(out[0][s, :, l], back[0][t]) and torch.equal(out[1][s, :, l], back[1][t])
    for first, n, length in ((5, 9, [37, 5, 11]), (36, 1, [0, 37, 100]), (0, 37, [-3, 1, 36]), (7, 0, [1, 1, 1])):
        part = [torch.full((n_seq, n_head, n, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        dm.dsmoe_quant_cache_read(cache, torch.tensor(length, dtype=torch.int32, device="cuda"), *part, first=first)
        for p, whole in zip(part, out):
            for s in range(n_seq):
                m = min(max(length[s] - first, 0), n)
                assert torch.equal(p[s, :, :m], whole[s, :, first:first + m]) and bool((p[s, :, m:] == 9.0).all())
    assert status.item() == 0


def test_any_bytes_are_read_as_they_are():
    """All bytes in all places, scales of any kind."""
    rng = np.random.default_rng(1)
    code = rng.integers(-8, 8, (2, 3, 50, 96))
    scale = np.exp2(rng.integers(-133, 119, (2, 3, 50, 3)).astype(float)) * rng.integers(1, 16, (2, 3, 50, 3))
    scale[0, 0, 0] = [np.nan, 0.0, -1.5]
    K, Ks = tensors(code, scale)
    V, Vs = tensors(code[::-1].copy(), scale[::-1].copy())
    assert same(Ks[..., :3].double().cpu().numpy(), scale)
    out = [torch.empty((2, 3, 50, 96), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dm.dsmoe_quant_cache_read(dm.make_quant_cache(K, V, Ks, Vs), None, *out)
    assert same(out[0].double().cpu().numpy(), values(code, scale)) and same(out[1].double().cpu().numpy(), values(code, scale)[::-1])


def test_values_at_borders():
    """Quotients that are halves and largest values that are sevenfold scales, at all magnitudes; zeros of both signs, the smallest numbers and the
    largest, and groups with values that are no numbers."""
    rng = np.random.default_rng(2)
    T, d = 600, 64
    scale = rng.integers(8, 16, (T, 1, 2, 1)) * np.exp2(rng.integers(-128, 117, (T, 1, 2, 1)).astype(float))
    half = rng.integers(-14, 15, (T, 1, 2, GROUP)) / 2.0
    x = half * scale
    x[::2, :, :, 0] = 7 * scale[::2, :, :, 0]                  # the scale is what it is taken to be: halves stay halves
    x[1::3] += rng.integers(-3, 4, x[1::3].shape) * scale[1::3] / 16
    x = x.reshape(T, 1, d)
    x[5] = 0.0
    x[6, 0, ::2] = -0.0
    x[7] = 2.0 ** -133 * rng.integers(-127, 128, d)            # below the smallest normal number
    x[8] = 3.3895313892515355e38 * rng.choice([-1, 1, 0.5], d)
    x[9, 0, 3], x[10, 0, 40], x[11, 0, 33] = np.nan, np.inf, -np.inf
    k = torch.from_numpy(x).to(torch.bfloat16).cuda()
    x = k.double().cpu().numpy()
    cache, held = empty(1, 1, T, d)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    back = torch.empty_like(k)
    dm.dsmoe_quant_cache_write(cache, k, k, None, pos, k_back=back)
    check(held, x, x, [(0, t) for t in range(T)], list(range(T)), d)
    code, sc = quantise(x)
    assert same(back.double().cpu().numpy(), values(code, sc))
    fine = np.isfinite(x).reshape(T, 1, 2, GROUP).all(-1)
    assert np.isnan(back.double().cpu().numpy().reshape(T, 1, 2, GROUP)[~fine]).all() and (~fine).sum() == 3
    # no value is off by more than half a scale (of more than 2^122 some are)
    off = np.abs(values(code, sc) - x).reshape(T, 1, 2, GROUP)
    small = fine & (sc < 2.0 ** 122) & (sc > 0)
    assert (off[small].max(-1) <= sc[small] / 2).all()


def test_padding_and_tokens_out_of_range():
    rng = np.random.default_rng(3)
    rows = [(0, 4), (1, -1), (2, 1), (-1, 2), (1, 20), (0, -2), (1, 19), (0, 0), (2 ** 31 - 1, 0), (0, 2 ** 31 - 1)]
    live = [0, 6, 7]
    cache, held = empty(2, 2, 20, 64)
    k, k_np = bf16(rng, len(rows), 2, 64)
    v, v_np = bf16(rng, len(rows), 2, 64)
    seq, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*rows))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    back = torch.full_like(k, 3.0)
    dm.dsmoe_quant_cache_write(cache, k, v, seq, pos, v_back=back, dev_status=status)
    check(held, k_np, v_np, rows, live, 64)
    assert status.item() == 1
    dead = [t for t in range(len(rows)) if t not in live]
    assert bool((back[dead] == 3.0).all()) and same(back[live].double().cpu().numpy(), values(*quantise(v_np[live])))
    # padding alone is no mistake
    status.zero_()
    dm.dsmoe_quant_cache_write(cache, k[:2], v[:2], seq[:2], pos[:2], dev_status=status)
    assert status.item() == 0
    dm.dsmoe_quant_cache_write(cache, k[:0], v[:0], None, pos[:0], dev_status=status)


@pytest.mark.parametrize("sinks,L", [(0, 8), (3, 11), (1, 40), (4, 5)])
def test_rolling_caches(sinks, L):
    """Single tokens far on, and prompts of several lengths of the ring, of which the latest stay."""
    rng = np.random.default_rng(L)
    ring, d, n_head = L - sinks, 128, 2
    starts = [0, sinks, L - 1, 1000, 2 ** 31 - 1 - 3 * ring]
    n = 3 * ring
    tokens = [(s, p0 + i) for s, p0 in enumerate(starts) for i in range(n)]
    cache, held = empty(len(starts), n_head, L, d)
    k, k_np = bf16(rng, len(tokens), n_head, d)
    v, v_np = bf16(rng, len(tokens), n_head, d)
    seq, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*tokens))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    back = torch.zeros_like(k)
    dm.dsmoe_quant_cache_write(cache, k, v, seq, pos, sinks, True, k_back=back, dev_status=status)
    last = {}
    for t, (s, p) in enumerate(tokens):
        last[s, slot_of(p, L, sinks, True)] = t
    rows = [(s, slot_of(p, L, sinks, True)) for s, p in tokens]
    check(held, k_np, v_np, rows, sorted(last.values()), d)
    assert same(back.double().cpu().numpy(), values(*quantise(k_np))) and status.item() == 0


def test_parts_of_larger_tensors():
    """Keys and values as they lie beside the queries, rows of a larger cache with gaps between them that are left as they were."""
    rng = np.random.default_rng(4)
    T, n_head, d, L = 17, 3, 96, 30
    both, both_np = bf16(rng, T, 4, n_head, d)
    k, v = both[:, 1], both[:, 3]
    codes = [torch.full((5, L + 9, n_head + 2, 80), 0x5a, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((5, L + 9, n_head + 2, 16), 0x5a, dtype=torch.uint8, device="cuda").view(torch.bfloat16) for _ in range(2)]
    part = [x[1:4, 4:4 + L, 2:].transpose(1, 2)[..., : x.shape[3] * w // 80] for x, w in zip((*codes, *scales), (48, 48, 40, 40))]
    cache = dm.make_quant_cache(*part)
    rows = [(t % 3, 29 - t) for t in range(T)]
    seq, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*rows))
    back = [torch.full((T, n_head, 2, d + 8), 3.0, dtype=torch.bfloat16, device="cuda")[:, :, i, 8:] for i in range(2)]
    dm.dsmoe_quant_cache_write(cache, k, v, seq, pos, k_back=back[0], v_back=back[1])
    check(part, both_np[:, 1], both_np[:, 3], rows, range(T), d)
    for x in codes + scales:
        x = x.view(torch.uint8).clone()
        wide = 48 if x.shape[3] == 80 else 6
        x[1:4, 4:4 + L, 2:, :wide] = 0x5a
        assert bool((x == 0x5a).all())
    out = torch.full((3, L, n_head, 2, d + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    dm.dsmoe_quant_cache_read(cache, None, out[..., 0, 8:].transpose(1, 2), out[..., 1, 8:].transpose(1, 2))
    for t, (s, l) in enumerate(rows):
        assert torch.equal(out[s, l, :, 0, 8:], back[0][t]) and torch.equal(out[s, l, :, 1, 8:], back[1][t])
    assert bool((out[..., :8] == 9.0).all())


def test_many_rows():
    """More rows than a grid has threads for at a time; tokens beyond one pass of anything."""
    n_seq, n_head, L, d = 3, 4, 30011, 64
    gen = torch.Generator(device="cuda").manual_seed(5)
    T = n_seq * L
    k = torch.randn((T, n_head, d), generator=gen, device="cuda").to(torch.bfloat16)
    cache, held = empty(n_seq, n_head, L, d)
    seq = torch.arange(n_seq, dtype=torch.int32, device="cuda").repeat_interleave(L)
    pos = torch.arange(L, dtype=torch.int32, device="cuda").repeat(n_seq)
    back = [torch.zeros_like(k) for _ in range(2)]
    dm.dsmoe_quant_cache_write(cache, k, k.flip(0), seq, pos, k_back=back[0], v_back=back[1])
    out = [torch.zeros((n_seq, n_head, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dm.dsmoe_quant_cache_read(cache, torch.tensor([L, 17, L - 1], dtype=torch.int32, device="cuda"), *out)
    for o, b in zip(out, back):
        want = b.view(n_seq, L, n_head, d).transpose(1, 2).clone()
        want[1, :, 17:] = 0
        want[2, :, L - 1] = 0
        assert torch.equal(o, want)
    at = np.random.default_rng(5).integers(0, T, 500)
    assert same(back[0][at].double().cpu().numpy(), values(*quantise(k[at].double().cpu().numpy())))


def test_offsets_beyond_32_bits():
    """Rows more than 2^32 bytes behind the first."""
    n_head, d, L = 2, 256, 9_000_000
    codes = [torch.zeros((1, L, n_head, d // 2), dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in range(2)]
    scales = [torch.zeros((1, L, n_head, 8), dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2)]
    assert 2 * L * d // 2 > 2 ** 31
    cache = dm.make_quant_cache(*codes, *scales)
    rng = np.random.default_rng(6)
    k, k_np = bf16(rng, 3, n_head, d)
    rows = [(0, L - 1), (0, L // 2), (0, 0)]
    pos = torch.tensor([l for _, l in rows], dtype=torch.int32, device="cuda")
    dm.dsmoe_quant_cache_write(cache, k, k, None, pos)
    for code, scale in written([*codes, *scales], rows, d):
        want, s = quantise(k_np)
        assert np.array_equal(code, want) and same(scale, s)
    wide = torch.zeros((1, n_head, 2, L * d), dtype=torch.bfloat16, device="cuda")          # positions L * d apart: 2^32 bytes
    out = torch.as_strided(wide, (1, n_head, 2, d), (0, 2 * L * d, L * d, 1))
    dm.dsmoe_quant_cache_read(cache, None, out, torch.as_strided(wide, (1, n_head, 2, d), (0, 2 * L * d, L * d, 1), d), first=L - 2)
    assert same(out[0, :, 1].double().cpu().numpy(), values(*quantise(k_np))[0])


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(7)
    cache, held = empty(1, 2, 40, 128)
    k, k_np = bf16(rng, 6, 2, 128)
    pos = torch.tensor([3, 39, 0, -1, 17, 8], dtype=torch.int32, device="cuda")
    out = [torch.zeros((1, 2, 40, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    dm.dsmoe_quant_cache_write(cache, k, k, None, pos, stream=stream)
    torch.cuda.synchronize()
    live = [0, 1, 2, 4, 5]
    check(held, k_np, k_np, [(0, int(p)) for p in pos.tolist()], live, 128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dm.dsmoe_quant_cache_write(cache, k, k, None, pos)
        dm.dsmoe_quant_cache_read(cache, None, *out)
    k.copy_(torch.from_numpy(k_np * 2).to(torch.bfloat16))
    pos += 0
    graph.replay()
    torch.cuda.synchronize()
    code, scale = quantise(k_np * 2)
    for t in live:
        assert same(out[0][0, :, int(pos[t])].double().cpu().numpy(), values(code, scale)[t])
