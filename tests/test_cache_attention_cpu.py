"""The attention steps on a key/value cache: the plain forms that the GPU tests compare with, and what the calls refuse (no GPU needed)."""
import copy
import ctypes

import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import attention, evict, visible
from paper_2404_05567_b200 import build as dm_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    dm_build.build()


def test_visible_keys():
    assert visible(5) == [0, 1, 2, 3, 4, 5] and visible(-1) == [] and visible(-1, 3, 2) == []
    assert visible(9, 3, 0) == [7, 8, 9] and visible(9, 3, 2) == [0, 1, 7, 8, 9] and visible(2, 3, 2) == [0, 1, 2]


def test_plain_attention():
    """Two keys with equal logits; a key that outweighs; nothing visible."""
    K, V = np.array([[1.0, 0], [1, 0], [0, 90]]), np.array([[2.0], [4], [7]])
    V = np.repeat(V, 2, 1)
    out, lse, p, _, _ = attention(np.array([[3.0, 0]]), K, V, 1.0, [0, 1])
    assert np.allclose(out, 3) and np.allclose(lse, 3 + np.log(2)) and np.allclose(p, 0.5)
    assert np.allclose(attention(np.array([[0.0, 1]]), K, V, 1.0, [0, 1, 2])[0], 7)
    out, lse = attention(np.ones((1, 2)), K, V, 1.0, [])[:2]
    assert (out == 0).all() and lse[0] == -np.inf


def test_plain_eviction():
    t = np.array([5, 1, 3, 3, 0, 9, 2], dtype=np.float32)
    assert evict(t, 7, 7, 0, 0) == list(range(7)) and evict(t, 3, 4, 1, 1) == [0, 1, 2]
    assert evict(t, 7, 3, 0, 0) == [0, 2, 5] and evict(t, 7, 4, 1, 1) == [0, 2, 5, 6] and evict(t, 7, 3, 1, 2) == [0, 5, 6]
    assert evict(np.array([np.nan, -np.inf, 0, np.nan], dtype=np.float32), 4, 2, 0, 0) == [1, 2]


def _desc(**kw):
    a = dict(T=4, n_head=2, group=3, d_head=64, n_seq=2, L=32, scale=0.125)
    strides = {k: kw.pop(k) for k in ("q_stride", "o_stride", "kv_stride") if k in kw}
    a.update(kw)
    d = dm.AttentionDesc(*a.values())
    row = a["n_head"] * a["group"] * a["d_head"]
    d.q_stride[:] = d.o_stride[:] = (row, a["group"] * a["d_head"], a["d_head"])
    d.kv_stride[:] = (a["n_head"] * a["L"] * a["d_head"], a["L"] * a["d_head"], a["d_head"])
    for k, v in strides.items():
        getattr(d, k)[:] = v
    return d


def _size(d, kind=0, P=0):
    n = ctypes.c_size_t(0)
    return dm.lib().dsmoe_attention_workspace_size(ctypes.byref(d), kind, P, ctypes.byref(n)), n.value


def test_descriptors_that_are_refused():
    assert _size(_desc())[0] == 0
    for kw in (dict(T=-1), dict(n_head=0), dict(group=0), dict(d_head=0), dict(n_seq=0), dict(L=0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(q_stride=(384, 192, 4)), dict(q_stride=(-384, 192, 64)), dict(kv_stride=(4096, 2048, 63)),
               dict(o_stride=(384, 192, 32)), dict(o_stride=(0, 192, 64)), dict(o_stride=(384, 0, 64)), dict(o_stride=(380, 192, 64)),
               dict(o_stride=(128, 64, 64))):
        assert _size(_desc(**kw))[0] == 1, kw
    for kw in (dict(d_head=48), dict(d_head=288), dict(group=65), dict(T=2 ** 30), dict(kv_stride=(2 ** 41, 2048, 64))):
        assert _size(_desc(**kw))[0] == 2, kw
    for kw in (dict(q_stride=(0, 0, 0)), dict(o_stride=(384, 64, 128)), dict(o_stride=(64, 64 * 4 * 3, 64 * 4)), dict(T=0, o_stride=(0, 192, 64)),
               dict(T=1, o_stride=(0, 192, 64))):
        assert _size(_desc(**kw))[0] == 0, kw
    assert _size(_desc(), 3)[0] == 1 and _size(_desc(), -1)[0] == 1 and _size(_desc(), 1, -1)[0] == 1
    assert _size(_desc(T=0)) == (0, 0)
    assert dm.lib().dsmoe_attention_workspace_size(None, 0, 0, ctypes.byref(ctypes.c_size_t(0))) == 1
    # more to hold: a prefix, the rows' sums
    assert _size(_desc(), 1, 1000)[1] > _size(_desc(), 1, 0)[1] >= _size(_desc(), 0)[1]
    assert _size(_desc(), 2)[1] > _size(_desc(), 0)[1]


A = 1 << 20       # addresses far apart, never looked at on the host


def _call(name, d, more=(), q=A, K=2 * A, V=3 * A, seq=4 * A, pos=5 * A, out=6 * A, lse=None, tail=(), ws=8 * A, n=1 << 40):
    return getattr(dm.lib(), name)(ctypes.byref(d) if d is not None else None, *more, q, K, V, seq, pos, out, lse, *tail, ws, n, None, None)


CALLS = [("dsmoe_window_attention", (16, 2, 0), ()), ("dsmoe_tally_attention", (), (None, 9 * A))]


@pytest.mark.parametrize("name,more,tail", CALLS)
def test_calls_that_are_refused(name, more, tail):
    d = _desc()
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(pos=None), dict(out=None), dict(q=A + 8), dict(K=2 * A + 2), dict(V=3 * A + 4),
               dict(out=6 * A + 8), dict(out=A), dict(out=A + 16), dict(out=2 * A + 4096), dict(out=3 * A)):
        assert _call(name, d, more, tail=tail, **kw) == 1, kw
    assert _call(name, None, more, tail=tail) == 1
    assert _call(name, _desc(d_head=40), more, tail=tail) == 2
    need = _size(d, 2 if "tally" in name else 0)[1]
    for kw in (dict(ws=None), dict(ws=8 * A + 8), dict(n=need - 1), dict(n=0)):
        assert _call(name, d, more, tail=tail, **kw) == 3, kw


def test_caches_of_more_positions_than_are_counted():
    assert _size(_desc(L=2 ** 30, kv_stride=(0, 0, 0)))[0] == 0 and _size(_desc(L=2 ** 30 + 1, kv_stride=(0, 0, 0)))[0] == 2
    assert _size(_desc(), dm.ATTENTION_PREFIX, 2 ** 30)[0] == 0 and _size(_desc(), dm.ATTENTION_PREFIX, 2 ** 30 + 1)[0] == 2
    # parts of 2^36 bytes and more
    big = dict(n_head=16, group=8, d_head=128, o_stride=(16384, 1024, 128))
    assert _size(_desc(T=2 ** 18, **big), dm.ATTENTION_PREFIX, 4096)[0] == 0 and _size(_desc(T=2 ** 22, **big), dm.ATTENTION_PREFIX, 4096)[0] == 2


def test_windows_that_are_refused():
    for window, sinks, rolling in ((0, 0, 0), (-1, 0, 0), (4, -1, 0), (4, 0, 2), (4, 0, -1), (31, 2, 1), (1, 32, 1), (33, 0, 1)):
        assert _call("dsmoe_window_attention", _desc(), (window, sinks, rolling)) == 1, (window, sinks, rolling)
    assert _call("dsmoe_window_attention", _desc(T=0), (4, 1, 0), q=None, out=None, ws=None, n=0) == 0


def test_prefixes_that_are_refused():
    def go(d=None, Kp=10 * A, Vp=11 * A, P=8, stride=(512, 64), **kw):
        p = dm.Prefix(Kp, Vp, P)
        p.stride[:] = stride
        return _call("dsmoe_prefix_attention", d or _desc(), (ctypes.byref(p),), **kw)
    for kw in (dict(P=-1), dict(Kp=None), dict(Vp=None), dict(Kp=10 * A + 2), dict(stride=(512, 60)), dict(stride=(-512, 64)), dict(out=10 * A),
               dict(out=11 * A + 64), dict(q=None), dict(out=A)):
        assert go(**kw) == 1, kw
    assert _call("dsmoe_prefix_attention", _desc(), (None,)) == 1
    assert go(stride=(2 ** 41, 64)) == 2
    assert go(n=_size(_desc(), 1, 8)[1] - 1) == 3
    assert go(d=_desc(T=0), q=None, ws=None, n=0) == 0


def test_tallies_that_are_refused():
    d = _desc()                                        # 2 * 2 * 32 tallies: 512 bytes
    for tail in ((None, None), (9 * A, 9 * A + 4), (9 * A + 508, 9 * A), (9 * A, 9 * A + 508)):
        assert _call("dsmoe_tally_attention", d, (), tail=tail) == 1, tail
    assert _call("dsmoe_tally_attention", _desc(T=0), (), tail=(9 * A, 9 * A), ws=None, n=0) == 0


def test_evictions_that_are_refused():
    def go(d=None, keep=16, sinks=2, recent=4, out_stride=(2048, 1024, 64), pitch=16, length=A, tally=2 * A, K=3 * A, V=4 * A, kept=5 * A,
           len_out=6 * A, tally_out=7 * A, K_out=8 * A, V_out=9 * A, ws=10 * A, n=1 << 20):
        a = dm.EvictArgs(keep, sinks, recent)
        a.out_stride[:] = out_stride
        a.tally_pitch = pitch
        return dm.lib().dsmoe_cache_evict(ctypes.byref(d or _desc()), ctypes.byref(a), length, tally, K, V, kept, len_out, tally_out, K_out, V_out,
                                          ws, n, None, None)
    same = dict(out_stride=(4096, 2048, 64), pitch=32)
    for kw in (dict(keep=0), dict(keep=33, pitch=33), dict(sinks=-1), dict(recent=-1), dict(sinks=10, recent=7), dict(pitch=15),
               dict(out_stride=(2048, 1024, 60)), dict(out_stride=(2048, 512, 64)), dict(out_stride=(0, 1024, 64)), dict(length=None),
               dict(tally=None), dict(K=None), dict(V=None), dict(kept=None), dict(len_out=None), dict(tally_out=None), dict(K_out=None),
               dict(V_out=None), dict(K=3 * A + 2), dict(V_out=9 * A + 8), dict(K_out=3 * A), dict(V_out=4 * A), dict(V_out=8 * A),
               dict(K_out=3 * A, V_out=4 * A), dict(K_out=3 * A + 64), dict(K_out=4 * A, V_out=3 * A, **same), dict(tally_out=2 * A),
               dict(tally_out=2 * A + 4, pitch=32)):
        assert go(**kw) == 1, kw
    assert go(out_stride=(2 ** 41, 1024, 64)) == 2
    assert go(ws=None) == 3 and go(ws=10 * A + 4) == 3 and go(n=8) == 3
    n = ctypes.c_size_t(0)
    assert dm.lib().dsmoe_evict_workspace_size(None, ctypes.byref(n)) == 1
    assert dm.lib().dsmoe_evict_workspace_size(ctypes.byref(_desc()), None) == 1
    assert dm.dsmoe_evict_workspace_size(_desc()) >= 16


def test_the_binding_checks_shapes_and_types():
    q = torch.zeros((4, 2, 3, 64), dtype=torch.bfloat16)
    K = torch.zeros((2, 2, 32, 64), dtype=torch.bfloat16)
    desc = dm.make_attention_desc(q, K, 0.125)
    assert _size(desc)[0] == 0
    args = lambda **kw: {**dict(q=q, K=K, V=K.clone(), tok_seq=None, pos=torch.zeros(4, dtype=torch.int32), out=torch.zeros_like(q), lse=None), **kw}
    for kw in (dict(q=q.float()), dict(q=q[:3]), dict(out=q.transpose(1, 2)), dict(K=K[:, :, :31]), dict(V=K.float()), dict(V=K.transpose(1, 2))):
        with pytest.raises(ValueError):
            dm.dsmoe_window_attention(desc, 4, 0, False, *args(**kw).values(), None)
    with pytest.raises(ValueError):
        dm.dsmoe_prefix_attention(desc, K[0, :, :, :32], K[0, :, :, :32], *args().values(), None)
    with pytest.raises(ValueError):
        dm.dsmoe_tally_attention(desc, *args().values(), None, torch.zeros((2, 2, 31)), None)
    with pytest.raises(ValueError):
        dm.dsmoe_cache_evict(desc, 8, 0, 0, None, torch.zeros((2, 2, 32)), K, K.clone(), torch.zeros((2, 2, 7), dtype=torch.int32), None,
                             torch.zeros((2, 2, 8)), K[:, :, :8].clone(), K[:, :, :8].clone(), None)


def test_the_binding_checks_tallies_and_places_for_what_stays():
    q = torch.zeros((4, 2, 3, 64), dtype=torch.bfloat16)
    K, V = (torch.zeros((2, 2, 32, 64), dtype=torch.bfloat16) for _ in range(2))
    desc, tally, pos = dm.make_attention_desc(q, K, 0.125), torch.zeros((2, 2, 32)), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        dm.dsmoe_tally_attention(desc, q, K, V, None, pos, torch.zeros_like(q), None, torch.zeros((1, 2, 32)), tally, None)
    out, room, kept, length = torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 8)), torch.zeros((2, 2, 8), dtype=torch.int32), pos[:2]
    for a, b, c in ((out, out[:, :, :7], room), (out.float(), out.float(), room), (out[..., :32], out[..., :32], room), (out[:1], out[:1], room),
                    (out, out, room[:1]), (out, out, room[:, :1]), (out, out, room[0]), (out.transpose(2, 3), out.transpose(2, 3), room)):
        with pytest.raises(ValueError):
            dm.dsmoe_cache_evict(desc, 8, 0, 0, length, tally, K, V, kept, length, c, a, b, None)
    for a, t in ((kept[..., :7], tally), (kept, tally[:, :, :31]), (kept, tally[:1])):
        with pytest.raises(ValueError):
            dm.dsmoe_cache_evict(desc, 8, 0, 0, length, t, K, V, a, length, room, out, out.clone(), None)
    with pytest.raises(ValueError):                      # in place: the whole cache's tallies are kept
        dm.dsmoe_cache_evict(desc, 8, 0, 0, length, tally[:, :, :8], K, V, kept, length, tally[:, :, :8], K, V, None)
    # nothing wrong with the shapes: what is missing is the workspace
    for place in ((tally, K, V), (room, out, out.clone())):
        with pytest.raises(dm.DsmoeError) as e:
            dm.dsmoe_cache_evict(desc, 8, 0, 0, length, tally, K, V, kept, length, *place, None, stream=type("S", (), {"cuda_stream": 0}))
        assert e.value.code == 3


def test_extents_beyond_64_bits_are_refused():
    """Strides and sizes that are allowed one by one, but lie further apart than addresses go."""
    far, ok = 2 ** 40, (384, 192, 64)
    for kw in (dict(L=2 ** 30, kv_stride=(0, 0, far)), dict(n_seq=2 ** 27, n_head=1, kv_stride=(far, 2048, 64)),
               dict(T=2 ** 26, group=1, o_stride=(128, 64, 64), q_stride=(far, 64, 64))):
        assert _call("dsmoe_window_attention", _desc(**kw), (4, 0, 0)) == 2, kw
        assert _call("dsmoe_tally_attention", _desc(**kw), tail=(None, 1 << 50)) == 2, kw
    p = dm.Prefix(10 * A, 11 * A, 2 ** 30)
    p.stride[:] = (512, far)
    assert _call("dsmoe_prefix_attention", _desc(o_stride=ok), (ctypes.byref(p),)) == 2
    for L, kv, out in ((2 ** 30, (0, 0, far), (2048, 1024, 64)), (2 ** 30, (64, 64, 128), (64, 128, far))):
        a = dm.EvictArgs(2 ** 28, 0, 0)
        a.out_stride[:], a.tally_pitch = out, 2 ** 30
        d = _desc(L=L, kv_stride=kv)
        assert dm.lib().dsmoe_cache_evict(ctypes.byref(d), ctypes.byref(a), A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 1 << 45, 1 << 50, 1 << 51, 10 * A, 1 << 20,
                                          None, None) == 2, kv


def test_places_for_what_stays_that_overlap():
    """Keys' and values' rows in part the same memory are refused, in place or not; rows that lie between one another are not."""
    def go(kv_stride, out_stride, K, V, K_out, V_out, keep=16, d=None):
        a = dm.EvictArgs(keep, 2, 4)
        a.out_stride[:], a.tally_pitch = out_stride, 32
        # (what is not refused lacks its workspace: 3)
        return dm.lib().dsmoe_cache_evict(ctypes.byref(d or _desc(kv_stride=kv_stride)), ctypes.byref(a), A, 2 * A, K, V, 5 * A, 6 * A, 7 * A, K_out, V_out, None, 0,
                                          None, None)
    whole, room, at = (4096, 2048, 64), (2048, 1024, 64), 8 * A
    for off, want in ((0, 1), (16, 1), (128, 1), (1024 * 2, 1), (2048 * 2 - 16, 1), (4096 * 2 - 16, 1), (4096 * 2, 3), (-16, 1), (-4096 * 2 + 16, 1), (-4096 * 2, 3)):
        assert go(whole, room, 3 * A, 4 * A, at, at + off) == want, off
    # keys and values side by side in each position, head or sequence: [n_seq][n_head][16][2][64] and so on
    for stride, step in (((4096, 2048, 128), 64), ((4096, 2048, 64), 1024), ((4096, 1024, 64), 2048)):
        for off, want in ((step * 2, 3), (step * 2 - 16, 1), (step * 2 + 16, 1), (-step * 2, 3), (step * 2 + stride[0] * 2, 3)):
            assert go(whole, stride, 3 * A, 4 * A, at, at + off) == want, (stride, off)
    # in place: [n_seq][n_head][32][2][64]
    both = (8192, 4096, 128)
    for off, want in ((128, 3), (-128, 3), (64, 1), (256, 1), (16, 1), (4096 * 2, 1), (4096 * 2 + 128, 3), (8192 * 2, 1), (2 * 8192 * 2, 3)):
        assert go(both, both, at, at + off, at, at + off) == want, off
    # rows of less than a stride: a place between them, and one that is too small
    for off, want in ((64 * 2, 3), (96 * 2, 3), (112 * 2, 1), (48 * 2, 1)):
        assert go(whole, (8192, 4096, 160), 3 * A, 4 * A, at, at + off) == want, off
    # any order of dimensions with any gaps, against the addresses themselves
    rng = np.random.default_rng(0)
    seen = set()
    for _ in range(1500):
        n = rng.integers(1, 4, 3)
        stride, span = np.zeros(3, dtype=np.int64), 32
        for i in rng.permutation(3):
            stride[i] = span + 8 * rng.integers(0, 12)
            span += stride[i] * (n[i] - 1)
        off = 8 * int(rng.integers(-span // 8 - 4, span // 8 + 5))
        d = _desc(d_head=32, n_seq=n[0], n_head=n[1], L=n[2], kv_stride=(0, 0, 32))
        a = dm.EvictArgs(n[2], 0, 0)
        a.out_stride[:], a.tally_pitch = stride.tolist(), 32
        got = dm.lib().dsmoe_cache_evict(ctypes.byref(d), ctypes.byref(a), A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A, at, at + 2 * off, None, 0, None, None)
        rows = [s * stride[0] + h * stride[1] + p * stride[2] for s in range(n[0]) for h in range(n[1]) for p in range(n[2])]
        meet = any(abs(x - y - off) < 32 for x in rows for y in rows)
        assert got == (1 if meet else 3), (n, stride, off)
        seen.add((meet, abs(off) < span))
    assert seen == {(True, True), (False, True), (False, False)}


def test_the_binding_checks_numbers_and_lengths():
    """What the kernels read as int32 and fp32 is that, and is long enough."""
    q, K = torch.zeros((4, 2, 3, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 32, 64), dtype=torch.bfloat16)
    desc, pos, tally = dm.make_attention_desc(q, K, 0.125), torch.zeros(4, dtype=torch.int32), torch.zeros((2, 2, 32))
    stream = type("S", (), {"cuda_stream": 0})
    Kp = torch.zeros((2, 8, 64), dtype=torch.bfloat16)

    def calls(**kw):
        a = dict(q=q, K=K, V=K.clone(), tok_seq=pos, pos=pos, out=torch.zeros_like(q), lse=torch.zeros(4, 2, 3))
        a.update({k: v for k, v in kw.items() if k in a})
        dev_status, tally_in, prefix = kw.get("dev_status"), kw.get("tally_in", tally), kw.get("Kp", Kp)
        yield lambda: dm.dsmoe_window_attention(desc, 4, 0, False, *a.values(), None, dev_status, stream)
        yield lambda: dm.dsmoe_prefix_attention(desc, prefix, prefix, *a.values(), None, dev_status, stream)
        yield lambda: dm.dsmoe_tally_attention(desc, *a.values(), tally_in, kw.get("tally_out", tally), None, dev_status, stream)

    for call in calls():                                  # nothing wrong but the missing workspace
        with pytest.raises(dm.DsmoeError):
            call()
    for kw in (dict(pos=pos.long()), dict(tok_seq=pos.long()), dict(pos=pos[:3]), dict(tok_seq=pos[:3]), dict(pos=torch.zeros((4, 2), dtype=torch.int32)[:, 0]),
               dict(lse=torch.zeros(4, 2, 3).double()), dict(lse=torch.zeros(4, 2, 2)), dict(lse=torch.zeros(4, 3, 2).transpose(1, 2)),
               dict(dev_status=torch.zeros(1, dtype=torch.int64)), dict(dev_status=pos[:0])):
        for call in calls(**kw):
            with pytest.raises(ValueError):
                call()
    for kw in (dict(tally_in=tally.double()), dict(tally_out=tally.bfloat16()), dict(tally_in=tally.half(), tally_out=tally.clone())):
        with pytest.raises(ValueError):
            list(calls(**kw))[2]()
    out, room, kept, length = torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 8)), torch.zeros((2, 2, 8), dtype=torch.int32), pos[:2]
    good = dict(length=length, tally=tally, K=K, V=K.clone(), kept=kept, len_out=length, tally_out=room, K_out=out, V_out=out.clone(), workspace=None, dev_status=None)
    for kw in (dict(length=length.long()), dict(length=pos[:1]), dict(len_out=length.long()), dict(len_out=pos[:1]), dict(kept=kept.long()),
               dict(kept=kept.float()), dict(tally=tally.double()), dict(tally_out=room.double()), dict(tally=tally.transpose(0, 1)),
               dict(dev_status=length.long())):
        with pytest.raises(ValueError):
            dm.dsmoe_cache_evict(desc, 8, 0, 0, *{**good, **kw}.values(), stream)
    with pytest.raises(dm.DsmoeError):
        dm.dsmoe_cache_evict(desc, 8, 0, 0, *good.values(), stream)


def test_the_binding_checks_devices(monkeypatch):
    """Tensors on several devices, and on another than the current one.  (There is one device here: some say that they are elsewhere.)"""
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1
    away = lambda x: x.as_subclass(Elsewhere)
    q, K = torch.zeros((4, 2, 3, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 32, 64), dtype=torch.bfloat16)
    desc, pos, tally = dm.make_attention_desc(q, K, 0.125), torch.zeros(4, dtype=torch.int32), torch.zeros((2, 2, 32))
    good = dict(q=q, K=K, V=K.clone(), tok_seq=pos, pos=pos, out=torch.zeros_like(q), lse=torch.zeros(4, 2, 3), workspace=torch.zeros(8, dtype=torch.uint8),
                dev_status=pos, stream=type("S", (), {"cuda_stream": 0}))
    for name in list(good)[:-1]:
        with pytest.raises(ValueError):
            dm.dsmoe_window_attention(desc, 4, 0, False, *{**good, name: away(good[name])}.values())
    Kp = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    for a, b in ((away(Kp), Kp), (Kp, away(Kp))):
        with pytest.raises(ValueError):
            dm.dsmoe_prefix_attention(desc, a, b, *good.values())
    with pytest.raises(ValueError):
        dm.dsmoe_tally_attention(desc, *list(good.values())[:7], tally, away(tally.clone()), *list(good.values())[7:])
    monkeypatch.setattr(dm.binding, "_current_device", lambda: 0)
    here = {k: away(v) if isinstance(v, torch.Tensor) else v for k, v in good.items()}
    with pytest.raises(ValueError, match="current"):
        dm.dsmoe_window_attention(desc, 4, 0, False, *{**here, "stream": None}.values())
    with pytest.raises(dm.DsmoeError):                    # one device, and a stream that the caller has chosen: what is missing is workspace
        dm.dsmoe_window_attention(desc, 4, 0, False, *here.values())


def test_workspaces_hold_what_the_calls_use():
    """Prompts of one sequence and heads of more than 128 have no room for parts that nobody leaves."""
    def one(T, d=128, n_seq=1, kind=0, P=0):
        row = 4 * 5 * d
        return _size(_desc(T=T, n_head=4, group=5, d_head=d, n_seq=n_seq, L=T, o_stride=(row, 5 * d, d), q_stride=(row, 5 * d, d),
                           kv_stride=(4 * T * d, T * d, d)), kind, P)[1]
    # (one part of the rows at most where there are enough tokens to fill the GPU)
    for T in (8192, 32768, 131072):
        rows = T * 20
        assert one(T) < 1 << 20
        assert one(T, kind=dm.ATTENTION_TALLY) < rows * 8 + T * 8 + 4 * T * 4 * 16 + (1 << 20)
        assert one(T, kind=dm.ATTENTION_PREFIX, P=1000) < 2 * rows * (128 + 2) * 4 + (64 << 20)
        assert one(T, n_seq=2) > 100 << 20               # tokens of short runs may be left to the other kernel
    # a pass of 512 tokens: for each warp of 148 CTAs two tiles of 16 rows
    assert one(512, 160, 512) < 2.1 * 148 * 4 * 16 * 162 * 4 + (1 << 20) < one(512, 128, 512)


def test_descriptors_can_be_copied():
    """A copy is a descriptor of its own, also behind a call."""
    q, K = torch.zeros((4, 2, 3, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 32, 64), dtype=torch.bfloat16)
    desc, pos, tally, stream = dm.make_attention_desc(q, K, 0.125), torch.zeros(4, dtype=torch.int32), torch.zeros((2, 2, 32)), type("S", (), {"cuda_stream": 0})
    kept = torch.zeros((2, 2, 8), dtype=torch.int32)

    def code(d, **kw):
        with pytest.raises(dm.DsmoeError) as e:
            if kw:
                dm.dsmoe_cache_evict(d, 8, kw["sinks"], 0, pos[:2], tally, K, V, kept, pos[:2], tally, K, V, None, None, stream)
            else:
                dm.dsmoe_window_attention(d, 4, 0, False, q, K, V, None, pos, torch.zeros_like(q), None, None, None, stream)
        return e.value.code
    V = K.clone()
    assert code(desc) == 3 and code(desc, sinks=2) == 3 and code(desc, sinks=9) == 1 and code(desc, sinks=2) == 3
    for other in (copy.copy(desc), copy.deepcopy(desc)):
        other.scale, other.kv_stride[1] = float("nan"), 4
        assert code(other) == 1 and code(other, sinks=2) == 1 and code(desc) == 3 and code(desc, sinks=2) == 3
