"""The key/value cache in 4 bits: the plain forms that the GPU tests compare with, and what the calls refuse (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from paper_2404_05567_b200 import build as dm_build
from quant_cache_reference import pack, places, quantise, scales_of, slot_of, unpack, values


@pytest.fixture(scope="module", autouse=True)
def _built():
    dm_build.build()


def test_plain_quantisation():
    x = np.zeros((4, 32))
    x[0, :4] = [7.0, 3.5, -2.5, 0.5]               # scale 1: halves to the even integer
    x[1, :3] = [1.0, -0.5, 0.1]                    # 1 / 7 = 0.142857 up to 10 / 64
    x[3, 0] = np.inf
    code, scale = quantise(x)
    assert scale[0, 0] == 1.0 and list(code[0, :4]) == [7, 4, -2, 0]
    assert scale[1, 0] == 10 / 64 and list(code[1, :3]) == [6, -3, 1]
    assert scale[2, 0] == 0 and (code[2] == 0).all() and np.isnan(scale[3, 0]) and np.isnan(values(code, scale)[3]).all()
    # four significant bits, times four: a bf16 holds s * c
    rng = np.random.default_rng(0)
    code, scale = quantise(torch.from_numpy(rng.standard_normal((500, 96))).to(torch.bfloat16).double().numpy())
    v = torch.from_numpy(values(code, scale))
    assert torch.equal(v.to(torch.bfloat16).double(), v)
    mantissa, _ = np.frexp(scale)
    assert (mantissa * 16 == np.rint(mantissa * 16)).all() and np.abs(code).max() == 7


def test_plain_layout():
    assert [scales_of(d) for d in (32, 64, 96, 128, 160, 256)] == [2, 2, 4, 4, 8, 8] == [dm.quant_scales(d) for d in (32, 64, 96, 128, 160, 256)]
    assert places(32)[:3] == [(0, 0), (0, 4), (1, 0)] and places(32)[31] == (15, 4)
    assert places(128)[32] == (4, 0) and places(128)[8] == (16, 0) and places(128)[127] == (63, 4)
    code = np.random.default_rng(1).integers(-8, 8, (3, 160))
    assert (unpack(pack(code)) == code).all() and pack(code).shape == (3, 80)
    assert slot_of(9, 8, 2, True) == 3 and slot_of(1, 8, 2, True) == 1 and slot_of(5, 8) == 5


A = 1 << 20       # addresses far apart, never looked at on the host


def _cache(**kw):
    a = dict(n_seq=2, n_head=2, L=32, d_head=64, K=2 * A, V=3 * A, K_scale=12 * A, V_scale=13 * A)
    strides = {k: kw.pop(k) for k in ("code_stride", "scale_stride") if k in kw}
    a.update(kw)
    c = dm.QuantCache(*a.values())
    sc = dm.quant_scales(a["d_head"])
    c.code_stride[:] = (a["n_head"] * a["L"] * a["d_head"] // 2, a["L"] * a["d_head"] // 2, a["d_head"] // 2)
    c.scale_stride[:] = (a["n_head"] * a["L"] * sc, a["L"] * sc, sc)
    for k, v in strides.items():
        getattr(c, k)[:] = v
    return c


def _desc(**kw):
    a = dict(T=4, n_head=2, group=3, d_head=64, n_seq=2, L=32, scale=0.125)
    strides = {k: kw.pop(k) for k in ("q_stride", "o_stride", "kv_stride") if k in kw}
    a.update(kw)
    d = dm.AttentionDesc(*a.values())
    d.q_stride[:] = d.o_stride[:] = (a["n_head"] * a["group"] * a["d_head"], a["group"] * a["d_head"], a["d_head"])
    for k, v in strides.items():
        getattr(d, k)[:] = v
    return d


def _write(c, T=4, sinks=0, rolling=0, stride=(128, 64), back=(128, 64), k=20 * A, v=21 * A, pos=22 * A, k_back=None, v_back=None):
    args = dm.QuantWriteArgs(T, sinks, rolling)
    args.in_stride[:], args.back_stride[:] = stride, back
    return dm.lib().dsmoe_quant_cache_write(ctypes.byref(c) if c is not None else None, ctypes.byref(args), k, v, None, pos, k_back, v_back, None, None)


def _read(c, first=0, rows=32, stride=(4096, 2048, 64), K=20 * A, V=21 * A):
    args = dm.QuantReadArgs(first, rows)
    args.out_stride[:] = stride
    return dm.lib().dsmoe_quant_cache_read(ctypes.byref(c), ctypes.byref(args), None, K, V, None)


def _attend(d, c, window=16, sinks=2, rolling=0, q=20 * A, pos=21 * A, out=22 * A, ws=30 * A, n=1 << 40):
    return dm.lib().dsmoe_quant_attention(ctypes.byref(d), ctypes.byref(c), window, sinks, rolling, q, None, pos, out, None, ws, n, None, None)


def _size(d):
    n = ctypes.c_size_t(0)
    return dm.lib().dsmoe_quant_attention_workspace_size(ctypes.byref(d), ctypes.byref(n)), n.value


@pytest.mark.parametrize("call", [lambda c: _write(c, T=0), lambda c: _read(c, rows=0), lambda c: _attend(_desc(T=0), c)])
def test_caches_that_are_refused(call):
    assert call(_cache()) == 0
    for kw in (dict(n_seq=0), dict(n_head=-1), dict(L=0), dict(d_head=0), dict(K=None), dict(V=None), dict(K_scale=None), dict(V_scale=None), dict(K=2 * A + 8),
               dict(V=3 * A + 4), dict(K_scale=12 * A + 2), dict(V_scale=13 * A + 1), dict(code_stride=(2048, 1024, 40)), dict(code_stride=(-2048, 1024, 32)),
               dict(scale_stride=(128, 64, 1)), dict(scale_stride=(128, -64, 2))):
        assert call(_cache(**kw)) == 1, kw
    for kw in (dict(d_head=48), dict(d_head=288), dict(L=2 ** 30 + 1), dict(n_seq=2 ** 20, n_head=2 ** 10), dict(code_stride=(2 ** 41, 1024, 32)),
               dict(scale_stride=(128, 2 ** 41, 2)), dict(n_seq=2 ** 12, code_stride=(2 ** 40, 1024, 32))):
        assert call(_cache(**kw)) == 2, kw


def test_writes_that_are_refused():
    c = _cache()
    assert _write(None) == 1 and dm.lib().dsmoe_quant_cache_write(ctypes.byref(c), None, *[20 * A] * 2, None, 22 * A, None, None, None, None) == 1
    for kw in (dict(T=-1), dict(sinks=-1), dict(rolling=2), dict(rolling=1, sinks=32), dict(stride=(128, 60)), dict(stride=(-128, 64)), dict(k=None), dict(v=None),
               dict(pos=None), dict(k=20 * A + 8), dict(v=21 * A + 2), dict(k_back=23 * A + 8), dict(k_back=23 * A, back=(128, 4)), dict(k_back=23 * A, back=(64, 64)),
               dict(v_back=23 * A, back=(0, 64)), dict(k_back=20 * A), dict(v_back=21 * A + 1024 - 16), dict(k_back=23 * A, v_back=23 * A), dict(k=2 * A + 4096 - 16),
               dict(v=13 * A), dict(k_back=3 * A), dict(v_back=12 * A)):
        assert _write(c, **kw) == 1, kw
    for kw in (dict(stride=(2 ** 41, 64)), dict(T=2 ** 30), dict(k_back=23 * A, back=(128, 2 ** 41)), dict(T=2 ** 12, stride=(2 ** 40, 64))):
        assert _write(c, **kw) == 2, kw
    # caches whose rows overlap, within a part of it or between parts
    for kw in (dict(code_stride=(2048, 1024, 16)), dict(code_stride=(0, 1024, 32)), dict(code_stride=(2048, 0, 32)), dict(V=2 * A), dict(V=2 * A + 16), dict(V=2 * A + 2048),
               dict(scale_stride=(128, 64, 0)), dict(V_scale=12 * A), dict(K_scale=2 * A), dict(V_scale=3 * A + 4096 - 4), dict(K_scale=3 * A + 64)):
        assert _write(_cache(**kw)) == 1, kw
    # nothing to write; nothing asked back
    assert _write(c, T=0, k=None, v=None, pos=None) == 0 and _write(c, T=0, rolling=1, sinks=31, back=(4, 4)) == 0


def test_reads_that_are_refused():
    c = _cache()
    for kw in (dict(first=-1), dict(rows=-1), dict(first=1), dict(first=32, rows=1), dict(first=2 ** 31 - 1, rows=2 ** 31 - 1), dict(stride=(4096, 2048, 60)),
               dict(stride=(4096, -2048, 64)), dict(stride=(4096, 2048, 32)), dict(stride=(0, 2048, 64)), dict(K=None), dict(V=None), dict(K=20 * A + 8),
               dict(V=21 * A + 2), dict(K=2 * A), dict(V=3 * A + 4096 - 16), dict(V=12 * A), dict(K=13 * A), dict(V=20 * A), dict(V=20 * A + 16)):
        assert _read(c, **kw) == 1, kw
    assert _read(c, stride=(2 ** 41, 2048, 64)) == 2
    assert _read(c, first=32, rows=0, K=None, V=None) == 0


def test_attention_calls_that_are_refused():
    d, c = _desc(), _cache()
    for kw in (dict(window=0), dict(window=-1), dict(sinks=-1), dict(rolling=2), dict(window=31, rolling=1), dict(window=1, sinks=32, rolling=1), dict(q=None),
               dict(pos=None), dict(out=None), dict(q=20 * A + 8), dict(out=22 * A + 4), dict(out=20 * A), dict(out=2 * A), dict(out=3 * A + 4096 - 16), dict(out=12 * A),
               dict(out=13 * A)):
        assert _attend(d, c, **kw) == 1, kw
    for kw in (dict(n_seq=1), dict(n_head=1), dict(L=31), dict(d_head=32)):
        assert _attend(_desc(**kw), c) == 1, kw
    for kw in (dict(T=-1), dict(group=0), dict(scale=float("nan")), dict(q_stride=(384, 192, 4)), dict(o_stride=(384, 0, 64))):
        assert _attend(_desc(**kw), c) == 1 and _size(_desc(**kw))[0] == 1, kw
    for kw in (dict(group=65), dict(T=2 ** 30)):
        assert _attend(_desc(**kw), c) == 2 and _size(_desc(**kw))[0] == 2, kw
    assert dm.lib().dsmoe_quant_attention(None, ctypes.byref(c), 1, 0, 0, *[A] * 5, None, A, 0, None, None) == 1
    assert dm.lib().dsmoe_quant_attention(ctypes.byref(d), None, 1, 0, 0, *[A] * 5, None, A, 0, None, None) == 1
    assert dm.lib().dsmoe_quant_attention_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == 1
    assert dm.lib().dsmoe_quant_attention_workspace_size(ctypes.byref(d), None) == 1
    need = _size(d)[1]
    for kw in (dict(ws=None), dict(ws=30 * A + 8), dict(n=need - 1), dict(n=0)):
        assert _attend(d, c, **kw) == 3, kw
    assert _attend(_desc(T=0), c, q=None, pos=None, out=None, ws=None, n=0) == 0 and _size(_desc(T=0)) == (0, 0)


def test_workspaces_of_prompts_hold_what_they_read_back():
    """4 d_head bytes a slot and head where a call is taken as one of prompts; the cache's 16-bit strides are not looked at."""
    from quant_cache_reference import taken_as_prompts
    a = dict(n_seq=2, n_head=2, d_head=64, scale=0.125, L=200000, group=8)
    copies = 4 * 64 * 2 * 2 * 200000
    for T, kw, prompts in ((16, {}, True), (15, {}, False), (16, dict(group=2), False), (64, dict(d_head=160), False), (64, dict(scale=-0.1), False)):
        got = {**a, **kw, "T": T}
        assert taken_as_prompts(got["T"], got["n_seq"], got["n_head"], got["group"], got["L"], got["d_head"], got["scale"]) == prompts
        size = _size(_desc(**got))[1]
        assert size >= copies if prompts else size < copies / 2, (T, kw)
    d = dict(T=15, group=8, L=200000)
    assert _size(_desc(**d, kv_stride=(1, -3, 2 ** 60))) == _size(_desc(**d))


def _tensors(n_seq=2, n_head=3, L=40, d=128, by_token=False):
    held = [torch.zeros((n_seq, n_head, L, w), dtype=t) for w, t in ((d // 2, torch.uint8), (d // 2, torch.uint8), (dm.quant_scales(d), torch.bfloat16),
                                                                     (dm.quant_scales(d), torch.bfloat16))]
    return [x.transpose(1, 2).contiguous().transpose(1, 2) for x in held] if by_token else held


def test_binding_refuses_other_types_shapes_and_layouts():
    good = _tensors()
    cache = dm.make_quant_cache(*good)
    assert (cache.n_seq, cache.n_head, cache.L, cache.d_head) == (2, 3, 40, 128) and list(cache.scale_stride) == [480, 160, 4]
    other = _tensors(by_token=True)
    for i, x in ((0, good[0].char()), (1, good[1][:, :, :39]), (1, other[1]), (2, good[2].half()), (2, good[2][..., :3]), (3, other[3]), (3, good[3][:1]),
                 (0, torch.zeros((2, 3, 40, 128), dtype=torch.uint8)[..., ::2])):
        bad = list(good)
        bad[i] = x
        with pytest.raises(ValueError):
            dm.make_quant_cache(*bad)
    q = torch.zeros((4, 3, 5, 128), dtype=torch.bfloat16)
    desc = dm.make_quant_attention_desc(q, cache, 0.1)
    for x in (q[:, :2], q[..., :64]):
        with pytest.raises(ValueError):
            dm.make_quant_attention_desc(x, cache)
    with pytest.raises(ValueError):
        dm.make_quant_attention_desc(q, cache, 1.0, q[:3])
    k, ints = torch.zeros((4, 3, 128), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for args in ((k.float(), k, None, ints), (k, k[:3], None, ints), (k, k.transpose(0, 1).contiguous().transpose(0, 1), None, ints), (k, k, ints[:3], ints),
                 (k, k, None, ints.long()), (k, k, None, ints, 0, False, k.half()), (k, k, None, ints, 0, False, None, k[:2]), (k[:, :2], k[:, :2], None, ints),
                 (k[..., ::2], k[..., ::2], None, ints)):
        with pytest.raises(ValueError):
            dm.dsmoe_quant_cache_write(cache, *args)
    out = torch.zeros((2, 3, 40, 128), dtype=torch.bfloat16)
    for args in ((ints, out.half(), out), (ints, out[:, :2], out[:, :2]), (ints[:1], out, out.clone()), (ints, out, out[:, :, :39]), (ints, out[..., ::2], out[..., ::2])):
        with pytest.raises(ValueError):
            dm.dsmoe_quant_cache_read(cache, *args)
    lse, ws = torch.zeros((4, 3, 5)), torch.zeros(16, dtype=torch.uint8)
    for args in ((q.half(), None, ints, q.clone(), lse), (q, None, ints, q[:3], lse), (q, None, ints[:3], q.clone(), lse), (q, None, ints, q.clone(), lse[:3])):
        with pytest.raises(ValueError):
            dm.dsmoe_quant_attention(desc, cache, 1, 0, False, *args, ws)
