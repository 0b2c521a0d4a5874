"""Attention over a cache in 4 bits where one key has nearly all of the weight and very many have the rest, each of them next to none, beside values of smaller scales:
what they add up to is there (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import BF16_HALF_STEP, attention
from quant_cache_reference import GROUP, quant_logit_error, tensors, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group,n,bits", [(32, 1, 65536, 24.6), (32, 1, 65535, 25.0), (32, 12, 65536, 24.6), (160, 5, 65536, 24.6), (32, 3, 5000, 20.0)])
def test_flat_tail_behind_one_key(d, group, n, bits):
    """As many pairs as there are warps, so that a warp has one's keys from the first to the last: key 0, of large values in the first place of each group and zeros in
    the others, and n - 1 keys of 2^-bits of its weight each, whose values' scales are 2^-6 times the size."""
    T = 1776
    rng = np.random.default_rng(n + d)
    q = torch.from_numpy(rng.standard_normal(d).astype(np.float32)).to(torch.bfloat16)
    G = d // GROUP
    kc, ks = np.zeros((1, 1, n, d), dtype=int), np.zeros((1, 1, n, G))
    vc, vs = np.zeros((1, 1, n, d), dtype=int), np.zeros((1, 1, n, G))
    kc[0, 0, 0], ks[0, 0, 0] = np.where(q.double().numpy() > 0, 5, -5), 0.5
    vc[0, 0, 0].reshape(G, GROUP)[:, 0], vs[0, 0, 0] = 7, 1.875
    vc[0, 0, 1:], vs[0, 0, 1:] = rng.integers(1, 8, (n - 1, d)), (rng.integers(8, 12, (n - 1, G)) / 8) * 2.0 ** -6
    vc[0, 0, 1:].reshape(n - 1, G, GROUP)[:, :, 0] = 0
    K, V = values(kc, ks)[0, 0], values(vc, vs)[0, 0]
    scale = float(np.float32(bits * np.log(2.0) / (q.double().numpy() @ K[0])))
    qs = q.double().numpy()[None]
    want, lse, weight, absolute, spread = attention(qs, K, V, scale, np.arange(n))
    error = quant_logit_error(qs, scale, ks[0, 0], spread, d)
    # Weights are off by exp(+-2 error) and 2^-20, and rounded to fp16 before and behind the product with a scale, 2^-11 each; or, in units in which the largest weight is
    # 2^10 and the largest scale, 1.875, at least 1 / 2 and below 1, by 2^-25 times the scale and by 2^-25: 2^-35 of the tail's scales, of at most 2^-5, and of 2, times codes of 7.  Sums in fp32: a step of 16
    # keys may cut each of its 17 terms 2^-23 below the largest, that is the sum so far, and the parts' sums add 2^8 steps of 2^-24.  The output is rounded to bf16.
    tol = (BF16_HALF_STEP * np.abs(want) * 1.01
           + absolute * (np.expm1(2 * error)[..., None] + 2.0 ** -20 + 2.0 ** -10 * 1.01 + 2.0 ** -16 + n / 16 * 17 * 2.0 ** -23)
           + n * 7 * 2.0 ** -35 * (2 + 2.0 ** -5))
    tail = (np.arange(d) % GROUP > 0)
    assert (want[:, tail] > 4 * tol[:, tail]).all()           # (the tolerance says something)
    (K_, K_scale), (V_, V_scale) = tensors(kc, ks), tensors(vc, vs)
    cache = dm.make_quant_cache(K_, V_, K_scale, V_scale)
    queries = q.cuda().expand(T, 1, group, d).contiguous()
    out, got_lse = torch.full_like(queries, 7.0), torch.full((T, 1, group), 7.0, device="cuda")
    pos = torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
    desc = dm.make_quant_attention_desc(queries, cache, scale)
    ws = torch.empty(dm.dsmoe_quant_attention_workspace_size(desc), dtype=torch.uint8, device="cuda")
    dm.dsmoe_quant_attention(desc, cache, 2 ** 31 - 1, 0, False, queries, None, pos, out, got_lse, ws)
    got = out.double().cpu().numpy()
    assert (np.abs(got - want[0]) <= tol[0]).all(), (np.abs(got - want[0]) / tol[0]).max()
    assert (np.abs(got_lse.double().cpu().numpy() - lse[0]) <= error[0] + 1e-4).all()
