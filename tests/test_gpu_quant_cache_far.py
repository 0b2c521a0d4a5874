"""Writing and reading a cache in 4 bits whose codes and scales lie more than 2^32 bytes apart, along each of its dimensions (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from quant_cache_reference import GROUP, quantise, scales_of, unpack, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [0, 1, 2])
def test_rows_more_than_32_bits_apart(far):
    d, steps = 96, 4
    shape = [2, 2, 2]
    shape[far] = steps
    held, spans = [], []
    for width, dtype, unit in ((d // 2, torch.uint8, 1), (scales_of(d), torch.bfloat16, 2)):
        apart = (2 ** 32 // (steps - 1) // unit // 64 + 1) * 64                         # the last step is behind 2^32 bytes
        stride = [256, 128, 64]
        stride[far] = apart
        rows = [int(sum(s * i for s, i in zip(stride, at))) for at in np.ndindex(*shape)]
        assert max(rows) * unit >= 2 ** 32
        for _ in range(2):
            x = torch.empty(max(rows) + width, dtype=dtype, device="cuda")
            part = torch.as_strided(x, (*shape, width), (*stride, 1))
            part.zero_()
            held.append(part)
    K, V, K_scale, V_scale = held
    cache = dm.make_quant_cache(K, V, K_scale, V_scale)
    rng = np.random.default_rng(far)
    n_seq, n_head, L = shape
    T = n_seq * L
    k, v = (torch.from_numpy(rng.standard_normal((T, n_head, d)).astype(np.float32)).to(torch.bfloat16) for _ in range(2))
    seq = torch.arange(n_seq, dtype=torch.int32, device="cuda").repeat_interleave(L)
    pos = torch.arange(L, dtype=torch.int32, device="cuda").repeat(n_seq)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dm.dsmoe_quant_cache_write(cache, k.cuda(), v.cuda(), seq, pos, dev_status=status)
    out = [torch.zeros((n_seq, n_head, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dm.dsmoe_quant_cache_read(cache, None, *out)
    for x, codes, scales, o in ((k, K, K_scale, out[0]), (v, V, V_scale, out[1])):
        code, scale = quantise(x.double().numpy().reshape(n_seq, L, n_head, d).transpose(0, 2, 1, 3))
        assert np.array_equal(unpack(codes.cpu().numpy()), code)
        assert np.array_equal(scales[..., : d // GROUP].double().cpu().numpy(), scale)
        assert np.array_equal(o.double().cpu().numpy(), values(code, scale))
    assert status.item() == 0


def test_outputs_more_than_32_bits_apart():
    """Rows that are read back, and rows that a write gives back."""
    d, L = 64, 3
    cache = dm.make_quant_cache(*(torch.zeros((1, 1, L, w), dtype=t, device="cuda") for w, t in ((d // 2, torch.uint8), (d // 2, torch.uint8),
                                                                                               (scales_of(d), torch.bfloat16), (scales_of(d), torch.bfloat16))))
    rng = np.random.default_rng(9)
    apart = 2 ** 31 + 64                                             # elements of two bytes
    k, v = (torch.from_numpy(rng.standard_normal((L, 1, d)).astype(np.float32)).to(torch.bfloat16) for _ in range(2))
    far = [torch.empty(2 * apart + d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rows = [torch.as_strided(x, (L, 1, d), (apart, d, 1)) for x in far]
    for x, y in zip(rows, (k, v)):
        x.copy_(y)
    back = [torch.zeros_like(k, device="cuda") for _ in range(2)]
    dm.dsmoe_quant_cache_write(cache, *rows, None, torch.arange(L, dtype=torch.int32, device="cuda"), k_back=back[0], v_back=back[1])
    for x in rows:
        x.zero_()
    dm.dsmoe_quant_cache_read(cache, None, *(x.view(L, 1, d).unsqueeze(0).transpose(1, 2) for x in rows))
    for x, b, o in ((k, back[0], rows[0]), (v, back[1], rows[1])):
        want = values(*quantise(x.double().numpy()))
        assert np.array_equal(b.double().cpu().numpy(), want) and np.array_equal(o.double().cpu().numpy(), want)
