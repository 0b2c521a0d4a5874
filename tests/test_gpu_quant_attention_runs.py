"""dsmoe_quant_attention of batches with about as many (token, head) pairs as a GPU has SMs, whose caches are as long as one launch takes them and longer (GPU required)."""
import pytest
import torch

import paper_2404_05567_b200 as dm
from quant_cache_reference import QuantCase

pytestmark = pytest.mark.gpu

ALL = 2 ** 31 - 1


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("n_head,group,L", [(2, 3, 2304), (2, 3, 2305), (4, 12, 1536), (4, 12, 1537)])
def test_one_long_cache_beside_short_ones(n_head, group, L, by_token):
    n = 74 // n_head * 2
    assert n * n_head <= 148
    tokens = [(0, L - 1)] + [(s, 3 * s) for s in range(1, n)]
    c = QuantCase(tokens, n_head, group, 32, n, L, seed=L, by_token=by_token)
    cache = c.cache()
    desc = dm.make_quant_attention_desc(c.q, cache, c.scale, c.out)
    ws = torch.full((dm.dsmoe_quant_attention_workspace_size(desc),), 0xff, dtype=torch.uint8, device="cuda")
    dm.dsmoe_quant_attention(desc, cache, ALL, 0, False, c.q, c.tok_seq, c.pos, c.out, c.lse, ws, c.status)
    c.check(c.expected())
    assert c.status.item() == 0
