"""dsmoe_quant_attention gives the same results every time, on any stream and from a graph, with workspaces that are filled before the stream may begin (GPU required)."""
import pytest
import torch

import paper_2404_05567_b200 as dm
from quant_cache_reference import QuantCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompt", [False, True])
def test_same_results_on_every_stream(prompt):
    tokens = [(s, 1000 + 77 * s) for s in range(9)] if not prompt else [(0, p) for p in range(200)] + [(1, p) for p in range(300, 500)]
    c = QuantCase(tokens, 4, 5, 128, 9, 2000, seed=14)
    assert c.prompts() == prompt
    cache = c.cache()
    desc = dm.make_quant_attention_desc(c.q, cache, c.scale, c.out)
    ws = torch.empty(dm.dsmoe_quant_attention_workspace_size(desc), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        dm.dsmoe_quant_attention(desc, cache, 900, 4, False, c.q, c.tok_seq, c.pos, c.out, c.lse, ws, c.status, stream=stream)

    def clear(stream):
        """What other calls may have left, before anything of `stream` that comes now."""
        ws.fill_(0xff)
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        stream.wait_stream(torch.cuda.current_stream())

    clear(torch.cuda.current_stream())
    call()
    c.check(c.expected(900, 4))
    first, lse = c.out.clone(), c.lse.clone()
    for i in range(3):
        stream = torch.cuda.Stream()
        clear(stream)
        call(stream)
        torch.cuda.current_stream().wait_stream(stream)
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        clear(torch.cuda.current_stream())
        graph.replay()
        assert torch.equal(c.out, first) and torch.equal(c.lse, lse)
    assert c.status.item() == 0
