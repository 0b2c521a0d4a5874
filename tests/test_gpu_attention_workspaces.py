"""What the attention steps do with their workspace (GPU required): they stay within the bytes that they ask for, and what lay there makes no difference."""
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import Case
from test_gpu_attention_tiles import prompt
from test_gpu_prefix_attention import run as run_prefix
from test_gpu_window_attention import run as run_window

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


def decoding(n, last):
    return [(s, last - 3 * s) for s in range(n)]


# tokens, heads, group, d_head, sequences, L, shared keys
CASES = {
    "one sequence's prompt": (prompt(0, 799, 800), 2, 5, 128, 1, 800, 0),
    "one sequence's prompt, keys in parts": (prompt(0, 2999, 60), 1, 5, 64, 1, 3000, 0),
    "... behind shared keys": (prompt(0, 1299, 60), 2, 5, 96, 1, 1300, 700),
    "prompts and single tokens": (prompt(0, 699, 90) + prompt(1, 400, 3) + [(2, 650), (3, 20)], 2, 5, 64, 4, 700, 0),
    "more tokens than a pass lists, of short runs": ([(i % 90, 10 + i // 90) for i in range(700)], 2, 4, 64, 90, 40, 0),
    "decoding": (decoding(20, 900), 4, 5, 128, 20, 901, 0),
    "decoding, wide heads": (decoding(20, 900), 2, 5, 160, 20, 901, 0),
    "decoding, wide heads of two tiles of rows": (decoding(3, 3000), 2, 20, 256, 3, 3001, 0),
    "many short pairs, wide heads": (decoding(300, 950), 4, 2, 192, 300, 951, 0),
    "decoding behind shared keys": (decoding(5, 300), 2, 5, 64, 5, 301, 2000),
    "decoding behind shared keys, wide heads": (decoding(30, 300), 2, 5, 224, 30, 301, 2000),
}


def calls(c, kind):
    desc = c.desc()
    size = dm.dsmoe_attention_workspace_size(desc, kind, c.P)
    common = c.q, c.K, c.V, c.tok_seq, c.pos, c.out, c.lse
    tally = torch.zeros((c.n_seq, c.n_head, c.L), device="cuda")

    def once(ws):
        if kind == dm.ATTENTION_WINDOW:
            dm.dsmoe_window_attention(desc, 600, 4, False, *common, ws, c.status)
        elif kind == dm.ATTENTION_PREFIX:
            dm.dsmoe_prefix_attention(desc, c.Kp, c.Vp, *common, ws, c.status)
        else:
            dm.dsmoe_tally_attention(desc, *common, None, tally, ws, c.status)
        torch.cuda.synchronize()
        assert c.status.item() == 0
        return c.out.clone(), c.lse.clone(), tally.clone()
    return size, once


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("plain_heads", [False, True])
def test_workspaces(name, plain_heads):
    """plain_heads: one head's shared keys, or caches, for all, which no tensor map describes."""
    tokens, n_head, group, d, n_seq, L, P = CASES[name]
    c = Case(tokens, n_head, group, d, n_seq, L, P=P, seed=len(tokens))
    if plain_heads and P:
        c.Kp, c.Vp = (x[:1].contiguous().expand(n_head, P, d) for x in (c.Kp, c.Vp))
    elif plain_heads:
        c.K, c.V = (x[:, :1].contiguous().expand(n_seq, n_head, L, d) for x in (c.K, c.V))
    for kind in ((dm.ATTENTION_PREFIX,) if P else (dm.ATTENTION_WINDOW, dm.ATTENTION_TALLY)):
        size, once = calls(c, kind)
        results = []
        for fill in (0, 255, 127):
            room = torch.full((size + GUARD,), fill, dtype=torch.uint8, device="cuda")
            results.append(once(room[:size]))
            assert (room[size:] == fill).all()
        for other in results[1:]:
            for a, b in zip(results[0], other):
                assert torch.equal(a, b)
        assert torch.isfinite(results[0][0].float()).all()


def test_a_long_pair_among_many_short_ones():
    """Runs of single warps, the last pair as long as 250 units and the others one: its parts are no more than the sum has places for."""
    run_window(Case([(0, 0)] * 1183 + [(1, 3999)], 1, 1, 32, 2, 4000, seed=1), 2 ** 31 - 1)
    tokens = [(0, 0)] * 31 + [(1, 3999)]
    run_prefix(Case(tokens, 40, 1, 32, 2, 4000, P=500, seed=2))
