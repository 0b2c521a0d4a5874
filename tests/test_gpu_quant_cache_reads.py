"""Reading caches in 4 bits back of which little is held, of many sequences at once, and prompts on such caches (GPU required)."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import visible
from quant_cache_reference import QuantCase, quantise, tensors, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("n_seq,n_head,L,d,first,rows", [(300, 2, 70, 96, 3, 60), (129, 1, 90, 32, 0, 90), (128, 3, 33, 256, 32, 1), (5, 4, 700, 64, 100, 555),
                                                         (1, 1, 1, 32, 0, 1), (1000, 1, 7, 160, 1, 5),
                                                         (300, 2, 530, 256, 7, 520), (3, 2, 52000, 224, 1, 51999), (257, 2, 900, 224, 7, 890)])
def test_what_is_held_of_many_sequences(n_seq, n_head, L, d, first, rows, by_token):
    """Lengths below nothing, of nothing, before the first slot that is asked for, within them, and beyond; all of a sequence beside none of its neighbours.  The last
    sizes are more than four to six times what a grid takes at once."""
    rng = np.random.default_rng(n_seq + d)
    parts = []
    for _ in range(2):                             # (rows out of 1009, in another order for each sequence and head)
        code, scale = quantise(rng.standard_normal((1009, d)))
        at = rng.integers(0, 1009, (n_seq, n_head, L))
        parts.append((code[at].astype(np.int8), scale[at]))
    (K, K_scale), (V, V_scale) = (tensors(*p, by_token) for p in parts)
    cache = dm.make_quant_cache(K, V, K_scale, V_scale)
    for length in (None, rng.integers(-2, L + 3, n_seq), np.where(np.arange(n_seq) % 7 == 0, 2 ** 31 - 1, 0), np.where(np.arange(n_seq) == n_seq - 1, L, -2 ** 31),
                   np.full(n_seq, first)):
        out = [torch.full((n_seq, rows, n_head, d + 8), 3.0, dtype=torch.bfloat16, device="cuda")[..., 8:].transpose(1, 2) for _ in range(2)]
        at = None if length is None else torch.tensor(length, dtype=torch.int32, device="cuda")
        dm.dsmoe_quant_cache_read(cache, at, *out, first=first)
        held = np.full(n_seq, L) if length is None else length
        for o, p in zip(out, parts):
            want = torch.from_numpy(values(*p)[:, :, first:first + rows]).to(torch.bfloat16)      # (exact)
            want[torch.from_numpy(np.arange(first, first + rows) >= held[:, None])[:, None].expand(n_seq, n_head, rows)] = 3.0
            assert torch.equal(o.cpu(), want)


@pytest.mark.parametrize("room", [300, 3000])
@pytest.mark.parametrize("window,sinks", [(40, 3), (2 ** 31 - 1, 0)])
def test_prompts_of_many_sequences_in_caches_that_hold_little(window, sinks, room):
    """Prompts of 16 tokens of most of 140 sequences, at the start of their caches, at the end and between; nothing else is any number."""
    n_seq, n_head, L, d = 140, 4, 300, 64
    ends = [(16 + 37 * s) % 284 + 16 for s in range(n_seq)]
    tokens = [(s, e - 16 + i if s % 9 else -1) for s, e in enumerate(ends) for i in range(16)]
    seen = {(s, l) for s, p in tokens for l in visible(p, window if window < L else None, sinks)}
    c = QuantCase(tokens, n_head, 4, d, n_seq, L, seed=31, hide=lambda s, l: (s, l) not in seen)
    assert c.prompts()
    want = c.expected(window if window < L else None, sinks)
    for name in ("K", "V", "K_scale", "V_scale"):
        x = getattr(c, name)
        wide = torch.full((n_seq, n_head, room, x.shape[3]), 0xff if x.dtype == torch.uint8 else float("nan"), dtype=x.dtype, device="cuda")
        wide[:, :, :L] = x
        setattr(c, name, wide)
    cache = c.cache()
    desc = dm.make_quant_attention_desc(c.q, cache, c.scale, c.out)
    ws = torch.full((dm.dsmoe_quant_attention_workspace_size(desc),), 0xff, dtype=torch.uint8, device="cuda")
    dm.dsmoe_quant_attention(desc, cache, window, sinks, False, c.q, c.tok_seq, c.pos, c.out, c.lse, ws, c.status)
    c.check(want)
    assert c.status.item() == 0
