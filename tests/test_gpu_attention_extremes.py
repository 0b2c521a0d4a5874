"""The attention steps where a row's logits jump far, and where queries, keys or values are no numbers: each row's result is its own formula's, whatever the
rows, tiles and parts beside it hold (GPU required)."""
import numpy as np
import pytest
import torch

import cache_attention_reference as ref
from cache_attention_reference import Case
from test_gpu_attention_tiles import prompt
from test_gpu_window_attention import run

pytestmark = pytest.mark.gpu

LN2 = float(np.float32(np.log(2)))


def with_logits(c, base, peaks):
    """Logits of `base` and at the keys `peaks` of theirs, in base 2, give or take what the other columns add; values far below 1."""
    q, K = c.q.float().cpu(), c.K.float().cpu()
    q[..., 1:] *= 2.0 ** -5
    q[..., 0], K[..., 0] = 1.0, base
    for l, x in peaks.items():
        K[:, :, l, 0] = x
    c.q, c.K, c.V = q.to(torch.bfloat16).cuda(), K.to(torch.bfloat16).cuda(), c.V * 2.0 ** -10
    c.q_np, c.K_np, c.V_np = (x.float().cpu().numpy() for x in (c.q, c.K, c.V))
    return c


@pytest.mark.parametrize("jump", [40.0, 100.0, 125.5, 126.5, 127.5, 140.0])
@pytest.mark.parametrize("at", [50, 140, 200, 300])
def test_logits_that_jump_within_a_tile(jump, at):
    """In the first, the middle and the last tile of keys, and a second key of half the weight in the tile after it."""
    peaks = {at: jump, min(at + 130, 320): jump - 1}
    run(with_logits(Case(prompt(0, 383, 60), 1, 5, 64, 1, 384, seed=at, scale=LN2), 0.0, peaks), 2 ** 31 - 1)


@pytest.mark.parametrize("jump", [40.0, 100.0, 125.5, 126.5, 127.5, 140.0])
@pytest.mark.parametrize("at", [140, 200, 900])
def test_logits_that_jump_within_a_part(jump, at):
    """Keys in four parts, and another part whose largest logit was there from its first tile on."""
    c = Case(prompt(0, 1023, 60), 1, 5, 128, 1, 1024, seed=at, scale=LN2)
    run(with_logits(c, -100.0, {at: jump - 100, 600: jump - 97}), 2 ** 31 - 1)
