"""Which kernels calls of dsmoe_quant_attention take (no GPU needed)."""
import ctypes

import pytest

import paper_2404_05567_b200 as dm
from paper_2404_05567_b200 import build as dm_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    dm_build.build()


def _whole(pairs, seen, warps=12, sms=148):
    f = getattr(dm.lib(), "_ZN5dsmoe11quant_wholeExxii")
    f.restype, f.argtypes = ctypes.c_bool, [ctypes.c_longlong, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return f(pairs, seen, warps, sms)


@pytest.mark.parametrize("sms", [7, 132, 148, 160])
@pytest.mark.parametrize("warps", [4, 6, 8, 12])
def test_a_cta_per_pair_takes_few_keys_of_any_number_of_pairs(warps, sms):
    """However many pairs there are: one of them may be the only one that has all of the keys, and then the call is as long as one CTA takes for them."""
    for pairs in range(1, sms + 1):
        assert not _whole(pairs, 6 * 32 * warps + 1, warps, sms) and not _whole(pairs, 131072, warps, sms) and not _whole(pairs, 1 << 30, warps, sms)
        assert _whole(pairs, 1, warps, sms) and _whole(pairs, 3 * 32 * warps, warps, sms)
    assert not _whole(sms + 1, 1, warps, sms)


def test_a_cta_per_pair_of_many_keys_only_where_few_ctas_stay_idle():
    assert _whole(148, 2304) and _whole(128, 2304) and not _whole(128, 2305) and not _whole(64, 2304) and _whole(64, 2029) and not _whole(64, 2030)
    assert _whole(4, 1184) and not _whole(4, 1185)


def _size(T, n_seq, n_head, group, d_head, L, scale):
    desc = dm.AttentionDesc(T, n_head, group, d_head, n_seq, L, scale)
    desc.q_stride[:] = desc.o_stride[:] = (n_head * group * d_head, group * d_head, d_head)
    return dm.dsmoe_quant_attention_workspace_size(desc)


def _as_prompts(*sizes):
    """Calls with a negative scale are never taken as prompts; the others' workspaces differ from theirs if they are."""
    return _size(*sizes, 0.1) != _size(*sizes, -0.1)


@pytest.mark.parametrize("T,n_head,group,d,L", [(64, 1, 16, 128, 1000), (64, 1, 16, 128, 1200), (32, 4, 16, 128, 1000), (128, 1, 12, 96, 640), (148, 1, 5, 128, 2000)])
def test_what_one_launch_takes_is_not_taken_as_a_prompt(T, n_head, group, d, L):
    assert not _as_prompts(T, 1, n_head, group, d, L)
    assert _as_prompts(2 * T + 100, 1, n_head, group, d, L)


@pytest.mark.parametrize("group,d,few,many", [(1, 64, 31, 32), (2, 64, 15, 16), (3, 128, 15, 16), (4, 128, 15, 16), (5, 128, 12, 13), (6, 96, 10, 11), (8, 128, 7, 8), (16, 128, 7, 8)])
def test_tokens_of_a_sequence_that_fill_little_of_a_tile_are_not_taken_as_prompts(group, d, few, many):
    for n_seq in (2, 32):
        assert not _as_prompts(few * n_seq, n_seq, 4, group, d, 24000) and _as_prompts(many * n_seq, n_seq, 4, group, d, 24000)


@pytest.mark.parametrize("T,n_seq,n_head,group,d,L", [(1024, 64, 64, 5, 128, 1 << 20), (64, 1, 512, 5, 128, 1 << 23), (1 << 17, 1 << 12, (1 << 13) - 1, 1, 128, 1 << 30)])
def test_copies_beyond_any_workspace_are_not_made(T, n_seq, n_head, group, d, L):
    """Rows of a cache may be shared (strides of 0), so that sizes go further than memory does: such calls are taken as single tokens, not refused."""
    size = _size(T, n_seq, n_head, group, d, L, 0.1)
    assert size == _size(T, n_seq, n_head, group, d, L, -0.1) < 2 ** 36
    assert _as_prompts(T, n_seq, min(n_head, 8), group, d, min(L, 1 << 12))
