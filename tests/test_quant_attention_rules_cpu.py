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
