"""fp32 4-bit attention of rows that one key takes for itself: every other weight is below 2^-86, also in whole halves of a tile.

Tolerance as derived in test_gpu_kv4_range.py.  Its other bar, 1e-5, cannot hold here: the scale times log2(e) is rounded to a float, so a score
of 200 is off by 200 2^-24 = 1.2e-5 from that alone, and so is, relative to itself, the weight of a key that lies that far below.  And a weight below 2^-126 is no normal float, with the exponents'
reference at most 2^4 above the largest one: what is below 2^-122 of the largest weight may be zero."""
import pytest
import torch

from tests.test_gpu_kv4_range import F32, SHAPES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("gap", [60, 70, 95, 200])
@pytest.mark.parametrize("key", [0, 5, 23])
def test_one_key_outweighs_all(shape, gap, key):
    """The slot's key `key` scores `gap` (natural units) above the others, and half of its values are zero."""
    case = Case(shape, F32, 20)
    key = min(key, case.L_c - 1)
    case.q[:, :, 0] = 8.0
    case.k[:, :, 0] = 0.0
    case.k[:, key, 0] = gap / (8.0 * case.scale)
    codes = case.k4[:case.H_k * (case.L + 5) * case.d // 2].view(case.H_k, case.L + 5, case.d // 2)
    codes[:, :case.L, 0] &= 0xf0                              # the clean rows have nothing there
    case.k_clean[:, :, 0] = 0
    case.v[:, key, ::2] = 0.0
    case.check(bar=1.0, least_weight=2.0 ** -122)
