"""The merge of ranges' partial results in 4-bit attention: what a range does not have takes no part."""
import pytest
import torch

from paper_2602_10825_amd import binding as B
from tests.test_gpu_kv4_attend import i32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,d,L_clean", [(12, 128, 4096), (3, 64, 2048), (1, 128, 1024), (40, 128, 640)])
def test_an_infinite_column_of_the_last_range_stays_infinite(H, d, L_clean):
    """32 rows, few heads: the keys are divided, and the slot's whole tile lies in the last range."""
    L_c = 32
    q, bufs, cap4, slots = make(H, H, d, 1, L_c, L_clean, 3)
    args = (*slots, L_c, L_clean, [0], i32(0), i32(1))
    plain = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *args)["out"].clone()
    slots[1][:, 0, 5] = float("inf")
    got = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *args)["out"]
    assert bool((got[..., 5] == float("inf")).all())
    others = [i for i in range(d) if i != 5]
    assert torch.equal(got[..., others], plain[..., others])
