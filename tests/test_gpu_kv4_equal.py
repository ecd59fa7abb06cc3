"""4-bit attention against flowcache_attend on the unpacked rows, bit for bit: where both take 256-row blocks and the clean region ends with a
tile of 64 keys, they form the same products in the same order, and nothing is rounded for the 4-bit rows."""
import pytest
import torch

from paper_2602_10825_amd import binding as B
from tests.test_gpu_kv4_attend import DEV, i32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grow", [False, True])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("H_q,H_k,d,A,L_c,L_clean", [(24, 24, 128, 2, 1024, 2048), (24, 24, 64, 2, 1024, 2048), (24, 4, 128, 4, 1024, 64), (48, 8, 64, 1, 2048, 4096)])
def test_same_bits_in_256_row_blocks(H_q, H_k, d, A, L_c, L_clean, reverse, grow):
    q, bufs, cap4, slots = make(H_q, H_k, d, A, L_c, L_clean, 3, grow=grow)
    caches = [torch.zeros((H_k, L_clean + A * L_c, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    B.flowcache_kv4_unpack(*bufs, cap4, *caches, L_clean)
    for c, s in zip(caches, slots):
        c[:, L_clean:] = s[:, :A * L_c]
    off, idx, n = [i * L_c for i in range(A)], i32(*range(A)), i32(A)
    if reverse:
        off.reverse()
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)                    # no room to divide the keys
    a = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *slots, L_c, L_clean, off, idx, n, workspace=ws)
    b = B.flowcache_attend(q, None, None, *caches, L_c, L_clean, [L_clean + o for o in off], idx, n, workspace=ws)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
