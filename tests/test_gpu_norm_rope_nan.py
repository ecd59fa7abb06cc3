"""A NaN of any payload in a norm's weight is a NaN in the output; every finite bf16 value goes through as it is where nothing turns."""
import numpy as np
import pytest
import torch

from paper_2602_10825_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [0x7fc00000, 0x7fffffff, 0xffffffff, 0x7fff8000, 0xffc00000])
def test_weights_that_are_no_number(dtype, bits):
    d, H, rows = 64, 2, 5
    w = np.ones(d, np.float32)
    w.view(np.uint32)[9] = bits
    w = torch.from_numpy(w).to(DEV)
    q = torch.ones((rows, H, d), dtype=dtype, device=DEV)
    cache = torch.zeros((H, rows, d), dtype=dtype, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    got = B.flowcache_qk_norm_rope(q, q, None, cache, None, rows, 0, [0], i32(0), i32(1), (24, 20, 20), (2, 2), [1], q_weight=w, k_weight=w)
    for x in (got, cache.transpose(0, 1)):
        bad = torch.isnan(x.float())
        assert bool(bad[..., 8:10].all()) and int(bad.sum()) == rows * H * 2        # the element and the one it is turned with


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_every_bf16_value_goes_through(pairing):
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.where(torch.isfinite(x.float()), x, torch.zeros_like(x)).view(-1, 2, 64).to(DEV)
    rows = x.shape[0]
    cache = torch.zeros((2, rows, 64), dtype=x.dtype, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    got = B.flowcache_qk_norm_rope(x, x, None, cache, None, rows, 0, [0], i32(0), i32(1), (0, 0, 0), (2, 2), [1], pairing=pairing, norm_eps=None)
    assert torch.equal(got, x) and torch.equal(cache.transpose(0, 1), x)          # (as numbers: a zero may change its sign)
