"""The heads' norm over the range of a float: y = x (mean x^2 + eps)^-1/2 has entries of at most sqrt(d), whatever x is.

Tolerance as in test_gpu_qk_norm_rope.py: 2^-19 of the length of a rotated pair, then half a step of the type (of an output below
the normal numbers, half of the least one)."""
import numpy as np
import pytest
import torch

from oracle import flowcache_oracle as O
from paper_2602_10825_amd import binding as B
from paper_2602_10825_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
LEAST = {"bf16": 2.0 ** -134, "f32": 2.0 ** -150}


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def both(dtype, x, eps, dims, grid=(2, 3), **kw):
    rows, H, d = x.shape
    q = B.to_device(x, dtype, DEV)
    cache = torch.zeros((H, rows, d), dtype=q.dtype, device=DEV)
    got = B.flowcache_qk_norm_rope(q, q, None, cache, None, rows, 0, [0], i32(0), i32(1), dims, grid, [3], norm_eps=eps, **kw)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(got.transpose(0, 1).view(bits), cache.view(bits))   # queries and keys take the same steps
    return O.widen(B.to_host(got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale,eps", [(1e18, 1e-6), (2e19, 1e-6), (1e25, 0.0), (1e30, 1e-6), (5e37, 0.0), (5e37, 1e30), (1e-12, 0.0), (1e-19, 0.0), (1e-23, 0.0),
                                       (1e-30, 0.0), (1e-37, 0.0), (1e-42, 0.0), (1e-20, 1e-6), (1e-16, 1e-32), (1e-20, 1e-42)])
def test_heads_of_any_magnitude(dtype, d, scale, eps):
    rows, H = 19, 3
    if dtype == "bf16":
        scale = max(scale, 1e-39)                                       # (below, all entries would be zero)
    rng = np.random.default_rng(d)
    x = rng.standard_normal((rows, H, d)) * scale
    x[3, 1] = 0
    x[3, 1, 5] = scale                                                  # one entry alone
    x[4, 2, 7] *= 100 if scale < 1e36 else 1
    x[5, 0] = rng.standard_normal(d)                                    # an ordinary head among them
    x = synth.to_storage(x.astype(np.float32), dtype)
    dims = (24, 20, 20)
    z = O.rotate(O.norm_heads(x, None, float(np.float32(eps))), O.token_positions(3, rows, 2, 3), dims, 10000.0, False)
    length = np.hypot(z[..., 0::2], z[..., 1::2]).repeat(2, -1)
    got = both(dtype, x, eps, dims)
    excess = np.abs(got - z) - STEP[dtype] * np.abs(z) - 2.0 ** -19 * length - LEAST[dtype]
    assert excess.max() <= 0, (excess.max(), np.unravel_index(excess.argmax(), excess.shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zeros_and_infinities(dtype):
    """eps = 0 makes a head of zeros NaN, an infinite entry makes NaN of its own pair; both stay in their heads."""
    x = np.ones((4, 3, 64), np.float32)
    x[1, 1] = 0
    x[2, 0, 6] = np.inf
    got = both(dtype, synth.to_storage(x, dtype), 0.0, (0, 0, 0))
    assert np.isnan(got[1, 1]).all() and np.isnan(got[2, 0, 6]) and np.array_equal(got[2, 0, 8:], np.zeros(56))
    bad = np.isnan(got)
    bad[1, 1] = bad[2, 0, 6:8] = False
    assert not bad.any()
    assert np.abs(got[0] - 1).max() <= 2.0 ** -19 + STEP[dtype]
