"""Attention on a clean region in 4 bits whose codes and scales are written out here: blocks of a row with scales of their own, keys and
values at both ends of the scale, and in fp32 the range that flowcache_attend has.

Tolerance, bf16: as in test_gpu_kv4_attend.py.  fp32, in units of 2^-24, relative to sum p |v|: a score is at most 130 additions (of
products in fp32; of three bf16 parts fewer) of products exact to 1, with the query's scaling 132 B, B the largest sum of |q k| times the
scale that the row sees, twice that for weight and sum; exponential, reference, parts and merge 60; the sums over n keys, one after
the other at worst, 2 n; and never more than the library's bar for fp32 attention, 1e-5.  Then half a
step of the output, and for sums below the normal numbers 2^-149 for each of the n keys; an infinity is expected where float64 rounds to one."""
import numpy as np
import pytest
import torch

from oracle import flowcache_oracle as O
from paper_2602_10825_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
# (H_q, H_k, d, A, L_c, L_clean): 32-row blocks, then 256-row blocks
SHAPES = [(2, 1, 64, 2, 40, 300), (4, 4, 128, 1, 33, 70), (12, 12, 128, 1, 1, 2049), (24, 12, 128, 2, 511, 95), (24, 24, 64, 2, 256, 640), (1, 1, 128, 3, 1500, 650)]


@pytest.fixture(scope="module", autouse=True)
def release_memory():
    """The blocks that these tests used go back to the device, not to the next test's torch.empty."""
    yield
    torch.cuda.empty_cache()


def rows4(rng, H, n, d, scales, spare=5):
    """Random codes with the given scale bytes [H, n, d / 32] -> (buffer with spare rows that are no numbers, values in float64)"""
    codes = rng.integers(0, 256, (H, n, d // 2), dtype=np.uint8)
    scales = np.broadcast_to(scales, (H, n, d // 32)).astype(np.uint8)
    pad = lambda x: np.concatenate([x, np.full((H, spare, x.shape[2]), 255, np.uint8)], 1).ravel()
    return torch.from_numpy(np.concatenate([pad(codes), pad(scales)])).to(DEV), O.kv4_values(codes, scales)


def normal(rng, *s):
    return rng.standard_normal(s)


class Case:
    """Inputs as float64 arrays, to be changed before check()."""

    def __init__(self, shape, dtype, seed=0, k_scales=127, v_scales=127):
        self.H_q, self.H_k, self.d, self.A, self.L_c, self.L = shape
        self.dtype, self.rng = dtype, np.random.default_rng(seed)
        rng, rows = self.rng, self.A * self.L_c
        self.k4, self.k_clean = rows4(rng, self.H_k, self.L, self.d, k_scales)
        self.v4, self.v_clean = rows4(rng, self.H_k, self.L, self.d, v_scales)
        self.q = normal(rng, rows, self.H_q, self.d)
        self.k, self.v = (normal(rng, self.H_k, rows, self.d) for _ in range(2))
        self.scale = 0.25 * self.d ** -0.5                    # (a code's root mean square is about 3)

    def check(self, k_ref=None, room=True, bar=1e-5, least_weight=0.0):
        dtype, A, L_c, L, d = self.dtype, self.A, self.L_c, self.L, self.d
        q, k, v = (torch.from_numpy(x.astype(np.float32)).to(DEV).to(dtype) for x in (self.q, self.k, self.v))
        idx, n, off = torch.arange(A, dtype=torch.int32, device=DEV), torch.tensor([A], dtype=torch.int32, device=DEV), [i * L_c for i in range(A)]
        ws = None if room else torch.empty(256, dtype=torch.uint8, device=DEV)
        got = B.flowcache_attend_kv4(q, None, None, self.k4, self.v4, L + 5, k, v, L_c, L, off, idx, n, softmax_scale=self.scale, workspace=ws)
        self.out, worst = got["out"].double(), 0.0
        kr = k.double() if k_ref is None else torch.from_numpy(k_ref.astype(np.float32)).to(DEV).to(dtype).double()
        scale = float(np.float32(self.scale))
        for c in range(A):
            seen, blk, g = (c + 1) * L_c, slice(c * L_c, (c + 1) * L_c), self.H_q // self.H_k
            kk = torch.cat([torch.from_numpy(self.k_clean).to(DEV), kr[:, :seen]], 1).repeat_interleave(g, 0)
            vv = torch.cat([torch.from_numpy(self.v_clean).to(DEV), v.double()[:, :seen]], 1).repeat_interleave(g, 0)
            qq = q[blk].double().transpose(0, 1)
            s = qq @ kk.transpose(1, 2).contiguous() * scale
            p = torch.softmax(s, -1)
            want, size = p @ vv, p @ vv.abs()
            want_lse = torch.logsumexp(s, -1)
            if dtype == BF:
                tol = 2.0 ** -8 * want.abs() + (2.0 ** -7 + 2.0 ** -13) * size + 2.0 ** -134
                lse_tol = torch.full_like(want_lse, 2.0 ** -8 + 1e-5)
            else:
                row = (qq.abs() @ kk.abs().transpose(1, 2).contiguous()).amax(-1) * scale
                u = (2.0 ** -24 * (2 * 132 * row + 60 + 2 * s.shape[-1])).clamp(max=bar)
                tol, lse_tol = 2.0 ** -24 * want.abs() + u[..., None] * size + 2.0 ** -149 * s.shape[-1] + least_weight * vv.abs().sum(1, keepdim=True), u + 2.0 ** -23 * want_lse.abs()
            inf = want.to(F32 if dtype == F32 else BF).isinf()
            have = self.out[blk].transpose(0, 1)
            assert torch.equal(have[inf], want[inf].to(have.dtype).sign() * float("inf"))
            err = torch.where(inf, torch.zeros_like(want), (have - want).abs() - torch.where(inf, torch.zeros_like(tol), tol))
            assert float(err.max()) <= 0, (c, float(err.max()), float(have[~inf].abs().max()))      # (a NaN fails too)
            assert not bool(have.isnan().any())
            assert float(((got["lse"][:, blk].double() - want_lse).abs() - lse_tol).max()) <= 0


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("room", [True, False])
def test_blocks_of_a_row_have_scales_of_their_own(shape, dtype, room):
    """Each of a row's blocks counts equally in the scores, at magnitudes up to 2^12 apart: another block's scale would show."""
    H_q, H_k, d, A, L_c, L = shape
    rng = np.random.default_rng(9)
    e = rng.permutation([-6, -1, 2, 6])[:d // 32]
    own = rng.integers(-1, 2, (H_k, L, d // 32))
    case = Case(shape, dtype, 1, k_scales=127 + e + own, v_scales=127 + rng.integers(-6, 7, (H_k, L, d // 32)))
    factor = np.exp2(e.astype(float)).repeat(32)
    case.q /= factor
    case.k *= factor
    case.check(room=room)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("low,high,power", [(1, 4, -124), (250, 253, 123), (1, 253, None)])
def test_keys_at_the_ends_of_the_scale(shape, dtype, low, high, power):
    """Scales of 2^-126 .. (half of it, the least code, is no normal bf16 number) and of 2^125; the last case mixes all."""
    H_q, H_k, d, A, L_c, L = shape
    rng = np.random.default_rng(3)
    bytes_ = rng.integers(low, high, (H_k, L, d // 32))
    case = Case(shape, dtype, 2, k_scales=bytes_)
    if power is None:                                    # block 0 small, the last one large, with queries to match
        at = np.concatenate([np.full(d // 64, -60), np.full(d // 64, 60)])
        case = Case(shape, dtype, 2, k_scales=127 + at + rng.integers(-1, 2, (H_k, L, d // 32)))
        case.q /= np.exp2(at.astype(float)).repeat(32)
        case.k *= np.exp2(at.astype(float)).repeat(32)
    else:
        case.k *= 2.0 ** power
        case.q *= 2.0 ** (-power // 2)
        case.scale *= 2.0 ** (-power - -power // 2)
    case.check()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,low,high,power", [(BF, 1, 4, -124), (F32, 1, 4, -124), (BF, 200, 203, 73), (F32, 225, 228, 100)])
def test_values_at_the_ends_of_the_scale(shape, dtype, low, high, power):
    """Sums of weights and values stay finite up to here (a weight before it is divided by their sum is at most 1 in fp32, 2^40 in bf16)."""
    H_q, H_k, d, A, L_c, L = shape
    case = Case(shape, dtype, 4, v_scales=np.random.default_rng(5).integers(low, high, (H_k, L, d // 32)))
    case.v *= 2.0 ** power
    case.check()


# ------------------------------------------------------------------ fp32: the range of flowcache_attend
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("power", [-120, -110, -100, 100, 120])
def test_queries_of_another_magnitude_than_the_keys(shape, power):
    case = Case(shape, F32, 6, k_scales=127 - power)
    case.q *= 2.0 ** power
    case.k *= 2.0 ** -power
    case.check()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("power", [-140, -128, -120])
def test_small_queries_with_a_large_scale(shape, power):
    """The scale is taken into the queries; what is small is so only before."""
    case = Case(shape, F32, 7)
    case.q *= 2.0 ** power
    case.scale *= 2.0 ** -(power // 2)
    case.k *= 2.0 ** -(power - power // 2)
    case.k4, case.k_clean = rows4(case.rng, case.H_k, case.L, case.d, 127 - (power - power // 2))
    case.check()


@pytest.mark.parametrize("shape", SHAPES)
def test_channels_of_opposite_magnitude(shape):
    H_q, H_k, d, A, L_c, L = shape
    e = np.concatenate([np.full(d // 64, 30), np.zeros(d // 64, int)])
    case = Case(shape, F32, 8, k_scales=127 + e)
    f = np.exp2(e.astype(float)).repeat(32)
    case.q /= f
    case.k *= f
    case.check()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("power", [24, 60, 100, -100, -106, -110, -112, -115, -118, -130, -140])
def test_a_value_column_of_another_magnitude(shape, power):
    """In the slots alone, and with the clean rows' values so small that only the column's own size counts."""
    case = Case(shape, F32, 9)
    case.v[:, :, 5] *= 2.0 ** power
    case.check()
    case = Case(shape, F32, 9, v_scales=np.where(np.arange(shape[2] // 32) == 0, max(1, 127 + min(power, 0) - 3), 127))
    case.v[:, :, :32] *= 2.0 ** min(power, 0)
    case.check()


@pytest.mark.parametrize("shape", SHAPES)
def test_the_largest_floats(shape):
    case = Case(shape, F32, 10)
    big = float(np.finfo(np.float32).max)
    case.v[:, 0, 3], case.v[:, case.L_c // 2, 4] = big, -big
    case.check()
    case = Case(shape, F32, 11)                       # a query of the largest float meets keys that have nothing there
    case.q[:, :, 7] = big
    case.k[:, :, 7] = 0
    case.scale = 2.0 ** -1 * case.scale
    codes = case.k4[:case.H_k * (case.L + 5) * case.d // 2].view(case.H_k, case.L + 5, case.d // 2)
    codes[:, :case.L, 3] &= 0x0f
    case.k_clean[:, :, 7] = 0
    case.check()


@pytest.mark.parametrize("shape", SHAPES)
def test_infinite_entries(shape):
    """A slot's key whose score is minus infinity has no weight; an infinite value makes its column infinite and nothing else."""
    case = Case(shape, F32, 12)
    case.q[:, :, 0] = np.abs(case.q[:, :, 0]) + 0.1
    far = case.k.copy()
    far[:, 0, 0] = -1e6
    if case.A * case.L_c > 1:
        case.k[:, 0, 0] = -np.inf
        case.check(k_ref=far)
    case = Case(shape, F32, 13)
    case.check()
    plain = case.out.clone()
    case.v[:, 0, 5] = np.inf
    args = case.q, case.k, case.v
    q, k, v = (torch.from_numpy(x.astype(np.float32)).to(DEV) for x in args)
    A, L_c = case.A, case.L_c
    got = B.flowcache_attend_kv4(q, None, None, case.k4, case.v4, case.L + 5, k, v, L_c, case.L, [i * L_c for i in range(A)],
                                 torch.arange(A, dtype=torch.int32, device=DEV), torch.tensor([A], dtype=torch.int32, device=DEV),
                                 softmax_scale=case.scale)["out"].double()
    assert bool((got[:, :, 5] == float("inf")).all())
    others = [i for i in range(case.d) if i != 5]
    assert float((got[..., others] - plain[..., others]).abs().max()) <= 1e-5 * float(plain.abs().max())
