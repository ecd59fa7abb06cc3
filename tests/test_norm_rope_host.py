"""Host side of the norm and rotation call.  CPU only."""
import ctypes
import decimal
import subprocess

import pytest

from paper_2602_10825_amd import build
from tests.test_oracle_rope_kv4 import INVALID, UNSUPPORTED, L, P, ints, rope  # noqa: F401  (L: the library, a fixture)

FAR = ctypes.c_void_p(0x10008000)


def test_queries_in_place_need_rows_without_gaps(L):  # noqa: F811
    """q_out = q over the rows of a fused projection would write a row's queries over rows that are not read yet."""
    row = 12 * 128
    assert rope(L, q=P, out=P, qs=3 * row) == INVALID
    assert rope(L, q=P, out=P, qs=row + 8) == INVALID
    one = dict(A=1, off=ints(500), frame0=ints(0))
    assert rope(L, q=P, out=P, qs=3 * row, L_c=2, **one) == INVALID
    # other calls get as far as the frame's size
    large = dict(gh=1 << 20, gw=1 << 20)
    for ok in (dict(qs=row), dict(qs=3 * row, out=FAR), dict(qs=3 * row, L_c=1, **one)):
        assert rope(L, **{**dict(q=P, out=P), **ok, **large}) == UNSUPPORTED


# ------------------------------------------------------------------ frequencies
DRIVER = r"""
#include "rope_turns.hpp"
extern "C" __attribute__((visibility("default"))) void turns(double theta, const int32_t* dims, double* turns, float* rest) {
    fc_rope_turns(theta, dims, turns, rest);
}
"""


@pytest.fixture(scope="module")
def turns(tmp_path_factory):
    d = tmp_path_factory.mktemp("turns")
    src, so = d / "turns.hip", d / "turns.so"
    src.write_text(DRIVER)
    subprocess.run([build.HIPCC, "--offload-host-only", *build.FLAGS, "-shared", str(src), "-o", str(so)], check=True)
    f = ctypes.CDLL(str(so)).turns
    f.argtypes, f.restype = [ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p], None
    return f


@pytest.mark.parametrize("theta", [1.0, 1.5, 2.0, 100.0, 1e4, 5e5, 1e9, 1.7e308])
@pytest.mark.parametrize("dims", [(128, 0, 0), (44, 42, 42), (2, 0, 62), (0, 64, 0), (0, 0, 0)])
def test_frequencies_hold_more_than_64_bits(turns, theta, dims):
    """Relative to the axis' first frequency: at most 64 products round by 2^-64, 2^-58; the ratio's exponent is off by three roundings of
    2^-64 of x / i, x = 2 i ln(theta) / dim, which becomes 3 x e^-x 2^-64; the second part rounds by 2^-77.  Below 2^-57."""
    hi, lo = (ctypes.c_double * 64)(*[-1.0] * 64), (ctypes.c_float * 64)(*[-1.0] * 64)
    turns(theta, ints(*dims), ctypes.addressof(hi), ctypes.addressof(lo))
    with decimal.localcontext() as ctx:
        ctx.prec, ctx.Emin, ctx.Emax = 60, -10 ** 6, 10 ** 6
        two_pi = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
        p = 0
        for dim in dims:
            for i in range(dim // 2):
                want = (decimal.Decimal(theta).ln() * decimal.Decimal(-2 * i) / decimal.Decimal(dim)).exp() / two_pi
                got = decimal.Decimal(hi[p]) + decimal.Decimal(lo[p])
                assert abs(got - want) <= decimal.Decimal(2) ** -57 / two_pi, (dim, i)
                p += 1
    assert list(hi[p:]) == [-1.0] * (64 - p) and list(lo[p:]) == [-1.0] * (64 - p)
