"""Host side of the norm and rotation call.  CPU only."""
import ctypes

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
