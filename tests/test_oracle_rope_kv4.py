"""Pins for the oracle's head norm, rotation by several axes and 4-bit rows, and the library's refusals of bad arguments
for the calls that compute them.  CPU only."""
import ctypes
import math
import os

import numpy as np
import pytest

from oracle import flowcache_oracle as O
from paper_2602_10825_amd import binding

INVALID, UNSUPPORTED = 1, 2
P, NULL = ctypes.c_void_p(0x10000), None       # P is never dereferenced: validation fails first


# ------------------------------------------------------------------ rotation and norm
@pytest.mark.parametrize("halves", [False, True])
def test_rotation_is_multiplication_by_a_complex_number(halves):
    rng = np.random.default_rng(0)
    x, dims = rng.standard_normal((5, 2, 64)), (24, 20, 16)
    pos = np.array([[0, 0, 0], [1, 0, 0], [0, 3, 0], [7, 1, 2], [-4, 9, 30]])
    y = O.rotate(x, pos, dims, 10000.0, halves)
    z = x[..., :32] + 1j * x[..., 32:] if halves else x[..., 0::2] + 1j * x[..., 1::2]
    angle = np.zeros((5, 32))
    angle[:, :12] = pos[:, :1] * 10000.0 ** (-np.arange(12) / 12)
    angle[:, 12:22] = pos[:, 1:2] * 10000.0 ** (-np.arange(10) / 10)
    angle[:, 22:30] = pos[:, 2:] * 10000.0 ** (-np.arange(8) / 8)       # two pairs are left as they are
    z = z * np.exp(1j * angle)[:, None]
    want = np.concatenate([z.real, z.imag], -1) if halves else np.stack([z.real, z.imag], -1).reshape(x.shape)
    assert np.allclose(y, want, rtol=0, atol=1e-13)
    assert np.array_equal(y[0], x[0])


def test_products_of_rotated_rows_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 128))
    dims = (44, 42, 42)
    turn = lambda x, p: O.rotate(x, np.array([p]), dims, 10000.0, False)[0, 0]
    a = turn(q, (5, 6, 7)) @ turn(k, (2, 1, 9))
    b = turn(q, (1005, 16, 27)) @ turn(k, (1002, 11, 29))
    assert abs(a - b) < 1e-9


def test_norm_gives_unit_mean_square():
    x = np.random.default_rng(2).standard_normal((3, 2, 64)) * 100
    y = O.norm_heads(x, None, 0.0)
    assert np.allclose((y * y).mean(-1), 1.0, rtol=1e-14)
    w = np.arange(64, dtype=np.float32)
    assert np.allclose(O.norm_heads(x, w, 0.0), y * w)
    assert np.array_equal(O.norm_heads(np.zeros((1, 1, 64)), None, 1e-6), np.zeros((1, 1, 64)))


def test_positions_walk_a_frame_row_by_row():
    p = O.token_positions(10, 14, 2, 3)
    assert p[0].tolist() == [10, 0, 0] and p[2].tolist() == [10, 0, 2] and p[3].tolist() == [10, 1, 0]
    assert p[6].tolist() == [11, 0, 0] and p[13].tolist() == [12, 0, 1]


# ------------------------------------------------------------------ 4 bits
def test_every_code_is_its_own_nearest():
    codes = np.zeros((1, 16, 32), np.uint8)
    for c in range(16):
        codes[0, c, :] = c | (c << 4)
        codes[0, c, 0] = 0x70 | c                    # a 6 keeps the scale
        codes[0, c, 16] = 0x70 | c
    for byte in (1, 2, 100, 127, 200, 252):
        scales = np.full((1, 16, 2), byte, np.uint8)
        v = O.kv4_values(codes, scales)
        got, s = O.kv4_pack(v)
        assert np.array_equal(s, scales) and np.array_equal(O.kv4_values(got, s), v)


def test_packing_is_nearest_with_ties_to_even_and_does_not_drift():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((2, 50, 64)) * np.exp2(rng.integers(-40, 40, (2, 50, 1)).astype(np.float64))
    codes, scales = O.kv4_pack(x)
    v = O.kv4_values(codes, scales)
    s = np.exp2(scales.astype(np.float64) - 127).repeat(32, -1)
    grid = np.array([m * g for m in O.KV4_MAGNITUDES for g in (1, -1)])
    best = np.abs(np.minimum(np.abs(x / s), 6)[..., None] * np.sign(x)[..., None] - grid).min(-1)
    assert np.allclose(np.abs(v / s - np.sign(x) * np.minimum(np.abs(x / s), 6)), best, atol=1e-15)
    top = np.abs(x).reshape(2, 50, 2, 32).max(-1) / np.exp2(scales.astype(np.float64) - 127)
    assert top.min() >= 3.5 and top.max() < 7.0
    again, s2 = O.kv4_pack(v)
    assert np.array_equal(s2, scales) and np.array_equal(O.kv4_values(again, s2), v)
    ties = np.zeros((1, 1, 64))
    ties[0, 0, :9] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -2.5]
    assert O.kv4_values(*O.kv4_pack(ties))[0, 0, :9].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, -2]


def test_extreme_blocks():
    x = np.zeros((1, 4, 32))
    x[0, 1, 3], x[0, 1, 4] = np.inf, 1.0
    x[0, 2, 0], x[0, 2, 1] = 255 * 2.0 ** 120, 2.0 ** 127       # the largest bf16 value is cut off at 1.5 2^127
    x[0, 3, 7] = 2.0 ** -149
    x = np.concatenate([x, x], -1)
    codes, scales = O.kv4_pack(x)
    v = O.kv4_values(codes, scales)
    assert scales[0, :, 0].tolist() == [1, 255, 252, 1] and not v[0, 0].any() and not v[0, 3].any()
    assert np.isnan(v[0, 1]).all() and v[0, 2, 0] == 1.5 * 2.0 ** 127 and v[0, 2, 1] == 2.0 ** 127


# ------------------------------------------------------------------ refusals
@pytest.fixture(scope="module")
def L():
    assert os.path.exists(binding.LIB_PATH)
    return binding.lib()


def ints(*x):
    return ctypes.cast((ctypes.c_int32 * len(x))(*x), ctypes.c_void_p)


def rope(L, **kw):
    a = dict(q=P, qs=12 * 128, k=P, v=P, ks=12 * 128, dtype=1, H_q=12, H_k=12, d=128, norm=1, eps=1e-6, wq=P, wk=NULL,
             dims=ints(44, 42, 42), pairing=0, theta=1e4, gh=34, gw=60, frame0=ints(0, 5), L_c=100, L_clean=500, A=2,
             off=ints(500, 600), idx=P, n=P, out=P, kc=P, vc=P, hs=700 * 128, ts=128, cap=700, stream=NULL)
    a.update(kw)
    return L.flowcache_qk_norm_rope(*a.values())


def test_qk_norm_rope_rejects_bad_arguments(L):
    for name in ("q", "k", "dims", "frame0", "off", "idx", "n", "out", "kc", "vc"):
        assert rope(L, **{name: NULL}) == INVALID, name
    assert rope(L, A=0) == INVALID and rope(L, A=17) == INVALID and rope(L, L_c=0) == INVALID and rope(L, L_clean=-1) == INVALID
    assert rope(L, H_q=0) == INVALID and rope(L, H_k=0) == INVALID and rope(L, dtype=2) == INVALID and rope(L, cap=0) == INVALID
    assert rope(L, d=96) == UNSUPPORTED
    assert rope(L, gh=0) == INVALID and rope(L, gw=-3) == INVALID
    assert rope(L, gh=1 << 20, gw=1 << 20) == UNSUPPORTED
    for theta in (0.0, -1.0, 0.99, math.inf, math.nan):
        assert rope(L, theta=theta) == INVALID
    for eps in (-1e-6, math.inf, math.nan):
        assert rope(L, eps=eps) == INVALID
    assert rope(L, pairing=2) == INVALID
    for dims in ((43, 42, 42), (-2, 42, 42), (44, 44, 42)):
        assert rope(L, dims=ints(*dims)) == INVALID
    assert rope(L, dims=ints(2 ** 31 - 2, 2 ** 31 - 2, 2)) == INVALID
    assert rope(L, off=ints(500, 601)) == INVALID                        # past the capacity
    assert rope(L, off=ints(500, 599)) == INVALID                        # overlapping
    assert rope(L, off=ints(499, 600)) == INVALID                        # in the clean region
    assert rope(L, qs=12 * 128 - 8) == INVALID and rope(L, ks=0) == INVALID
    assert rope(L, qs=12 * 128 + 4) == UNSUPPORTED and rope(L, ks=12 * 128 + 2) == UNSUPPORTED
    assert rope(L, hs=100) == INVALID and rope(L, ts=64) == INVALID
    for name in ("q", "k", "v", "out", "kc", "vc"):
        assert rope(L, **{name: ctypes.c_void_p(0x10008)}) == UNSUPPORTED, name
    assert rope(L, L_c=2 ** 27 - 7, A=1, off=ints(0), frame0=ints(0), cap=2 ** 28, hs=2 ** 28 * 128, L_clean=0) == UNSUPPORTED
    assert rope(L, L_c=2 ** 30, A=2, off=ints(0, 2 ** 30 - 1), cap=2 ** 31 - 1, hs=2 ** 40, L_clean=0) == INVALID


def test_kv4_rejects_bad_arguments(L):
    assert L.flowcache_kv4_bytes(12, 1000, 128) == 12 * 1000 * 68 and L.flowcache_kv4_bytes(3, 7, 64) == 3 * 7 * 34
    assert L.flowcache_kv4_bytes(24, 2 ** 31 - 1, 128) == 24 * (2 ** 31 - 1) * 68
    for bad in ((0, 10, 128), (1, 0, 128), (1, -5, 64), (1, 10, 96)):
        assert L.flowcache_kv4_bytes(*bad) == 0

    def pack(**kw):
        a = dict(kc=P, vc=P, hs=500 * 64, ts=64, cap=500, dtype=1, H=2, d=64, pos=0, kept=NULL, count=100, k4=P, v4=P,
                 cap4=300, pos4=0, stream=NULL)
        a.update(kw)
        return L.flowcache_kv4_pack(*a.values())

    def unpack(**kw):
        a = dict(k4=P, v4=P, cap4=300, pos4=0, count=100, kc=P, vc=P, hs=500 * 64, ts=64, cap=500, dtype=1, H=2, d=64, pos=0,
                 stream=NULL)
        a.update(kw)
        return L.flowcache_kv4_unpack(*a.values())

    for call in (pack, unpack):
        assert call(k4=NULL) == INVALID and call(kc=NULL) == INVALID and call(v4=NULL) == INVALID and call(vc=NULL) == INVALID
        assert call(pos=401) == INVALID and call(pos=-1) == INVALID and call(pos4=201) == INVALID and call(pos4=-1) == INVALID
        assert call(count=-1) == INVALID and call(pos=2 ** 31 - 1) == INVALID and call(pos4=2 ** 31 - 1) == INVALID
        assert call(cap=0) == INVALID and call(cap4=0) == INVALID and call(H=0) == INVALID and call(dtype=3) == INVALID
        assert call(d=32) == UNSUPPORTED and call(hs=499 * 64) == INVALID and call(ts=63) == INVALID and call(ts=68, hs=500 * 68) == UNSUPPORTED
        assert call(k4=ctypes.c_void_p(0x10004)) == UNSUPPORTED and call(vc=ctypes.c_void_p(0x10002)) == UNSUPPORTED
        assert call(H=65536) == UNSUPPORTED
        assert call(count=2 ** 27 - 7, cap=2 ** 27, hs=2 ** 33, cap4=2 ** 27) == UNSUPPORTED
        assert call(count=0) == 0                                        # nothing to do, nothing launched
        assert call(count=0, v4=NULL, vc=NULL) == 0                      # K alone
    assert pack(kept=P, pos=1) == INVALID                                # rows from a list start nowhere
    assert pack(kept=P, count=301) == INVALID


def test_attend_kv4_rejects_bad_arguments(L):
    def attend(**kw):
        a = dict(q=P, k_new=P, v_new=P, k4=P, v4=P, cap4=600, kc=P, vc=P, hs=256 * 64, ts=64, cap=256, dtype=1, H_q=4, H_k=1, d=64,
                 L_c=128, L_clean=512, A=2, off=ints(0, 128), idx=P, n=P, scale=0.0, out=P, lse=P, ws=P, wsb=1 << 24, stream=NULL)
        a.update(kw)
        return L.flowcache_attend_kv4(*a.values())

    for name in ("q", "k_new", "v_new", "k4", "v4", "kc", "vc", "off", "idx", "n", "out"):
        assert attend(**{name: NULL}) == INVALID, name
    assert attend(dtype=5) == INVALID and attend(dtype=0, ts=66, hs=256 * 66) == UNSUPPORTED
    assert attend(cap4=511) == INVALID and attend(L_clean=-1) == INVALID
    assert attend(H_q=3, H_k=2) == INVALID and attend(A=0) == INVALID and attend(A=17) == INVALID and attend(L_c=0) == INVALID
    assert attend(d=96) == UNSUPPORTED and attend(ts=32) == INVALID and attend(hs=100) == INVALID
    assert attend(off=ints(0, 129)) == INVALID and attend(off=ints(0, 127)) == INVALID and attend(off=ints(-1, 128)) == INVALID
    for scale in (-1.0, math.inf, math.nan):
        assert attend(scale=scale) == INVALID
    for name in ("q", "k_new", "v_new", "k4", "v4", "kc", "vc", "out"):
        assert attend(**{name: ctypes.c_void_p(0x10004)}) == UNSUPPORTED, name
    assert attend(L_clean=2 ** 31 - 200, cap4=2 ** 31 - 1) == UNSUPPORTED  # positions beyond 32 bits
    assert attend(L_clean=2 ** 31 - 256 - 256, cap4=2 ** 31 - 1) == UNSUPPORTED     # or so near that a tile passes them
    for dtype in (0, 1):                                 # a launch of 2^32 threads
        assert attend(dtype=dtype, L_c=2 ** 24, off=ints(0, 2 ** 24), cap=2 ** 25, hs=2 ** 31, H_q=16) == UNSUPPORTED
    assert L.flowcache_attend_kv4_workspace(2, 128, 4, 64) == L.flowcache_attend_workspace(2, 128, 4, 1, 64, 0, 50)
    assert L.flowcache_attend_kv4_workspace(0, 128, 4, 64) == 0 and L.flowcache_attend_kv4_workspace(2, 128, 4, 96) == 0
