"""K/V rows to 4 bits and back, bit for bit against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import flowcache_oracle as O
from paper_2602_10825_amd import binding as B
from paper_2602_10825_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def release_memory():
    """The blocks that these tests used go back to the device, not to the next test's torch.empty."""
    yield
    torch.cuda.empty_cache()


def rows(dtype, H, n, d, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((H, n, d))
    if kind == "wide":                                # every exponent, zeros, whole blocks of them
        x *= np.exp2(rng.integers(-150, 128, (H, n, d // 16)).astype(np.float64)).repeat(16, -1)
        x *= rng.random((H, n, d)) < 0.9
        x[:, ::7, :32] = 0
    if kind == "halves":                              # halfway between two magnitudes, and the scale's borders
        x = rng.choice([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 8], (H, n, d)) * rng.choice([-1, 1], (H, n, d))
        x *= np.exp2(rng.integers(-20, 20, (H, n, 1)).astype(np.float64))
    with np.errstate(over="ignore"):
        return synth.to_storage(np.clip(x, -3e38, 3e38).astype(np.float32), dtype)


def planes(buf, H, cap4, d):
    b = buf.cpu().numpy()
    split = H * cap4 * d // 2
    return b[:split].reshape(H, cap4, d // 2), b[split:].reshape(H, cap4, d // 32)


def filled(H, cap4, d, value=0xAB):
    return B.kv4_buffer(H, cap4, d, DEV).fill_(value)


@pytest.mark.parametrize("kind", ["normal", "wide", "halves"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,d,cap,pos,count,cap4,pos4", [
    (2, 64, 50, 0, 50, 50, 0), (3, 128, 77, 5, 64, 100, 31), (1, 128, 1, 0, 1, 1, 0), (12, 64, 333, 300, 33, 40, 7), (4, 128, 700, 1, 699, 701, 2),
])
def test_pack_and_unpack(dtype, kind, H, d, cap, pos, count, cap4, pos4):
    e = 4 if dtype == "f32" else 8
    k, v = (rows(dtype, H, cap, d, s, kind) for s in (1, 2))
    strided = [torch.zeros((H, cap + 1, d + e), dtype=TORCH[dtype], device=DEV)[:, :cap, :d] for _ in range(2)]
    for t, x in zip(strided, (k, v)):
        t.copy_(B.to_device(x, dtype, DEV))
    bufs = [filled(H, cap4, d) for _ in range(2)]
    B.flowcache_kv4_pack(*strided, *bufs, cap4, count, cache_pos=pos, pos4=pos4)
    back = [torch.full((H, cap + 1, d + e), 9.0, dtype=TORCH[dtype], device=DEV) for _ in range(2)]
    views = [t[:, :cap, :d] for t in back]
    B.flowcache_kv4_unpack(*bufs, cap4, *views, count, pos4=pos4, cache_pos=pos)
    for x, buf, t in zip((k, v), bufs, back):
        codes, scales = O.kv4_pack(x[:, pos:pos + count])
        got_c, got_s = planes(buf, H, cap4, d)
        assert np.array_equal(got_s[:, pos4:pos4 + count], scales) and np.array_equal(got_c[:, pos4:pos4 + count], codes)
        for p in (got_c, got_s):                       # the rows around are as they were
            assert (p[:, :pos4] == 0xAB).all() and (p[:, pos4 + count:] == 0xAB).all()
        val = O.kv4_values(codes, scales)
        whole = O.widen(B.to_host(t))
        assert np.array_equal(whole[:, pos:pos + count, :d], val)
        whole[:, pos:pos + count, :d] = 9
        assert (whole == 9).all()
    again = [filled(H, cap4, d) for _ in range(2)]
    B.flowcache_kv4_pack(*views, *again, cap4, count, cache_pos=pos, pos4=pos4)
    for a, b in zip(again, bufs):                      # (the sign of a zero is kept too)
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_byte_unpacks_to_its_value(dtype):
    """All 256 scales with all 16 codes, as another writer may have made them."""
    H, d, n = 1, 64, 256
    codes = np.tile(np.arange(16, dtype=np.uint8) * 17, (1, n, 2))
    scales = np.repeat(np.arange(256, dtype=np.uint8), 2).reshape(1, n, 2)
    buf = torch.from_numpy(np.concatenate([codes.ravel(), scales.ravel()])).to(DEV)
    out = torch.zeros((H, n, d), dtype=TORCH[dtype], device=DEV)
    B.flowcache_kv4_unpack(buf, None, n, out, None, n)
    with np.errstate(over="ignore"):
        want = O.kv4_values(codes, scales).astype(np.float32).astype(np.float64)
    got = O.widen(B.to_host(out))
    assert np.array_equal(got[:, 1:], want[:, 1:], equal_nan=True)
    assert np.array_equal(got[:, 0], want[:, 0])       # 2^-127, below the normal range


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_blocks_that_are_not_finite(dtype, bad):
    x = rows("f32", 1, 4, 64, 5)
    x[0, 1, 40], x[0, 2, 0] = bad, bad
    k = torch.from_numpy(x).to(DEV).to(TORCH[dtype])
    buf, out = filled(1, 4, 64), torch.zeros_like(k)
    B.flowcache_kv4_pack(k, None, buf, None, 4, 4)
    B.flowcache_kv4_unpack(buf, None, 4, out, None, 4)
    nan = torch.isnan(out)[0].view(4, 2, 32)
    assert nan.all(-1).tolist() == nan.any(-1).tolist() == [[False, False], [False, True], [True, False], [False, False]]
    again = filled(1, 4, 64)
    B.flowcache_kv4_pack(out, None, again, None, 4, 4)
    assert torch.equal(again, buf)


def test_a_selection_is_packed_where_it_lies():
    """Rows of a list: the same buffers as compacting the cache and packing its start; entries outside are skipped."""
    H, L, n, d = 3, 900, 401, 128
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v = (torch.randn((H, L, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    mass = torch.rand((H, L), generator=g, device=DEV)
    kept = B.flowcache_kv_select(k, L, n, mass)
    a = [filled(H, n, d) for _ in range(2)]
    B.flowcache_kv4_pack(k, v, *a, n, n, kept_idx=kept)
    k2, v2 = k.clone(), v.clone()
    B.flowcache_kv_compact(k2, v2, L, n, kept)
    b = [filled(H, n, d) for _ in range(2)]
    B.flowcache_kv4_pack(k2, v2, *b, n, n)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    bad = kept.clone()
    bad[0, 5], bad[1, 7], bad[2, 400], bad[2, 3] = -1, L, 2 ** 31 - 1, -2 ** 31
    c = [filled(H, n, d) for _ in range(2)]
    B.flowcache_kv4_pack(k, v, *c, n, n, kept_idx=bad)
    for x, y in zip(c, a):
        for p, q in zip(planes(x, H, n, d), planes(y, H, n, d)):
            q = q.copy()
            for h, i in ((0, 5), (1, 7), (2, 400), (2, 3)):
                q[h, i] = 0xAB
            assert np.array_equal(p, q)


def test_long_buffers_and_no_rows():
    """Bytes and elements past 2^31; nothing is touched by a count of zero."""
    H, d, cap = 2, 128, 1 << 23
    k = torch.zeros((H, cap, d), dtype=torch.bfloat16, device=DEV)
    x = torch.randn((H, 64, d), device=DEV).to(torch.bfloat16)
    k[:, -64:] = x
    cap4 = 1 << 26                                     # codes alone 2^33 bytes
    buf = B.kv4_buffer(H, cap4, d, DEV)
    small = filled(H, 64, d)
    B.flowcache_kv4_pack(k, None, buf, None, cap4, 64, cache_pos=cap - 64, pos4=cap4 - 64)
    B.flowcache_kv4_pack(x, None, small, None, 64, 64)
    k[:, -64:] = 0
    B.flowcache_kv4_unpack(buf, None, cap4, k, None, 64, pos4=cap4 - 64, cache_pos=cap - 64)
    y = torch.zeros_like(x)
    B.flowcache_kv4_unpack(small, None, 64, y, None, 64)
    assert torch.equal(k[:, -64:], y) and bool(y.any()) and not bool(k[:, :64].any())
    before = small.clone()
    B.flowcache_kv4_pack(x, None, small, None, 64, 0, cache_pos=64, pos4=64)
    B.flowcache_kv4_unpack(small, None, 64, y, None, 0)
    assert torch.equal(small, before)


def test_refusals():
    k = torch.zeros((2, 10, 64), dtype=torch.bfloat16, device=DEV)
    buf = B.kv4_buffer(2, 10, 64, DEV)
    B.flowcache_kv4_pack(k, None, buf, None, 10, 10)
    with pytest.raises(ValueError):
        B.flowcache_kv4_pack(k, None, buf, None, 11, 10)              # the buffer is smaller than that
    with pytest.raises(ValueError):
        B.flowcache_kv4_unpack(buf.cpu(), None, 10, k, None, 10)
    with pytest.raises(ValueError):
        B.flowcache_kv4_pack(k, None, buf.view(torch.int8), None, 10, 10)
    for kw in (dict(count=11), dict(count=1, pos4=10), dict(count=1, cache_pos=10), dict(count=-1), dict(count=1, cache_pos=-1)):
        with pytest.raises(B.FlowCacheError):
            B.flowcache_kv4_pack(k, None, buf, None, 10, **kw)
        with pytest.raises(B.FlowCacheError):
            B.flowcache_kv4_unpack(buf, None, 10, k, None, **kw)
    with pytest.raises(AssertionError):
        B.flowcache_kv4_pack(k, None, buf, None, 10, 4, kept_idx=torch.zeros((2, 5), dtype=torch.int32, device=DEV))
    with pytest.raises(B.FlowCacheError):
        B.kv4_buffer(2, 0, 64, DEV)
