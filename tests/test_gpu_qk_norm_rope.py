"""Head norm and rotation by (time, height, width) into query rows and K/V slots, against float64.

Tolerance.  In units of u = 2^-24, relative to the length of a rotated pair: the sum of 128 squares is off by at most 14 u,
its root by half of that; root, mean and eps 3 u, the two factors of an element 2 u, an angle's last bits 2 u (a float's half
turn), sine and cosine 4 u, product and sum of the rotation 2 u: 20 u, bound 32 u = 2^-19; then one rounding to the type, half a step."""
import numpy as np
import pytest
import torch

from oracle import flowcache_oracle as O
from paper_2602_10825_amd import binding as B
from paper_2602_10825_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def release_memory():
    """The blocks that these tests used go back to the device, not to the next test's torch.empty."""
    yield
    torch.cuda.empty_cache()


def inputs(dtype, rows, H, d, seed, scale=1.0):
    x = (np.random.default_rng(seed).standard_normal((rows, H, d)) * scale).astype(np.float32)
    return synth.to_storage(x, dtype)


def reference(x, pos, w, eps, dims, theta, halves):
    y = O.widen(x) if eps is None else O.norm_heads(x, w, eps)
    z = O.rotate(y, pos, dims, theta, halves)
    d = z.shape[-1]
    if halves:
        r = np.hypot(z[..., :d // 2], z[..., d // 2:])
        return z, np.concatenate([r, r], -1)
    return z, np.hypot(z[..., 0::2], z[..., 1::2]).repeat(2, -1)


def run(dtype, H_q, H_k, d, A, L_c, rec, grid, dims, frame0, halves=False, weights=True, eps=1e-6, theta=10000.0, L_clean=40, gap=8,
        with_v=True, fused=True, scale=1.0, tok_pad=0, idx=None, n=None, seed=0, reverse=False, stream=None):
    rows, e = A * L_c, 4 if dtype == "f32" else 8
    q, k, v = (inputs(dtype, rows, H, d, seed + i, scale) for i, H in enumerate((H_q, H_k, H_k)))
    if fused:
        x = torch.cat([B.to_device(t, dtype, DEV) for t in (q, k, v)], 1)
        if tok_pad:                       # rows of a wider tensor still
            wide = torch.full((rows, x.shape[1] * d + tok_pad), 7.0, dtype=x.dtype, device=DEV)
            wide[:, :x.shape[1] * d] = x.reshape(rows, -1)
            x = wide.as_strided((rows, x.shape[1], d), (wide.stride(0), d, 1))
        tq, tk, tv = x.split((H_q, H_k, H_k), 1)
    else:
        tq, tk, tv = (B.to_device(t, dtype, DEV) for t in (q, k, v))
    rng = np.random.default_rng(seed + 9)
    wq, wk = (None, None) if not weights else (rng.uniform(-2, 2, d).astype(np.float32) for _ in range(2))
    off = [L_clean + i * (L_c + gap) for i in range(A)]
    if reverse:
        off.reverse()
    cap = L_clean + A * (L_c + gap)
    caches = [torch.full((H_k, cap + 3, d + e), 3.0, dtype=TORCH[dtype], device=DEV)[:, :cap, :d] for _ in range(2)]
    t_idx = torch.tensor(list(rec) + [-1] * (A - len(rec)) if idx is None else idx, dtype=torch.int32, device=DEV)
    t_n = torch.tensor([len(rec) if n is None else n], dtype=torch.int32, device=DEV)
    q_out = torch.full((rows, H_q, d), 5.0, dtype=TORCH[dtype], device=DEV)
    torch.cuda.synchronize()
    got = B.flowcache_qk_norm_rope(tq, tk, tv if with_v else None, caches[0], caches[1] if with_v else None, L_c, L_clean, off, t_idx, t_n,
                                   dims, grid, frame0, theta, "halves" if halves else "interleaved",
                                   *(None if w is None else torch.from_numpy(w).to(DEV) for w in (wq, wk)), norm_eps=eps, q_out=q_out,
                                   stream=stream)
    torch.cuda.synchronize()
    assert got is q_out
    ref_q = np.full((rows, H_q, d), 5.0)
    tol_q = np.zeros_like(ref_q)
    ref_k, ref_v = np.full((H_k, cap, d), 3.0), np.full((H_k, cap, d), 3.0)
    tol_k = np.zeros_like(ref_k)
    listed = list(rec) + [-1] * (A - len(rec)) if idx is None else idx
    for r in range(min(A, len(rec) if n is None else n)):
        c = listed[r]
        if not 0 <= c < A:
            continue
        pos, blk = O.token_positions(frame0[c], L_c, *grid), slice(r * L_c, (r + 1) * L_c)
        for x, w, out, tol in ((q, wq, ref_q, tol_q), (k, wk, ref_k, tol_k)):
            z, length = reference(x[blk], pos, w, eps, dims, theta, halves)
            t = STEP[dtype] * np.abs(z) + 2.0 ** -19 * length
            if out is ref_q:
                out[blk], tol[blk] = z, t
            else:
                s = slice(off[c], off[c] + L_c)
                out[:, s], tol[:, s] = z.transpose(1, 0, 2), t.transpose(1, 0, 2)
        if with_v:
            ref_v[:, off[c]:off[c] + L_c] = O.widen(v[blk]).transpose(1, 0, 2)
    got_q, got_k, got_v = (O.widen(B.to_host(t)) for t in (q_out, caches[0], caches[1]))
    assert np.array_equal(np.isnan(got_q), np.isnan(ref_q)) and np.array_equal(np.isnan(got_k), np.isnan(ref_k))
    for g, ref, tol in ((got_q, ref_q, tol_q), (got_k, ref_k, tol_k)):
        worst = np.nanmax(np.abs(g - ref) - tol)
        assert worst <= 0, (worst, np.nanmax(np.abs(g - ref)))
    assert np.array_equal(got_v, ref_v)
    for t in caches:                       # the padding of the rows, and the rows past the capacity
        whole = torch.as_strided(t, (H_k, cap + 3, d + e), t.stride())
        assert bool((whole[:, cap:] == 3).all()) and bool((whole[..., d:] == 3).all())
    return q_out, caches


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H_q,H_k,d,A,L_c,rec,grid,dims", [
    (12, 12, 128, 2, 101, [1], (5, 7), (44, 42, 42)),
    (8, 2, 128, 3, 64, [0, 2], (4, 4), (44, 42, 42)),
    (4, 1, 64, 2, 128, [0, 1], (8, 16), (24, 20, 20)),
    (3, 3, 64, 4, 37, [0, 1, 2, 3], (1, 1), (64, 0, 0)),      # time alone, every token its own frame
    (5, 5, 128, 1, 1, [0], (34, 60), (0, 64, 64)),            # one token
    (1, 1, 64, 16, 3, list(range(16)), (2, 1), (16, 16, 16)), # a quarter of the head is left as it is
    (2, 2, 128, 1, 9, [0], (3, 3), (0, 0, 0)),                # nothing turns
])
def test_matches_float64(dtype, halves, H_q, H_k, d, A, L_c, rec, grid, dims):
    frame0 = [3 + 11 * i for i in range(A)]
    run(dtype, H_q, H_k, d, A, L_c, rec, grid, dims, frame0, halves=halves, tok_pad=8 * (A % 2), reverse=A == 3, seed=L_c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("frame0", [-17, 65535, 10 ** 7, 2 ** 31 - 100])
def test_far_positions_keep_their_angles(dtype, frame0):
    run(dtype, 2, 1, 128, 1, 50, [0], (1, 1), (128, 0, 0), [frame0], seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_options(dtype):
    case = (dtype, 3, 3, 64, 2, 33, [0, 1], (4, 4), (24, 20, 20), [0, 9])
    run(*case, eps=None)                              # rotation alone
    run(*case, weights=False)
    run(*case, eps=0.0, scale=1e-3)
    run(*case, eps=0.5, scale=0.1, theta=100.0)
    run(*case, eps=1e-6, scale=3e4)                   # squares of 1e9, sums beyond 1e11
    run(*case, with_v=False, fused=False)
    run(*case, scale=0.0)                             # zero rows stay zero


def test_a_nan_stays_in_its_head():
    dtype, d, H = "bf16", 128, 3
    x = torch.randn(8, H, d, device=DEV, dtype=torch.bfloat16)
    x[2, 1, 5] = float("nan")
    k = torch.randn(8, 2, d, device=DEV, dtype=torch.bfloat16)
    cache = torch.zeros(2, 8, d, device=DEV, dtype=torch.bfloat16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    out = B.flowcache_qk_norm_rope(x, k, None, cache, None, 8, 0, [0], i32(0), i32(1), (44, 42, 42), (2, 2), [0])
    bad = torch.isnan(out).any(-1)
    assert bad.nonzero().tolist() == [[2, 1]] and bool(torch.isfinite(cache).all())


@pytest.mark.parametrize("idx,n", [([1, -1, -1], 1), ([0, 1, 2], 0), ([-1, 7, 2], 3), ([2, -5, 10 ** 9], 99), ([0, 1, 2], -4)])
def test_bad_lists_touch_nothing_else(idx, n):
    run("bf16", 4, 2, 64, 3, 20, [0], (3, 3), (24, 20, 20), [0, 4, 8], idx=idx, n=n)


def test_queries_in_place_and_a_second_stream():
    run("bf16", 12, 12, 128, 2, 700, [0, 1], (5, 7), (44, 42, 42), [0, 20], stream=torch.cuda.Stream())
    q = torch.randn(66, 4, 64, device=DEV, dtype=torch.bfloat16)
    k = torch.randn(66, 4, 64, device=DEV, dtype=torch.bfloat16)
    caches = [torch.zeros(4, 66, 64, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    args = (66, 0, [0], i32(0), i32(1), (24, 20, 20), (5, 5), [3])
    for pairing in ("interleaved", "halves"):
        want = B.flowcache_qk_norm_rope(q, k, k, *caches, *args, pairing=pairing)
        same = q.clone()
        got = B.flowcache_qk_norm_rope(same, k, k, *caches, *args, pairing=pairing, q_out=same)
        assert got is same and torch.equal(got, want) and not torch.equal(got, q)


def test_without_a_norm_the_weights_are_not_read():
    q = torch.randn(5, 2, 64, device=DEV)
    cache = torch.zeros(2, 5, 64, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    w = torch.full((64,), float("nan"), device=DEV)
    args = (q, q, None, cache, None, 5, 0, [0], i32(0), i32(1), (24, 20, 20), (2, 2), [9])
    a, b = (B.flowcache_qk_norm_rope(*args, q_weight=x, k_weight=x, norm_eps=None) for x in (None, w))
    assert torch.equal(a, b) and bool(torch.isfinite(cache).all())


def test_many_tokens_of_many_heads():
    """A launch over more tokens than the chip holds, and offsets beyond 2^31 elements in the cache."""
    H, d, L_c, cap = 24, 128, 9361, 1 << 20
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn(L_c, 3 * H, d, generator=g, device=DEV).to(torch.bfloat16)
    cache = [torch.zeros(H, cap, d, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    off = cap - L_c
    q, k, v = x.split(H, 1)
    out = B.flowcache_qk_norm_rope(q, k, v, *cache, L_c, 0, [off], i32(0), i32(1), (44, 42, 42), (30, 52), [1000])
    pos = O.token_positions(1000, L_c, 30, 52)
    rows = np.array([0, 1, 1559, 1560, 5000, L_c - 1])
    for got, src in ((out[rows], q), (cache[0][:, off + rows].transpose(0, 1), k)):
        z, length = reference(B.to_host(src[rows]), pos[rows], None, 1e-6, (44, 42, 42), 10000.0, False)
        assert np.all(np.abs(O.widen(B.to_host(got)) - z) <= 2.0 ** -8 * np.abs(z) + 2.0 ** -19 * length)
    assert torch.equal(cache[1][:, off:], v.transpose(0, 1)) and not bool(cache[0][:, :off].any())


def test_refusals():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, device=DEV, dtype=dtype)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)

    def call(q=z(8, 4, 64), k=z(8, 2, 64), v=z(8, 2, 64), kc=z(2, 8, 64), vc=z(2, 8, 64), L_c=8, off=(0,), frame0=(0,), dims=(24, 20, 20),
             grid=(2, 2), **kw):
        return B.flowcache_qk_norm_rope(q, k, v, kc, vc, L_c, 0, off, i32(0), i32(1), dims, grid, frame0, **kw)

    call()
    for kw in (dict(q=z(8, 4, 64, dtype=torch.float32)), dict(k=z(8, 2, 32)), dict(v=z(7, 2, 64)), dict(q=z(8, 64, 4).transpose(1, 2)),
               dict(pairing="pairs"), dict(frame0=(0, 1)), dict(L_c=4), dict(q_weight=z(64)), dict(k_weight=z(32, dtype=torch.float32)),
               dict(kc=z(2, 8, 64).cpu()), dict(q=z(8, 4, 64).cpu()), dict(dims=(32, 32)), dict(grid=(2, 2, 2)),
               dict(v=z(8, 4, 64)[:, :2])):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(dims=(25, 20, 19)), dict(norm_eps=-1.0), dict(theta=0.0), dict(off=(1,)), dict(grid=(0, 2))):
        with pytest.raises(B.FlowCacheError):
            call(**kw)
    with pytest.raises(TypeError):
        h = torch.float16
        call(q=z(8, 4, 64, dtype=h), k=z(8, 2, 64, dtype=h), v=z(8, 2, 64, dtype=h), kc=z(2, 8, 64, dtype=h), vc=z(2, 8, 64, dtype=h))
