"""Attention on a clean region in 4 bits against float64 on the values that the 4-bit rows stand for.

Tolerance.  A weight is rounded to bf16, half a step of 2^-8, and so is its share of the row's sum: the row is off by at most
2^-8 (sum p |v| + |out|) <= 2^-7 sum p |v|.  Scores, exponentials and sums in fp32 add about 2^-16 of that: 2^-13.  Then the output's rounding,
2^-8 |out|.  The logarithm of the sum: 2^-8 for the weights, 1e-5 for the rest.

fp32, in units of 2^-24.  A score is 24 (a slot's key 48) additions of products that are exact to 1: 48 B, B the largest sum of
|q k| times the scale that the row sees; twice that for weight and sum.  Exponential, weight's parts and reference 16.  The row's sums over the
tiles of one wavefront, an 8th of them, 12 additions each of 32 keys, and the merge of 8 wavefronts and up to 32 ranges 40 (256-row
blocks: one addition per tile, of all tiles, and 12 within a tile, which is less): all times sum p |v|."""
import numpy as np
import pytest
import torch

from paper_2602_10825_amd import binding as B
from tests.test_gpu_kv4 import filled

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def release_memory():
    """The blocks that these tests used go back to the device, not to the next test's torch.empty."""
    yield
    torch.cuda.empty_cache()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def make(H_q, H_k, d, A, L_c, L_clean, seed, spare=9, grow=False, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    q = n(A * L_c, H_q, d).to(dtype)
    clean = [n(H_k, max(L_clean, 1), d) for _ in range(2)]
    slots = [n(H_k, A * L_c + 16, d) for _ in range(2)]
    if grow:                                            # scores that grow along the keys: the reference is raised again and again
        clean[0] *= torch.linspace(0.05, 4, max(L_clean, 1), device=DEV)[None, :, None]
        slots[0] *= torch.linspace(3, 6, A * L_c + 16, device=DEV)[None, :, None]
    clean, slots = [x.to(torch.bfloat16) for x in clean], [x.to(dtype) for x in slots]
    cap4 = L_clean + spare
    bufs = []
    for x in clean:
        b = filled(H_k, cap4, d, 255)                   # rows past the clean region are not numbers
        if L_clean:
            tmp = filled(H_k, L_clean, d)
            B.flowcache_kv4_pack(x[:, :L_clean].contiguous(), None, tmp, None, L_clean, L_clean)
            split = H_k * L_clean * d // 2
            b[:H_k * cap4 * d // 2].view(H_k, cap4, -1)[:, :L_clean] = tmp[:split].view(H_k, L_clean, -1)
            b[H_k * cap4 * d // 2:].view(H_k, cap4, -1)[:, :L_clean] = tmp[split:].view(H_k, L_clean, -1)
        bufs.append(b)
    return q, bufs, cap4, slots


def reference(q, values, slots, off, L_c, rec, scale):
    """(out, its tolerance, log sum exp and its tolerance) of the listed row blocks, [rows, H_q, d] and [H_q, rows]"""
    H_q, d = q.shape[1:]
    H_k = slots[0].shape[0]
    out, tol, lse, lse_tol = [], [], [], []
    for r, c in enumerate(rec):
        k, v = (torch.cat([x] + [s[:, o:o + L_c].double() for o in off[:c + 1]], 1) for x, s in zip(values, slots))
        k, v = (x.repeat_interleave(H_q // H_k, 0) for x in (k, v))
        s = q[r * L_c:(r + 1) * L_c].double().transpose(0, 1) @ k.transpose(1, 2).contiguous() * scale
        p = torch.softmax(s, -1)
        o = p @ v
        out.append(o.transpose(0, 1))
        if q.dtype == torch.bfloat16:
            t = 2.0 ** -8 * o.abs() + (2.0 ** -7 + 2.0 ** -13) * (p @ v.abs())
            t_lse = torch.full_like(s[..., 0], 2.0 ** -8 + 1e-5)
        else:
            row = (q[r * L_c:(r + 1) * L_c].double().abs().transpose(0, 1) @ k.abs().transpose(1, 2).contiguous()).amax(-1) * scale
            u = 2.0 ** -24 * (2 * 48 * row + 16 + 40 + 12 * (s.shape[-1] / 256 + 1))
            t = 2.0 ** -24 * o.abs() + u[..., None] * (p @ v.abs())
            t_lse = u + 2.0 ** -23 * torch.logsumexp(s, -1).abs()
        tol.append(t.transpose(0, 1))
        lse.append(torch.logsumexp(s, -1))
        lse_tol.append(t_lse)
    return torch.cat(out), torch.cat(tol), torch.cat(lse, 1), torch.cat(lse_tol, 1)


def check(H_q, H_k, d, A, L_c, L_clean, rec, seed=0, scale=0.0, reverse=False, grow=False, new=False, ws=None, idx=None, n=None, stream=None,
          dtype=torch.bfloat16):
    q, bufs, cap4, slots = make(H_q, H_k, d, A, L_c, L_clean, seed, grow=grow, dtype=dtype)
    off = [3 + i * L_c for i in range(A)]
    if reverse:
        off.reverse()
    values = [torch.zeros((H_k, max(L_clean, 1), d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    B.flowcache_kv4_unpack(*bufs, cap4, *values, L_clean)
    values = [x[:, :L_clean].double() for x in values]
    kn = vn = None
    if new:
        kn, vn = (torch.randn((A * L_c, H_k, d), device=DEV).to(dtype) for _ in range(2))
    out = torch.full_like(q, 7.0)
    t_idx, t_n = i32(*(list(rec) + [-1] * (A - len(rec)) if idx is None else idx)), i32(len(rec) if n is None else n)
    if ws is not None:
        ws = torch.empty(ws, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    got = B.flowcache_attend_kv4(q, kn, vn, *(bufs if L_clean else (None, None)), cap4 if L_clean else 0, *slots, L_c, L_clean, off,
                                 t_idx, t_n, softmax_scale=scale, out=out, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    if new:
        for r, c in enumerate(rec):
            for s, x in zip(slots, (kn, vn)):
                assert torch.equal(s[:, off[c]:off[c] + L_c], x[r * L_c:(r + 1) * L_c].transpose(0, 1))
    rows = len(rec) * L_c
    if rows:
        ref, tol, lse, lse_tol = reference(q, values, slots, off, L_c, rec, scale or d ** -0.5)
        err = (got["out"][:rows].double() - ref).abs()
        assert float((err - tol).max()) <= 0, (float(err.max()), float(tol.max()))
        assert float(((got["lse"][:, :rows].double() - lse).abs() - lse_tol).max()) <= 0
        if dtype == torch.float32 and not grow:             # the library's bar for fp32 attention
            assert float(err.max() / ref.abs().max()) <= 1e-5
            assert float((err.norm(dim=-1) / ref.norm(dim=-1)).max()) <= 1e-5
    assert bool((out[rows:] == 7).all())
    return got["out"]


@pytest.mark.parametrize("H_q,H_k,d,A,L_c,L_clean,rec", [
    (2, 2, 128, 1, 1, 1, [0]), (2, 1, 64, 1, 1, 0, [0]), (12, 12, 128, 1, 1, 4097, [0]),
    (4, 4, 64, 2, 33, 31, [1]), (4, 2, 128, 3, 40, 32, [0, 2]), (3, 1, 64, 2, 65, 63, [0, 1]),
    (8, 2, 128, 2, 328, 1311, [1]), (2, 2, 128, 2, 257, 64, [0, 1]), (2, 2, 64, 2, 300, 65, [1]),
    (1, 1, 128, 4, 130, 129, [0, 1, 2, 3]), (1, 1, 64, 16, 20, 500, [3, 15]),
    (24, 24, 64, 2, 256, 640, [0, 1]), (12, 12, 128, 4, 385, 1025, [0, 1, 2, 3]), (24, 4, 64, 4, 330, 333, [0, 1, 2, 3]),
    (96, 8, 64, 1, 300, 700, [0]), (1, 1, 128, 1, 64, 20011, [0]), (64, 8, 128, 2, 520, 100, [0, 1]),
])
@pytest.mark.parametrize("form", ["plain", "grow", "other"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matches_float64(H_q, H_k, d, A, L_c, L_clean, rec, form, dtype):
    if form == "other":                                 # slots in reverse, new rows, a scale, no room to divide the keys
        check(H_q, H_k, d, A, L_c, L_clean, rec, seed=2, scale=0.11, reverse=True, new=True, ws=256, dtype=dtype)
    else:
        check(H_q, H_k, d, A, L_c, L_clean, rec, seed=1, grow=form == "grow", dtype=dtype)


@pytest.mark.parametrize("idx,n,rec", [([0, 1, 2], 0, []), ([2, -1, -1], 1, [2]), ([1, 2, 10 ** 9], 2, [1, 2]), ([0, 1, 2], 77, [0, 1, 2]), ([0, 1, 2], -3, [])])
@pytest.mark.parametrize("L_c", [20, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lists(idx, n, rec, L_c, dtype):
    check(4, 2, 64, 3, L_c, 100, rec, idx=idx, n=n, dtype=dtype)


@pytest.mark.parametrize("H_q,H_k,d", [(1, 1, 128), (2, 1, 64)])
@pytest.mark.parametrize("L_clean", [0, 1, 31, 32, 33, 650, 5000])
@pytest.mark.parametrize("rec", [(0, 1, 2), (2, 0), (1,)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_rows(H_q, H_k, d, L_clean, rec, dtype):
    """256-row blocks: tiles of codes alone, the last of them before a slot's, slots alone; keys in ranges and, without room, whole."""
    check(H_q, H_k, d, 3, 1500, L_clean, rec, seed=L_clean, grow=L_clean == 650, reverse=len(rec) == 2, dtype=dtype)
    if len(rec) == 3:
        check(H_q, H_k, d, 3, 1500, L_clean, rec, seed=L_clean + 1, ws=256, dtype=dtype)


def test_an_entry_that_is_no_chunk_is_skipped():
    q, bufs, cap4, slots = make(4, 2, 64, 3, 50, 130, 5)
    off, outs = [0, 50, 100], []
    for idx, blocks in (([5, 1, -9], [1]), ([0, 1, 2], [0, 1, 2])):
        out = torch.full_like(q, 7.0)
        B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *slots, 50, 130, off, i32(*idx), i32(3), out=out)
        outs.append(out)
    assert bool((outs[0][:50] == 7).all()) and bool((outs[0][100:] == 7).all())
    a, b = (o[50:100].double() for o in outs)
    assert float((a - b).norm() / b.norm()) < 2.0 ** -7      # the plans may differ: a rounding of weights and of the result


@pytest.mark.parametrize("H_q,H_k,d,A,L_c,L_clean", [(12, 12, 128, 2, 1024, 4096), (4, 4, 64, 1, 40, 640), (8, 2, 128, 2, 328, 1280)])
def test_equals_the_bf16_attention_of_the_unpacked_rows(H_q, H_k, d, A, L_c, L_clean):
    """The clean region in whole tiles, keys undivided: the same products in the same order, hence the same bits wherever both
    calls take blocks of the same kind, and a rounding of weights apart where they do not."""
    q, bufs, cap4, slots = make(H_q, H_k, d, A, L_c, L_clean, 3)
    caches = [torch.zeros((H_k, L_clean + A * L_c, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    B.flowcache_kv4_unpack(*bufs, cap4, *caches, L_clean)
    for c, s in zip(caches, slots):
        c[:, L_clean:] = s[:, :A * L_c]
    off, idx, n = [i * L_c for i in range(A)], i32(*range(A)), i32(A)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    a = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *slots, L_c, L_clean, off, idx, n, workspace=ws)
    b = B.flowcache_attend(q, None, None, *caches, L_c, L_clean, [L_clean + o for o in off], idx, n, workspace=ws)
    if not torch.equal(a["out"], b["out"]):
        x, y = a["out"].double(), b["out"].double()
        assert float((x - y).norm() / y.norm()) < 2.0 ** -7
        assert float((a["lse"] - b["lse"]).abs().max()) < 2.0 ** -7


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L_c", [1, 300])
def test_a_block_that_is_no_number_shows_only_where_it_is_seen(L_c, dtype):
    """A NaN beyond the clean region's end (make() puts one in every spare row) and in slots of later chunks changes nothing."""
    H, d, A, L_clean = 2, 128, 2, 100
    q, bufs, cap4, slots = make(H, H, d, A, L_c, L_clean, 7, dtype=dtype)
    off = [0, L_c]
    args = (L_c, L_clean, off, i32(0, -1), i32(1))
    want = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *slots, *args)["out"][:L_c].clone()
    for s in slots:
        s[:, L_c:] = float("nan")
    got = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *slots, *args)["out"][:L_c]
    assert bool(torch.isfinite(want).all()) and torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_buffers(dtype):
    """Codes past 2^32 bytes: a buffer of 2^27 rows, of which the call sees the first, for head 1."""
    H, d, cap4, L_clean, L_c = 2, 64, 1 << 27, 3000, 2
    q, bufs, small, slots = make(H, H, d, 1, L_c, L_clean, 8, dtype=dtype)
    big = []
    for b in bufs:
        x = torch.empty(H * cap4 * (d // 2 + d // 32), dtype=torch.uint8, device=DEV)
        split, big_split = H * small * d // 2, H * cap4 * d // 2
        x[:big_split].view(H, cap4, -1)[:, :L_clean] = b[:split].view(H, small, -1)[:, :L_clean]
        x[big_split:].view(H, cap4, -1)[:, :L_clean] = b[split:].view(H, small, -1)[:, :L_clean]
        big.append(x)
    args = (*slots, L_c, L_clean, [0], i32(0), i32(1))
    a = B.flowcache_attend_kv4(q, None, None, *bufs, small, *args)["out"]
    b = B.flowcache_attend_kv4(q, None, None, *big, cap4, *args)["out"]
    assert torch.equal(a, b)


@pytest.mark.parametrize("H_q,H_k,d,A,L_c,L_clean", [(12, 12, 128, 2, 300, 2050), (8, 2, 64, 2, 40, 700), (2, 2, 128, 1, 1, 9000)])
def test_fp32_agrees_with_the_fp32_attention_of_the_unpacked_rows(H_q, H_k, d, A, L_c, L_clean):
    """Two roundings of the same sums, each within 1e-5 of the norm."""
    q, bufs, cap4, slots = make(H_q, H_k, d, A, L_c, L_clean, 3, dtype=torch.float32)
    caches = [torch.zeros((H_k, L_clean + A * L_c, d), device=DEV) for _ in range(2)]
    B.flowcache_kv4_unpack(*bufs, cap4, *caches, L_clean)
    for c, s in zip(caches, slots):
        c[:, L_clean:] = s[:, :A * L_c]
    off, idx, n = [i * L_c for i in range(A)], i32(*range(A)), i32(A)
    a = B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *slots, L_c, L_clean, off, idx, n)
    b = B.flowcache_attend(q, None, None, *caches, L_c, L_clean, [L_clean + o for o in off], idx, n)
    assert float((a["out"] - b["out"]).norm() / b["out"].norm()) <= 2e-6
    assert float((a["lse"] - b["lse"]).abs().max()) <= 1e-5


def test_another_stream():
    check(8, 2, 128, 2, 328, 1311, [1], stream=torch.cuda.Stream())


def test_refusals():
    q, bufs, cap4, slots = make(4, 2, 64, 1, 8, 40, 1)
    args = lambda **kw: {**dict(q=q, k_new=None, v_new=None, k4=bufs[0], v4=bufs[1], capacity4=cap4, k_cache=slots[0], v_cache=slots[1], L_c=8,
                                L_clean=40, active_off=[0], recompute_idx=i32(0), n_recompute=i32(1)), **kw}
    B.flowcache_attend_kv4(**args())
    for kw in (dict(capacity4=cap4 + 1), dict(k4=bufs[0].cpu()), dict(q=q.cpu()), dict(v4=bufs[1][1:])):
        with pytest.raises(ValueError):
            B.flowcache_attend_kv4(**args(**kw))
    for kw in (dict(L_clean=cap4 + 1), dict(active_off=[17]), dict(softmax_scale=-1.0), dict(k4=None, v4=None),
               dict(L_clean=-1)):
        with pytest.raises(B.FlowCacheError):
            B.flowcache_attend_kv4(**args(**kw))
    for kw in (dict(q=q.float()), dict(k4=None), dict(L_c=4)):
        with pytest.raises(AssertionError):
            B.flowcache_attend_kv4(**args(**kw))


def sweep(n, seed):
    rng = np.random.default_rng(seed)
    for i in range(n):
        d = int(rng.choice([64, 128]))
        H_k = int(rng.choice([1, 2, 3, 8]))
        H_q = H_k * int(rng.choice([1, 1, 2, 4]))
        A = int(rng.choice([1, 2, 3, 5]))
        L_c = int(np.exp(rng.uniform(0, np.log(700))))
        # around the edges of 32- and 64-key tiles, and of the three tiles that K runs ahead
        L_clean = int(rng.choice([0, 1, 64, 128, 192, 256, 320, 384])) + int(rng.integers(-2, 3)) if rng.random() < 0.6 else int(np.exp(rng.uniform(0, 9)))
        rec = sorted(rng.choice(A, size=int(rng.integers(1, A + 1)), replace=False).tolist())
        yield i, (H_q, H_k, d, A, L_c, max(L_clean, 0), rec), bool(rng.random() < 0.5)


@pytest.mark.parametrize("i,shape,grow", sweep(48, 7))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sweep(i, shape, grow, dtype):
    check(*shape, seed=i, grow=grow, reverse=bool(i & 1), new=bool(i & 2), ws=256 if i % 3 == 0 else None, dtype=dtype)


@pytest.mark.parametrize("L_c,L_clean", [(1, 70), (40, 0), (300, 200), (520, 650)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_slots(L_c, L_clean, dtype):
    """Slots whose rows are parts of wider ones, heads with a gap: the result of contiguous ones."""
    H, d, A = 3, 128, 2
    q, bufs, cap4, slots = make(H, H, d, A, L_c, L_clean, 4, dtype=dtype)
    wide = [torch.full((H, s.shape[1] + 5, d + 24), float("nan"), device=DEV, dtype=dtype)[:, :s.shape[1], 8:8 + d] for s in slots]
    for w, s in zip(wide, slots):
        w.copy_(s)
    args = (L_c, L_clean, [L_c + 2, 0], i32(0, 1), i32(2))
    a, b = (B.flowcache_attend_kv4(q, None, None, *bufs, cap4, *c, *args) for c in (slots, wide))
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"]) and bool(torch.isfinite(a["out"]).all())


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    case = (12, 12, 128, 1, 40, 9000)
    data = [make(*case, seed) for seed in (1, 2)]
    args = lambda x: (x[0], None, None, *x[1], x[2], *x[3], 40, 9000, [0], i32(0), i32(1))
    want = [B.flowcache_attend_kv4(*args(x))["out"] for x in data]
    calls = [args(x) for x in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [[B.flowcache_attend_kv4(*c, stream=s)["out"] for c, s in zip(calls, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        assert all(torch.equal(x, y) for x, y in zip(pair, want))
