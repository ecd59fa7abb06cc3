"""The rollout with head norm, rotation and a clean region in 4 bits, all together: a host mirror built from the oracle follows
layer 0 through every tick and commit (what the calls do alone is tested beside them)."""
import numpy as np
import pytest
import torch

from oracle import flowcache_oracle as O
from paper_2602_10825_amd import binding as B
from paper_2602_10825_amd.rollout import RolloutConfig, run_rollout
from tests._checks import assert_mass_close
from tests.test_gpu_kv4 import planes

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(600)]


@pytest.fixture(scope="module", autouse=True)
def release_memory():
    """The blocks that these tests used go back to the device, not to the next test's torch.empty."""
    yield
    torch.cuda.empty_cache()


def config(**kw):
    return RolloutConfig(**{**dict(H=2, d=64, L_c=96, n_layers=2, n_units=6, steps=8, stagger=4, budget_chunks=2, warmup_m=2, eps=0.08,
                                   obs_window=20, delta0=0.03, decay=0.8, seed=3, grid=(5, 7), kv4=True), **kw})


def mirror_of(cfg, seen):
    H, d, L_c, budget = cfg.H, cfg.d, cfg.L_c, cfg.budget_chunks * cfg.L_c
    base, frames = budget + L_c, -(-L_c // (cfg.grid[0] * cfg.grid[1])) if cfg.grid else 0
    codes = [np.zeros((H, budget, d // 2), np.uint8) for _ in range(2)]
    scales = [np.zeros((H, budget, d // 32), np.uint8) for _ in range(2)]

    def same(x, c, s, n):
        got_c, got_s = planes(x, H, budget, d)
        assert np.array_equal(got_c[:, :n], c[:, :n]) and np.array_equal(got_s[:, :n], s[:, :n])

    def observer(event, info):
        tk = info["tick"]
        seen.append(event)
        if event == "attend":
            rec, off = info["rec"], [x - base for x in tk["active_off"]]
            q, k, v = (O.widen(B.to_host(info[n])) for n in ("q", "k_cache", "v_cache"))
            if cfg.grid:
                new = O.widen(B.to_host(info["qkv"])).reshape(-1, 3, H, d)
                w = [x.cpu().numpy() for x in info["norm_w"]]
                for r, c in enumerate(rec):
                    pos = O.token_positions(tk["unit"][c] * frames, L_c, *cfg.grid)
                    blk, slot = slice(r * L_c, (r + 1) * L_c), slice(off[c], off[c] + L_c)
                    for i, got in ((0, q[blk]), (1, k[:, slot].transpose(1, 0, 2))):
                        z = O.rotate(O.norm_heads(new[blk, i], w[i], 1e-6), pos, cfg.axis_dims, 10000.0, False)
                        length = np.hypot(z[..., 0::2], z[..., 1::2]).repeat(2, -1)
                        assert np.all(np.abs(got - z) <= 2.0 ** -8 * np.abs(z) + 2.0 ** -19 * length), tk["tick"]
                    assert np.array_equal(v[:, slot], new[blk, 2].transpose(1, 0, 2))
            L = tk["L_clean"]
            for x, c, s in zip((info["k4"], info["v4"]), codes, scales):
                same(x, c, s, L)
            kk, vv = (np.concatenate([O.kv4_values(c[:, :L], s[:, :L]), x], 1) for c, s, x in zip(codes, scales, (k, v)))
            ref, _ = O.attend(q[:len(rec) * L_c], kk, vv, L, [L + x for x in off], L_c, rec)
            # |v| is about 1: weights and output rounded to bf16, 2^-7 sum p |v| + 2^-8 |out|
            bound, _ = O.attend(q[:len(rec) * L_c], kk, np.abs(vv), L, [L + x for x in off], L_c, rec)
            err = np.abs(O.widen(B.to_host(info["out"]))[:len(rec) * L_c] - ref)
            assert np.all(err <= (2.0 ** -7 + 2.0 ** -13) * bound + 2.0 ** -8 * np.abs(ref)), tk["tick"]
        elif event == "commit":
            src, dst, merged = tk["commit_src_off"] - base, tk["commit_dst_off"], tk["merged_len"]
            rows = [O.widen(B.to_host(info[n]))[:, src:src + L_c] for n in ("k_cache", "v_cache")]
            if tk["compress"]:
                whole = [np.concatenate([O.kv4_values(c[:, :dst], s[:, :dst]), x], 1) for c, s, x in zip(codes, scales, rows)]
                m = info["mass"].cpu().numpy()
                assert_mass_close(m, O.attention_mass(B.to_host(info["q_obs"]), whole[0], merged), "bf16", f"tick {tk['tick']}")
                kept, k, v, _ = O.kv_compress(*whole, merged, budget, m, cfg.pool_k, cfg.lam)
                assert np.array_equal(info["kept"].cpu().numpy(), kept), tk["tick"]
                packed = [O.kv4_pack(x[:, :budget]) for x in (k, v)]
                at = 0
            else:
                packed, at = [O.kv4_pack(x) for x in rows], dst
            for c, s, (pc, ps) in zip(codes, scales, packed):
                c[:, at:at + pc.shape[1]], s[:, at:at + pc.shape[1]] = pc, ps
            for x, c, s in zip((info["k4"], info["v4"]), codes, scales):
                same(x, c, s, tk["L_clean_after"])

    return observer


@pytest.mark.parametrize("kw", [{}, {"grid": None}, {"d": 128, "H": 3, "L_c": 70, "stagger": 3, "eps": 0.0}])
def test_rollout_matches_host_mirror(kw):
    cfg, seen = config(**kw), []
    res = run_rollout(cfg, observer=mirror_of(cfg, seen), keep_indices=True)
    assert res.stats["commits"] == cfg.n_units == seen.count("commit") and len(res.kept) == cfg.n_units - cfg.budget_chunks
    assert seen.count("attend") > cfg.n_units


def test_rotation_alone_and_the_ratio_of_sizes():
    """With the clean region in bf16 and the rotation on; and what the 4-bit region saves."""
    res = run_rollout(config(kv4=False))
    assert res.stats["commits"] == 6 and res.stats["norm_rope_ms"] > 0
    assert B.kv4_buffer(12, 40800, 128).numel() * 256 == 12 * 40800 * 256 * 68


def test_captured_tick_and_commit_replay_to_the_eager_bits():
    """Norm and rotation, attention and a commit's unpacking, selection and packing in one graph, replayed with other work between."""
    H, d, L_c, L_clean, A, budget = 4, 128, 200, 600, 2, 600
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    rows, clean = n(A * L_c, 3 * H, d), [n(H, L_clean, d) for _ in range(2)]
    slots0 = [n(H, A * L_c, d) for _ in range(2)]
    slots = [x.clone() for x in slots0]
    bufs0, bufs = ([B.kv4_buffer(H, budget, d) for _ in range(2)] for _ in range(2))
    B.flowcache_kv4_pack(*clean, *bufs0, budget, L_clean)
    scratch = [torch.zeros(H, L_clean + L_c, d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    idx, count = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 1], [2]))
    q, out, kept = torch.zeros_like(rows[:, :H]).contiguous(), n(A * L_c, H, d), torch.zeros((H, budget), dtype=torch.int32, device="cuda")
    L = B.lib()
    ws = [torch.empty(max(x, 256), dtype=torch.uint8, device="cuda") for x in (
        L.flowcache_attend_kv4_workspace(A, L_c, H, d), L.flowcache_attention_mass_workspace(50, H, H, d, L_clean + L_c),
        L.flowcache_kv_compress_workspace(H, L_clean + L_c, d, budget, B.FC_BF16))]
    off, merged = [0, L_c], L_clean + L_c

    def step():
        for x, y in zip((*slots, *bufs), (*slots0, *bufs0)):
            x.copy_(y)
        B.flowcache_qk_norm_rope(*rows.split(H, 1), *slots, L_c, 0, off, idx, count, (44, 42, 42), (5, 7), [7, 13], q_out=q)
        res = B.flowcache_attend_kv4(q, None, None, *bufs, budget, *slots, L_c, L_clean, off, idx, count, out=out, workspace=ws[0])
        B.flowcache_kv4_unpack(*bufs, budget, *scratch, L_clean)
        for s, x in zip(scratch, slots):
            s[:, L_clean:] = x[:, :L_c]
        mass = B.flowcache_attention_mass(q[-50:], scratch[0], merged, workspace=ws[1])
        B.flowcache_kv_select(scratch[0], merged, budget, mass, kept_idx=kept, workspace=ws[2])
        B.flowcache_kv4_pack(*scratch, *bufs, budget, budget, kept_idx=kept)
        return res["lse"], mass

    lse, mass = step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (q, out, lse, mass, kept, *bufs, *slots)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lse, mass = step()
    for replay in range(3):
        assert np.isfinite(torch.randn(1 << 20, device="cuda").sum().item())
        for x in (q, out, kept, *bufs, *slots, *scratch):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip((q, out, lse, mass, kept, *bufs, *slots), want)):
            assert torch.equal(x, y), (replay, i)
