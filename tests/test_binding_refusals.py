"""What the Python calls refuse before the library is asked: tensors whose type would be misread.  CPU only; the library
is stood in for, so a call that is let through shows as one and touches nothing."""
import pytest
import torch

from paper_2602_10825_amd import binding as B

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class LetThrough(Exception):
    pass


class Library:
    """Answers the size queries; any other call has been let through."""

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *a: 256

        def call(*a):
            raise LetThrough(name)
        return call


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    monkeypatch.setattr(B, "_lib", Library())
    monkeypatch.setattr(B, "_same_device", lambda *a: None)
    monkeypatch.setattr(B, "_stream", lambda stream: 0)


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def attend(**kw):
    args = dict(q=z(16, 4, 64), k_new=None, v_new=None, k4=None, v4=None, capacity4=0, k_cache=z(2, 16, 64), v_cache=z(2, 16, 64),
                L_c=8, L_clean=0, active_off=[0, 8], recompute_idx=z(2, dtype=I32), n_recompute=z(1, dtype=I32))
    return B.flowcache_attend_kv4(**{**args, **kw})


def test_valid_calls_are_let_through():
    with pytest.raises(LetThrough):
        attend()


@pytest.mark.parametrize("k,v", [(F32, BF), (BF, F32)])
def test_attention_without_clean_rows_wants_one_type_for_both_caches(k, v):
    with pytest.raises(AssertionError):
        attend(q=z(16, 4, 64, dtype=k), k_cache=z(2, 16, 64, dtype=k), v_cache=z(2, 16, 64, dtype=v))


def rope(**kw):
    args = dict(q=z(16, 4, 64), k=z(16, 2, 64), v=z(16, 2, 64), k_cache=z(2, 16, 64), v_cache=z(2, 16, 64), L_c=8, L_clean=0,
                active_off=[0, 8], recompute_idx=z(2, dtype=I32), n_recompute=z(1, dtype=I32), dims=(24, 20, 20), grid=(2, 4), frame0=[0, 1])
    return B.flowcache_qk_norm_rope(**{**args, **kw})


@pytest.mark.parametrize("call", [attend, rope])
@pytest.mark.parametrize("bad", [dict(recompute_idx=z(2, dtype=torch.int64)), dict(n_recompute=z(1, dtype=torch.int64)),
                                 dict(recompute_idx=z(2, dtype=F32)), dict(n_recompute=z(1, dtype=torch.uint8)),
                                 dict(recompute_idx=z(4, dtype=I32)[::2])])
def test_recompute_lists_are_int32_and_without_gaps(call, bad):
    """Two entries 0, 1 of 64 bits would be read as chunks 0, 0: two row blocks for one slot."""
    with pytest.raises(LetThrough):
        call()
    with pytest.raises(LetThrough):
        call(n_recompute=torch.tensor(1, dtype=I32))               # a number without dimensions is one entry
    with pytest.raises(ValueError):
        call(**bad)


def pack(**kw):
    args = dict(k_cache=z(2, 16, 64), v_cache=None, k4=z(2 * 16 * 34, dtype=torch.uint8), v4=None, capacity4=16, count=4, cache_pos=1, pos4=2)
    return B.flowcache_kv4_pack(**{**args, **kw})


def unpack(**kw):
    args = dict(k4=z(2 * 16 * 34, dtype=torch.uint8), v4=None, capacity4=16, k_cache=z(2, 16, 64), v_cache=None, count=4, cache_pos=1, pos4=2)
    return B.flowcache_kv4_unpack(**{**args, **kw})


@pytest.mark.parametrize("call,names", [(pack, ("count", "cache_pos", "pos4")), (unpack, ("count", "cache_pos", "pos4")),
                                        (attend, ("L_clean", "capacity4")), (rope, ("L_clean",))])
@pytest.mark.parametrize("more", [1 << 32, -(1 << 32), 1 << 40])
def test_numbers_beyond_32_bits_are_refused(call, names, more):
    """The library takes them as int: 2^32 + 3 rows would be 3."""
    with pytest.raises(LetThrough):
        call()
    for name in names:
        with pytest.raises(ValueError):
            call(**{name: more + 3})


def test_a_frame_beyond_32_bits_is_refused():
    for grid in ((1 << 32, 4), (2, (1 << 32) + 4)):
        with pytest.raises(ValueError):
            rope(grid=grid)
