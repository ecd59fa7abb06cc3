"""The cases of perf/operators.py hand the calls what they take, and give with them what their plain forms give."""
import importlib.util
import os

import pytest
import torch

from paper_2602_10825_amd import binding as B
from paper_2602_10825_amd.build import ROOT

SMALL = ("qk tiny f32", "qk small grouped", "pack small f32", "unpack small", "attend small grouped")


@pytest.fixture
def cases():
    spec = importlib.util.spec_from_file_location("operator_cases", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("name,call", [("unpack small", "flowcache_kv4_unpack"), ("attend small grouped", "flowcache_attend_kv4")])
def test_buffers_are_handed_over_as_bytes(cases, monkeypatch, name, call):
    """On the CPU, with the call stood in for."""
    got = []

    def stand_in(*args, **kw):
        got.extend(x for x in args if isinstance(x, torch.Tensor) and x.dim() == 1 and x.numel() > 2)
        return {"out": None}

    monkeypatch.setattr(cases, "DEV", "cpu")
    monkeypatch.setattr(B, call, stand_in)
    case = next(c for c in cases.listed() if c["name"] == name)
    state = cases.prepare(case, 1)
    cases.own = True
    cases.run(state)
    heads, rows, d = (case["H"], case["L"], case["d"]) if name == "unpack small" else (case["H_k"], case["L_clean"], case["d"])
    buffers = [x for x in got if x.numel() == heads * rows * (d // 2 + d // 32)]
    assert len(buffers) == 2 and all(x.dtype == torch.uint8 and x.is_contiguous() for x in buffers)
    assert all(torch.equal(x, state[k].to(x.dtype)) and torch.equal(x.long(), state[k].long()) for x, k in zip(buffers, ("k4", "v4")))


@pytest.mark.gpu
@pytest.mark.parametrize("name", SMALL)
def test_calls_give_what_the_plain_forms_give(cases, name):
    """Differences of at most what two roundings of the type and the kernels' own tests allow, as a share of the norm: 2^-8 for bf16, 2e-6 for fp32."""
    case = next(c for c in cases.listed() if c["name"] == name)
    outs = []
    for own in (False, True):
        cases.own = own
        x = cases.run(cases.prepare(case, 5))
        outs.append({k: v.double().clone() for k, v in (x if isinstance(x, dict) else {"out": x}).items()})
    for k, plain in outs[0].items():
        exact = case["kind"] in ("pack", "unpack")
        bar = 0.0 if exact else 2.0 ** -8 if case["dtype"] == "bf16" else 2e-6
        assert float((outs[1][k] - plain).norm()) <= bar * float(plain.norm()), k
