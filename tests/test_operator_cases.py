"""The cases of perf/operators.py: whatever sizes they are drawn with, no call gets a scratch that is too small for it (no GPU: the calls are recorded)."""
import importlib.util
import os
import random

import pytest
import torch

import paper_2502_15779_amd as rcp

FILE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")


@pytest.fixture
def cases():
    spec = importlib.util.spec_from_file_location("operator_cases", FILE)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.own = True
    return module


def _empty(*shape, dtype=torch.float16):
    return torch.empty(shape, dtype=dtype, device="meta")


def _room(cases, case, monkeypatch):
    """(bytes of the scratch that the call is given, or None where it makes its own; bytes that it takes)"""
    given = []
    s = {"kind": case["kind"], "work": _empty(cases.WORKSPACE, dtype=torch.uint8)}
    if case["kind"] == "lowrank":
        monkeypatch.setattr(rcp, "lowrank_add", lambda *a, workspace, **k: given.append(workspace))
        s |= dict.fromkeys(("x", "A", "B", "which", "scaling", "base", "out"))
        need = rcp.lowrank_workspace_bytes(case["m"], case["n"], case["k"], case["r"])
    else:
        monkeypatch.setattr(rcp, "kv8_attn", lambda *a, workspace, **k: given.append(workspace))
        _, new = cases._requests(case, 0)
        b, one = case["b"], case["one"]
        s |= dict.fromkeys(("table", "ks", "vc", "vs", "scale", "out"))
        s |= {"q": _empty(sum(new), case["hq"], case["d"]), "kc": _empty(3, case["hkv"], case["page"], case["d"]),
              "lengths": _empty(b, dtype=torch.int32), "starts": None if one else _empty(b + 1, dtype=torch.int32)}
        need = rcp.kv8_workspace_bytes(sum(new), b, case["hq"], case["hkv"], case["d"], one)
    cases.run(s)
    return given[0] if given[0] is None else given[0].numel(), need


def test_a_prompt_that_just_leaves_the_device_unfilled(cases, monkeypatch):
    """3990 rows of 16 over 2 heads: two parts of every row, 67.4 MB of partial results."""
    case = {"kind": "attn", "b": 1, "hq": 16, "hkv": 2, "d": 128, "page": 64, "lmin": 3990, "lmax": 3990, "nmin": 3990, "nmax": 3990, "one": False}
    given, need = _room(cases, case, monkeypatch)
    assert need > cases.WORKSPACE and (given is None or given >= need)


def test_every_case_has_room(cases, monkeypatch):
    rng = random.Random(3)
    drawn = [c for c in cases.listed() + [cases.draw(rng) for _ in range(3000)] if c["kind"] != "append"]
    for case in drawn:
        given, need = _room(cases, case, monkeypatch)
        assert need > 0 and (given is None or given >= need), case
