"""perf/operators.py: its plain forms, the framework's calls, and its definitions in 64 bits give the same, on small cases of the ranges that it draws from.

Tolerances: a bf16 result has one rounding, 2^-8 / sqrt(3) of it in the 2-norm over many values, gradients with an activation two (dz is rounded for the products): both stay below 2^-8.  In "train" the
values in front of the activation are kept in 8 bits: where their float32 sums and the exact ones lie on two sides of a code's border they differ by 2^-3 at most, in one of 2^13 or more values (K * 2^-24 over
half a step of 2^-4, K up to 5600 and sums in any direction, root of K): 2^-3 * 2^-6.5 in the norm of the slopes, which move by at most 1.2 of it, below 2^-9."""
import importlib.util
import os
import random

import pytest
import torch

import _block_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _module(device):
    spec = importlib.util.spec_from_file_location("operator_cases", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.DEVICE = device
    return m


def _small(m, each, most, seed):
    """`each` drawn cases of every kind that take little."""
    rng, got = random.Random(seed), {op: [] for op in ("rope_table", "rope", "rope_grad", "save", "load", "linear", "train", "grad")}
    for _ in range(10_000):
        c = m.draw(rng)
        w = m.work(c)
        if w["bytes"] < most and w["flops"] < 100 * most and len(got[c["op"]]) < each:
            got[c["op"]].append(c)
    assert all(len(cases) == each for cases in got.values())
    return [c for op in sorted(got) for c in got[op]]


def _flat(x):
    return list(x.values()) if isinstance(x, dict) else list(x) if isinstance(x, (list, tuple)) else [x]


def _check(c, got, want, what):
    if isinstance(want, dict):
        assert set(got) == set(want), what
        got, want = [got[k] for k in want], [want[k] for k in want]
    for a, b in zip(_flat(got), _flat(want)):
        if b is None:
            continue
        assert a.shape == b.shape, what
        a, b = a.double(), b.double()
        assert a.isfinite().all(), what
        off, norm = float((a - b).norm()), float(b.norm())
        if c["op"] in ("save", "load"):
            assert torch.equal(a, b), what
        elif c["op"] == "rope_table":
            places = max(c["T"], c["H"], c["W"])
            assert float((a - b).abs().max()) <= 2.0 ** -25 * 1.6 + 6 * ref.F32 + places * 2.0 ** -48, what
        elif c.get("dtype") == "fp32":
            assert off <= 4 * ref.F32 * norm, (what, off, norm)
        else:
            assert off <= (ref.BF16 + (2.0 ** -9 if c["op"] == "train" else 0)) * norm, (what, off, norm)


def test_plain_forms_against_their_definition():
    m = _module("cpu")
    assert m.own is False
    for i, c in enumerate(_small(m, 2, 3e6, 11)):
        st = m.prepare(c, 100 + i)
        _check(c, m.run(st), m.exact(c, 100 + i), c)


@pytest.mark.gpu
def test_calls_against_the_definition_and_the_plain_forms():
    m = _module("cuda")
    for i, c in enumerate(_small(m, 6, 6e7, 12)):
        print(c, flush=True)
        st = m.prepare(c, 200 + i)
        m.own = False
        plain = m.run(st)
        m.own = True
        got = m.run(st)
        m.own = False
        exact = m.exact(c, 200 + i)
        _check(c, plain, exact, ("plain", c))
        _check(c, got, exact, ("calls", c))
        if c["op"] == "save":
            assert torch.equal(got["codes"].view(torch.uint8), plain["codes"].view(torch.uint8)) and torch.equal(got["scales"], plain["scales"])
