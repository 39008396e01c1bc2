"""perf/more_operators.py: its plain forms, the framework's calls, and its definitions in 64 bits give the same, on small cases of the ranges that it draws from.

Tolerances: a bf16 result has one rounding, 2^-8 / sqrt(3) of it in the 2-norm over many values, and stays below 2^-8.  float32 results: 64 * 2^-24 (_norm_ref.py).  Codes: a value that the two sides see on two sides of a
border has codes one apart, so what is made of them differs by a step of the largest value in one of 2^12 values or fewer; that is far below the rounding of a bf16 result."""
import importlib.util
import os
import random

import pytest
import torch

import _block_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OPS = ("norm", "norm_grad", "quant", "linear8", "sublayer8")


def _module(device):
    spec = importlib.util.spec_from_file_location("more_operator_cases", os.path.join(ROOT, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.DEVICE = device
    return m


def _small(m, each, most, seed):
    """`each` drawn cases of every kind that take little."""
    rng, got = random.Random(seed), {op: [] for op in OPS}
    for _ in range(10_000):
        c = m.draw(rng)
        w = m.work(c)
        if w["bytes"] < most and w["flops"] < 100 * most and len(got[c["op"]]) < each:
            got[c["op"]].append(c)
    assert all(len(cases) == each for cases in got.values())
    return [c for op in OPS for c in got[op]]


def _check(got, want, what):
    if not isinstance(want, dict):
        got, want = dict(out=got), dict(out=want)
    assert set(got) == set(want), what
    for name, b in want.items():
        a = got[name]
        if b is None:
            continue
        assert a.shape == b.shape, what
        off, norm = float((a.double() - b.double()).norm()), float(b.double().norm())
        assert a.isfinite().all() and off <= (ref.BF16 if a.dtype is torch.bfloat16 else 64 * ref.F32) * norm, (what, name, off, norm)


def test_plain_forms_against_their_definition():
    m = _module("cpu")
    assert m.own is False
    for i, c in enumerate(_small(m, 2, 3e6, 11)):
        st = m.prepare(c, 100 + i)
        _check(m.run(st), m.exact(c, 100 + i), c)


@pytest.mark.gpu
def test_calls_against_the_definition_and_the_plain_forms():
    m = _module("cuda")
    for i, c in enumerate(_small(m, 8, 6e7, 12)):
        print(c, flush=True)
        st = m.prepare(c, 200 + i)
        m.own = False
        plain = m.run(st)
        m.own = True
        got = m.run(st)
        m.own = False
        exact = m.exact(c, 200 + i)
        _check(plain, exact, ("plain", c))
        _check(got, exact, ("calls", c))
        if c["op"] == "quant":
            assert torch.equal(got["codes"], plain["codes"]), c
