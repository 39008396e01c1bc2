"""GPU: tables whose base and factors are no 32-bit numbers, at far places, where the nearest of them would show."""
import ctypes

import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu


def _bound(lengths, attention):
    # an angle of at most an eighth of a turn is rounded once (2^-25 pi / 2), then the function (4 ulp) and the factor; a turn's 64 bits, of up to `places` radians, are off by some
    # ulp (2^-52 each) of the powers and products in front, here and in the reference: 16 of them
    return attention * (2.0 ** -25 * 1.6 + 6 * ref.F32 + max(lengths) * 2.0 ** -48)


@pytest.mark.parametrize("scaling, factor, trained, fast, slow", [
    ("none", (1.0, 1.0, 1.0), (0, 0, 0), 32.0, 1.0), ("linear", (1.3, 10 / 3, 1.6), (0, 0, 0), 32.0, 1.0), ("ntk", (1.3, 1.1, 10 / 3), (0, 0, 0), 32.0, 1.0),
    ("yarn", (1.3, 2.7, 10 / 3), (21, 48, 8192), 32.0, 1.0), ("yarn", (1.1, 1.6, 6.7), (300, 100, 4096), 31.9, 1.1)])
@pytest.mark.parametrize("theta", [10000.0, 10000.7, 499.3])
@pytest.mark.parametrize("lengths, axes", [((1, 1, 131072), (0, 0, 128)), ((32768, 1, 9), (32, 0, 20)), ((21, 80, 80), (44, 42, 42))])
def test_base_and_factors_in_64_bits(lengths, axes, theta, scaling, factor, trained, fast, slow):
    import paper_2605_28691_amd as sk

    got = sk.skiparse_rope_table(lengths, axes, theta=theta, scaling=scaling, factor=factor, trained=trained, fast=fast, slow=slow, attention=0.7)
    parts = []
    for n, r, s, t in zip(lengths, axes, factor, trained):
        a = torch.arange(n, dtype=torch.float64)[:, None] * ref.frequencies(r, theta, scaling, s, t, fast, slow)[None]
        parts.append(torch.stack((a.cos(), a.sin()), -1).reshape(-1) * 0.7)
    assert (got.data.double().cpu() - torch.cat(parts)).abs().max() <= _bound(lengths, 0.7)


def test_the_general_way_and_the_call_in_32_bits():
    """By way of ctypes the same bits; the call with 32-bit arguments is that of their values."""
    import paper_2605_28691_amd as sk

    lengths, axes, f = (1, 40, 5000), (0, 16, 48), ctypes.c_float
    want = sk.skiparse_rope_table(lengths, axes, theta=10000.7, scaling="linear", factor=1.3)
    out = torch.empty_like(want.data)
    at = (*lengths, *axes)
    sk._general("skiparse_rope_table_ex", out, *at, 10000.7, 1, 1.3, 1.3, 1.3, 0, 0, 0, 32.0, 1.0, 1.0, sk._stream())
    assert torch.equal(out, want.data)
    rounded = {v: f(v).value for v in (10000.7, 1.3)}
    want = sk.skiparse_rope_table(lengths, axes, theta=rounded[10000.7], scaling="linear", factor=rounded[1.3])
    code = sk.lib().skiparse_rope_table(ctypes.c_void_p(out.data_ptr()), *at, f(10000.7), 1, *map(f, (1.3,) * 3), 0, 0, 0, f(32), f(1), f(1), ctypes.c_void_p(sk._stream()))
    assert code == 0 and torch.equal(out, want.data)
