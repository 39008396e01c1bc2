"""GPU: products of 8-bit integers whose scales lie far from 1: what is an ordinary number as a whole is one, whatever a sum times one of the scales would be.

The bounds are those of _norm_ref.py: the sum's conversion, one product and one fused product and sum, three roundings of the four that it counts."""
import pytest
import torch

import _norm_ref as nr
from test_gpu_linear_int8 import _inputs

pytestmark = pytest.mark.gpu

# one row, few rows of one and two blocks, tiles of 64, 128 and 256, and tiles that are cut along k
SIZES = [(1, 5120, 40), (5, 1536, 72), (16, 5120, 4104), (20, 5120, 264), (20, 528, 4104), (33, 144, 520), (40, 8016, 264), (300, 1008, 1000), (390, 1536, 8960), (528, 8016, 3616), (3650, 1920, 1248)]


@pytest.mark.parametrize("act", ["none", "gelu_tanh"])
@pytest.mark.parametrize("M, K, N", SIZES)
def test_scales_far_from_one(M, K, N, act):
    import paper_2605_28691_amd as sk

    x, w, bias, residual = _inputs(M, K, N, M + K + N)
    near = sk.skiparse_linear_fwd_int8(x, w, bias, residual, act=act)
    # some tokens' scales times 2^e, all channels' times 2^-e: those tokens' results are the ordinary ones
    for e in (63, 64, 70, 100, 120, -60, -100):
        far = torch.arange(M, device="cuda") % 3 == 0
        xs = torch.where(far, x.scales * 2.0 ** e, x.scales)
        xe, we = sk.Quantized(x.codes, xs), sk.Quantized(w.codes, w.scales * 2.0 ** -e)
        assert xs.isfinite().all() and we.scales.isfinite().all()
        got = sk.skiparse_linear_fwd_int8(xe, we, bias, residual, act=act)
        y, slack = nr.linear(xe.codes, xe.scales, we.codes, we.scales, bias, residual, act)
        y, slack = y[far], slack[far]
        nr.close(got[far], y, nr.BF16 * y.abs() + slack, (M, K, N, act, e))
        if abs(e) < 100:  # powers of two change no rounding where nothing leaves the range of normal numbers
            assert torch.equal(got[far], near[far]), e
    # a token does not see which scales the others have
    xs = torch.where(torch.arange(M, device="cuda") % 3 == 0, torch.full_like(x.scales, 2.0 ** 120), x.scales)
    got = sk.skiparse_linear_fwd_int8(sk.Quantized(x.codes, xs), w, bias, residual, act=act)
    keep = torch.arange(M, device="cuda") % 3 != 0
    assert torch.equal(got[keep], near[keep])


@pytest.mark.parametrize("M, K, N", SIZES)
def test_both_scales_large(M, K, N):
    """Sums of zero stay zero; all others are beyond any range, with their sign."""
    import paper_2605_28691_amd as sk

    codes = torch.zeros(M, K, dtype=torch.int8, device="cuda")
    codes[1::3, 0], codes[2::3, 0] = 1, -1
    x = sk.Quantized(codes, torch.full((M,), 2.0 ** 120, device="cuda"))
    w = sk.Quantized(torch.ones(N, K, dtype=torch.int8, device="cuda"), torch.full((N,), 2.0 ** 120, device="cuda"))
    bias = torch.randn(N, device="cuda").bfloat16()
    got = sk.skiparse_linear_fwd_int8(x, w, bias)
    assert torch.equal(got[0::3], bias.expand_as(got[0::3])) and (got[1::3] == float("inf")).all() and (got[2::3] == -float("inf")).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_token_of_large_values(dtype):
    """Values of 2^100 quantised, times weights of 2^-100: what a norm of such a row, or the row itself, is followed by."""
    import paper_2605_28691_amd as sk

    g = torch.Generator(device="cuda").manual_seed(2)
    for M in (1, 7, 200):
        x = torch.randn(M, 1536, generator=g, device="cuda") * 2.0 ** 120
        q, w = sk.skiparse_quantize_int8(x.to(dtype)), sk.skiparse_quantize_int8((torch.randn(72, 1536, generator=g, device="cuda") * 2.0 ** -115).to(dtype))
        assert (q.scales > 2.0 ** 97).all()
        y, slack = nr.linear(q.codes, q.scales, w.codes, w.scales, None, None, "none")
        nr.close(sk.skiparse_linear_fwd_int8(q, w), y, nr.BF16 * y.abs() + slack, M)
