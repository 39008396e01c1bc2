"""GPU: slices of rows in 8-bit integers, whose scales begin at any multiple of 4 bytes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _some(M, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(M, K, generator=g, device="cuda").bfloat16()


def _rows(sk, q, at, n):
    return sk.Quantized(q.codes[at:at + n], q.scales[at:at + n])


@pytest.mark.parametrize("K, N", [(64, 72), (1536, 264), (8016, 520)])
def test_products_of_a_slice(K, N):
    """Of the tokens, of the channels, and of both: the whole product's rows and channels, bit for bit."""
    import paper_2605_28691_amd as sk

    q, w = sk.skiparse_quantize_int8(_some(300, K, 1)), sk.skiparse_quantize_int8(_some(N, K, 2))
    whole = sk.skiparse_linear_fwd_int8(q, w)
    for at, n in ((1, 1), (2, 1), (3, 5), (5, 20), (7, 33), (1, 299), (4, 64)):
        assert torch.equal(sk.skiparse_linear_fwd_int8(_rows(sk, q, at, n), w), whole[at:at + n]), (at, n)
        out = torch.empty(n, N, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(sk.skiparse_linear_fwd_int8(_rows(sk, q, at, n), w, out=out), whole[at:at + n])
    for at, n in ((1, 8), (2, 64), (3, 56), (8, 64)):
        for rows in (1, 20, 300):
            assert torch.equal(sk.skiparse_linear_fwd_int8(_rows(sk, q, 0, rows), _rows(sk, w, at, n)), whole[:rows, at:at + n]), (at, n, rows)
    assert torch.equal(sk.skiparse_linear_fwd_int8(_rows(sk, q, 3, 40), _rows(sk, w, 5, 64)), whole[3:43, 5:69])
    # in strides they are refused, wherever they begin
    for at in (0, 1):
        strided = torch.ones(80, device="cuda")[at::2]
        with pytest.raises(ValueError):
            sk.skiparse_linear_fwd_int8(sk.Quantized(q.codes[:40], strided), w)


def test_a_slice_in_a_graph():
    import paper_2605_28691_amd as sk

    x = _some(60, 528, 3)
    q, w = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(_some(264, 528, 4))
    sk.skiparse_linear_fwd_int8(_rows(sk, q, 3, 40), w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sk.skiparse_linear_fwd_int8(_rows(sk, q, 3, 40), w)
    for seed in (5, 6, 7):
        sk.skiparse_quantize_int8(_some(60, 528, seed), out=q)
        want = sk.skiparse_linear_fwd_int8(q, w)[3:43]
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", [32, 528, 5136])
def test_results_into_a_slice(K, dtype):
    """The quantiser and the norm write rows of a larger Quantized, and nothing beside them."""
    import paper_2605_28691_amd as sk

    x = _some(40, K, 8).to(dtype)
    weight = _some(1, K, 9)[0].to(dtype)
    for f in (lambda out: sk.skiparse_quantize_int8(x, out=out), lambda out: sk.skiparse_rmsnorm_fwd(x, weight, quantize=True, out=out), lambda out: sk.skiparse_rmsnorm_fwd(x, weight, x, quantize=True, out=out)[0]):
        want = f(None)
        for at in (1, 2, 3, 4):
            q = sk.Quantized(torch.full((48, K), 77, dtype=torch.int8, device="cuda"), torch.full((48,), 77.0, device="cuda"))
            part = _rows(sk, q, at, 40)
            assert f(part) is part
            assert torch.equal(part.codes, want.codes) and torch.equal(part.scales, want.scales)
            for t in q:
                assert (t[:at] == 77).all() and (t[at + 40:] == 77).all(), at
    # half a float's address is none
    odd = torch.empty(4 * 40 + 2, dtype=torch.uint8, device="cuda")[2:].view(40, 4)
    assert odd.data_ptr() % 4 == 2
    with pytest.raises(sk.SkiparseError):
        sk._skiparse_quantize_int8(x, torch.empty(40, K, dtype=torch.int8, device="cuda"), odd, 1, 1, 1, 40, K, 1, 0, 0, 0 if dtype is torch.bfloat16 else 1, sk._stream())
