"""GPU: a sparse attention block in 8-bit integers as a user writes it, and the training step of its norms, against float64.

The block: the stream's sum and its norm in codes, in the sparse layout; q, k and v from them; the norm and positions of q and k; attention; its result in codes, back in the original order; the output projection added to the stream;
the norm in codes; the widening product with GELU; its result in codes; the narrowing product added to the stream.

Tolerances: what the reference does not share with the calls is rounding: it takes the codes as the calls have them (a code's step is no error of theirs: each quantiser is checked by itself), and everything else in float64."""
import pytest
import torch

import _block_ref as ref
import _norm_ref as nr

pytestmark = pytest.mark.gpu

B, T, H, W, s = 1, 3, 8, 12, 2
HEADS, D, C, F = 4, 64, 256, 528
PATTERN = "token"


def _weights(g):
    r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    w = dict(n1=1 + 0.2 * r(C), n2=1 + 0.2 * r(C), nq=1 + 0.2 * r(D), nk=1 + 0.2 * r(D))
    w = {k: v.bfloat16() for k, v in w.items()}
    for name, (n, k) in dict(q=(C, C), k=(C, C), v=(C, C), o=(C, C), up=(F, C), down=(C, F)).items():
        w[name] = (r(n, k) * k ** -0.5).bfloat16()
        w["b" + name] = (r(n) * 0.2).bfloat16()
    return w


def _dequantized(q):
    return q.codes.double() * q.scales.double()[..., None]


def _near(got, want, what, terms=1.0):
    """One rounding to bf16 a step, 2^-8 / sqrt(3) of it in the 2-norm; `terms` of them add up by their squares."""
    rel = float((got.double() - want).norm() / want.norm())
    assert got.isfinite().all() and rel <= terms ** 0.5 * ref.BF16 / 3 ** 0.5 * 1.1, (what, rel)


def test_block_in_8_bits():
    import paper_2605_28691_amd as sk

    g = torch.Generator(device="cuda").manual_seed(9)
    w = _weights(g)
    w8 = {n: sk.skiparse_quantize_int8(w[n]) for n in ("q", "k", "v", "o", "up", "down")}
    N = T * H * W
    x, branch = (torch.randn(B, N, C, generator=g, device="cuda").bfloat16() for _ in range(2))
    grid = dict(T=T, H=H, W=W, s=s, pattern=PATTERN)
    to, back = dict(order="to_sparse", **grid), dict(order="to_original", **grid)
    table = sk.skiparse_rope_table((T, H, W), (24, 20, 20))

    # the calls
    codes, h = sk.skiparse_rmsnorm_fwd(branch, w["n1"], residual=x, quantize=True, **to)
    q, k, v = (sk.skiparse_linear_fwd_int8(codes, w8[n], w["b" + n]).unflatten(-1, (HEADS, D)) for n in "qkv")
    qn, kn = sk.skiparse_rmsnorm_fwd(q, w["nq"]), sk.skiparse_rmsnorm_fwd(k, w["nk"])
    qr, kr = sk.skiparse_rope(qn, kn, table, T, H, W, s, PATTERN, order="stay_sparse")
    a = sk.skiparse_attn_fwd_sparse(qr, kr, v, T, H, W, s, PATTERN, out_layout="same")
    a8 = sk.skiparse_quantize_int8(a.flatten(2), **back)
    h2 = sk.skiparse_linear_fwd_int8(a8, w8["o"], w["bo"], residual=h)
    u8 = sk.skiparse_rmsnorm_fwd(h2, w["n2"], quantize=True)
    y = sk.skiparse_linear_fwd_int8(u8, w8["up"], w["bup"], act="gelu_tanh")
    y8 = sk.skiparse_quantize_int8(y)
    h3 = sk.skiparse_linear_fwd_int8(y8, w8["down"], w["bdown"], residual=h2)

    # step by step, each from what the step before it gave
    moved = lambda t, order: ref.moved(t, order, (B, T, H, W), s, PATTERN)  # noqa: E731
    hd = x.double() + branch.double()
    assert torch.equal(h, hd.bfloat16())
    n1 = moved(nr.norm(branch, w["n1"], x, 1e-6)[0], "to_sparse")
    step = codes.scales.double()[..., None]
    assert ((_dequantized(codes) - n1).abs() <= step * (0.5 + 127 * nr.ROW) * (1 + nr.ROW)).all()
    for got, n in ((q, "q"), (k, "k"), (v, "v")):
        _near(got.flatten(2), _dequantized(codes) @ _dequantized(w8[n]).t() + w["b" + n].double(), n)
    for got, src, n in ((qn, q, "nq"), (kn, k, "nk")):
        want, _ = nr.norm(src, w[n], None, 1e-6)
        nr.close(got, want, nr.norm_bound(want, torch.bfloat16), n)
    tab = table.data.double()
    for got, src in ((qr, qn), (kr, kn)):
        turned = ref.rope(moved(src.double(), "to_original"), tab, (T, H, W), (24, 20, 20), (B, T, H, W), (0, 0, 0), "interleaved", 1.0)
        _near(moved(got, "to_original"), turned, "positions")
    qd, kd, vd = (t.double().transpose(1, 2) for t in (qr, kr, v))
    att = torch.softmax(qd @ kd.transpose(-1, -2) * D ** -0.5, -1) @ vd
    _near(a, att.transpose(1, 2), "attention", 2.5)  # probabilities and the result are rounded
    ad = moved(a.flatten(2).double(), "to_original")
    assert ((_dequantized(a8) - ad).abs() <= a8.scales.double()[..., None] * (0.5 + 1e-4)).all()
    _near(h2, _dequantized(a8) @ _dequantized(w8["o"]).t() + w["bo"].double() + h.double(), "stream")
    n2, _ = nr.norm(h2, w["n2"], None, 1e-6)
    assert ((_dequantized(u8) - n2).abs() <= u8.scales.double()[..., None] * (0.5 + 127 * nr.ROW) * (1 + nr.ROW)).all()
    _near(y, ref.act("gelu_tanh", _dequantized(u8) @ _dequantized(w8["up"]).t() + w["bup"].double()), "widened")
    assert ((_dequantized(y8) - y.double()).abs() <= y8.scales.double()[..., None] * (0.5 + 1e-4)).all()
    _near(h3, _dequantized(y8) @ _dequantized(w8["down"]).t() + w["bdown"].double() + h2.double(), "stream's end")

    # the same once more in a captured graph, whatever lies in its buffers
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c_, h_ = sk.skiparse_rmsnorm_fwd(branch, w["n1"], residual=x, quantize=True, **to)
        q_, k_, v_ = (sk.skiparse_linear_fwd_int8(c_, w8[n], w["b" + n]).unflatten(-1, (HEADS, D)) for n in "qkv")
        q_, k_ = sk.skiparse_rope(sk.skiparse_rmsnorm_fwd(q_, w["nq"]), sk.skiparse_rmsnorm_fwd(k_, w["nk"]), table, T, H, W, s, PATTERN, order="stay_sparse")
        a_ = sk.skiparse_quantize_int8(sk.skiparse_attn_fwd_sparse(q_, k_, v_, T, H, W, s, PATTERN, out_layout="same").flatten(2), **back)
        h_ = sk.skiparse_linear_fwd_int8(a_, w8["o"], w["bo"], residual=h_, out=h_)
        y_ = sk.skiparse_quantize_int8(sk.skiparse_linear_fwd_int8(sk.skiparse_rmsnorm_fwd(h_, w["n2"], quantize=True), w8["up"], w["bup"], act="gelu_tanh"))
        end = sk.skiparse_linear_fwd_int8(y_, w8["down"], w["bdown"], residual=h_)
    for _ in range(3):
        end.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(end, h3)


def test_training_step_of_the_norms():
    """out = linear(norm(x + branch) in the sparse layout), back in the original order and added to the stream: the gradients of x, branch and all weights, by these calls and by float64's autograd of the same."""
    import paper_2605_28691_amd as sk

    g = torch.Generator(device="cuda").manual_seed(4)
    N = T * H * W
    x, branch, dout = (torch.randn(B, N, C, generator=g, device="cuda").bfloat16() for _ in range(3))
    n1 = (1 + 0.2 * torch.randn(C, generator=g, device="cuda")).bfloat16()
    w1 = (torch.randn(C, C, generator=g, device="cuda") * C ** -0.5).bfloat16()
    grid = dict(T=T, H=H, W=W, s=s, pattern=PATTERN)
    to, back = dict(order="to_sparse", **grid), dict(order="to_original", **grid)
    u, h = sk.skiparse_rmsnorm_fwd(branch, n1, residual=x, **to)
    out = sk.skiparse_linear_fwd(u, w1, residual=h, **back)
    du, dw1, _ = sk.skiparse_linear_bwd(dout, u, w1, need_db=False, **back)
    dx, dn1 = sk.skiparse_rmsnorm_bwd(du, h, n1, dx_add=dout, **to)

    leaves = [t.double().cpu().requires_grad_() for t in (x, branch, n1, w1)]
    xd, bd, nd, wd = leaves
    hd = xd + bd
    y = hd / torch.sqrt((hd * hd).mean(-1, keepdim=True) + 1e-6) * nd
    z = hd + y @ wd.t()
    z.backward(dout.double().cpu())
    _near(out.cpu(), z.detach(), "out", 3)                                 # u and the result; h in between
    _near(dx.cpu(), xd.grad, "dx", 4)                                      # h, du and dx are rounded
    assert torch.equal(xd.grad, bd.grad)
    _near(dw1.cpu(), wd.grad, "dw", 3)
    _near(dn1.cpu(), nd.grad, "dweight", 4)
