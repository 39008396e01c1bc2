"""Refusals of the norm and of the products in 8-bit integers, without a GPU: the C ABI's checks and the binding's; and the definition of codes."""
import ctypes

import numpy as np
import pytest
import torch

import _norm_ref as nr
import paper_2605_28691_amd as sk

P = [ctypes.c_void_p(0x10000 + i * (1 << 44)) for i in range(12)]  # addresses far apart; never dereferenced because validation fails first
ODD = ctypes.c_void_p(0x10004)
EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE = -1, -2, -3, -4
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    return sk.lib()


def _near(p, by=16):
    return ctypes.c_void_p(p.value + by)


def test_norm_refusals(lib):
    def call(x=P[0], residual=P[1], weight=P[2], total=P[3], out=P[4], scales=None, B=1, T=2, H=8, W=8, cols=64, eps=1e-6, s=2, pattern=0, order=1, dtype=0):
        return lib.skiparse_rmsnorm_fwd(x, residual, weight, total, out, scales, B, T, H, W, cols, ctypes.c_float(eps), s, pattern, order, dtype, None)

    q = dict(scales=P[5])
    for bad in (dict(x=None), dict(out=None), dict(residual=None), dict(eps=0), dict(eps=-1e-6), dict(eps=NAN), dict(eps=INF), dict(eps=1e-40), dict(eps=2e30), dict(order=3), dict(order=-1), dict(dtype=7), dict(B=0), dict(T=-1),
                dict(cols=0), dict(pattern=2), dict(s=0), dict(x=ODD), dict(residual=ODD), dict(weight=ODD), dict(total=ODD), dict(out=ODD), dict(scales=ODD),
                # buffers that overlap: rows move here, so not even whole ones may
                dict(out=P[0]), dict(out=_near(P[0])), dict(out=P[1]), dict(out=P[2]), dict(out=P[3]), dict(total=_near(P[0])), dict(total=_near(P[1])), dict(total=P[2]),
                dict(order=0, out=_near(P[0])), dict(order=0, out=P[1]), dict(order=0, out=P[0], total=P[0]), dict(order=0, out=P[0], **q), dict(out=P[5], **q), dict(scales=P[0]),
                dict(scales=P[1]), dict(scales=P[2]), dict(scales=P[3])):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(H=7), dict(H=6, pattern=1), dict(T=1 << 12, H=1 << 10, W=1 << 10), dict(order=0, T=1 << 16, H=1 << 10, W=1 << 10)):
        assert call(**bad) == ESHAPE, bad
    for bad in (dict(dtype=2), dict(cols=60), dict(cols=32776)):
        assert call(**bad) == EUNSUPPORTED, bad


def test_quantize_refusals(lib):
    def call(x=P[0], codes=P[1], scales=P[2], B=1, T=2, H=8, W=8, cols=64, s=2, pattern=0, order=1, dtype=0):
        return lib.skiparse_quantize_int8(x, codes, scales, B, T, H, W, cols, s, pattern, order, dtype, None)

    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(order=3), dict(dtype=4), dict(W=0), dict(cols=-8), dict(x=ODD), dict(codes=ODD), dict(scales=ODD), dict(codes=P[0]), dict(codes=P[2]),
                dict(scales=P[0]), dict(scales=_near(P[1]))):
        assert call(**bad) == EINVAL, bad
    assert call(H=7) == ESHAPE
    for bad in (dict(dtype=2), dict(cols=4), dict(cols=32776)):
        assert call(**bad) == EUNSUPPORTED, bad


def test_norm_gradient_refusals(lib):
    def call(dy=P[0], h=P[1], weight=P[2], add=P[3], dx=P[4], dw=P[5], B=1, T=2, H=8, W=8, cols=64, eps=1e-6, s=2, pattern=0, order=1, dtype=0, ws=P[6], size=1 << 30):
        return lib.skiparse_rmsnorm_bwd(dy, h, weight, add, dx, dw, B, T, H, W, cols, ctypes.c_float(eps), s, pattern, order, dtype, ws, size, None)

    for bad in (dict(dy=None), dict(h=None), dict(dx=None), dict(dx=None, dw=None, add=None), dict(eps=0), dict(eps=NAN), dict(order=4), dict(dtype=9), dict(H=0), dict(dy=ODD), dict(h=ODD), dict(weight=ODD),
                dict(add=ODD), dict(dx=ODD), dict(dw=ODD), dict(dx=P[0]), dict(dx=P[1]), dict(dx=P[2]), dict(dx=_near(P[3])), dict(dx=P[5]), dict(dx=P[6]), dict(dw=P[0]), dict(dw=P[1]), dict(dw=P[2]),
                dict(dw=P[3]), dict(dw=P[6]), dict(ws=P[0]), dict(ws=P[1]), dict(ws=P[2]), dict(ws=P[3]), dict(order=0, dx=P[0])):
        assert call(**bad) == EINVAL, bad
    need = lib.skiparse_rmsnorm_bwd_workspace_bytes(128, 64)
    assert need >= 64 * 4
    for bad in (dict(ws=None), dict(ws=ODD), dict(size=need - 1)):
        assert call(**bad) == EWORKSPACE, bad
    assert call(H=7) == ESHAPE and call(cols=60) == EUNSUPPORTED and call(dtype=2) == EUNSUPPORTED
    assert lib.skiparse_rmsnorm_bwd_workspace_bytes(0, 64) == lib.skiparse_rmsnorm_bwd_workspace_bytes(5, -8) == lib.skiparse_rmsnorm_bwd_workspace_bytes(5, 40000) == 0


def test_product_refusals(lib):
    def call(x=P[0], xs=P[1], w=P[2], ws=P[3], bias=P[4], residual=P[5], out=P[6], B=1, T=2, H=8, W=8, K=64, N=128, s=2, pattern=0, order=1, act=1, space=P[7], size=1 << 40):
        return lib.skiparse_linear_fwd_int8(x, xs, w, ws, bias, residual, out, B, T, H, W, K, N, s, pattern, order, act, space, size, None)

    for bad in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(out=None), dict(order=3), dict(act=3), dict(act=-1), dict(B=0), dict(K=0), dict(N=-8), dict(pattern=5), dict(x=ODD), dict(xs=ODD),
                dict(w=ODD), dict(ws=ODD), dict(bias=ODD), dict(residual=ODD), dict(out=ODD), dict(out=P[0]), dict(out=P[1]), dict(out=P[2]), dict(out=P[3]), dict(out=P[4]), dict(out=_near(P[5]))):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(H=7), dict(H=6, pattern=1), dict(K=131072), dict(N=1 << 23), dict(T=256, H=256, W=256, K=1024), dict(order=0, T=1, H=1, W=1 << 30, N=1024, K=16)):
        assert call(**bad) == ESHAPE, bad
    for bad in (dict(K=72), dict(K=20), dict(N=100)):
        assert call(**bad) == EUNSUPPORTED, bad
    for M, K, N in ((300, 8016, 264), (40, 131056, 72), (528, 8016, 3616)):
        need = lib.skiparse_linear_fwd_int8_workspace_bytes(M, K, N)
        at = dict(order=0, B=1, T=1, H=1, W=M, K=K, N=N)
        if need:
            for bad in (dict(space=None), dict(space=ODD), dict(size=need - 1)):
                assert call(**at, **bad) == EWORKSPACE, bad
            for other in P[:7]:
                assert call(**at, space=other) == EINVAL
    assert lib.skiparse_linear_fwd_int8_workspace_bytes(0, 64, 64) == lib.skiparse_linear_fwd_int8_workspace_bytes(4, -1, 64) == 0


def test_binding_refusals():
    """In front of any GPU work."""
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q = lambda *s: sk.Quantized(torch.zeros(*s, dtype=torch.int8), torch.zeros(s[:-1]))  # noqa: E731
    norm, grad, quant, prod = sk.skiparse_rmsnorm_fwd, sk.skiparse_rmsnorm_bwd, sk.skiparse_quantize_int8, sk.skiparse_linear_fwd_int8
    for call in (lambda: norm(b(4, 64), b(32)), lambda: norm(b(4, 64), torch.zeros(64)), lambda: norm(b(4, 64), None, b(5, 64)), lambda: norm(b(4, 64), None, torch.zeros(4, 64)),
                 lambda: norm(b(4, 64), total=b(4, 64)), lambda: norm(b(4, 64), out=b(4, 32)), lambda: norm(b(4, 64), out=torch.zeros(4, 64)), lambda: norm(b(4, 64), None, b(4, 64), total=b(5, 64)),
                 lambda: norm(b(4, 64), quantize=True, out=b(4, 64)), lambda: norm(b(4, 64), quantize=True, out=q(4, 32)), lambda: norm(b(1, 12, 64), order="to_sparse", T=1, H=4, W=4, s=2),
                 lambda: grad(b(4, 64), b(4, 32)), lambda: grad(b(4, 64), b(5, 64)), lambda: grad(b(4, 64), b(4, 64), b(32)), lambda: grad(b(4, 64), torch.zeros(4, 64)),
                 lambda: grad(b(4, 64), b(4, 64), dx_add=b(64)), lambda: grad(b(4, 64), b(4, 64), dw=b(32)), lambda: grad(b(4, 64), b(4, 64), dx=b(4, 32)),
                 lambda: quant(b(4, 64), out=q(4, 32)), lambda: quant(b(4, 64), out=sk.Quantized(q(4, 64).codes, torch.zeros(5))), lambda: quant(b(1, 12, 64), order="to_original", T=1, H=4, W=4, s=2),
                 lambda: prod(b(4, 64), q(8, 64)), lambda: prod(q(4, 64), b(8, 64)), lambda: prod(q(4, 64), q(8, 32)), lambda: prod(q(4, 64), q(2, 8, 64)), lambda: prod(q(4, 64), q(8, 64), b(4)),
                 lambda: prod(q(4, 64), q(8, 64), torch.zeros(8)), lambda: prod(q(4, 64), q(8, 64), None, b(4, 16)), lambda: prod(q(4, 64), q(8, 64), out=torch.zeros(4, 8)),
                 lambda: prod(sk.Quantized(q(4, 64).codes, torch.zeros(4, dtype=torch.float64)), q(8, 64)), lambda: prod(sk.Quantized(b(4, 64), torch.zeros(4)), q(8, 64))):
        with pytest.raises(ValueError):
            call()
    assert grad(b(4, 64), b(4, 64), need_dx=False, need_dw=False) == (None, None)


def test_definition_of_codes():
    """The test's own form of it, on values worked out by hand."""
    x = torch.tensor([[127.0, 0.5, 1.5, -2.5, -127.0, 3.0, 0.0, -0.0], [0.0] * 8, [1.0, float("nan")] + [0.0] * 6, [-2.0, 1.0] + [0.0] * 6, [2.0 ** -120] + [0.0] * 7])
    codes, scales = nr.codes(x)
    assert codes[0].tolist() == [127, 0, 2, -2, -127, 3, 0, 0] and scales[0] == 1
    assert not codes[1].any() and scales[1] == 1 and not codes[2].any() and np.isnan(scales[2])
    assert codes[3].tolist()[:2] == [-127, 64] and float(scales[3]) == float(np.float32(2) / np.float32(127))  # 63.5 goes to the even code
    assert codes[4, 0] == 32 and float(scales[4]) == float(np.float32(2.0 ** -118) / np.float32(127))           # 31.75


def test_whole_calls_answer_only_what_is_plain():
    """On the CPU nothing is: the native module says so without a look at the device."""
    native = sk._marshal
    assert sk.lib() and native is not None and sk._plain_rmsnorm_fwd is native.plain_rmsnorm_fwd

    def never(*args):
        raise AssertionError("asked for the device")

    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    q = sk.Quantized(x.to(torch.int8), torch.zeros(4))
    for call, good in ((native.plain_rmsnorm_fwd, (x, None, None, 1e-6, False, sk.Quantized, None, never, never)), (native.plain_quantize_int8, (x, sk.Quantized, None, never, never)),
                       (native.plain_linear_fwd_int8, (q, q, None, None, 0, sk.Quantized, None, never, never)), (native.plain_rmsnorm_bwd, (x, x, None, None, 1e-6, True, True, never, never))):
        assert call(*good) is call(*good[:-1]) is call(*good, 1) is call() is NotImplemented
        for i in range(len(good)):
            for bad in (None, 5, 1.5, "x", (), (1,) * 9, [x], torch.zeros(2), sk.Quantized, object()):
                assert call(*good[:i], bad, *good[i + 1:]) is NotImplemented
