"""GPU: the calls that the native module has as a whole against the same calls by way of the binding's Python: results, classes, refusals, references."""
import gc
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

WHOLE = ("_plain_rmsnorm_fwd", "_plain_rmsnorm_bwd", "_plain_quantize_int8", "_plain_linear_fwd_int8")
GRID = dict(T=2, H=8, W=8)


@pytest.fixture()
def both(monkeypatch):
    """f -> (its result with the whole calls, how many of them had an answer, its result without)."""
    import paper_2605_28691_amd as sk

    sk.lib()
    native = {name: getattr(sk, name) for name in WHOLE}
    assert all(f is getattr(sk._marshal, name[1:]) for name, f in native.items())

    def run(f):
        answered = []

        def watched(g):
            def call(*args):
                r = g(*args)
                answered.append(r is not NotImplemented)
                return r
            return call

        for name, g in native.items():
            monkeypatch.setattr(sk, name, watched(g))
        a = f(sk)
        for name in WHOLE:
            monkeypatch.setattr(sk, name, sk._not_plain)
        b = f(sk)
        for name, g in native.items():
            monkeypatch.setattr(sk, name, g)
        return a, answered, b

    return run


def _same(a, b):
    assert type(a) is type(b)
    if isinstance(a, tuple):
        assert len(a) == len(b)
        for x, y in zip(a, b):
            _same(x, y)
    elif a is not None:
        assert a.shape == b.shape and a.dtype == b.dtype and a.is_contiguous() and not a.requires_grad and torch.equal(a, b)


def _tensors(dtype, lead=(2, 128), cols=64, out=40):
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return new(*lead, cols), new(*lead, cols), new(cols), new(*lead, cols), new(out, cols), new(out), new(*lead, out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["same", "to_sparse", "to_original"])
def test_results(both, order, dtype):
    lead = (8, 32) if order == "to_original" else (2, 128)
    place = {} if order == "same" else dict(order=order, s=2, pattern="group", **GRID)
    x, r, w, dy, wide, bias, res = _tensors(dtype, lead)
    back = {"same": (2, 128), "to_sparse": (8, 32), "to_original": (2, 128)}[order]
    for weight in (w, None, torch.nn.Parameter(w)):
        for residual in (r, None):
            for quantize in (False, True):
                a, yes, b = both(lambda sk: sk.skiparse_rmsnorm_fwd(x, weight, residual, 1e-5, quantize=quantize, **place))
                _same(a, b)
                assert yes == [True]
    a, yes, b = both(lambda sk: sk.skiparse_quantize_int8(x, **place))
    _same(a, b)
    assert yes == [True]
    q = a
    if dtype is torch.bfloat16:
        import paper_2605_28691_amd as sk

        rows, w8 = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(wide)
        for bi in (bias, None):
            for residual in (res.reshape(*back, 40), None):
                for act in ("none", "silu"):
                    a, yes, b = both(lambda sk: sk.skiparse_linear_fwd_int8(rows, w8, bi, residual, act, **place))
                    _same(a, b)
                    assert yes == [True]
        assert sk.skiparse_linear_fwd_int8(q, w8).shape == (*q.codes.shape[:-1], 40)
    for kw in ({}, dict(need_dx=False), dict(need_dw=False)):
        for add in (r, None):
            if add is not None and not kw.get("need_dx", True):
                continue
            a, yes, b = both(lambda sk: sk.skiparse_rmsnorm_bwd(dy.reshape(*back, 64), x, w, add, 1e-5, **kw, **place))
            _same(a, b)
            assert yes == ([True] if order == "same" else [])


def test_shapes(both):
    import paper_2605_28691_amd as sk

    for shape in ((64,), (1, 64), (3, 5, 7, 16), (1, 1, 5120)):
        x = torch.randn(shape, device="cuda").bfloat16()
        for f in (lambda sk: sk.skiparse_rmsnorm_fwd(x), lambda sk: sk.skiparse_rmsnorm_fwd(x, None, x), lambda sk: sk.skiparse_quantize_int8(x), lambda sk: sk.skiparse_rmsnorm_bwd(x, x)):
            a, yes, b = both(f)
            _same(a, b)
            assert yes == [True]
        q, w = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(torch.randn(24, shape[-1], device="cuda").bfloat16())
        a, yes, b = both(lambda sk: sk.skiparse_linear_fwd_int8(q, w))
        _same(a, b)
        assert yes == [True] and a.shape == (*shape[:-1], 24)
    # cut along k: with a workspace
    x, w = (sk.skiparse_quantize_int8(torch.randn(*s, device="cuda").bfloat16()) for s in ((40, 8192), (264, 8192)))
    assert sk.skiparse_linear_fwd_int8_workspace_bytes(40, 8192, 264) > 0
    a, yes, b = both(lambda sk: sk.skiparse_linear_fwd_int8(x, w))
    _same(a, b)
    assert yes == [True]


def test_what_is_not_plain_goes_on(both):
    """Tensors of a subclass, buffers of the caller's, numbers that are like a float: by the other way, with the same results."""
    class Sub(torch.Tensor):
        pass

    x, r, w, dy, wide, bias, res = _tensors(torch.bfloat16)
    plain = lambda t: tuple(map(plain, t)) if isinstance(t, tuple) else t.as_subclass(torch.Tensor)  # noqa: E731
    want = both(lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r))[0]
    for f in (lambda sk: sk.skiparse_rmsnorm_fwd(x.as_subclass(Sub), w, r), lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r.as_subclass(Sub)),
              lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r, out=torch.empty_like(x)), lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r, total=torch.empty_like(x)),
              lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r, quantize=0), lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r, torch.tensor(1e-6))):
        a, yes, b = both(f)
        assert yes in ([], [False])
        for got in (a, b):
            assert all(torch.equal(u, v) for u, v in zip(plain(got), want))


def _refused(f, sk):
    try:
        f(sk)
    except Exception as e:  # noqa: BLE001
        return type(e), str(e)
    raise AssertionError("not refused")


def test_refusals_are_the_same(both):
    import paper_2605_28691_amd as sk

    x, r, w, dy, wide, bias, res = _tensors(torch.bfloat16)
    q, w8 = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(wide)
    strided, odd = torch.empty(2, 128, 128, dtype=torch.bfloat16, device="cuda")[..., ::2], torch.empty(2 * 128 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 128, 64)
    part = sk.Quantized(q.codes, q.scales[:1])
    calls = [lambda sk, kw=kw: sk.skiparse_rmsnorm_fwd(**{**dict(x=x, weight=w, residual=r), **kw}) for kw in (
        dict(x=x.cpu()), dict(x=strided), dict(x=odd), dict(x=x.half()), dict(x=5), dict(x=x[:0]), dict(weight=w[:32]), dict(weight=w.float()), dict(weight=w.cpu()), dict(weight=w[None]), dict(residual=r[:1]),
        dict(residual=r.float()), dict(residual=strided), dict(residual=odd), dict(eps=0.0), dict(eps=float("nan")), dict(eps="one"), dict(pattern="none"), dict(order="none"), dict(order="to_sparse"),
        dict(order="to_sparse", s=2, **GRID, x=x[:, :96].contiguous(), residual=None), dict(x=x[..., :60].contiguous(), weight=None, residual=None), dict(quantize=True, x=x.double()))]
    calls += [lambda sk, t=t: sk.skiparse_quantize_int8(t) for t in (x.cpu(), strided, odd, x.half(), x[:0], 5, x[..., :4].contiguous())]
    calls += [lambda sk, kw=kw: sk.skiparse_linear_fwd_int8(**{**dict(x=q, w=w8, bias=bias, residual=res), **kw}) for kw in (
        dict(x=x), dict(x=tuple(q)), dict(x=part), dict(x=sk.Quantized(q.codes.cpu(), q.scales.cpu())), dict(x=sk.Quantized(x, q.scales)), dict(x=sk.Quantized(q.codes, q.scales.bfloat16())),
        dict(w=sk.Quantized(w8.codes[:, :32].contiguous(), w8.scales)), dict(w=q), dict(bias=bias[:8]), dict(bias=bias.float()), dict(residual=res[:1]), dict(residual=res.float()), dict(act="relu"),
        dict(order="to_sparse"), dict(residual=strided), dict(w=sk.Quantized(w8.codes[:36], w8.scales[:36])))]
    calls += [lambda sk, kw=kw: sk.skiparse_rmsnorm_bwd(**{**dict(dy=dy, h=x, weight=w, dx_add=r), **kw}) for kw in (
        dict(dy=dy.float()), dict(dy=dy[:1]), dict(h=strided), dict(h=None), dict(weight=w[:8]), dict(dx_add=r[:1]), dict(dx_add=odd), dict(eps=0.0), dict(need_dx=False), dict(pattern="none"))]
    for i, f in enumerate(calls):
        print(i, flush=True)
        a, yes, b = both(lambda sk: _refused(f, sk))
        assert a == b, i
    gc.collect()


def test_references():
    """Nothing is kept and nothing given away: neither tensors nor None."""
    import paper_2605_28691_amd as sk

    x, r, w, dy, wide, bias, res = _tensors(torch.bfloat16)
    q, w8 = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(wide)

    def calls():
        sk.skiparse_rmsnorm_fwd(x, w, r, quantize=True)
        sk.skiparse_rmsnorm_fwd(x, None, None)
        sk.skiparse_quantize_int8(x, order="to_sparse", s=2, **GRID)
        sk.skiparse_linear_fwd_int8(q, w8, bias, res)
        sk.skiparse_rmsnorm_bwd(dy, x, w, need_dx=False)
        sk.skiparse_rmsnorm_bwd(dy, x, w, need_dw=False)
        _refused(lambda sk: sk.skiparse_rmsnorm_fwd(x, w, r, eps=0.0), sk)

    held = (x, r, w, dy, bias, res, q, q.codes, w8.scales, sk.Quantized)
    calls()
    gc.collect()
    memory, counts, none = torch.cuda.memory_allocated(), [sys.getrefcount(t) for t in held], sys.getrefcount(None)
    for _ in range(200):
        calls()
    gc.collect()
    assert torch.cuda.memory_allocated() == memory and [sys.getrefcount(t) for t in held] == counts and abs(sys.getrefcount(None) - none) < 100
