"""GPU: the native module's whole calls on tensors that only look like plain ones."""
import pytest
import torch

from test_gpu_whole_calls import _refused, _tensors, both  # noqa: F401

pytestmark = pytest.mark.gpu


def _inside(transform, f, t):
    """f of what `transform` hands on in t's place; the gradient needs a number to begin from."""
    def g(a):
        assert type(a) is torch.Tensor and a.is_contiguous() and a.is_cuda
        f(a)
        return a.sum()

    return transform(g)(t)


@pytest.mark.parametrize("transform", [torch.func.vmap, torch.func.grad])
def test_tensors_without_storage(both, transform):  # noqa: F811
    """A tensor inside vmap or grad has no memory of its own: each call says so, by the native way as by the other, and the process lives on."""
    import paper_2605_28691_amd as sk

    x, r, w, dy, wide, bias, res = _tensors(torch.bfloat16)
    q, w8 = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(wide)
    calls = [(lambda sk, t: sk.skiparse_rmsnorm_fwd(t, w), x), (lambda sk, t: sk.skiparse_rmsnorm_fwd(t, w, quantize=True), x), (lambda sk, t: sk.skiparse_rmsnorm_fwd(x[0], t), r[0].expand(2, 128, 64)[:, 0].contiguous()),
             (lambda sk, t: sk.skiparse_rmsnorm_fwd(x[0], w, t), r), (lambda sk, t: sk.skiparse_quantize_int8(t), x), (lambda sk, t: sk.skiparse_rmsnorm_bwd(t, x[0], w), dy),
             (lambda sk, t: sk.skiparse_rmsnorm_bwd(dy[0], t, w, need_dx=False), x), (lambda sk, t: sk.skiparse_rmsnorm_bwd(dy[0], x[0], w, t), r), (lambda sk, t: sk.skiparse_linear_fwd_int8(q, w8, t), bias.expand(2, 40).contiguous())]
    for i, (f, t) in enumerate(calls):
        print(i, flush=True)
        a, yes, b = both(lambda sk: _refused(lambda sk: _inside(transform, lambda a: f(sk, a), t if transform is torch.func.vmap else t[0].contiguous()), sk))
        assert a == b and yes == [False] and issubclass(a[0], RuntimeError), (i, a, yes, b)
    if transform is torch.func.vmap:
        a, yes, b = both(lambda sk: _refused(lambda sk: torch.func.vmap(lambda c, s: sk.skiparse_linear_fwd_int8(sk.Quantized(c, s), w8))(q.codes, q.scales), sk))
        assert a == b and yes == [False] and issubclass(a[0], RuntimeError)
    assert torch.equal(sk.skiparse_quantize_int8(x).codes, q.codes)
