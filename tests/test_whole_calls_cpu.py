"""The native module's whole calls on the host: which arguments they answer and with what, and what becomes of tensors that have no memory of their own."""
import os
import subprocess
import sys

import pytest
import torch

import _host_marshal as hm
import paper_2605_28691_amd as sk

HERE = os.path.dirname(os.path.abspath(__file__))
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def path(tmp_path_factory):
    if not os.path.exists(sk._LIB_PATH):
        from paper_2605_28691_amd import build

        build.build()
    return hm.build(str(tmp_path_factory.mktemp("marshal")))


@pytest.fixture()
def host(path):
    return hm.Host(path)


# Each whole call inside vmap and inside grad, where a tensor is a torch.Tensor itself, contiguous, and without memory of its own.
WITHOUT_STORAGE = """
import sys
import torch
import _host_marshal as hm
import paper_2605_28691_amd as sk

n = hm.Host(sys.argv[1])
at = (hm.device, hm.stream)
x, w = torch.randn(3, 4, 64), torch.randn(64)
codes, scales = torch.zeros(3, 4, 64, dtype=torch.int8), torch.ones(3, 4)
weights, bias = sk.Quantized(torch.zeros(8, 64, dtype=torch.int8), torch.ones(8)), torch.randn(3, 8).bfloat16()
q = sk.Quantized(codes[0], scales[0])
calls = dict(
    norm=lambda x: n.native.plain_rmsnorm_fwd(x, w, None, 1e-6, False, sk.Quantized, None, *at),
    norm_residual=lambda x: n.native.plain_rmsnorm_fwd(torch.ones(4, 64), w, x, 1e-6, True, sk.Quantized, None, *at),
    quantize=lambda x: n.native.plain_quantize_int8(x, sk.Quantized, None, *at),
    bwd=lambda x: n.native.plain_rmsnorm_bwd(x, torch.ones(4, 64), w, None, 1e-6, True, True, *at),
    bwd_add=lambda x: n.native.plain_rmsnorm_bwd(torch.ones(4, 64), torch.ones(4, 64), w, x, 1e-6, True, False, *at),
)
seen = []


def inside(f):
    def g(*args):
        assert all(type(a) is torch.Tensor and a.is_contiguous() for a in args)
        seen.append(f(*args))
        return args[0].sum()
    return g


for name, f in calls.items():
    torch.func.vmap(inside(f))(x)
    torch.func.grad(inside(f))(x[0])
    print(name, flush=True)
torch.func.vmap(inside(lambda c, s: n.native.plain_linear_fwd_int8(sk.Quantized(c, s), weights, None, None, 0, sk.Quantized, None, *at)))(codes, scales)
for f in (torch.func.vmap, torch.func.grad):
    f(inside(lambda b: n.native.plain_linear_fwd_int8(q, weights, b, None, 0, sk.Quantized, None, *at)))(bias if f is torch.func.vmap else bias[0])
assert len(seen) == 2 * len(calls) + 3 and all(r is NotImplemented for r in seen), seen
assert not n.calls
# and the same calls of ordinary tensors are answered
assert calls["norm"](x[0]).shape == (4, 64) and calls["quantize"](x[0]).scales.shape == (4,) and len(n.calls) == 2
"""


def test_tensors_without_storage(path):
    """They go on to the Python, which says what is the matter, instead of ending the process (so: in one of its own)."""
    done = subprocess.run([sys.executable, "-c", WITHOUT_STORAGE, path], cwd=HERE, env={**os.environ, "PYTHONPATH": os.path.dirname(HERE)}, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert done.returncode == 0, (done.returncode, done.stdout, done.stderr)


def _calls(host):
    """(whole call, arguments that it answers, which of them may be None)"""
    n, at = host.native, (hm.device, hm.stream)
    x, r, w = torch.randn(4, 64).bfloat16(), torch.randn(4, 64).bfloat16(), torch.randn(64).bfloat16()
    q, w8 = sk.Quantized(torch.zeros(4, 64, dtype=torch.int8), torch.ones(4)), sk.Quantized(torch.zeros(8, 64, dtype=torch.int8), torch.ones(8))
    place = (4, 1, 1, 1, 2, 2, 2, 0, 1)
    return ((n.plain_rmsnorm_fwd, (x, w, r, 1e-6, True, sk.Quantized, None, *at), {1, 2, 6}),
            (n.plain_rmsnorm_fwd, (x, w, r, 1e-6, False, sk.Quantized, place, *at), {1, 2, 6}),
            (n.plain_quantize_int8, (x, sk.Quantized, None, *at), {2}),
            (n.plain_quantize_int8, (x, sk.Quantized, place, *at), {2}),
            (n.plain_linear_fwd_int8, (q, w8, torch.randn(8).bfloat16(), torch.randn(4, 8).bfloat16(), 1, sk.Quantized, None, *at), {2, 3, 6}),
            (n.plain_rmsnorm_bwd, (x, r, w, r, 1e-6, True, True, *at), {2, 3}))


def test_every_argument_counts(host):
    """What is answered as it stands is not with any one argument that does not fit the others: nothing is launched then."""
    strided, cuda_like = torch.randn(4, 128).bfloat16()[:, ::2], torch.zeros(4, 64, dtype=BF16, device="meta")
    bad = (None, 5, 1.5, "x", (), (1,) * 9, (1,) * 8, (1,) * 8 + (1.5,), (1 << 31,) + (1,) * 8, [], torch.zeros(2), torch.zeros(0), torch.zeros(4, 63), torch.zeros(4, 64, dtype=torch.float16), strided, cuda_like,
           sk.Quantized(torch.zeros(4, 64, dtype=torch.int8), torch.ones(3)), sk.Quantized(torch.zeros(4, 64), torch.ones(4)), sk.Quantized(torch.zeros(4, 64, dtype=torch.int8), torch.ones(4).double()),
           sk.Quantized(torch.zeros(4, 64, dtype=torch.uint8), torch.ones(4)), torch.int8, object())
    for call, good, optional in _calls(host):
        assert call(*good) is not NotImplemented and len(host.calls) == 1
        host.calls.clear()
        for i in range(len(good)):
            for b in bad:
                # the module takes any PLACE of nine numbers, which the binding has made; with a residual the result's shape has to be its
                place = isinstance(b, tuple) and not isinstance(b, sk.Quantized) and b == (1,) * 9 and good[i - 1] is sk.Quantized and call.__name__ != "plain_linear_fwd_int8"
                fits = place or (b is None and i in optional) or (type(b) is type(good[i]) is float) or (type(b) is type(good[i]) is int)
                # any rows can be quantised: how many channels they may have is the library's to say
                fits = fits or (call.__name__ == "plain_quantize_int8" and i == 0 and type(b) is torch.Tensor and b.dtype is F32 and b.numel() > 0)
                got = call(*good[:i], b, *good[i + 1:])
                if fits:
                    host.calls.clear()
                else:
                    assert got is NotImplemented and not host.calls, (call.__name__, i, b)
        assert call(*good[:-1]) is call(*good, 1) is call() is NotImplemented and not host.calls


def _at(t):
    return t.data_ptr()


def test_what_reaches_the_library(host):
    """Every argument in its place, results that are shaped as the call says, and a workspace of the size that was asked for."""
    n, at = host.native, (hm.device, hm.stream)
    x, r, w = torch.randn(2, 8, 64), torch.randn(2, 8, 64), torch.randn(64)
    place = (8, 2, 2, 1, 4, 2, 2, 1, 1)
    out, total = n.plain_rmsnorm_fwd(x, w, r, 0.25, False, sk.Quantized, None, *at)
    assert host.calls.pop() == ("skiparse_rmsnorm_fwd", (_at(x), _at(r), _at(w), _at(total), _at(out), None, 1, 1, 1, 16, 64, 0.25, 1, 0, 0, 1, 5))
    assert out.shape == total.shape == x.shape and out.dtype == total.dtype == F32
    q = n.plain_rmsnorm_fwd(x.bfloat16(), None, None, 0.5, True, sk.Quantized, place, *at)
    name, args = host.calls.pop()
    assert args[1:] == (None, None, None, _at(q.codes), _at(q.scales), 2, 1, 4, 2, 64, 0.5, 2, 1, 1, 0, 5)
    assert type(q) is sk.Quantized and q.codes.shape == (8, 2, 64) and q.scales.shape == (8, 2) and q.codes.dtype == torch.int8 and q.scales.dtype == F32
    q = n.plain_quantize_int8(x, sk.Quantized, place, *at)
    assert host.calls.pop() == ("skiparse_quantize_int8", (_at(x), _at(q.codes), _at(q.scales), 2, 1, 4, 2, 64, 2, 1, 1, 1, 5)) and q.codes.shape == (8, 2, 64)
    w8, bias, res = sk.Quantized(torch.zeros(24, 64, dtype=torch.int8), torch.ones(24)), torch.randn(24).bfloat16(), torch.randn(8, 2, 24).bfloat16()
    out = n.plain_linear_fwd_int8(q, w8, bias, res, 2, sk.Quantized, None, *at)
    name, args = host.calls.pop()
    assert args[:7] == tuple(map(_at, (*q, *w8, bias, res, out))) and args[7:17] == (1, 1, 1, 16, 64, 24, 1, 0, 0, 2) and args[17] is not None and args[18:] == (hm.SPACE, 5)
    assert out.shape == res.shape and out.dtype == BF16
    dx, dw = n.plain_rmsnorm_bwd(x, r, w, x, 0.5, True, True, *at)
    name, args = host.calls.pop()
    assert args[:6] == tuple(map(_at, (x, r, w, x, dx, dw))) and args[6:16] == (1, 1, 1, 16, 64, 0.5, 1, 0, 0, 1) and args[16] is not None and args[17:] == (hm.SPACE, 5)
    assert dx.shape == r.shape and dw.shape == (64,)
    assert n.plain_rmsnorm_bwd(x, r, None, None, 0.5, True, False, *at)[1] is None and host.calls.pop()[1][16:] == (None, 0, 5)
    assert not host.calls


def test_refused_by_the_library(host):
    """A code becomes the binding's exception, with nothing left behind."""
    host.code = -2
    for call, good, _ in _calls(host):
        with pytest.raises(sk.SkiparseError):
            call(*good)


def test_scales_of_a_slice_are_the_bindings(host):
    """Scales that begin off 16 bytes are copied there; the module leaves them alone."""
    n, at = host.native, (hm.device, hm.stream)
    q, w8 = sk.Quantized(torch.zeros(9, 64, dtype=torch.int8), torch.ones(9)), sk.Quantized(torch.zeros(16, 64, dtype=torch.int8), torch.ones(16))
    assert q.scales.data_ptr() % 16 == w8.scales.data_ptr() % 16 == 0
    for i, j, answered in ((0, 0, True), (4, 4, True), (1, 0, False), (0, 2, False), (3, 5, False), (5, 8, False)):
        got = n.plain_linear_fwd_int8(sk.Quantized(q.codes[i:], q.scales[i:]), sk.Quantized(w8.codes[j:j + 8], w8.scales[j:j + 8]), None, None, 0, sk.Quantized, None, *at)
        assert (got is not NotImplemented) == answered == bool(host.calls)
        host.calls.clear()


# A daemon thread that does nothing but a whole call, of a function that returns at once, and no code that it has: no tensor comes back, since where the last reference to one goes torch lets go of the lock by itself.
AT_THE_END = """
import ctypes
import sys
import threading
import time
import torch
import _host_marshal as hm
import paper_2605_28691_amd as sk

n = hm.Host(sys.argv[1]).native
n.bind("skiparse_quantize_int8", ctypes.cast(ctypes.CDLL(None).getpid, ctypes.c_void_p).value)
x, calls = torch.randn(4, 64), []


def loop():
    while True:
        try:
            n.plain_quantize_int8(x, sk.Quantized, None, hm.device, hm.stream)
        except sk.SkiparseError:
            calls[:] = [True]


threading.Thread(target=loop, daemon=True).start()
while not calls:
    time.sleep(0.01)
time.sleep(0.1)
"""


def test_a_daemon_thread_at_the_end_of_the_process(path):
    """It is ended where it asks for the interpreter's lock, and the process with the code of its own."""
    for _ in range(3):
        done = subprocess.run([sys.executable, "-c", AT_THE_END, path], cwd=HERE, env={**os.environ, "PYTHONPATH": os.path.dirname(HERE)}, stderr=subprocess.PIPE, text=True, timeout=100)
        assert done.returncode == 0, (done.returncode, done.stderr)
