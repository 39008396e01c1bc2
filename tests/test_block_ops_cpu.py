"""Refusals of the operators round the attention, without a GPU: the C ABI's checks and the binding's."""
import ctypes

import pytest
import torch

import paper_2605_28691_amd as sk

P = [ctypes.c_void_p(0x10000 + i * (1 << 36)) for i in range(12)]  # addresses far apart; never dereferenced because validation fails first
ODD = ctypes.c_void_p(0x10004)
EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    return sk.lib()


def test_rope_table_refusals(lib):
    f = ctypes.c_float

    def call(table=P[0], T=2, H=3, W=4, r=(4, 4, 8), theta=1e4, scaling=0, factor=(1, 1, 1), trained=(0, 0, 0), fast=32, slow=1, attention=1):
        return lib.skiparse_rope_table(table, T, H, W, *r, f(theta), scaling, *map(f, factor), *trained, f(fast), f(slow), f(attention), None)

    inf, nan = float("inf"), float("nan")
    for bad in (dict(table=None), dict(table=ODD), dict(T=0), dict(W=-1), dict(r=(0, 0, 0)), dict(r=(3, 4, 8)), dict(r=(-2, 4, 8)), dict(theta=0), dict(theta=-1),
                dict(theta=nan), dict(theta=inf), dict(scaling=4), dict(scaling=-1), dict(attention=nan), dict(scaling=1, factor=(1, 0.5, 1)),
                dict(scaling=2, factor=(1, 1, inf)), dict(scaling=3, factor=(2, 2, 2), trained=(5, 0, 5)), dict(scaling=3, factor=(2, 2, 2), trained=(5, 5, 5), fast=1, slow=1)):
        assert call(**bad) == EINVAL, bad
    assert call(r=(514, 0, 0)) == EUNSUPPORTED
    assert call(W=1 << 30) == ESHAPE
    assert lib.skiparse_rope_table_bytes(2, 3, 4, 4, 4, 8) == 8 * (2 * 2 + 3 * 2 + 4 * 4)
    assert lib.skiparse_rope_table_bytes(2, 3, 4, 4, 3, 8) == 0 and lib.skiparse_rope_table_bytes(0, 3, 4, 4, 4, 8) == 0
    assert lib.skiparse_rope_table_bytes(1, 1, 1 << 30, 0, 0, 4) == 0


def test_rope_refusals(lib):
    def call(q=P[0], k=P[1], qo=P[2], ko=P[3], table=P[4], B=1, heads=2, T=2, H=8, W=8, D=64, r=(16, 16, 32), length=(2, 8, 8), at=(0, 0, 0), s=2, pattern=0, order=1,
             layout=0, inverse=0, dtype=0):
        return lib.skiparse_rope(q, k, qo, ko, table, B, heads, T, H, W, D, *r, *length, *at, s, pattern, order, layout, inverse, dtype, None)

    near = ctypes.c_void_p(P[0].value + 64)
    for bad in (dict(q=None), dict(qo=None), dict(table=None), dict(k=None), dict(ko=None), dict(q=ODD), dict(ko=ODD), dict(table=ODD), dict(order=4), dict(order=-1),
                dict(layout=2), dict(inverse=2), dict(dtype=7), dict(B=0), dict(heads=0), dict(pattern=3), dict(r=(0, 0, 0)), dict(r=(2, 3, 2)), dict(r=(32, 32, 2)),
                dict(r=(66, 0, 0)), dict(at=(-1, 0, 0)), dict(length=(2, 0, 8)), dict(qo=P[0]), dict(qo=near), dict(qo=P[1]), dict(ko=P[2]), dict(ko=P[0]), dict(qo=P[4]),
                dict(order=0, qo=near), dict(order=0, qo=P[1], k=P[1])):
        assert call(**bad) == EINVAL, bad
    for bad in (dict(H=7), dict(H=6, pattern=1), dict(at=(1, 0, 0)), dict(length=(2, 7, 8)), dict(at=(0, 0, 2147483647)), dict(T=1 << 12, H=1 << 10, W=1 << 10)):
        assert call(**bad) == ESHAPE, bad
    for bad in (dict(dtype=2), dict(D=68), dict(D=520)):
        assert call(**bad) == EUNSUPPORTED, bad
    # an axis without channels has no places to fit; the next check is reached
    assert call(r=(0, 16, 16), length=(1, 8, 8), at=(5, 0, 0), qo=P[4]) == EINVAL


def test_checkpoint_refusals(lib):
    for f, first in ((lib.skiparse_checkpoint_save, True), (lib.skiparse_checkpoint_load, False)):
        def call(x=P[0], codes=P[1], scales=P[2], rows=4, cols=64, dtype=0):
            return f(*((x, codes, scales) if first else (codes, scales, x)), rows, cols, dtype, None)

        for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(rows=0), dict(cols=0), dict(rows=-1), dict(dtype=5), dict(x=ODD), dict(codes=ODD), dict(codes=P[0]),
                    dict(scales=P[1]), dict(scales=ctypes.c_void_p(P[0].value + 3))):
            assert call(**bad) == EINVAL, bad
        assert call(dtype=2) == EUNSUPPORTED and call(cols=60) == EUNSUPPORTED
        assert call(rows=2147483647, cols=2147483640) == ESHAPE


def _fwd(lib, x=P[0], w=P[1], bias=P[2], residual=P[3], out=P[4], pre=P[5], scales=P[6], B=1, T=2, H=8, W=8, K=64, N=128, s=2, pattern=0, order=1, act=1, dtype=0, ws=P[7],
         size=1 << 34):
    return lib.skiparse_linear_fwd(x, w, bias, residual, out, pre, scales, B, T, H, W, K, N, s, pattern, order, act, dtype, ws, size, None)


def test_linear_refusals(lib):
    near = ctypes.c_void_p(P[3].value + 16)
    for bad in (dict(x=None), dict(w=None), dict(out=None), dict(pre=None), dict(order=3), dict(order=-1), dict(act=3), dict(act=-1), dict(dtype=9), dict(B=0), dict(K=0),
                dict(N=-8), dict(pattern=2), dict(x=ODD), dict(w=ODD), dict(bias=ODD), dict(residual=ODD), dict(out=ODD), dict(pre=ODD), dict(out=P[0]), dict(out=P[1]),
                dict(out=P[2]), dict(out=near), dict(pre=P[4]), dict(pre=P[3]), dict(scales=P[5]), dict(scales=P[0])):
        assert _fwd(lib, **bad) == EINVAL, bad
    for bad in (dict(H=7), dict(H=6, pattern=1), dict(K=1 << 23), dict(N=1 << 23), dict(T=1 << 12, H=1 << 10, W=1 << 10), dict(T=256, H=128, W=128, K=512)):
        assert _fwd(lib, **bad) == ESHAPE, bad
    for bad in (dict(dtype=1), dict(dtype=2), dict(K=60), dict(N=100)):
        assert _fwd(lib, **bad) == EUNSUPPORTED, bad
    assert _fwd(lib, K=(1 << 23) - 8, N=(1 << 23) - 8, s=1) == ESHAPE  # weights of 2^40 elements and more
    # a product that is cut along k needs the workspace, clear of everything else
    large = dict(T=1, H=16, W=8, s=1, K=5120, N=5120)
    need = lib.skiparse_linear_workspace_bytes(128, 5120, 5120)
    assert need > 0
    for bad in (dict(ws=None), dict(size=need - 1), dict(ws=ODD)):
        assert _fwd(lib, **large, **bad) == EWORKSPACE, bad
    for at in (0, 1, 2, 3, 4, 5, 6):
        assert _fwd(lib, **large, ws=P[at]) == EINVAL, at


def test_linear_backward_refusals(lib):
    def call(dy=P[0], x=P[1], xs=P[2], w=P[3], pre=P[4], ps=P[5], add=P[6], dx=P[7], dw=P[8], db=P[9], B=1, T=2, H=8, W=8, K=64, N=128, s=2, pattern=0, order=1, act=1,
             dtype=0, ws=P[10], size=1 << 34):
        return lib.skiparse_linear_bwd(dy, x, xs, w, pre, ps, add, dx, dw, db, B, T, H, W, K, N, s, pattern, order, act, dtype, ws, size, None)

    near = ctypes.c_void_p(P[6].value + 16)
    for bad in (dict(dy=None), dict(dx=None, dw=None, db=None, add=None), dict(w=None), dict(x=None), dict(pre=None), dict(add=P[6], dx=None), dict(act=7), dict(order=3),
                dict(pre=None, ps=None), dict(dx=P[0]), dict(dx=P[1]), dict(dx=P[3]), dict(dx=near), dict(dx=P[8]), dict(dw=P[6]), dict(db=P[5]), dict(dw=P[9]),
                dict(ws=P[0]), dict(ws=P[8]), dict(ws=P[2]), dict(dx=ODD), dict(db=ODD), dict(dy=ODD)):
        assert call(**bad) == EINVAL, bad
    need = lib.skiparse_linear_bwd_workspace_bytes(128, 64, 128, 1, 1, 1)
    assert need >= 128 * 128 * 2 + 128 * 64 * 2
    assert call(size=0) == EWORKSPACE and call(ws=None) == EWORKSPACE and call(ws=ODD) == EWORKSPACE
    assert call(H=7) == ESHAPE and call(K=12) == EUNSUPPORTED
    for bad in ((0, 64, 128, 1, 1, 1), (128, -1, 128, 1, 1, 1), (128, 64, 128, 3, 1, 1), (128, 64, 128, 1, 5, 1)):
        assert lib.skiparse_linear_bwd_workspace_bytes(*bad) == 0


def test_what_may_be_left_out_is_what_the_native_module_takes(monkeypatch):
    """The binding's table of optional tensors against the module's: None there must not send the call the general way, None elsewhere must."""
    assert set(sk._OPTIONAL) <= set(sk._TENSORS)
    for name, optional in sk._OPTIONAL.items():
        assert optional <= {i for i, _ in sk._TENSORS[name]}
    source = open(sk._HERE + "/csrc/marshal.cpp").read()
    import re

    listed = {m[0]: {int(i) for i in m[1].split(",")} for m in re.findall(r"X\((\w+), at\(([\d, ]+)\)\)", source)}
    assert listed == sk._OPTIONAL


def test_binding_refusals(monkeypatch):
    monkeypatch.setattr(sk, "_stream", lambda: 0)
    monkeypatch.setattr(sk, "_here", lambda *t: None)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    x, w = bf(4, 64), bf(32, 64)
    for args, kw in (((x, bf(32, 56)), {}), ((x, w, bf(64)), {}), ((x, w, None, bf(4, 64)), {}), ((x.float(), w), {}), ((x, w.float()), {}), ((x, w), dict(keep="fp8")),
                     ((x, w), dict(pre=bf(4, 32))), ((x, w), dict(out=bf(5, 32))), ((x, w), dict(order="to_sparse", T=1, H=2, W=2, s=2)),
                     ((x, w), dict(keep="checkpoint", pre=sk.Checkpoint(torch.zeros(4, 32), torch.zeros(4, 1)))), ((x, w), {})):
        with pytest.raises(ValueError):  # the last one: tensors on the CPU
            sk.skiparse_linear_fwd(*args, **kw)
    dy = bf(4, 32)
    for args, kw in (((dy, bf(4, 56), w), {}), ((bf(4, 40), x, w), {}), ((dy, x, w), dict(act="silu")), ((dy, x, w), dict(act="silu", pre=bf(3, 32))), ((bf(3, 32), x, w), {}),
                     ((dy, x, w), dict(dx_add=bf(4, 32))), ((dy, x, w), dict(dw=bf(64, 32))), ((dy, x.float(), w), {})):
        with pytest.raises(ValueError):
            sk.skiparse_linear_bwd(*args, **kw)
    with pytest.raises(KeyError):
        sk.skiparse_linear_fwd(x, w, act="relu")
    q = bf(1, 128, 2, 64)
    table = sk.RopeTable(torch.zeros(2 * (2 * 8 + 8 * 8 + 8 * 16)), (2, 8, 8), (16, 16, 32))
    for args, kw in (((q, None, table, 2, 8, 7), {}), ((q, bf(1, 128, 1, 64), table, 2, 8, 8), {}), ((q, q.float(), table, 2, 8, 8), {}), ((q[0], None, table, 2, 8, 8), {}),
                     ((q, None, table, 2, 8, 8, 2, "token", "to_original"), {}), ((q, None, table._replace(data=table.data[1:]), 2, 8, 8), {}),
                     ((q, None, table._replace(data=table.data.double()), 2, 8, 8), {}), ((q, None, table, 2, 8, 8), dict(q_out=bf(128, 1, 2, 64))),
                     ((q, None, table, 0, 8, 8), {}), ((q, None, table, 2, 8, 8), {})):
        with pytest.raises(ValueError):
            sk.skiparse_rope(*args, **kw)
    for bad in (((0, 1, 1), (2, 2, 2)), ((1, 1, 1), (1, 2, 2)), ((1, 1, 1), (0, 0, 0))):
        with pytest.raises(ValueError):
            sk.skiparse_rope_table(*bad, device="cpu")
    with pytest.raises(ValueError):
        sk.skiparse_checkpoint_load(sk.Checkpoint(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)))
    with pytest.raises(ValueError):
        sk.skiparse_checkpoint_save(x)  # on the CPU


def test_tensors_of_another_device_are_refused(monkeypatch):
    class Far:
        device = "cuda:1"

        @staticmethod
        def get_device():
            return 1

    monkeypatch.setattr(sk, "_get_device", lambda: 0)
    sk._here(None, torch.zeros(1))
    with pytest.raises(ValueError):
        sk._here(Far)
