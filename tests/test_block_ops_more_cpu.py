"""The operators round the attention, without a GPU: arguments at the ends of their types, in the C ABI and the binding."""
import ctypes

import pytest
import torch

import paper_2605_28691_amd as sk

P = [ctypes.c_void_p(0x10000 + i * (1 << 44)) for i in range(8)]  # addresses far apart; never dereferenced because validation fails first
EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE = -1, -2, -3, -4


def test_rope_table_takes_its_base_and_factors_in_64_bits():
    """Refusals of the call in 64 bits, and the types that the binding hands over."""
    L = sk.lib()
    types = L.skiparse_rope_table_ex.argtypes
    assert [i for i, t in enumerate(types) if t is ctypes.c_double] == [7, 9, 10, 11, 15, 16, 17] and ctypes.c_float not in types
    assert "skiparse_rope_table_ex" in sk._TENSORS

    def call(T=2, r=(4, 4, 8), theta=1e4, scaling=0, factor=(1, 1, 1), trained=(0, 0, 0), fast=32, slow=1, attention=1):
        return L.skiparse_rope_table_ex(P[0], T, 3, 4, *r, theta, scaling, *factor, *trained, fast, slow, attention, None)

    inf, nan = float("inf"), float("nan")
    for bad in (dict(T=0), dict(r=(0, 0, 0)), dict(r=(3, 4, 8)), dict(theta=0), dict(theta=nan), dict(theta=inf), dict(theta=1e300), dict(attention=nan), dict(attention=-inf),
                dict(scaling=1, factor=(1, 1 - 2.0 ** -40, 1)), dict(scaling=2, factor=(1, 1, inf)), dict(scaling=2, factor=(nan, 1, 1)),
                dict(scaling=3, factor=(2, 2, 2), trained=(5, 0, 5)), dict(scaling=3, factor=(2, 2, 2), trained=(5, 5, 5), fast=1, slow=1),
                dict(scaling=3, factor=(2, 2, 2), trained=(5, 5, 5), fast=nan)):
        assert call(**bad) == EINVAL, bad
    # channels whose sum passes 31 bits
    assert call(r=(2147483646, 2147483646, 2147483646)) == EUNSUPPORTED


def test_integers_beyond_the_c_types_are_refused(monkeypatch):
    """2^32 + 1 rows are not one row: what a C type does not hold is refused, by the calls and by the functions of sizes, and not cut."""
    meta = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="meta")  # noqa: E731
    monkeypatch.setattr(sk, "_stream", lambda: 0)
    monkeypatch.setattr(sk, "_here", lambda *t: None)
    for rows in ((1 << 32) + 1, 1 << 31, (1 << 32) + 128):
        x, w = meta(rows, 8), meta(16, 8)
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_checkpoint_save(x)
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_checkpoint_load(sk.Checkpoint(meta(rows, 8, dtype=torch.uint8), meta(rows, 1, dtype=torch.uint8)))
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_linear_fwd(x, w)
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_linear_bwd(meta(rows, 16), x, w)
        for f in (sk.skiparse_linear_workspace_bytes, sk.skiparse_linear_bwd_workspace_bytes):
            with pytest.raises(ValueError, match="does not fit the 32 bits"):
                f(rows, 5120, 5120)
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_rope_table((1, 1, rows), (0, 0, 8), device="meta")
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_workspace_bytes(rows, 1, 1, 8, 8, 64, 2, False)
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk.skiparse_lse_shape(rows, 1, 1, 8, 8, 64, 2, "token")
    table = sk.RopeTable(meta(2 * 16 * 4, dtype=torch.float32), (1, 1, 16), (0, 0, 8))
    q = meta(1, 4, 1, 8)
    with pytest.raises(ValueError, match="does not fit the 32 bits"):
        sk.skiparse_rope(q, None, table, 1, 1, 4, at=(0, 0, 1 << 32))
    with pytest.raises(ValueError, match="does not fit the 64 bits"):  # bytes of a workspace
        sk._general("skiparse_linear_fwd", q, q, None, None, q, None, None, 1, 1, 1, 4, 8, 8, 1, 0, 0, 0, 0, None, -1, 0)
    with pytest.raises(ctypes.ArgumentError):  # no integer
        sk.skiparse_linear_workspace_bytes(4.0, 8, 8)


def test_backward_asks_for_what_it_reads_only(monkeypatch):
    """x is read for dw and w for dx, as in the C call: a program that wants one of them need not have kept the other."""
    calls = []
    monkeypatch.setattr(sk, "_stream", lambda: 0)
    monkeypatch.setattr(sk, "_here", lambda *t: None)
    monkeypatch.setattr(sk, "_skiparse_linear_bwd", lambda *a: calls.append(a))
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    dy, x, w = bf(5, 32), bf(5, 64), bf(32, 64)
    dx, dw, db = sk.skiparse_linear_bwd(dy, None, w, need_dw=False)
    assert dx.shape == x.shape and dw is None and db.shape == (32,)
    a = calls.pop()
    assert a[1] is None and a[3] is w and a[10:16] == (1, 1, 1, 5, 64, 32)
    dx, dw, db = sk.skiparse_linear_bwd(dy, x, None, need_dx=False)
    assert dx is None and dw.shape == w.shape
    a = calls.pop()
    assert a[1] is x and a[3] is None and a[14:16] == (64, 32)
    assert sk.skiparse_linear_bwd(dy, None, None, need_dx=False, need_dw=False)[2].shape == (32,)
    # rows that move: the other side's shape follows from dy's
    dy = bf(4, 8, 32)
    at = dict(order="to_sparse", T=2, H=4, W=4, s=2)
    assert sk.skiparse_linear_bwd(dy, None, w, need_dw=False, **at)[0].shape == (1, 32, 64)
    at["order"] = "to_original"
    assert sk.skiparse_linear_bwd(dy.view(1, 32, 32), None, w, need_dw=False, dx_add=bf(4, 8, 64), **at)[0].shape == (4, 8, 64)
    calls.clear()
    for args, kw in (((dy, None, w), {}), ((dy, bf(4, 8, 64), None), {}), ((dy, None, w), dict(need_dx=False)), ((dy, bf(4, 8, 56), w), dict(need_dw=False)),
                     ((dy, bf(4, 7, 64), None), dict(need_dx=False)), ((dy, None, bf(64)), dict(need_dw=False)), ((dy, None, bf(24, 64)), dict(need_dw=False)),
                     ((dy, None, w), dict(need_dw=False, dx_add=bf(4, 8, 56))), ((dy, None, w), dict(need_dw=False, order="to_sparse", T=2, H=4, W=3, s=2))):
        with pytest.raises(ValueError):
            sk.skiparse_linear_bwd(*args, **kw)
    assert not calls


def test_arguments_of_another_number_are_refused(monkeypatch):
    """A place with more or fewer than three numbers does not move the arguments behind it; nor does any call by the general way."""
    monkeypatch.setattr(sk, "_stream", lambda: 0)
    monkeypatch.setattr(sk, "_here", lambda *t: None)
    q = torch.zeros(1, 4, 1, 8, dtype=torch.bfloat16)
    table = sk.RopeTable(torch.zeros(2 * 16 * 4), (1, 1, 16), (0, 0, 8))
    calls = []
    with monkeypatch.context() as m:
        m.setattr(sk, "_skiparse_rope", lambda *a: calls.append(a))
        sk.skiparse_rope(q, None, table, 1, 1, 4, at=(0, 0, 5))
        assert len(calls[0]) == len(sk.lib().skiparse_rope.argtypes) and calls.pop()[17:20] == (0, 0, 5)
        for at in ((0, 0), (0, 0, 0, 0), ()):
            with pytest.raises(ValueError):
                sk.skiparse_rope(q, None, table, 1, 1, 4, at=at)
    assert not calls
    for name, tensors in sk._TENSORS.items():
        n = len(getattr(sk.lib(), name).argtypes)
        for count in (0, n - 1, n + 1):
            with pytest.raises(TypeError, match="arguments"):
                sk._general(name, *[1] * count)
