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
