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
