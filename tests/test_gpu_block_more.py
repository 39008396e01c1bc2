"""GPU: the operators round the attention, at the ends of what their calls take."""
import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu


def test_integers_beyond_the_c_types_do_not_reach_the_library():
    """By the native way: 2^32 + 4 rows are not four."""
    import paper_2605_28691_amd as sk

    assert sk._marshal is not None
    x = torch.randn(4, 64, device="cuda").bfloat16()
    codes, scales = torch.full((4, 64), 0xAB, dtype=torch.uint8, device="cuda"), torch.full((4, 2), 0xAB, dtype=torch.uint8, device="cuda")
    for rows in ((1 << 32) + 4, (1 << 64) + 4, 4 - (1 << 32)):
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk._skiparse_checkpoint_save(x, codes, scales, rows, 64, 0, sk._stream())
    assert (codes == 0xAB).all() and (scales == 0xAB).all()
    q = torch.randn(1, 4, 1, 64, device="cuda").bfloat16()
    table = sk.skiparse_rope_table((1, 1, 16), (0, 0, 64))
    with pytest.raises(ValueError, match="does not fit the 32 bits"):
        sk.skiparse_rope(q, None, table, 1, 1, 4, at=(0, 0, 1 << 32))
    # flags are unsigned, a workspace's bytes have 64 bits
    out, ws = torch.empty_like(x), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    w = torch.eye(64, device="cuda").bfloat16()
    call = (x, w, None, None, out, None, None, 1, 1, 1, 4, 64, 64, 1, 0, 0, 0, 0, ws)
    for size in (1 << 20, (1 << 63) - 1, (1 << 64) - 1):
        sk._skiparse_linear_fwd(*call, size, sk._stream())
    assert torch.equal(out, x)
    for size in (-1, 1 << 64):
        with pytest.raises(ValueError, match="does not fit the 64 bits"):
            sk._skiparse_linear_fwd(*call, size, sk._stream())
    for flags in (-1, 1 << 32):
        with pytest.raises(ValueError, match="does not fit the 32 bits"):
            sk._skiparse_attn_fwd(q, q, q, torch.empty_like(q), 1, 1, 1, 2, 2, 64, 2, 0, 0.0, 0, flags, None, 0, sk._stream())
