"""GPU: 8-bit activation checkpoints against their definition in float64, code by code."""
import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu


def _values(rows, cols, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(6 * torch.randn(rows, cols, generator=g))
    flat = x.view(-1)
    special = torch.tensor([0.0, -0.0, 448.0, 464.0, 465.0, 2.0 ** -9, 2.0 ** -10, 1e-42, 3.0e38, -3.0e38, 2.0 ** -126, 1.75, 1.7500001])
    flat[torch.randperm(flat.numel(), generator=g)[: len(special)]] = special[: flat.numel()]
    if rows > 2:
        x[1] = 0.0
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, cols", [(1, 8), (1, 32), (3, 40), (5, 64), (2, 1000), (7, 1536), (513, 96), (130, 72), (1, 33000)])
def test_codes_scales_and_values(rows, cols, dtype):
    import paper_2605_28691_amd as sk

    x = _values(rows, cols, rows * 7 + cols).to(dtype)
    codes, scales, values = ref.checkpoint(x.double())
    got = sk.skiparse_checkpoint_save(x.cuda())
    assert torch.equal(got.scales.cpu(), scales)
    assert torch.equal(got.codes.cpu(), codes)
    for back in (torch.bfloat16, torch.float32):
        y = sk.skiparse_checkpoint_load(got, dtype=back)
        # four bits and a power of two: exact, but for rounding among the type's smallest numbers
        assert torch.equal(y.cpu(), values.float().to(back))


def test_values_that_are_not_finite():
    """They become NaN and leave the scale of their block to the others."""
    import paper_2605_28691_amd as sk

    x = torch.randn(4, 96, generator=torch.Generator().manual_seed(3))
    x[0, 5], x[1, 40], x[2, 64:] = float("inf"), float("nan"), float("-inf")
    for dtype in (torch.bfloat16, torch.float32):
        t = x.to(dtype)
        _, scales, values = ref.checkpoint(t.double())
        got = sk.skiparse_checkpoint_save(t.cuda())
        assert torch.equal(got.scales.cpu(), scales) and got.scales[2, 2] == 127
        y = sk.skiparse_checkpoint_load(got, dtype=torch.float32).cpu()
        assert torch.equal(y.isnan(), ~t.isfinite())
        assert torch.equal(y.nan_to_num(), values.float().nan_to_num())


def test_every_code_and_scale():
    """Reading: all 256 codes under all 256 scale bytes, 255 being NaN."""
    import paper_2605_28691_amd as sk

    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 8)
    want = ref.values(codes, scales)
    want[255] = float("nan")
    for dtype in (torch.bfloat16, torch.float32):
        got = sk.skiparse_checkpoint_load(sk.Checkpoint(codes.cuda(), scales.cuda()), dtype=dtype).cpu()
        same = torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.0).double(), want.float().to(dtype).nan_to_num(nan=0.0).double())
        assert same, dtype


def test_rows_behind_the_last_are_left_alone():
    import paper_2605_28691_amd as sk

    x = torch.randn(37, 72, device="cuda", dtype=torch.bfloat16)
    codes, scales = torch.full((40, 72), 0xAB, dtype=torch.uint8, device="cuda"), torch.full((40, 3), 0xAB, dtype=torch.uint8, device="cuda")
    sk.skiparse_checkpoint_save(x, out=sk.Checkpoint(codes[:37], scales[:37]))
    assert (codes[37:] == 0xAB).all() and (scales[37:] == 0xAB).all()
    y = torch.full((40, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    sk.skiparse_checkpoint_load(sk.Checkpoint(codes[:37], scales[:37]), out=y[:37])
    assert (y[37:] == 7.0).all() and y[:37].isfinite().all()


def test_attention_backward_from_checkpoints():
    """The attention's saved tensors in 8 bits: the backward pass of what they stand for, bit for bit."""
    import paper_2605_28691_amd as sk
    import synth_inputs as si

    w = si.make_shape("ckpt", 1, 3, 64, 3, 8, 12, 2, seed=71)
    q, k, v = (t.cuda() for t in si.make_qkv(w))
    dout = si.make_dout(w).cuda()
    at = (w.T, w.H, w.W, w.s, "group")
    out, lse = sk.skiparse_attn_fwd_lse(q, k, v, *at)
    kept = [sk.skiparse_checkpoint_save(t) for t in (q, k, v, out)]
    restored = [sk.skiparse_checkpoint_load(c) for c in kept]
    for r, t in zip(restored, (q, k, v, out)):
        _, _, want = ref.checkpoint(t.double().cpu().reshape(-1, w.D))
        assert torch.equal(r.double().cpu().reshape(-1, w.D), want)
    got = sk.skiparse_attn_bwd(*restored, dout, lse, *at)
    assert all(g.isfinite().all() for g in got)
