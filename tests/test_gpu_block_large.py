"""GPU: tensors whose offsets pass 32 bits, and others that are long along one side, through the operators round the attention; samples against float64."""
import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu


def _fill(t, seed):
    """Values that depend on the place, without a tensor of random numbers as large again."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    row = torch.randn(1, *t.shape[1:], generator=g, device="cuda").to(t.dtype)
    t.copy_(row.expand_as(t))
    t.mul_(torch.rand(t.shape[0], generator=g, device="cuda").add_(0.5).to(t.dtype).view(-1, *[1] * (t.dim() - 1)))
    return t


ROWS = 300_000  # times 8192 channels: 4.9 GB in bf16, 2.5 * 10^9 elements


def test_linear_beyond_32_bits():
    import paper_2605_28691_amd as sk

    K, N = 8192, 24
    x = _fill(torch.empty(ROWS, K, dtype=torch.bfloat16, device="cuda"), 1)
    w = (torch.randn(N, K, device="cuda") * K ** -0.5).bfloat16()
    at = torch.tensor([0, 1, 131071, 131072, 262143, 262144, ROWS - 2, ROWS - 1], device="cuda")
    out = sk.skiparse_linear_fwd(x, w)
    want = x[at].double() @ w.double().t()
    bound = ref.BF16 * want.abs() + (K + 4) * ref.F32 * (x[at].double().abs() @ w.double().abs().t())
    assert ((out[at].double() - want).abs() <= bound).all() and out.isfinite().all()
    dy = torch.randn(ROWS, N, device="cuda").bfloat16()
    dx, dw, db = sk.skiparse_linear_bwd(dy, x, w)
    want = dy[at].double() @ w.double()
    assert ((dx[at].double() - want).abs() <= ref.BF16 * want.abs() + (N + 4) * ref.F32 * (dy[at].double().abs() @ w.double().abs())).all()
    want, size = torch.zeros(N, K, dtype=torch.float64, device="cuda"), torch.zeros(N, K, dtype=torch.float64, device="cuda")
    for i in range(0, ROWS, 20_000):
        a, b = dy[i : i + 20_000].double(), x[i : i + 20_000].double()
        want += a.t() @ b
        size += a.abs().t() @ b.abs()
    # float32 sums in up to 16 parts of ROWS / 16 rows: their error grows with the root of the rows at random, and is bounded by it times the sum of sizes / rows
    assert ((dw.double() - want).abs() <= ref.BF16 * want.abs() + ROWS * ref.F32 * size).all()
    assert float((dw.double() - want).norm() / want.norm()) <= ref.BF16
    del dx
    # the other way round: results of that size
    up = sk.skiparse_linear_fwd(dy, w.t().contiguous(), act="silu")
    z = dy[at].double() @ w.double()
    assert ((up[at].double() - ref.act("silu", z)).abs() <= ref.BF16 * ref.act("silu", z).abs() + (N + 4) * 1.2 * ref.F32 * (dy[at].double().abs() @ w.double().abs()) + 2.0 ** -19 * z.abs()).all()
    assert up.isfinite().all()


def test_rope_and_checkpoints_beyond_32_bits():
    import paper_2605_28691_amd as sk

    q = _fill(torch.empty(ROWS, 64, 128, dtype=torch.bfloat16, device="cuda"), 2).view(1, ROWS, 64, 128)
    table = sk.skiparse_rope_table((1, 1, ROWS), (0, 0, 128))
    at = torch.tensor([0, 131071, 262144, ROWS - 1], device="cuda")
    got, _ = sk.skiparse_rope(q, None, table, 1, 1, ROWS)
    cs = table.data.view(ROWS, 64, 2)[at].double()
    z = torch.view_as_complex(q[0, at].double().view(4, 64, 64, 2)) * torch.view_as_complex(cs.contiguous())[:, None]
    want = torch.view_as_real(z).reshape(4, 64, 128)
    assert ((got[0, at].double() - want).abs() <= ref.BF16 * want.abs() + 8 * ref.F32 * q[0, at].double().abs().amax()).all()
    del got
    x = q.view(ROWS, 8192)
    kept = sk.skiparse_checkpoint_save(x)
    codes, scales, values = ref.checkpoint(x[at].double())
    assert torch.equal(kept.codes[at], codes) and torch.equal(kept.scales[at], scales)
    assert torch.equal(sk.skiparse_checkpoint_load(kept)[at].double(), values)


def test_many_short_rows():
    """More rows than a grid's tiles have numbers to spare, and 8 channels."""
    import paper_2605_28691_amd as sk

    M = 4_000_003
    x, w = torch.randn(M, 8, device="cuda").bfloat16(), torch.randn(8, 8, device="cuda").bfloat16()
    dy = torch.randn(M, 8, device="cuda").bfloat16()
    out = sk.skiparse_linear_fwd(x, w)
    want = x.double() @ w.double().t()
    assert ((out.double() - want).abs() <= ref.BF16 * want.abs() + 12 * ref.F32 * (x.double().abs() @ w.double().abs().t())).all()
    dx, dw, db = sk.skiparse_linear_bwd(dy, x, w)
    want = dy.double() @ w.double()
    assert ((dx.double() - want).abs() <= ref.BF16 * want.abs() + 12 * ref.F32 * (dy.double().abs() @ w.double().abs())).all()
    want, size = dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs()
    # a random walk of M roundings of partial sums, each at most 2^-24 of the sum of sizes: 8 times its root, or 8 sqrt(M) / M of the bound for the worst case
    assert ((dw.double() - want).abs() <= ref.BF16 * want.abs() + 8 * M ** 0.5 * ref.F32 * size).all()
    want, size = dy.double().sum(0), dy.double().abs().sum(0)
    assert ((db.double() - want).abs() <= ref.BF16 * want.abs() + 8 * M ** 0.5 * ref.F32 * size).all()


@pytest.mark.parametrize("M", [1, 5, 20, 40])
def test_weights_beyond_32_bits(M):
    """Few rows against 4.4 GB of weights: the kernels that read them once, and tiles."""
    import paper_2605_28691_amd as sk

    K, N = 1 << 22, 520
    w = _fill(torch.empty(N, K, dtype=torch.bfloat16, device="cuda"), 3)
    x = torch.randn(M, K, device="cuda").bfloat16()
    out = sk.skiparse_linear_fwd(x, w)
    for i in range(0, N, 104):
        part = w[i : i + 104].double()
        want, size = x.double() @ part.t(), x.double().abs() @ part.abs().t()
        assert ((out[:, i : i + 104].double() - want).abs() <= ref.BF16 * want.abs() + (K + 4) * ref.F32 * size).all()
        # 8 times the root of K roundings, each at most 2^-24 of the sum of sizes at that point
        assert ((out[:, i : i + 104].double() - want).abs() <= ref.BF16 * want.abs() + 8 * K ** 0.5 * ref.F32 * size).all()


def test_checkpoints_in_more_than_one_launch():
    """More places of 8 channels than a launch takes: 9 * 10^8 rows of 8 channels, whose blocks of 32 are a quarter full."""
    import paper_2605_28691_amd as sk

    rows = 900_000_001
    x = torch.empty(rows, 8, dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.linspace(-3, 3, 8, device="cuda").bfloat16().expand_as(x))
    x[::3] *= 0.25
    kept = sk.skiparse_checkpoint_save(x)
    at = torch.cat([torch.arange(i - 3, i + 3, device="cuda") for i in (3, 1 << 29, 1 << 28, 3 << 28, rows - 3)])  # 4 places a row: 2^31 of them are 2^29 rows
    codes, scales, values = ref.checkpoint(x[at].double())
    assert torch.equal(kept.codes[at], codes) and torch.equal(kept.scales[at], scales)
    got = sk.skiparse_checkpoint_load(kept)
    assert torch.equal(got[at].double(), values)
    assert bool((kept.scales[::3] == kept.scales[0]).all() and (kept.scales[1::3] == kept.scales[1]).all() and (kept.scales[2::3] == kept.scales[1]).all())
    assert torch.equal(got[2::3], got[1:2].expand_as(got[2::3])) and torch.equal(got[::3], got[:1].expand_as(got[::3]))
