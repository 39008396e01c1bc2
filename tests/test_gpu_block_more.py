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


def test_more_rows_than_small_tiles_fit_a_grid():
    """2^30 + 5 rows of 8 channels: 2^24 tiles of 64 rows, and more, are not a launch; larger tiles are.  All rows are looked at, 17 GB a tensor."""
    import paper_2605_28691_amd as sk

    M, step = (1 << 30) + 5, 1 << 25
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.empty(M, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        for i in range(0, M, step):
            t[i : i + step] = torch.randn(min(step, M - i), 8, generator=g, device="cuda")
    w = torch.randn(8, 8, generator=g, device="cuda").bfloat16()
    w64 = w.double()
    close = lambda got, want, size: bool(((got.double() - want).abs() <= ref.BF16 * want.abs() + 12 * ref.F32 * size).all())  # noqa: E731
    out = sk.skiparse_linear_fwd(x, w)
    for i in range(0, M, step):
        a = x[i : i + step].double()
        assert close(out[i : i + step], a @ w64.t(), a.abs() @ w64.abs().t()), i
    del out
    dx, dw, db = sk.skiparse_linear_bwd(dy, x, w)
    sums = [torch.zeros(8, 8, dtype=torch.float64, device="cuda") for _ in range(2)] + [torch.zeros(8, dtype=torch.float64, device="cuda") for _ in range(2)]
    for i in range(0, M, step):
        a, b = dy[i : i + step].double(), x[i : i + step].double()
        assert close(dx[i : i + step], a @ w64, a.abs() @ w64.abs()), i
        for n in range(8):  # one channel of dy at a time: as a product of 2^25 terms an element it is the library's slowest
            v = a[:, n : n + 1] * b
            sums[0][n] += v.sum(0)
            sums[1][n] += v.abs_().sum(0)
        sums[2] += a.sum(0)
        sums[3] += a.abs_().sum(0)
    # at most M roundings of partial sums, each at most 2^-24 of the sum of sizes, in any direction: 8 times the root of their number
    for got, want, size in ((dw, *sums[:2]), (db, *sums[2:])):
        assert ((got.double() - want).abs() <= ref.BF16 * want.abs() + 8 * M ** 0.5 * ref.F32 * size).all()


def test_more_tokens_than_a_launch_of_positions_has_wavefronts():
    """67 million tokens of one head of 264 channels, a wavefront each: 2^24 workgroups, and more, are not a launch."""
    import paper_2605_28691_amd as sk

    B, W, D, step = 65729, 1021, 264, 1 << 22
    rows = B * W
    assert rows > 1 << 26
    g = torch.Generator(device="cuda").manual_seed(6)
    q = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, step):
        q[i : i + step] = torch.randn(min(step, rows - i), D, generator=g, device="cuda")
    table = sk.skiparse_rope_table((1, 1, W), (0, 0, 260))
    out = torch.full_like(q, float("nan"))
    sk.skiparse_rope(q.view(B, W, 1, D), None, table, 1, 1, W, q_out=out.view(B, W, 1, D))
    for i in range(0, rows, step):
        assert bool(out[i : i + step].isfinite().all()), i
    at = torch.cat([torch.randint(0, rows, (20_000,), generator=g, device="cuda")] + [torch.arange(max(0, i - 8), min(rows, i + 8), device="cuda") for i in (0, 1 << 25, 1 << 26, rows)])
    x = q[at].double()
    z = torch.view_as_complex(x[:, :260].reshape(-1, 130, 2)) * torch.view_as_complex(table.data.view(W, 130, 2)[at % W].double())
    want = torch.cat((torch.view_as_real(z).reshape(-1, 260), x[:, 260:]), 1)
    got = out[at].double()
    # one rounding of the result; products and their sum in float32
    assert bool(((got - want).abs() <= ref.BF16 * want.abs() + 8 * ref.F32 * x.abs().amax(1, keepdim=True)).all())
    assert torch.equal(got[:, 260:], x[:, 260:])


@pytest.mark.parametrize("order", ["same", "to_sparse", "to_original"])
def test_gradients_without_what_they_do_not_read(order):
    import paper_2605_28691_amd as sk

    T, H, W, s, K, N = 3, 4, 8, 2, 72, 136
    n = T * H * W
    sparse, plain = (4, n // 4), (1, n)
    lead = sparse if order == "to_sparse" else plain
    back = sparse if order == "to_original" else plain
    g = torch.Generator(device="cuda").manual_seed(8)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    dy, pre, x, w = r(*lead, N), r(*lead, N), r(*back, K), r(N, K)
    kw = dict(pre=pre, act="silu", order=order, T=T, H=H, W=W, s=s)
    want = sk.skiparse_linear_bwd(dy, x, w, **kw)
    dx, dw, db = sk.skiparse_linear_bwd(dy, None, w, need_dw=False, **kw)
    assert dw is None and torch.equal(dx, want[0]) and torch.equal(db, want[2])
    dx, dw, db = sk.skiparse_linear_bwd(dy, x, None, need_dx=False, **kw)
    assert dx is None and torch.equal(dw, want[1]) and torch.equal(db, want[2])
    assert torch.equal(sk.skiparse_linear_bwd(dy, None, None, need_dx=False, need_dw=False, **kw)[2], want[2])


@pytest.mark.parametrize("pattern", ["token", "group"])
def test_attention_gradients_from_checkpoints(pattern):
    """The attention's backward on saved tensors that went through 8 bits, against its formulas in float64 on the same values: P = exp(q k^T c - lse), dV = P^T dO,
    dS = P (dO V^T - rowsum(dO O)), dQ = c dS K, dK = c dS^T Q.  P and dS are rounded to bf16 for the products and the gradients once more: three roundings of 2^-8 at most, below 1e-2 in the
    2-norm as everywhere in the backward's tests."""
    import paper_2605_28691_amd as sk
    import synth_inputs as si

    w = si.make_shape("ckpt_grad", 1, 3, 64, 3, 8, 12, 2, seed=72)
    q, k, v = (t.cuda() for t in si.make_qkv(w))
    dout = si.make_dout(w).cuda()
    grid, H, W = (w.T, w.H, w.W), w.H, w.W
    if pattern == "group":
        assert H % (w.s * w.s) == 0 and W % (w.s * w.s) == 0
    at = (*grid, w.s, pattern)
    out, lse = sk.skiparse_attn_fwd_lse(q, k, v, *at)
    restored = [sk.skiparse_checkpoint_load(sk.skiparse_checkpoint_save(t)) for t in (q, k, v, out)]
    assert not torch.equal(restored[0], q)
    got = sk.skiparse_attn_bwd(*restored, dout, lse, *at)
    to = lambda t: ref.moved(t.double(), "to_sparse", (w.B, *grid), w.s, pattern).transpose(1, 2)  # noqa: E731  [sequences][heads][positions][D]
    q64, k64, v64, o64, d64 = (to(t) for t in (*restored, dout))
    c = w.D ** -0.5
    p = torch.exp(q64 @ k64.transpose(-1, -2).contiguous() * c - lse.double()[..., None])
    ds = p * (d64 @ v64.transpose(-1, -2).contiguous() - (d64 * o64).sum(-1, keepdim=True))
    want = ds @ k64 * c, ds.transpose(-1, -2).contiguous() @ q64 * c, p.transpose(-1, -2).contiguous() @ d64
    for a, b, name in zip(got, want, ("dq", "dk", "dv")):
        a = to(a)
        assert float((a - b).norm()) <= 1e-2 * float(b.norm()) and float((a - b).abs().max()) <= 3e-2 * float(b.abs().max()), name


def test_bias_gradient_of_many_rows():
    """300,000 rows, in parts of 128 that a second launch adds up."""
    import paper_2605_28691_amd as sk

    M, N = 300_000, 1000
    g = torch.Generator(device="cuda").manual_seed(9)
    dy = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    pre = (2 * torch.randn(M, N, generator=g, device="cuda")).bfloat16()
    for act in ("none", "silu"):
        _, _, db = sk.skiparse_linear_bwd(dy, None, None, pre=None if act == "none" else pre, act=act, need_dx=False, need_dw=False)
        want, size, off = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(3))
        for i in range(0, M, 30_000):
            d = dy[i : i + 30_000].double()
            t = d if act == "none" else d * ref.slope(act, pre[i : i + 30_000].double())
            want += t.sum(0)
            size += t.abs().sum(0)
            off += d.abs().sum(0)
        # float32 sums of 16, 8, up to 147 and 16 terms one after the other; the slope's own arithmetic is good to 2^-19
        assert ((db.double() - want).abs() <= ref.BF16 * want.abs() + (16 + 8 + 147 + 16) * ref.F32 * size + (2.0 ** -19 * off if act != "none" else 0)).all(), act
