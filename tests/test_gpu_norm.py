"""GPU: the root-mean-square norm, its gradients, and rows in 8-bit integers, against float64 (bounds: _norm_ref.py)."""
import pytest
import torch

import _block_ref as ref
import _norm_ref as nr

pytestmark = pytest.mark.gpu

EPS = 1e-6


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, *shape, dtype=torch.bfloat16):
    """Channels and rows of different sizes."""
    x = torch.randn(*shape, generator=g, device="cuda") * torch.exp2(2 * torch.randn(shape[-1], generator=g, device="cuda"))
    return (x * torch.exp2(3 * torch.randn(*shape[:-1], 1, generator=g, device="cuda"))).to(dtype)


def _weight(g, cols, dtype):
    return (1 + 0.5 * torch.randn(cols, generator=g, device="cuda")).to(dtype)


SIZES = [(1, 8), (1, 5120), (3, 16), (2, 24), (5, 40), (7, 64), (130, 72), (1000, 128), (33, 136), (9, 256), (70, 264), (20, 504), (65, 512), (66, 520), (17, 1000), (12, 1024), (40, 1032), (31, 1536),
         (8, 2048), (5, 2056), (3, 4008), (300, 5120), (6, 8192), (4, 13824), (2, 20480), (3, 32760), (2, 32768), (70001, 64), (2049, 1536), (1500, 1000), (1100, 5120), (1030, 264), (1024, 10008)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_forward(rows, cols, dtype):
    import paper_2605_28691_amd as sk

    g = _gen(rows * 7 + cols)
    x, res, w = _rows(g, rows, cols, dtype=dtype), _rows(g, rows, cols, dtype=dtype), _weight(g, cols, dtype)
    for weight in (w, None):
        y, _ = nr.norm(x, weight, None, EPS)
        nr.close(sk.skiparse_rmsnorm_fwd(x, weight), y, nr.norm_bound(y, dtype), "y")
        y, h = nr.norm(x, weight, res, EPS)
        out, total = sk.skiparse_rmsnorm_fwd(x, weight, res)
        nr.close(out, y, nr.norm_bound(y, dtype), "y of the sum")
        assert torch.equal(total, (x.float() + res.float()).to(dtype))
        again, _ = sk.skiparse_rmsnorm_fwd(x, weight, res)
        assert torch.equal(out, again)
    # in 8-bit integers: the nearest code of y 127 / max |y|, but for what float32 loses on the way
    y, _ = nr.norm(x, w, res, EPS)
    q, total8 = sk.skiparse_rmsnorm_fwd(x, w, res, quantize=True)
    assert torch.equal(total8, total)
    top = y.abs().amax(-1, keepdim=True)
    nr.close(q.scales, top[..., 0] / 127, nr.ROW * top[..., 0] / 127, "scales")
    nr.close(q.codes, y / top * 127, 0.5 + 127 * nr.ROW, "codes")
    assert q.codes.abs().amax(-1).eq(127).all()
    # what is written in place
    a, b = x.clone(), res.clone()
    got, t = sk.skiparse_rmsnorm_fwd(a, w, b, total=b)
    assert t is b and torch.equal(b, total) and torch.equal(got, sk.skiparse_rmsnorm_fwd(x, w, res)[0])
    got, t = sk.skiparse_rmsnorm_fwd(a, w, res, total=a)
    assert t is a and torch.equal(a, total)
    a = x.clone()
    assert torch.equal(sk.skiparse_rmsnorm_fwd(a, w, out=a), sk.skiparse_rmsnorm_fwd(x, w))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_quantized_rows(rows, cols, dtype):
    """Bit for bit: every decision of the definition is in float32."""
    import paper_2605_28691_amd as sk

    x = _rows(_gen(rows + cols), rows, cols, dtype=dtype)
    x[rows // 2, : cols // 2] = 0
    x[rows // 3] = 0
    got = sk.skiparse_quantize_int8(x)
    codes, scales = nr.codes(x.float())
    assert torch.equal(got.codes.cpu(), codes) and torch.equal(got.scales.cpu(), scales)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_gradients(rows, cols, dtype):
    import paper_2605_28691_amd as sk

    g = _gen(3 * rows + cols)
    h, w = _rows(g, rows, cols, dtype=dtype), _weight(g, cols, dtype)
    dy, add = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    for weight, a in ((w, add), (w, None), (None, add), (None, None)):
        ex, ew, bx, bw = nr.norm_grads(dy, h, weight, a, EPS)
        dx, dw = sk.skiparse_rmsnorm_bwd(dy, h, weight, dx_add=a)
        nr.close(dx, ex, nr.ROUND[dtype] * ex.abs() + bx, "dx")
        nr.close(dw, ew, nr.ROUND[dtype] * ew.abs() + bw, "dw")
        again = sk.skiparse_rmsnorm_bwd(dy, h, weight, dx_add=a)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    # one alone, and into what is added
    assert torch.equal(sk.skiparse_rmsnorm_bwd(dy, h, w, dx_add=add, need_dw=False)[0], sk.skiparse_rmsnorm_bwd(dy, h, w, dx_add=add)[0])
    assert torch.equal(sk.skiparse_rmsnorm_bwd(dy, h, w, need_dx=False)[1], sk.skiparse_rmsnorm_bwd(dy, h, w, dx_add=add)[1])
    want, into = sk.skiparse_rmsnorm_bwd(dy, h, w, dx_add=add)[0], add.clone()
    assert sk.skiparse_rmsnorm_bwd(dy, h, w, dx_add=into, dx=into)[0] is into and torch.equal(into, want)


def test_gradients_against_differences():
    """Of the forward call itself, in float32: (f(h + d) - f(h - d)) / 2 d with d = 2^-7.  A result may be off by ROW = 2^-18 of its size (_norm_ref.py), two of them over 2 d make 2^-11 of
    the sum of |dy y|; what the third derivative, at most 15 |dy w|, adds is d^2 / 6 of it, below 2^-12.  Twice that is allowed.  In the weights the result is linear."""
    import paper_2605_28691_amd as sk

    g = _gen(5)
    h, w = torch.randn(4, 40, generator=g, device="cuda"), _weight(g, 40, torch.float32)
    dy = torch.randn(4, 40, generator=g, device="cuda")
    dx, dw = sk.skiparse_rmsnorm_bwd(dy, h, w)
    y = nr.norm(h, w, None, EPS)[0]
    loss = lambda h, w: (sk.skiparse_rmsnorm_fwd(h, w).double() * dy.double()).sum(-1)  # noqa: E731
    for c in range(40):
        d = torch.zeros(4, 40, device="cuda")
        d[:, c] = 2.0 ** -7
        num = (loss(h + d, w) - loss(h - d, w)) / ((h + d).double() - (h - d).double())[:, c]
        size = (dy.double().abs() * (y.abs() + w.double().abs())).sum(-1)
        assert ((num - dx[:, c].double()).abs() <= 2.0 ** -10 * size).all(), c
        e = torch.zeros(40, device="cuda")
        e[c] = 2.0 ** -7
        num = (loss(h, w + e) - loss(h, w - e)).sum() / ((w + e).double() - (w - e).double())[c]
        assert (num - dw[c].double()).abs() <= 2.0 ** -10 * (dy.double() * y).abs().sum(), c


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, cols", [(700_000, 64), (300_001, 264), (70_003, 1000), (45_001, 1536), (13_002, 5120), (5_003, 13824), (2_100, 32768)])
def test_a_row_depends_on_nothing_but_itself(rows, cols, dtype):
    """Whichever lanes have it, and whether the tensors go past the caches (256 MB moved and more) or not: its bits are those of a call of few rows."""
    import paper_2605_28691_amd as sk

    g = _gen(cols)
    x, res, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(3))
    w = _weight(g, cols, dtype)
    out, total = sk.skiparse_rmsnorm_fwd(x, w, res)
    q, _ = sk.skiparse_rmsnorm_fwd(x, w, res, quantize=True)
    z = sk.skiparse_quantize_int8(x)
    dx, dw = sk.skiparse_rmsnorm_bwd(dy, total, w, dx_add=res)
    for first, n in ((0, 1), (rows - 1, 1), (rows // 3, 5), (rows // 2, 300), (rows - 1025, 1025)):
        part = slice(first, first + n)
        xs, rs, ds = x[part].clone(), res[part].clone(), dy[part].clone()
        o, t = sk.skiparse_rmsnorm_fwd(xs, w, rs)
        assert torch.equal(o, out[part]) and torch.equal(t, total[part]), n
        p, _ = sk.skiparse_rmsnorm_fwd(xs, w, rs, quantize=True)
        assert torch.equal(p.codes, q.codes[part]) and torch.equal(p.scales, q.scales[part]), n
        p = sk.skiparse_quantize_int8(xs)
        assert torch.equal(p.codes, z.codes[part]) and torch.equal(p.scales, z.scales[part]), n
        assert torch.equal(sk.skiparse_rmsnorm_bwd(ds, t, w, dx_add=rs)[0], dx[part]), n
    # and in place
    t = res.clone()
    assert torch.equal(sk.skiparse_rmsnorm_fwd(x, w, t, total=t)[0], out) and torch.equal(t, total)
    t = res.clone()
    assert torch.equal(sk.skiparse_rmsnorm_bwd(dy, total, w, dx_add=t, dx=t)[0], dx)
    _, ew, _, bw = nr.norm_grads(dy, total, w, None, EPS)
    nr.close(dw, ew, nr.ROUND[dtype] * ew.abs() + bw, "dw")


@pytest.mark.parametrize("rows, cols", [(1_400_003, 64), (3_800_001, 24), (360_001, 256), (11_000_001, 8)])
def test_two_rows_of_a_lane(rows, cols):
    """bf16 without a residual, 256 MB moved and more: the lanes of a short row have two, the last ones one or none."""
    import paper_2605_28691_amd as sk

    g = _gen(cols)
    x, w = torch.randn(rows, cols, generator=g, device="cuda").bfloat16(), _weight(g, cols, torch.bfloat16)
    out, q, z = sk.skiparse_rmsnorm_fwd(x, w), sk.skiparse_rmsnorm_fwd(x, w, quantize=True), sk.skiparse_quantize_int8(x)
    into = x.clone()
    assert torch.equal(sk.skiparse_rmsnorm_fwd(into, w, out=into), out)
    for part in (slice(0, 300_000), slice(rows // 2, rows // 2 + 77_777), slice(rows - 100_001, rows), slice(rows - 1, rows)):
        xs = x[part].clone()
        assert torch.equal(sk.skiparse_rmsnorm_fwd(xs, w), out[part])
        for p, whole in ((sk.skiparse_rmsnorm_fwd(xs, w, quantize=True), q), (sk.skiparse_quantize_int8(xs), z)):
            assert torch.equal(p.codes, whole.codes[part]) and torch.equal(p.scales, whole.scales[part])
    # rows that move: B = 2 grids of 4 x H x 2, H as long as it takes
    H = rows // 16 // 4 * 4
    n = 2 * 4 * H * 2
    place = dict(T=4, H=H, W=2, s=2, pattern="token")
    v = x[:n].view(2, n // 2, cols)
    moved = sk.skiparse_rmsnorm_fwd(v, w, order="to_sparse", **place)
    assert torch.equal(moved, ref.moved(out[:n].view(2, n // 2, cols), "to_sparse", (2, 4, H, 2), 2, "token"))
    assert torch.equal(sk.skiparse_rmsnorm_fwd(moved, order="to_original", **place), sk.skiparse_rmsnorm_fwd(sk.skiparse_rmsnorm_fwd(v, w).contiguous()))


GRIDS = [(1, (2, 4, 8), 2, "token"), (2, (1, 8, 4), 2, "group"), (3, (1, 9, 18), 3, "token"), (2, (2, 9, 9), 3, "group"), (1, (3, 16, 16), 4, "group"), (1, (21, 30, 52), 2, "token")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["to_sparse", "to_original"])
@pytest.mark.parametrize("B, grid, s, pattern", GRIDS)
@pytest.mark.parametrize("cols", [40, 264, 1536])
def test_rows_that_move(B, grid, s, pattern, order, cols, dtype):
    import paper_2605_28691_amd as sk

    T, H, W = grid
    n = T * H * W
    lead = (B, n) if order == "to_sparse" else (s * s * B, n // (s * s))
    g = _gen(n + cols)
    x, res, w = _rows(g, *lead, cols, dtype=dtype), _rows(g, *lead, cols, dtype=dtype), _weight(g, cols, dtype)
    at, to = dict(order=order, T=T, H=H, W=W, s=s, pattern=pattern), ((B, *grid), s, pattern)
    out, total = sk.skiparse_rmsnorm_fwd(x, w, res, **at)
    plain, plain_total = sk.skiparse_rmsnorm_fwd(x, w, res)
    assert torch.equal(total, plain_total) and torch.equal(out, ref.moved(plain, order, *to))
    q, _ = sk.skiparse_rmsnorm_fwd(x, w, res, quantize=True, **at)
    p, _ = sk.skiparse_rmsnorm_fwd(x, w, res, quantize=True)
    assert torch.equal(q.codes, ref.moved(p.codes, order, *to)) and torch.equal(q.scales, ref.moved(p.scales, order, *to))
    q, p = sk.skiparse_quantize_int8(x, **at), sk.skiparse_quantize_int8(x)
    assert torch.equal(q.codes, ref.moved(p.codes, order, *to)) and torch.equal(q.scales, ref.moved(p.scales, order, *to))
    add = _rows(g, *lead, cols, dtype=dtype)
    dy = torch.randn(*out.shape, generator=g, device="cuda").to(dtype)
    dx, dw = sk.skiparse_rmsnorm_bwd(dy, total, w, dx_add=add, **at)
    ex, ew = sk.skiparse_rmsnorm_bwd(ref.moved(dy, nr.INVS[order], *to).contiguous(), total, w, dx_add=add)
    assert torch.equal(dx, ex) and torch.equal(dw, ew)


@pytest.mark.parametrize("cols", [40, 1536, 5120])
def test_rows_far_from_one(cols):
    """Squares that leave float32's range, on either side, and rows of zeros."""
    import paper_2605_28691_amd as sk

    g = _gen(cols)
    base = torch.randn(9, cols, generator=g, device="cuda")
    size = torch.tensor([1.0, 2.0 ** 70, 2.0 ** 120, 2.0 ** -40, 2.0 ** -70, 2.0 ** -100, 0.0, 2.0 ** 60, 1.0], device="cuda")[:, None]
    x = base * size
    add = torch.zeros_like(x)
    for eps in (1e-6, 1.2e-38):
        y, _ = nr.norm(x, None, None, eps)
        # where the squares are beyond float32's range 1 / sqrt() may be a denormal number: half of 2^-149 over 2^-123, 2^-27 of it, is no more than a rounding more
        nr.close(sk.skiparse_rmsnorm_fwd(x, eps=eps), y, nr.norm_bound(y, torch.float32), ("y", eps))
        q = sk.skiparse_rmsnorm_fwd(x, eps=eps, quantize=True)
        top = y.abs().amax(-1)
        normal = (x.abs().amax(-1) >= 2.0 ** -118)
        nr.close(q.scales[normal], top[normal] / 127, nr.ROW * top[normal] / 127, "scales")
        nr.close(q.codes[normal], (y / top[:, None] * 127)[normal], 0.5 + 127 * nr.ROW, "codes")
        assert q.scales[6] == 1 and not q.codes[6].any()
        dy = torch.randn(9, cols, generator=g, device="cuda")
        for a in (None, add):
            dx, dw = sk.skiparse_rmsnorm_bwd(dy, x, None, dx_add=a, eps=eps)
            ex, ew, bx, bw = nr.norm_grads(dy, x, None, a, eps)
            nr.close(dx, ex, 2 * nr.F32 * ex.abs() + bx + 2.0 ** -149, "dx")
            nr.close(dw, ew, nr.F32 * ew.abs() + bw, "dw")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [40, 1000, 1536, 20480])
def test_gradients_far_from_one(cols, dtype):
    """Products of dy and h beyond float32's range, whose gradients are in it; rows between them are as they are alone."""
    import paper_2605_28691_amd as sk

    g = _gen(cols)
    h, dy = (torch.randn(9, cols, generator=g, device="cuda") for _ in range(2))
    sizes = [(0, 0), (62, 100), (50, 120), (90, 60), (-70, 20), (100, 110), (20, 122), (0, 0), (61, -100)]
    h = (h * torch.tensor([2.0 ** a for a, _ in sizes], device="cuda")[:, None]).to(dtype)
    dy = (dy * torch.tensor([2.0 ** b for _, b in sizes], device="cuda")[:, None]).to(dtype)
    w = _weight(g, cols, dtype)
    dx, dw = sk.skiparse_rmsnorm_bwd(dy, h, w)
    ex, ew, bx, bw = nr.norm_grads(dy, h, w, None, EPS)
    nr.close(dx, ex, (nr.ROUND[dtype] + 2 * nr.F32) * ex.abs() + bx + 2.0 ** (-149 if dtype is torch.float32 else -134), "dx")
    nr.close(dw, ew, nr.ROUND[dtype] * ew.abs() + bw, "dw")
    for i in (0, 3, 7):
        assert torch.equal(dx[i:i + 1], sk.skiparse_rmsnorm_bwd(dy[i:i + 1].clone(), h[i:i + 1].clone(), w)[0]), i


@pytest.mark.parametrize("cols", [24, 520, 5120])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_are_not_finite(cols, dtype):
    """They spoil themselves and no other row."""
    import paper_2605_28691_amd as sk

    g = _gen(cols)
    x, w = _rows(g, 12, cols, dtype=dtype), _weight(g, cols, dtype)
    bad = x.clone()
    bad[3, cols - 1], bad[5, 0], bad[9, cols // 2] = float("nan"), float("inf"), -float("inf")
    keep = [i for i in range(12) if i not in (3, 5, 9)]
    y, z = sk.skiparse_rmsnorm_fwd(x, w), sk.skiparse_rmsnorm_fwd(bad, w)
    assert torch.equal(y[keep], z[keep]) and z[3].isnan().all() and z[5, 0].isnan() and z[9, cols // 2].isnan()
    for make in (lambda t: sk.skiparse_quantize_int8(t), lambda t: sk.skiparse_rmsnorm_fwd(t, w, quantize=True)):
        p, q = make(x), make(bad)
        assert torch.equal(p.codes[keep], q.codes[keep]) and torch.equal(p.scales[keep], q.scales[keep])
        assert q.scales[[3, 5, 9]].isnan().all() and not q.codes[[3, 5, 9]].any()
    dy = torch.randn(12, cols, generator=g, device="cuda").to(dtype)
    assert torch.equal(sk.skiparse_rmsnorm_bwd(dy, x, w)[0][keep], sk.skiparse_rmsnorm_bwd(dy, bad, w)[0][keep])
    # a weight that is none spoils its channel of y, and in 8 bits every row
    w[cols // 3] = float("nan")
    z = sk.skiparse_rmsnorm_fwd(x, w)
    assert z[:, cols // 3].isnan().all() and int(z.isnan().sum()) == 12
    assert sk.skiparse_rmsnorm_fwd(x, w, quantize=True).scales.isnan().all()


def test_smallest_scales():
    """Rows below 2^-118 share its scale; codes at the border of two."""
    import paper_2605_28691_amd as sk

    x = torch.zeros(6, 16, device="cuda")
    x[0, 0], x[1, 1], x[2, 2] = 2.0 ** -118, 2.0 ** -120, 2.0 ** -149
    x[3, :4] = torch.tensor([127.0, 0.5, 1.5, -2.5], device="cuda")   # ties go to the even code
    x[4, :3] = torch.tensor([3.4e38, -3.4e38, 1e38], device="cuda")
    x[5, 0] = -1.0
    q = sk.skiparse_quantize_int8(x)
    codes, scales = nr.codes(x)
    assert torch.equal(q.codes.cpu(), codes) and torch.equal(q.scales.cpu(), scales)
    assert q.codes[3, :4].tolist() == [127, 0, 2, -2] and q.codes[5, 0] == -127 and q.scales[0] == q.scales[1] == q.scales[2]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_beyond_32_bit_offsets(dtype):
    import paper_2605_28691_amd as sk

    cols = 32768
    rows = (1 << 32) // cols + 37
    x = torch.empty(rows, cols, dtype=dtype, device="cuda")
    g = _gen(1)
    some = _rows(g, 64, cols, dtype=dtype)
    for i in range(0, rows, 64):
        x[i:i + 64] = some[: rows - i]
    w = _weight(g, cols, dtype)
    last = slice((rows - 1) // 64 * 64, rows)
    n = last.stop - last.start
    y = sk.skiparse_rmsnorm_fwd(x, w)
    assert torch.equal(y[last], sk.skiparse_rmsnorm_fwd(some[:n].contiguous(), w)) and torch.equal(y[:64], y[64:128])
    q, p = sk.skiparse_quantize_int8(x), sk.skiparse_quantize_int8(some)
    assert torch.equal(q.codes[last], p.codes[:n]) and torch.equal(q.scales[last], p.scales[:n])
    del q
    dx, _ = sk.skiparse_rmsnorm_bwd(y, x, w)
    assert torch.equal(dx[last], sk.skiparse_rmsnorm_bwd(y[:n].contiguous(), x[:n].contiguous(), w, need_dw=False)[0])


def test_what_lies_round_the_results():
    """Nothing is written before or behind a result, its scales or the workspace."""
    import paper_2605_28691_amd as sk

    for rows, cols in ((1, 8), (7, 40), (33, 1000), (5, 5120), (3, 32768)):
        g = _gen(cols)
        x, res, w = _rows(g, rows, cols), _rows(g, rows, cols), _weight(g, cols, torch.bfloat16)

        def room(shape, dtype):
            n = int(torch.tensor(shape).prod())
            pad = 256
            buf = torch.full((n + 2 * pad,), 77, dtype=dtype, device="cuda")
            return buf, buf[pad:pad + n].view(shape), pad

        def untouched(buf, pad):
            return bool((buf[:pad] == 77).all() and (buf[-pad:] == 77).all())

        rooms = [room((rows, cols), torch.bfloat16) for _ in range(3)] + [room((rows, cols), torch.int8), room((rows,), torch.float32), room((cols,), torch.bfloat16)]
        out, total, dx, codes, scales, dw = (r[1] for r in rooms)
        sk.skiparse_rmsnorm_fwd(x, w, res, out=out, total=total)
        sk.skiparse_rmsnorm_fwd(x, w, res, total=total, quantize=True, out=sk.Quantized(codes, scales))
        sk.skiparse_quantize_int8(x, out=sk.Quantized(codes, scales))
        size = sk.skiparse_rmsnorm_bwd_workspace_bytes(rows, cols)
        space = room((size,), torch.uint8)
        sk.skiparse_rmsnorm_bwd(out, total, w, dx=dx, dw=dw, workspace=space[1])
        for buf, _, pad in rooms + [space]:
            assert untouched(buf, pad), (rows, cols)


@pytest.mark.parametrize("rows, cols", [(1, 5120), (390, 1536), (2049, 264), (30, 20480), (513, 64)])
def test_two_graphs_and_two_streams(rows, cols):
    """A training step's calls in two captured graphs that run at once, each with a workspace of its own; replays with other inputs in the same places."""
    import paper_2605_28691_amd as sk

    g = _gen(rows)
    sets = []
    for _ in range(2):
        x, res, dy = (torch.randn(rows, cols, generator=g, device="cuda").bfloat16() for _ in range(3))
        w = _weight(g, cols, torch.bfloat16)
        out, total = sk.skiparse_rmsnorm_fwd(x, w, res)
        q = sk.skiparse_quantize_int8(out)
        dx, dw = sk.skiparse_rmsnorm_bwd(dy, total, w, dx_add=dy)
        sets.append((x, res, dy, w, out, total, q, dx, dw, torch.empty(sk.skiparse_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")))

    def step(x, res, dy, w, out, total, q, dx, dw, ws):
        sk.skiparse_rmsnorm_fwd(x, w, res, out=out, total=total)
        sk.skiparse_quantize_int8(out, out=q)
        sk.skiparse_rmsnorm_bwd(dy, total, w, dx_add=dy, dx=dx, dw=dw, workspace=ws)

    graphs = []
    for s in sets:
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(*s)
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in sets]
    for turn in range(4):
        for s in sets:
            for t in s[:3]:
                t.copy_(t.roll(1, -1) if turn % 2 else -t.flip(-1))
        want = []
        for s in sets:
            fresh = [*s[:4], *(torch.empty_like(t) for t in s[4:6]), sk.Quantized(*(torch.empty_like(t) for t in s[6])), *(torch.empty_like(t) for t in s[7:])]
            step(*fresh)
            want.append(fresh)
            for t in (*s[4:6], *s[6], *s[7:]):
                t.zero_()
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for s, f in zip(sets, want):
            for a, b in zip((*s[4:6], *s[6], *s[7:9]), (*f[4:6], *f[6], *f[7:9])):
                assert torch.equal(a, b), turn


def test_tensors_that_are_refused():
    """On the CPU, or not in one piece, or of another type."""
    import paper_2605_28691_amd as sk

    x, w = torch.randn(4, 64).bfloat16(), torch.randn(8, 64).bfloat16().cuda()
    d, qw = x.cuda(), sk.skiparse_quantize_int8(w)
    qx = sk.skiparse_quantize_int8(d)
    host = sk.Quantized(qx.codes.cpu(), qx.scales.cpu())
    apart = torch.randn(4, 128, device="cuda").bfloat16()[:, ::2]
    for call in (lambda: sk.skiparse_rmsnorm_fwd(x), lambda: sk.skiparse_rmsnorm_fwd(apart), lambda: sk.skiparse_rmsnorm_fwd(d, x[0]), lambda: sk.skiparse_rmsnorm_fwd(d, None, x),
                 lambda: sk.skiparse_rmsnorm_bwd(d, apart), lambda: sk.skiparse_rmsnorm_bwd(x, d), lambda: sk.skiparse_quantize_int8(apart), lambda: sk.skiparse_quantize_int8(x),
                 lambda: sk.skiparse_linear_fwd_int8(host, qw), lambda: sk.skiparse_linear_fwd_int8(qx, sk.Quantized(qw.codes, qw.scales.cpu())),
                 lambda: sk.skiparse_linear_fwd_int8(sk.Quantized(qx.codes, qx.scales.cpu()), qw), lambda: sk.skiparse_linear_fwd_int8(qx, qw, torch.zeros(8).bfloat16())):
        with pytest.raises(ValueError, match="contiguous device tensor"):
            call()
    with pytest.raises(KeyError):
        sk.skiparse_rmsnorm_fwd(d.half())
    with pytest.raises(sk.SkiparseError):
        sk.skiparse_rmsnorm_fwd(d, eps=0.0)
