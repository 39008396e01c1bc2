"""GPU: rotary positions against float64, table and rotation, every layout, order and type."""
import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scaling, factor, trained", [("none", 1.0, 0), ("linear", 4.0, 0), ("ntk", (1.0, 2.0, 8.0), 0), ("yarn", (1.0, 2.5, 16.0), (21, 48, 4096))])
@pytest.mark.parametrize("lengths, axes", [((1, 1, 1), (0, 0, 2)), ((21, 48, 80), (44, 42, 42)), ((5, 1, 131072), (6, 0, 128)), ((3, 7, 9), (2, 2, 4)), ((1, 700, 1), (0, 512, 0))])
def test_table(lengths, axes, scaling, factor, trained):
    import paper_2605_28691_amd as sk

    got = sk.skiparse_rope_table(lengths, axes, theta=500.0, scaling=scaling, factor=factor, trained=trained, attention=1.25)
    assert got.lengths == lengths and got.axes == axes
    as3 = lambda v: tuple(v) if isinstance(v, tuple) else (v,) * 3  # noqa: E731
    want = ref.table(lengths, axes, 500.0, scaling, as3(factor), as3(trained), 1.25)
    # the angle, at most an eighth of a turn after the reduction, is rounded once (2^-25 pi / 2), then the function (4 ulp) and the factor
    assert (got.data.double().cpu() - want).abs().max() <= 1.25 * (2.0 ** -25 * 1.6 + 6 * ref.F32)


SHAPES = [  # B, heads, D, (T, H, W), s, axes, at
    (1, 1, 8, (1, 1, 1), 1, (0, 0, 2), (0, 0, 0)),
    (1, 12, 128, (1, 1, 1), 1, (0, 0, 128), (0, 0, 1000)),
    (2, 3, 64, (2, 4, 8), 2, (16, 20, 28), (3, 0, 5)),
    (1, 40, 128, (2, 8, 8), 2, (44, 42, 42), (0, 0, 0)),
    (1, 2, 96, (3, 4, 4), 2, (6, 10, 14), (0, 1, 0)),    # five heads would fit a wavefront, four lanes are over; halves begin in the middle of a chunk
    (3, 5, 128, (1, 9, 18), 3, (0, 22, 10), (0, 0, 0)),   # a part of the head
    (1, 17, 40, (1, 4, 4), 1, (2, 2, 2), (0, 0, 0)),
    (1, 2, 512, (1, 2, 3), 1, (100, 100, 312), (0, 0, 0)),
    (1, 2, 64, (1, 1, 70001), 1, (0, 0, 64), (0, 0, 61000)),  # a line longer than the index maps' divisions allow: rows that stay need none
    (1, 9, 256, (1, 1, 37), 1, (0, 0, 250), (0, 0, 0)),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotation(shape, layout, dtype):
    import paper_2605_28691_amd as sk

    B, heads, D, (T, H, W), s, axes, at = shape
    lengths = (T + at[0] + 1, H + at[1], W + at[2] + 2)
    table = sk.skiparse_rope_table(lengths, axes, attention=0.75)
    t64 = table.data.double().cpu()
    g = torch.Generator().manual_seed(B * heads + D)
    grid = (B, T, H, W)
    q, k = (torch.randn(B, T * H * W, heads, D, generator=g).to(dtype) for _ in range(2))
    rounding = ref.BF16 if dtype == torch.bfloat16 else ref.F32
    R = sum(axes)
    for inverse in (False, True):
        want = [ref.rope(x.double(), t64, lengths, axes, grid, at, layout, -1.0 if inverse else 1.0) for x in (q, k)]
        top = [(x.double().abs().amax(-1, keepdim=True)) for x in (q, k)]
        orders = ["same"] + (["to_sparse", "to_original", "stay_sparse"] if s > 1 else [])
        patterns = ["token"] + (["group"] if s > 1 and H % (s * s) == 0 and W % (s * s) == 0 else [])
        for pattern in patterns:
            def to(x, name):
                return ref.moved(x, name, grid, s, pattern)

            for order in orders:
                ins = [x if order in ("same", "to_sparse") else to(x, "to_sparse") for x in (q, k)]
                outs = [x if order in ("same", "to_original") else to(x, "to_sparse") for x in want]
                big = [x if order in ("same", "to_original") else to(x, "to_sparse") for x in top]
                args = (table, T, H, W, s, pattern, order, layout, inverse, at)
                dev = [x.contiguous().cuda() for x in ins]
                got = sk.skiparse_rope(*dev, *args)
                for y, w_, x, m in zip(got, outs, dev, big):
                    y = y.double().cpu()
                    # one rounding of the result; products and their sum in float32
                    assert ((y - w_).abs() <= rounding * w_.abs() + 4 * ref.F32 * 2 * m).all(), (order, pattern, inverse)
                    if R < D:  # copied bit for bit
                        assert torch.equal(y[..., R:], (w_[..., R:]))
                alone, none = sk.skiparse_rope(dev[0], None, *args)
                assert none is None and torch.equal(alone, got[0])
                if order in ("same", "stay_sparse"):
                    again = sk.skiparse_rope(dev[0], dev[1], *args, q_out=dev[0], k_out=dev[1])
                    assert again[0] is dev[0] and all(torch.equal(x, y) for x, y in zip(again, got))


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_values_that_are_not_finite_stay_in_their_pair(layout):
    import paper_2605_28691_amd as sk

    q = torch.randn(1, 6, 2, 64, device="cuda").to(torch.bfloat16)
    table = sk.skiparse_rope_table((1, 1, 6), (0, 0, 32))
    clean, _ = sk.skiparse_rope(q, None, table, 1, 1, 6, layout=layout)
    bad = q.clone()
    bad[0, 2, 1, 5] = float("nan")
    bad[0, 3, 0, 40] = float("inf")  # behind the turned channels
    got, _ = sk.skiparse_rope(bad, None, table, 1, 1, 6, layout=layout)
    pair = {"interleaved": (4, 5), "half": (5, 21)}[layout]
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[0, 2, 1, list(pair)] = True
    assert torch.equal(got.isnan(), hit) and got[0, 3, 0, 40] == float("inf")
    hit[0, 3, 0, 40] = True
    assert torch.equal(got[~hit], clean[~hit])


def test_gradient_by_differences():
    """The derivative of <g, rope(x)> along d, by float64 differences of the plain form, is <rope_inverse(g), d>."""
    import paper_2605_28691_amd as sk

    T, H, W, axes, gen = 2, 4, 4, (4, 8, 12), torch.Generator().manual_seed(5)
    table = sk.skiparse_rope_table((T, H, W), axes)
    t64 = table.data.double().cpu()
    x, g, d = (torch.randn(1, T * H * W, 3, 32, generator=gen).float() for _ in range(3))
    f = lambda y: (g.double() * ref.rope(y, t64, (T, H, W), axes, (1, T, H, W), (0, 0, 0), "half", 1.0)).sum()  # noqa: E731
    h = 1e-3
    slope = (f(x.double() + h * d.double()) - f(x.double() - h * d.double())) / (2 * h)
    dx, _ = sk.skiparse_rope(g.cuda(), None, table, T, H, W, layout="half", inverse=True)
    size = (g.double().abs() * d.double().abs()).sum() * 2
    assert abs(float((dx.double().cpu() * d.double()).sum() - slope)) <= float(size) * 8 * ref.F32 + 1e-9 * float(size)


def test_back_and_forth_through_the_sparse_layout():
    import paper_2605_28691_amd as sk

    T, H, W, s, axes = 3, 8, 12, 2, (20, 22, 22)
    table = sk.skiparse_rope_table((T, H, W), axes)
    q, k = (torch.randn(2, T * H * W, 4, 64, device="cuda") for _ in range(2))
    qs, ks = sk.skiparse_rope(q, k, table, T, H, W, s, "token", "to_sparse")
    q2, k2 = sk.skiparse_rope(qs, ks, table, T, H, W, s, "token", "to_original", inverse=True)
    for a, b in ((q, q2), (k, k2)):
        assert (a - b).abs().max() <= a.abs().max() * 16 * ref.F32
