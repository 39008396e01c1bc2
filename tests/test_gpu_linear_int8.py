"""GPU: products of 8-bit integers with a scale for each token and channel, against float64 (bounds: _norm_ref.py)."""
import pytest
import torch

import _block_ref as ref
import _norm_ref as nr

pytestmark = pytest.mark.gpu


def _inputs(M, K, N, seed, lead=None):
    import paper_2605_28691_amd as sk

    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lead = lead or (M,)
    x = torch.randint(-127, 128, (*lead, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    xs, ws = torch.exp2(r(*lead)) / 73, torch.exp2(r(N)) / 73 * K ** -0.5
    return sk.Quantized(x, xs), sk.Quantized(w, ws), (r(N) * 0.5).bfloat16(), r(*lead, N).bfloat16()


def _check(x, w, bias, residual, act, got):
    y, slack = nr.linear(x.codes, x.scales, w.codes, w.scales, bias, residual, act)
    nr.close(got, y, nr.BF16 * y.abs() + slack, (tuple(got.shape), x.codes.shape[-1], act))


SIZES = [(1, 16, 8), (1, 5120, 40), (1, 1536, 4104), (2, 64, 128), (3, 80, 136), (5, 5120, 520), (16, 1008, 96), (17, 256, 72), (31, 528, 4104), (32, 5120, 264), (33, 144, 520), (64, 64, 64), (65, 208, 264),
         (100, 1536, 128), (127, 128, 8), (128, 128, 128), (129, 32, 384), (257, 272, 256), (390, 1008, 1000), (600, 2064, 232), (1025, 80, 520), (6566, 4112, 536), (528, 8016, 3616), (70001, 64, 72),
         (512, 256, 512), (1, 131056, 8), (40, 131056, 72), (923, 64, 4464), (6764, 4800, 80), (3650, 1920, 1248), (636, 5696, 4792), (7004, 64, 1392), (3726, 5696, 688),
         (1124, 4592, 3632), (5616, 4992, 728), (48, 1408, 88), (9, 64, 264), (20, 528, 4104), (3, 4112, 4104), (5535, 5696, 72), (1187, 7488, 3488), (10505, 288, 1200), (3046, 624, 4312), (48, 1568, 80)]


@pytest.mark.parametrize("act", ["none", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M, K, N", SIZES)
def test_forward(M, K, N, act):
    import paper_2605_28691_amd as sk

    x, w, bias, residual = _inputs(M, K, N, M + K + N)
    for b, r in ((bias, residual), (None, None), (bias, None), (None, residual)):
        _check(x, w, b, r, act, sk.skiparse_linear_fwd_int8(x, w, b, r, act=act))
    got = sk.skiparse_linear_fwd_int8(x, w, bias, residual, act=act)
    inplace = residual.clone()
    assert sk.skiparse_linear_fwd_int8(x, w, bias, inplace, act=act, out=inplace) is inplace and torch.equal(got, inplace)


@pytest.mark.parametrize("K, N", [(64, 72), (1536, 264), (5120, 5120), (8016, 520)])
def test_a_row_depends_on_nothing_but_itself(K, N):
    """The sums are whole numbers: however many rows share the call, and whatever kernel takes them, a row's bits are the same."""
    import paper_2605_28691_amd as sk

    x, w, bias, residual = _inputs(700, K, N, K + N)
    for act, b, r in (("gelu_tanh", bias, residual), ("none", None, None), ("silu", bias, None)):
        whole = sk.skiparse_linear_fwd_int8(x, w, b, r, act=act)
        for first, n in ((0, 1), (699, 1), (3, 2), (10, 5), (100, 16), (200, 17), (33, 32), (300, 33), (400, 130), (0, 512)):
            part = sk.Quantized(x.codes[first:first + n].contiguous(), x.scales[first:first + n].contiguous().clone())
            got = sk.skiparse_linear_fwd_int8(part, w, b, None if r is None else r[first:first + n].contiguous(), act=act)
            assert torch.equal(got, whole[first:first + n]), (act, first, n)


@pytest.mark.parametrize("M", [1, 4, 20, 300])
@pytest.mark.parametrize("K", [16, 1008, 131056])
def test_largest_sums(M, K):
    """All codes -128, or 127 against -128: nothing overflows, and no rounding happens before the scales."""
    import paper_2605_28691_amd as sk

    for a, b in ((-128, -128), (127, -128), (-128, 127), (127, 127)):
        x = sk.Quantized(torch.full((M, K), a, dtype=torch.int8, device="cuda"), torch.full((M,), 2.0 ** -20, device="cuda"))
        w = sk.Quantized(torch.full((24, K), b, dtype=torch.int8, device="cuda"), torch.full((24,), 0.5, device="cuda"))
        want = (torch.tensor(float(a * b * K), dtype=torch.float32) * 2.0 ** -21).bfloat16()
        got = sk.skiparse_linear_fwd_int8(x, w)
        assert got.eq(want.cuda()).all(), (a, b, got[0, 0], want)


@pytest.mark.parametrize("order", ["to_sparse", "to_original"])
@pytest.mark.parametrize("B, grid, s, pattern", [(1, (2, 4, 8), 2, "token"), (2, (1, 8, 4), 2, "group"), (1, (1, 4, 4), 2, "token"), (1, (1, 2, 2), 2, "token"), (3, (1, 9, 18), 3, "token"), (2, (2, 9, 9), 3, "group"),
                                                 (1, (3, 16, 16), 4, "group"), (1, (21, 30, 52), 2, "token")])
def test_rows_that_move(B, grid, s, pattern, order):
    import paper_2605_28691_amd as sk

    T, H, W = grid
    n, K, N = T * H * W, 112, 136
    lead = (B, n) if order == "to_sparse" else (s * s * B, n // (s * s))
    x, w, bias, _ = _inputs(B * n, K, N, n, lead=lead)
    to = (order, (B, *grid), s, pattern)
    xm = sk.Quantized(ref.moved(x.codes, *to).contiguous(), ref.moved(x.scales, *to).contiguous())
    residual = torch.randn(*xm.codes.shape[:2], N, device="cuda").bfloat16()
    got = sk.skiparse_linear_fwd_int8(x, w, bias, residual, act="silu", order=order, T=T, H=H, W=W, s=s, pattern=pattern)
    assert got.shape == residual.shape
    assert torch.equal(got, sk.skiparse_linear_fwd_int8(xm, w, bias, residual, act="silu"))
    _check(xm, w, bias, residual, "silu", got)


@pytest.mark.parametrize("M", [1, 7, 40, 400])
def test_scales_that_are_not_finite(M):
    """What a quantiser makes of a row that is not finite: its results are NaN, and no others."""
    import paper_2605_28691_amd as sk

    x, w, bias, residual = _inputs(M, 256, 264, M)
    good = sk.skiparse_linear_fwd_int8(x, w, bias, residual)
    x.scales[M // 2], x.codes[M // 2] = float("nan"), 0
    got = sk.skiparse_linear_fwd_int8(x, w, bias, residual)
    keep = torch.arange(M, device="cuda") != M // 2
    assert got[M // 2].isnan().all() and torch.equal(got[keep], good[keep])
    x, w, bias, residual = _inputs(M, 256, 264, M)
    w.scales[5], w.codes[5] = float("nan"), 0
    got = sk.skiparse_linear_fwd_int8(x, w, bias, residual)
    keep = torch.arange(264, device="cuda") != 5
    assert got[:, 5].isnan().all() and torch.equal(got[:, keep], good[:, keep])


def test_beyond_32_bit_offsets():
    import paper_2605_28691_amd as sk

    # codes beyond 4 GiB
    M, K, N = 66000, 65552, 72
    some, w, bias, _ = _inputs(600, K, N, 1)
    x = sk.Quantized(some.codes.repeat(M // 600, 1), some.scales.repeat(M // 600))
    got = sk.skiparse_linear_fwd_int8(x, w, bias)
    want = sk.skiparse_linear_fwd_int8(some, w, bias)
    assert torch.equal(got[-600:], want) and torch.equal(got.view(-1, 600, N), want.expand(M // 600, 600, N))
    del x, got
    # results and residual beyond 4 GiB
    M, K, N = 300000, 64, 8200
    some, w, bias, residual = _inputs(600, K, N, 2)
    x = sk.Quantized(some.codes.repeat(M // 600, 1), some.scales.repeat(M // 600))
    got = sk.skiparse_linear_fwd_int8(x, w, bias, residual.repeat(M // 600, 1), act="silu")
    want = sk.skiparse_linear_fwd_int8(some, w, bias, residual, act="silu")
    assert torch.equal(got[-600:], want) and torch.equal(got[:600], want) and torch.equal(got.view(-1, 600, N)[250], want)


def test_what_lies_round_the_results():
    import paper_2605_28691_amd as sk

    for M, K, N in ((1, 64, 8), (5, 1536, 72), (20, 5120, 40), (70, 208, 264), (300, 1008, 520), (528, 8016, 3616)):
        x, w, bias, residual = _inputs(M, K, N, M)
        pad = 512
        buf = torch.full((M * N + 2 * pad,), 77, dtype=torch.bfloat16, device="cuda")
        out = buf[pad:-pad].view(M, N)
        size = sk.skiparse_linear_fwd_int8_workspace_bytes(M, K, N)
        space = torch.full((size + 2 * pad,), 77, dtype=torch.uint8, device="cuda")
        want = sk.skiparse_linear_fwd_int8(x, w, bias, residual)
        assert torch.equal(sk.skiparse_linear_fwd_int8(x, w, bias, residual, out=out, workspace=space[pad:pad + size] if size else None), want)
        for b in (buf, space):
            assert (b[:pad] == 77).all() and (b[-pad:] == 77).all(), (M, K, N)


@pytest.mark.parametrize("M, K, N", [(1, 5120, 5120), (9, 1536, 520), (40, 8016, 264), (300, 1008, 1000)])
def test_two_graphs_and_two_streams(M, K, N):
    """Calls that overlap, each with a workspace of its own; replays with other inputs in the same places."""
    import paper_2605_28691_amd as sk

    sets = [_inputs(M, K, N, seed) for seed in (1, 2)]
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in sets]
    size = sk.skiparse_linear_fwd_int8_workspace_bytes(M, K, N)
    spaces = [torch.empty(max(size, 16), dtype=torch.uint8, device="cuda") for _ in sets]
    graphs = []
    for (x, w, b, r), o, ws in zip(sets, outs, spaces):
        sk.skiparse_linear_fwd_int8(x, w, b, r, out=o, workspace=ws)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            sk.skiparse_linear_fwd_int8(x, w, b, r, out=o, workspace=ws)
        graphs.append(gr)
    side = [torch.cuda.Stream() for _ in sets]
    for turn in range(4):
        for x, w, b, r in sets:
            x.codes.copy_(x.codes.roll(1, 0) if turn % 2 else x.codes.flip(-1))
        want = [sk.skiparse_linear_fwd_int8(*s) for s in sets]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for gr, st in zip(graphs, side):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for o, w_ in zip(outs, want):
            assert torch.equal(o, w_), turn
