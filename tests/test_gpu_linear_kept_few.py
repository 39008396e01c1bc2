"""GPU: few rows whose values in front of the activation are kept as a checkpoint.  What is kept changes no bit of the result."""
import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu

ROWS = [1, 2, 5, 15, 16, 17, 31, 32, 33]


def _inputs(M, K, N, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return r(M, K).bfloat16(), (r(N, K) * K ** -0.5).bfloat16(), (r(N) * 0.5).bfloat16(), r(M, N).bfloat16()


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("K, N", [(8, 8), (72, 40), (1032, 8200), (4104, 4120), (5120, 5120), (5128, 24), (520, 1000)])
def test_the_result_does_not_depend_on_what_is_kept(M, K, N):
    import paper_2605_28691_amd as sk

    x, w, bias, residual = _inputs(M, K, N, M + K + N)
    for act, b, r in (("gelu_tanh", bias, residual), ("silu", None, residual), ("none", bias, None)):
        plain = sk.skiparse_linear_fwd(x, w, b, r, act=act)
        kept16, pre = sk.skiparse_linear_fwd(x, w, b, r, act=act, keep="bf16")
        kept8, ckpt = sk.skiparse_linear_fwd(x, w, b, r, act=act, keep="checkpoint")
        assert torch.equal(plain, kept16) and torch.equal(plain, kept8)
        z = x.double() @ w.double().t() + (0 if b is None else b.double())
        # z is known to float32 sums of K exact products
        sums = (K + 4) * ref.F32 * (x.double().abs() @ w.double().abs().t() + (0 if b is None else b.double().abs()))
        blocks = -(-N // 32)
        pad = lambda t: torch.nn.functional.pad(t, (0, blocks * 32 - N)).reshape(M, blocks, 32)  # noqa: E731
        top, slack = pad(z.abs()).amax(-1), pad(sums).amax(-1)
        byte = lambda a: ref.checkpoint(a.reshape(-1, 1))[1].reshape(M, blocks)  # noqa: E731
        assert ((ckpt.scales >= byte((top - slack).clamp(min=0))) & (ckpt.scales <= byte(top + slack))).all()
        step = torch.exp2(ckpt.scales.double() - 127).repeat_interleave(32, -1)[:, :N] * 2.0 ** -10  # half a step of the smallest codes
        got = ref.values(ckpt.codes, ckpt.scales)
        assert ((got - z).abs() <= ref.E4M3 * z.abs() + step + 1.1 * sums).all()


@pytest.mark.parametrize("M", [1, 5, 20])
@pytest.mark.parametrize("K, N", [(64, 40), (520, 104), (1536, 4104)])
def test_nothing_else_is_written_and_nothing_behind_the_operands_counts(M, K, N):
    """Operands in the middle of NaN, results and kept values in the middle of other bytes, scales at an odd address; no workspace."""
    import paper_2605_28691_amd as sk

    x0, w0, bias, residual = _inputs(M, K, N, M * N)
    xb, wb = torch.full((M + 2, K), float("nan"), device="cuda").bfloat16(), torch.full((N + 40, K), float("nan"), device="cuda").bfloat16()
    x, w = xb[1 : M + 1], wb[8 : N + 8]
    x.copy_(x0)
    w.copy_(w0)
    assert sk.skiparse_linear_workspace_bytes(M, K, N) == 0
    want, ckpt = sk.skiparse_linear_fwd(x0, w0, bias, residual, act="silu", keep="checkpoint")

    def room(n, dtype, skip):
        buf = torch.full((n + 2048,), 7, dtype=dtype, device="cuda")
        return buf, buf[skip : skip + n]

    blocks = -(-N // 32)
    (ob, out), (cb, codes), (sb, scales) = room(M * N, torch.bfloat16, 1024), room(M * N, torch.uint8, 1024), room(M * blocks, torch.uint8, 1021)
    pre = sk.Checkpoint(codes.view(M, N), scales.view(M, blocks))
    got, kept = sk.skiparse_linear_fwd(x, w, bias, residual, act="silu", keep="checkpoint", out=out.view(M, N), pre=pre)
    assert torch.equal(got, want) and torch.equal(kept.codes, ckpt.codes) and torch.equal(kept.scales, ckpt.scales)
    for buf, n, skip in ((ob, M * N, 1024), (cb, M * N, 1024), (sb, M * blocks, 1021)):
        assert (buf[:skip] == 7).all() and (buf[skip + n :] == 7).all()
    # in place of the residual, and a row that is no number spoils its own blocks only
    inplace = residual.clone()
    sk.skiparse_linear_fwd(x, w, bias, inplace, act="silu", keep="checkpoint", out=inplace)
    assert torch.equal(inplace, want)
    if M > 1:
        x1 = x0.clone()
        x1[1, 3] = float("nan")
        got, kept = sk.skiparse_linear_fwd(x1, w0, bias, residual, act="silu", keep="checkpoint")
        others = [i for i in range(M) if i != 1]
        assert torch.equal(got[others], want[others]) and torch.equal(kept.codes[others], ckpt.codes[others]) and torch.equal(kept.scales[others], ckpt.scales[others])
        assert got[1].isnan().all() and (kept.codes[1] & 0x7F == 0x7F).all() and (kept.scales[1] == 127).all()


@pytest.mark.parametrize("M", [1, 3, 30])
@pytest.mark.parametrize("N", [24, 96, 520])
def test_kept_values_that_are_not_finite(M, N):
    """They become NaN and leave the scale of their block to the others, as in a checkpoint that is saved."""
    import paper_2605_28691_amd as sk

    K = 520
    x, w, bias, _ = _inputs(M, K, N, M + N)
    bias[5], bias[N // 2], bias[N - 1] = float("inf"), float("nan"), float("-inf")
    clean = bias.isfinite()
    _, kept = sk.skiparse_linear_fwd(x, w, bias, keep="checkpoint")
    w0, b0 = w.clone(), bias.clone()
    w0[~clean] = 0
    b0[~clean] = 0
    _, want = sk.skiparse_linear_fwd(x, w0, b0, keep="checkpoint")
    assert torch.equal(kept.scales, want.scales) and torch.equal(kept.codes[:, clean], want.codes[:, clean])
    assert (kept.codes[:, ~clean] & 0x7F == 0x7F).all()


@pytest.mark.parametrize("order", ["to_sparse", "to_original"])
@pytest.mark.parametrize("M", [4, 16, 32])
def test_rows_that_move(M, order):
    import paper_2605_28691_amd as sk

    K, N = 1032, 264
    T, H, W = (M // 4, 2, 2) if M < 32 else (4, 2, 4)
    lead = (1, M) if order == "to_sparse" else (4, M // 4)
    x, w, bias, _ = _inputs(M, K, N, M)
    x = x.view(*lead, K)
    got, kept = sk.skiparse_linear_fwd(x, w, bias, act="silu", keep="checkpoint", order=order, T=T, H=H, W=W, s=2)
    want, ckpt = sk.skiparse_linear_fwd(ref.moved(x, order, (1, T, H, W), 2, "token").contiguous(), w, bias, act="silu", keep="checkpoint")
    assert torch.equal(got, want) and torch.equal(kept.codes, ckpt.codes) and torch.equal(kept.scales, ckpt.scales)


@pytest.mark.parametrize("M", [1, 5, 20])
def test_captured_and_replayed(M):
    """A few rows forward with a checkpoint, and dx from it without x, in a HIP graph, replayed on new inputs with eager work between."""
    import paper_2605_28691_amd as sk

    K, N = 520, 1000
    x, w, bias, dy = _inputs(M, K, N, 40 + M)

    def step():
        out, pre = sk.skiparse_linear_fwd(x, w, bias, act="silu", keep="checkpoint")
        dx, _, db = sk.skiparse_linear_bwd(dy, None, w, pre=pre, act="silu", need_dw=False)
        return out, *pre, dx, db

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for trial in range(3):
        for t, new in zip((x, w, bias, dy), _inputs(M, K, N, 50 + trial)):
            t.copy_(new)
        for t in kept:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in kept]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), trial
