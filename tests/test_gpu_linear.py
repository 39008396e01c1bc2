"""GPU: the linear layer with its epilogue, and its gradients, against float64.

Tolerances, element by element: the result's one rounding (2^-8 of it), float32 sums of K exact products (K * 2^-24 of the sum of their sizes), and in the backward pass
the rounding of dz (2^-8 of every term).  Over a whole tensor roundings are independent: 2^-8 / sqrt(3) each at most, so two of them stay below 2^-8 in the 2-norm."""
import pytest
import torch

import _block_ref as ref
from test_linear_plan import WIDE

pytestmark = pytest.mark.gpu


def _close(got, want, bound, what, norm=True):
    got = got.double()
    assert got.isfinite().all(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), f"{what}: {float(over.max()):.3e} over its bound, {int((over > 0).sum())} of {over.numel()}"
    if norm and want.numel() >= 256:
        rel = float((got - want).norm() / want.norm())
        assert rel <= ref.BF16, f"{what}: 2-norm {rel:.3e}"


def _inputs(M, K, N, seed, bias=True, residual=True, lead=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lead = lead or (M,)
    x, w = r(*lead, K).bfloat16(), (r(N, K) * K ** -0.5).bfloat16()
    return x, w, (r(N) * 0.5).bfloat16() if bias else None, r(*lead, N).bfloat16() if residual else None, r(*lead, N).bfloat16()


def _check_forward(x, w, bias, residual, act, got, z=None):
    """x: [M][K] in the order of the result's rows."""
    K = x.shape[-1]
    x64, w64 = x.double(), w.double()
    z = x64 @ w64.t() + (0 if bias is None else bias.double())
    sums = (x64.abs() @ w64.abs().t() + (0 if bias is None else bias.double().abs())) * (K + 4) * ref.F32
    # the activation's slope is at most 1.13; its own arithmetic is good to 2^-19 of z
    y = ref.act(act, z) + (0 if residual is None else residual.double())
    _close(got, y, ref.BF16 * y.abs() + 1.2 * sums + (2.0 ** -19 * z.abs() if act != "none" else 0) + 2 * ref.F32 * y.abs(), f"out {tuple(got.shape)} K {K} {act}")
    return z, sums


SIZES = [(1, 8, 8), (1, 5120, 40), (2, 64, 128), (3, 72, 136), (16, 1000, 96), (17, 256, 72), (33, 136, 520), (64, 64, 64), (65, 200, 264), (100, 1536, 128),
         (127, 128, 8), (128, 128, 128), (129, 32, 384), (257, 264, 256), (390, 1000, 1000), (600, 2056, 232), (1025, 72, 520), (70001, 64, 72)]


@pytest.mark.parametrize("act", ["none", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M, K, N", SIZES)
def test_forward(M, K, N, act):
    import paper_2605_28691_amd as sk

    x, w, bias, residual, _ = _inputs(M, K, N, M + K + N)
    for b, r in ((bias, residual), (None, None), (bias, None), (None, residual)):
        _check_forward(x, w, b, r, act, sk.skiparse_linear_fwd(x, w, b, r, act=act))
    got = sk.skiparse_linear_fwd(x, w, bias, residual, act=act)
    assert torch.equal(got, sk.skiparse_linear_fwd(x, w, bias, residual, act=act))  # the same bits every time
    inplace = residual.clone()
    assert sk.skiparse_linear_fwd(x, w, bias, inplace, act=act, out=inplace) is inplace and torch.equal(got, inplace)


@pytest.mark.parametrize("M, K, N", [(1, 72, 32), (5, 64, 40), (130, 200, 264), (257, 1000, 96), (70, 512, 1024)])
def test_kept_values(M, K, N):
    """What is kept for the backward pass: z in bf16, or the checkpoint of z; the result is the same."""
    import paper_2605_28691_amd as sk

    x, w, bias, residual, _ = _inputs(M, K, N, 3 * M + K)
    plain = sk.skiparse_linear_fwd(x, w, bias, residual, act="gelu_tanh")
    out, pre = sk.skiparse_linear_fwd(x, w, bias, residual, act="gelu_tanh", keep="bf16")
    z, sums = _check_forward(x, w, bias, residual, "gelu_tanh", out)
    assert torch.equal(out, plain)
    _close(pre, z, ref.BF16 * z.abs() + sums, "pre")
    out, kept = sk.skiparse_linear_fwd(x, w, bias, residual, act="gelu_tanh", keep="checkpoint")
    assert torch.equal(out, plain)
    # scale: that of the block's largest |z|, which is known to `sums`
    blocks = -(-N // 32)
    pad = lambda t: torch.nn.functional.pad(t, (0, blocks * 32 - N)).reshape(M, blocks, 32)  # noqa: E731
    top, slack = pad(z.abs()).amax(-1), pad(sums).amax(-1)
    byte = lambda a: ref.checkpoint(a.reshape(-1, 1))[1].reshape(M, blocks)  # noqa: E731
    assert ((kept.scales >= byte(top - slack)) & (kept.scales <= byte(top + slack))).all()
    step = torch.exp2(kept.scales.double() - 127).repeat_interleave(32, -1)[:, :N] * 2.0 ** -10  # half a step of the smallest codes
    got = ref.values(kept.codes, kept.scales)
    assert ((got - z).abs() <= ref.E4M3 * z.abs() + step + 1.1 * sums).all()


GRIDS = [(1, (2, 4, 8), 2, "token"), (2, (1, 8, 4), 2, "group"), (3, (1, 9, 18), 3, "token"), (2, (2, 9, 9), 3, "group"), (1, (3, 16, 16), 4, "group"), (1, (21, 30, 52), 2, "token")]


@pytest.mark.parametrize("order", ["to_sparse", "to_original"])
@pytest.mark.parametrize("B, grid, s, pattern", GRIDS)
def test_rows_that_move(B, grid, s, pattern, order):
    import paper_2605_28691_amd as sk

    T, H, W = grid
    n, K, N = T * H * W, 104, 136
    lead = (B, n) if order == "to_sparse" else (s * s * B, n // (s * s))
    x, w, bias, _, _ = _inputs(B * n, K, N, n, lead=lead)
    at = dict(order=order, T=T, H=H, W=W, s=s, pattern=pattern)
    xm = ref.moved(x, order, (B, T, H, W), s, pattern)
    residual = torch.randn(*xm.shape[:2], N, device="cuda").bfloat16()
    got = sk.skiparse_linear_fwd(x, w, bias, residual, act="silu", **at)
    assert got.shape == residual.shape
    assert torch.equal(got, sk.skiparse_linear_fwd(xm.contiguous(), w, bias, residual, act="silu"))
    _check_forward(xm.reshape(-1, K), w, bias, residual.reshape(-1, N), "silu", got.reshape(-1, N))
    # and back
    _, pre = sk.skiparse_linear_fwd(x, w, bias, act="silu", keep="checkpoint", **at)
    dy = torch.randn_like(residual)
    back = {"to_sparse": "to_original", "to_original": "to_sparse"}[order]
    for act, p in (("silu", pre), ("none", None)):
        dx, dw, db = sk.skiparse_linear_bwd(dy, x, w, pre=p, act=act, **at)
        ex, ew, eb = sk.skiparse_linear_bwd(dy, xm.contiguous(), w, pre=p, act=act)
        assert torch.equal(dx, ref.moved(ex, back, (B, T, H, W), s, pattern))
        _close(dw, ew.double(), 2 * ref.BF16 * ew.double().abs() + 2e-4 * ew.double().abs().max(), "dw of moved rows", norm=False)
        _close(db, eb.double(), 2 * ref.BF16 * eb.double().abs() + 2e-4 * eb.double().abs().max(), "db of moved rows", norm=False)


def _check_backward(dy, x64, w, z64, act, dx, dw, db, add=None):
    """z64: the values in front of the activation that the call was given."""
    M, K = x64.shape
    N = w.shape[0]
    w64 = w.double()
    dz = dy.double() * (ref.slope(act, z64) if act != "none" else 1.0)
    # with an activation: rounding of dz, and its slope's arithmetic (2^-19 of dy times at most 1.2)
    off = dz.abs() * ref.BF16 + dy.double().abs() * 2.0 ** -19 if act != "none" else torch.zeros_like(dz)
    if dx is not None:
        want = dz @ w64 + (0 if add is None else add.double())
        bound = ref.BF16 * want.abs() + off @ w64.abs() + (N + 4) * ref.F32 * (dz.abs() @ w64.abs() + (0 if add is None else add.double().abs()))
        _close(dx, want, bound, f"dx {M} {K} {N} {act}")
    if dw is not None:
        want = dz.t() @ x64
        _close(dw, want, ref.BF16 * want.abs() + off.t() @ x64.abs() + (M + 4) * ref.F32 * (dz.abs().t() @ x64.abs()), f"dw {M} {K} {N} {act}")
    if db is not None:
        want = dz.sum(0)
        _close(db, want, ref.BF16 * want.abs() + ((M + 4) * ref.F32 * dz.abs() + (2.0 ** -19 * dy.double().abs() if act != "none" else 0)).sum(0), f"db {M} {N} {act}")


@pytest.mark.parametrize("act", ["none", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M, K, N", SIZES)
def test_backward(M, K, N, act):
    import paper_2605_28691_amd as sk

    x, w, bias, add, dy = _inputs(M, K, N, M * 3 + N)
    add = torch.randn_like(x)
    pre = None if act == "none" else (2 * torch.randn_like(dy.float())).bfloat16()
    z64 = None if pre is None else pre.double()
    got = sk.skiparse_linear_bwd(dy, x, w, pre=pre, act=act)
    _check_backward(dy, x.double(), w, z64, act, *got)
    assert all(torch.equal(a, b) for a, b in zip(got, sk.skiparse_linear_bwd(dy, x, w, pre=pre, act=act)))
    with_add = sk.skiparse_linear_bwd(dy, x, w, pre=pre, act=act, dx_add=add, need_dw=False, need_db=False)
    assert with_add[1] is None and with_add[2] is None
    _check_backward(dy, x.double(), w, z64, act, with_add[0], None, None, add)
    buf = add.clone()
    assert sk.skiparse_linear_bwd(dy, x, w, pre=pre, act=act, dx_add=buf, dx=buf, need_dw=False, need_db=False)[0] is buf
    assert torch.equal(buf, with_add[0])
    alone = sk.skiparse_linear_bwd(dy, x, w, pre=pre, act=act, need_dx=False, need_db=False)
    assert alone[0] is None and torch.equal(alone[1], got[1])
    alone = sk.skiparse_linear_bwd(dy, x, w, pre=pre, act=act, need_dx=False, need_dw=False)
    assert alone[:2] == (None, None) and torch.equal(alone[2], got[2])


@pytest.mark.parametrize("M, K, N", [(1, 40, 72), (130, 200, 264), (390, 1000, 96)])
def test_backward_from_checkpoints(M, K, N):
    """x and z in 8 bits: the gradients of the values that the checkpoints stand for."""
    import paper_2605_28691_amd as sk

    x, w, bias, _, dy = _inputs(M, K, N, M + 5 * N)
    out, pre = sk.skiparse_linear_fwd(x, w, bias, act="gelu_tanh", keep="checkpoint")
    kept = sk.skiparse_checkpoint_save(x)
    got = sk.skiparse_linear_bwd(dy, kept, w, pre=pre, act="gelu_tanh")
    _check_backward(dy, ref.values(kept.codes, kept.scales), w, ref.values(pre.codes, pre.scales), "gelu_tanh", *got)


def test_gradients_by_differences():
    """Directional derivatives of <g, act(x w^T + b)> by float64 differences of the plain form."""
    import paper_2605_28691_amd as sk

    M, K, N = 40, 72, 48
    x, w, bias, _, g = _inputs(M, K, N, 9)
    out, pre = sk.skiparse_linear_fwd(x, w, bias, act="gelu_tanh", keep="bf16")
    grads = sk.skiparse_linear_bwd(g, x, w, pre=pre, act="gelu_tanh")
    at = [t.double() for t in (x, w, bias)]
    f = lambda a, b, c: (g.double() * ref.act("gelu_tanh", a @ b.t() + c)).sum()  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i, grad in enumerate(grads):
        d = torch.randn(at[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        h = 1e-4
        up, down = [list(at) for _ in range(2)]
        up[i], down[i] = at[i] + h * d, at[i] - h * d
        slope = (f(*up) - f(*down)) / (2 * h)
        # z was rounded to bf16 (2^-8 of it; the slope's slope is at most 1.13 / 1), dz and the gradient too: three relative errors of 2^-8, independent from element to
        # element, and twice that for chance
        size = (grad.double() * d).norm() + (grad.double().norm() * d.norm()) / d.numel() ** 0.5
        assert abs(float((grad.double() * d).sum() - slope)) <= 6 * ref.BF16 * float(size), i


@pytest.mark.parametrize("M", [3, 70, 200])
def test_what_lies_beside_the_operands_does_not_count(M):
    """Rows of 72 channels, no multiple of a step's 64, in the middle of NaN; a row that holds NaN spoils its own results only; what lies behind a result stays."""
    import paper_2605_28691_amd as sk

    K, N = 72, 40
    big = torch.full((M + 4, K), float("nan"), device="cuda").bfloat16()
    wide = torch.full((N + 4, K), float("nan"), device="cuda").bfloat16()
    x, w, dy_all = big[2 : M + 2], wide[1 : N + 1], torch.full((M + 4, N), float("nan"), device="cuda").bfloat16()
    x.copy_(torch.randn(M, K, device="cuda"))
    w.copy_(torch.randn(N, K, device="cuda"))
    dy = dy_all[1 : M + 1]
    dy.copy_(torch.randn(M, N, device="cuda"))
    if x.data_ptr() % 16 == 0 and w.data_ptr() % 16 == 0:
        out = torch.full((M + 3, N), 7.0, device="cuda").bfloat16()
        sk.skiparse_linear_fwd(x, w, out=out[:M])
        _check_forward(x, w, None, None, "none", out[:M])
        assert (out[M:] == 7.0).all()
        dx_all, dw_all, db_all = torch.full((M + 3, K), 7.0, device="cuda").bfloat16(), torch.full((N + 3, K), 7.0, device="cuda").bfloat16(), torch.full((N + 8,), 7.0, device="cuda").bfloat16()
        got = sk.skiparse_linear_bwd(dy, x, w, dx=dx_all[:M], dw=dw_all[:N], db=db_all[:N])
        _check_backward(dy, x.double(), w, None, "none", *got)
        assert (dx_all[M:] == 7.0).all() and (dw_all[N:] == 7.0).all() and (db_all[N:] == 7.0).all()
    x2 = x.clone()
    x2[1, 70] = float("nan")
    got = sk.skiparse_linear_fwd(x2, w.contiguous())
    assert got[1].isnan().all() and got[[i for i in range(M) if i != 1]].isfinite().all()
    w2 = w.clone()
    w2[3, 71] = float("inf")
    got = sk.skiparse_linear_fwd(x.contiguous(), w2)
    assert not got[:, 3].isfinite().any() and got[:, [i for i in range(N) if i != 3]].isfinite().all()
    dx, dw, db = sk.skiparse_linear_bwd(dy, x2, w.contiguous())
    assert dx.isfinite().all() and dw[:, 70].isnan().all() and dw[:, [i for i in range(K) if i != 70]].isfinite().all()


def test_values_far_out():
    """Activations and slopes at the ends of the range: limits, not 0 * inf."""
    import paper_2605_28691_amd as sk

    z = torch.tensor([[-float("inf"), -3e38, -1e20, -200.0, -90.0, -20.0, -0.0, 0.0, 20.0, 90.0, 1e20, 3e38, float("inf"), 1e-30, -1e-30, 1.0]], device="cuda")
    for act in ("gelu_tanh", "silu"):
        eye = torch.eye(16, device="cuda").bfloat16()
        zero = torch.zeros(1, 16, device="cuda").bfloat16()
        got = sk.skiparse_linear_fwd(zero, eye, z[0].bfloat16(), act=act)
        zz = z.bfloat16().double()
        want = torch.where(zz == -float("inf"), 0.0, ref.act(act, zz).nan_to_num(nan=0.0, posinf=float("inf")))
        want = torch.where(zz < -100, 0.0, want)
        fin = want.isfinite()
        assert torch.equal(got.double().isfinite(), fin) and ((got.double() - want)[fin].abs() <= ref.BF16 * want[fin].abs() + 1e-6 * zz[fin].abs().clamp(max=100)).all()
        one = torch.ones(1, 16, device="cuda").bfloat16()
        dx, _, _ = sk.skiparse_linear_bwd(one, zero, eye, pre=z.bfloat16(), act=act, need_dw=False, need_db=False)
        want = torch.where(zz > 50, 1.0, torch.where(zz < -80, 0.0, ref.slope(act, zz.clamp(-80, 50))))
        assert ((dx.double() - want).abs() <= 2 * ref.BF16 * want.abs() + 1e-5).all()


def test_captured_and_replayed():
    """A training step of the layer in a HIP graph, replayed on new inputs with eager work between."""
    import paper_2605_28691_amd as sk

    M, K, N = 300, 200, 264
    x, w, bias, residual, dy = _inputs(M, K, N, 77)
    out, pre = torch.empty_like(residual), sk.Checkpoint(torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(M, 9, dtype=torch.uint8, device="cuda"))
    grads = torch.empty_like(x), torch.empty_like(w), torch.empty_like(bias)
    kept = sk.skiparse_checkpoint_save(x)
    fw = torch.empty(max(1, sk.skiparse_linear_workspace_bytes(M, K, N)), dtype=torch.uint8, device="cuda")
    bw = torch.empty(sk.skiparse_linear_bwd_workspace_bytes(M, K, N, "same", "silu", True), dtype=torch.uint8, device="cuda")

    def step():
        sk.skiparse_linear_fwd(x, w, bias, residual, act="silu", keep="checkpoint", out=out, pre=pre, workspace=fw)
        sk.skiparse_checkpoint_save(x, out=kept)
        sk.skiparse_linear_bwd(dy, kept, w, pre=pre, act="silu", dx=grads[0], dw=grads[1], db=grads[2], workspace=bw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for trial in range(3):
        gen = torch.Generator(device="cuda").manual_seed(trial)
        for t in (x, w, bias, residual, dy):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        for t in (out, *grads):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, *grads)]
        o, p = sk.skiparse_linear_fwd(x, w, bias, residual, act="silu", keep="checkpoint")
        want = (o, *sk.skiparse_linear_bwd(dy, sk.skiparse_checkpoint_save(x), w, pre=p, act="silu"))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), trial


def test_two_streams_at_once():
    """Calls on two streams share nothing."""
    import paper_2605_28691_amd as sk

    sets = [_inputs(500, 264, 520, i) for i in range(2)]
    want = [(sk.skiparse_linear_fwd(x, w, b, r, act="silu"), *sk.skiparse_linear_bwd(dy, x, w)) for x, w, b, r, dy in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for i, (st, (x, w, b, r, dy)) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(st):
                got[i] = (sk.skiparse_linear_fwd(x, w, b, r, act="silu"), *sk.skiparse_linear_bwd(dy, x, w))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("M, N", [(3, 96), (70, 72), (300, 520)])
def test_kept_values_that_are_not_finite(M, N):
    """In a checkpoint that a product writes they become NaN and leave the scale of their block to the others; as in one that is saved."""
    import paper_2605_28691_amd as sk

    K = 64
    x, w, bias, _, _ = _inputs(M, K, N, M)
    bias[5], bias[40], bias[41] = float("inf"), float("nan"), float("-inf")
    out, pre = sk.skiparse_linear_fwd(x, w, bias, keep="bf16")
    assert torch.equal(pre.isnan(), torch.isnan(bias).expand(M, N)) and torch.equal(pre.isfinite(), bias.isfinite().expand(M, N))
    _, kept = sk.skiparse_linear_fwd(x, w, bias, keep="checkpoint")
    got = sk.skiparse_checkpoint_load(kept, dtype=torch.float32)
    assert torch.equal(got.isnan(), ~bias.isfinite().expand(M, N))
    b0 = bias.clone()
    b0[[5, 40, 41]] = 0
    z = x.double() @ w.double().t() + b0.double()
    z[:, [5, 40, 41]] = 0.0
    sums = (K + 4) * ref.F32 * (x.double().abs() @ w.double().abs().t() + b0.double().abs())
    step = torch.exp2(kept.scales.double() - 127).repeat_interleave(32, -1)[:, :N] * 2.0 ** -10
    fine = bias.isfinite()
    assert ((got.double() - z).abs() <= ref.E4M3 * z.abs() + step + 1.1 * sums)[:, fine].all()
    blocks = -(-N // 32)
    top = torch.nn.functional.pad(z.abs(), (0, blocks * 32 - N)).reshape(M, blocks, 32).amax(-1)
    assert (torch.exp2(kept.scales.double() - 127) * 448 >= top * (1 - 1e-3)).all() and (torch.exp2(kept.scales.double() - 127) * 224 <= top * (1 + 1e-3)).all()


@pytest.mark.parametrize("M", [1, 2, 4, 5, 15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("K, N", [(8, 8), (72, 40), (520, 4104), (1032, 8200), (4104, 4120), (5128, 24)])
def test_few_rows(M, K, N):
    """The kernel for one row, with one, two and four channels a wavefront; those for up to 16 and 32, with 16 and 32 channels a workgroup; and the first size beyond them; in the order
    they come and moved."""
    import paper_2605_28691_amd as sk

    x, w, bias, residual, _ = _inputs(M, K, N, M + K)
    for act in ("none", "silu"):
        out, pre = sk.skiparse_linear_fwd(x, w, bias, residual, act=act, keep="bf16")
        z, sums = _check_forward(x, w, bias, residual, act, out)
        _close(pre, z, ref.BF16 * z.abs() + sums, "pre")
    if M in (4, 16, 32):
        T, H, W = M // 4 if M < 32 else 4, 2, 2 if M < 32 else 4
        at = dict(T=T, H=H, W=W, s=2, pattern="token")
        still = sk.skiparse_linear_fwd(x, w, bias)
        got = sk.skiparse_linear_fwd(x.reshape(1, M, K), w, bias, order="to_sparse", **at)
        assert got.shape == (4, M // 4, N) and torch.equal(got, ref.moved(still.reshape(1, M, N), "to_sparse", (1, T, H, W), 2, "token"))
        back = sk.skiparse_linear_fwd(x.reshape(4, M // 4, K), w, bias, order="to_original", **at)
        assert torch.equal(back, ref.moved(still.reshape(4, M // 4, N), "to_original", (1, T, H, W), 2, "token"))


def test_rows_and_channels_at_the_edges_of_all_tiles():
    """Results of the square tiles, whole and cut along k, with and without everything that the epilogue does."""
    import paper_2605_28691_amd as sk

    for M, K, N in ((513, 4096, 264), (1030, 2176, 1032), (5000, 192, 2056), (7700, 520, 1544), (2600, 7000, 520), (60, 9000, 72)):
        x, w, bias, residual, dy = _inputs(M, K, N, M)
        _check_forward(x, w, None, None, "none", sk.skiparse_linear_fwd(x, w))
        out, kept = sk.skiparse_linear_fwd(x, w, bias, residual, act="silu", keep="checkpoint")
        z, sums = _check_forward(x, w, bias, residual, "silu", out)
        step = torch.exp2(kept.scales.double() - 127).repeat_interleave(32, -1)[:, :N] * 2.0 ** -10
        assert ((ref.values(kept.codes, kept.scales) - z).abs() <= ref.E4M3 * z.abs() + step + 1.1 * sums).all()
        _check_backward(dy, x.double(), w, None, "none", *sk.skiparse_linear_bwd(dy, x, w))


@pytest.mark.parametrize("M, N, K", WIDE)
def test_wide_tiles(M, N, K):
    """Products with tiles of 128 x 256: forward, and each of the gradients, whose rows, channels and sum are other sizes of the layer."""
    import paper_2605_28691_amd as sk

    x, w, bias, residual, _ = _inputs(M, K, N, M)
    _check_forward(x, w, None, None, "none", sk.skiparse_linear_fwd(x, w))
    out, kept = sk.skiparse_linear_fwd(x, w, bias, residual, act="gelu_tanh", keep="checkpoint")
    z, sums = _check_forward(x, w, bias, residual, "gelu_tanh", out)
    step = torch.exp2(kept.scales.double() - 127).repeat_interleave(32, -1)[:, :N] * 2.0 ** -10
    assert ((ref.values(kept.codes, kept.scales) - z).abs() <= ref.E4M3 * z.abs() + step + 1.1 * sums).all()
    x, w, _, _, dy = _inputs(M, N, K, M + 1)  # dx: M x N, summed over K
    _check_backward(dy, x.double(), w, None, "none", *sk.skiparse_linear_bwd(dy, x, w))
    if M % 8 == 0:
        x, w, _, _, dy = _inputs(K, N, M, M + 2)  # dw: M x N, summed over K
        _check_backward(dy, x.double(), w, None, "none", *sk.skiparse_linear_bwd(dy, x, w))


@pytest.mark.parametrize("skip", [1, 2, 3])
@pytest.mark.parametrize("M, K, N", [(1, 72, 40), (70, 104, 136), (300, 200, 520)])
def test_scales_at_any_address(M, K, N, skip):
    """A checkpoint's scales lie at any address: written by save and by the product, read by load and by the backward pass; and nothing round them is touched."""
    import paper_2605_28691_amd as sk

    def at(scales):
        buf = torch.full((scales.numel() + 64,), 0xAB, dtype=torch.uint8, device="cuda")
        inner = buf[skip : skip + scales.numel()].view(scales.shape)
        assert inner.data_ptr() % 4 == skip
        return buf, inner

    def untouched(buf, n):
        return bool((buf[:skip] == 0xAB).all() and (buf[skip + n :] == 0xAB).all())

    x, w, bias, _, dy = _inputs(M, K, N, M)
    want = sk.skiparse_checkpoint_save(x)
    buf, scales = at(want.scales)
    kept = sk.skiparse_checkpoint_save(x, out=sk.Checkpoint(torch.empty_like(want.codes), scales))
    assert torch.equal(kept.scales, want.scales) and torch.equal(kept.codes, want.codes) and untouched(buf, scales.numel())
    assert torch.equal(sk.skiparse_checkpoint_load(kept), sk.skiparse_checkpoint_load(want))
    out, pre = sk.skiparse_linear_fwd(x, w, bias, act="silu", keep="checkpoint")
    buf, scales = at(pre.scales)
    got, odd = sk.skiparse_linear_fwd(x, w, bias, act="silu", keep="checkpoint", pre=sk.Checkpoint(torch.empty_like(pre.codes), scales))
    assert torch.equal(got, out) and torch.equal(odd.scales, pre.scales) and torch.equal(odd.codes, pre.codes) and untouched(buf, scales.numel())
    for a, b in zip(sk.skiparse_linear_bwd(dy, want, w, pre=pre, act="silu"), sk.skiparse_linear_bwd(dy, kept, w, pre=odd, act="silu")):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M, K, N", [(5, 64, 40), (20, 520, 4104), (70, 104, 136), (6566, 2056, 536)])
def test_what_lies_behind_the_results_is_left_alone(M, K, N):
    """Results in the middle of larger buffers: bytes in front of them and behind the last row stay, in every form, with everything that the epilogue writes."""
    import paper_2605_28691_amd as sk

    def room(*shape, dtype=torch.bfloat16):
        n = 1
        for d in shape:
            n *= d
        buf = torch.full((n + 4096,), 7, dtype=dtype, device="cuda")
        return buf, buf[2048 : 2048 + n].view(shape)

    def untouched(buf, n):
        return bool((buf[:2048] == 7).all() and (buf[2048 + n :] == 7).all())

    x, w, bias, residual, dy = _inputs(M, K, N, M)
    pairs = [room(M, N), room(M, N, dtype=torch.uint8), room(M, -(-N // 32), dtype=torch.uint8), room(M, N), room(M, K), room(N, K), room(N)]
    out, codes, scales, pre, dx, dw, db = (p[1] for p in pairs)
    sk.skiparse_linear_fwd(x, w, bias, residual, act="gelu_tanh", keep="checkpoint", out=out, pre=sk.Checkpoint(codes, scales))
    first = out.clone()
    sk.skiparse_linear_fwd(x, w, bias, residual, act="gelu_tanh", keep="bf16", out=out, pre=pre)
    sk.skiparse_linear_bwd(dy, x, w, pre=sk.Checkpoint(codes, scales), act="gelu_tanh", dx=dx, dw=dw, db=db)
    for buf, t in pairs:
        assert untouched(buf, t.numel())
    assert float((first.double() - out.double()).norm()) <= 2 * ref.BF16 * float(out.double().norm())


@pytest.mark.parametrize("M, K, N", [(40, 5120, 520), (528, 4008, 3616), (3000, 1536, 1536)])
def test_workspaces_of_exactly_their_size(M, K, N):
    """Products that are cut along k, forward and backward, in the bytes that they ask for: nothing behind these is touched, and dirty workspaces give the same results."""
    import paper_2605_28691_amd as sk

    x, w, bias, residual, dy = _inputs(M, K, N, M)
    kept = sk.skiparse_checkpoint_save(x)
    pre = (2 * torch.randn_like(dy.float())).bfloat16()
    n = sk.skiparse_linear_workspace_bytes(M, K, N)
    nb = sk.skiparse_linear_bwd_workspace_bytes(M, K, N, act="silu", x_checkpoint=True)
    assert nb > 0
    want = sk.skiparse_linear_fwd(x, w, bias, residual), *sk.skiparse_linear_bwd(dy, kept, w, pre=pre, act="silu")
    for byte in (0xFF, 0x7F):
        buf = torch.full((max(n, nb) + 4096,), byte, dtype=torch.uint8, device="cuda")
        got = [sk.skiparse_linear_fwd(x, w, bias, residual, workspace=buf[:n] if n else None)]
        assert (buf[n:] == byte).all()
        buf.fill_(byte)
        got += sk.skiparse_linear_bwd(dy, kept, w, pre=pre, act="silu", workspace=buf[:nb])
        assert (buf[nb:] == byte).all()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError):
        sk.skiparse_linear_bwd(dy, kept, w, pre=pre, act="silu", workspace=buf[: nb - 256])
