"""GPU: the operators together, as a sparse transformer block uses them: projections into the sparse layout, positions, attention, projection back with the residual, a
feed-forward of two products; forward and backward, from 8-bit checkpoints, eager and as a captured graph."""
import pytest
import torch

import _block_ref as ref

pytestmark = pytest.mark.gpu

B, T, H, W, S, PATTERN = 1, 2, 8, 8, 2, "group"
HEADS, D, HIDDEN = 2, 64, 320
C, N = HEADS * D, T * H * W
AXES = (16, 24, 24)


def _parameters(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n, k: (torch.randn(n, k, generator=g, device="cuda") * k ** -0.5).bfloat16()  # noqa: E731
    b = lambda n: (torch.randn(n, generator=g, device="cuda") * 0.2).bfloat16()  # noqa: E731
    p = {name: (r(C, C), b(C)) for name in "qkvo"}
    p["up"], p["down"] = (r(HIDDEN, C), b(HIDDEN)), (r(C, HIDDEN), b(C))
    x = torch.randn(B, N, C, generator=g, device="cuda").bfloat16()
    dy = torch.randn(B, N, C, generator=g, device="cuda").bfloat16()
    return p, x, dy


def _step(sk, p, x, dy, table):
    """One training step of the block: result, gradient of x, gradients of all weights and biases."""
    grid = dict(T=T, H=H, W=W, s=S, pattern=PATTERN)
    sparse, sub = (S * S * B, N // (S * S)), N // (S * S)
    heads = lambda t: t.view(*t.shape[:2], HEADS, D)  # noqa: E731
    flat = lambda t: t.view(*t.shape[:2], C)  # noqa: E731
    # forward
    kx = sk.skiparse_checkpoint_save(x)
    q, k, v = (sk.skiparse_linear_fwd(x, *p[n], order="to_sparse", **grid) for n in "qkv")
    q, k = sk.skiparse_rope(heads(q), heads(k), table, T, H, W, S, PATTERN, "stay_sparse", q_out=heads(q), k_out=heads(k))
    v = heads(v)
    o, lse = sk.skiparse_attn_fwd_lse(q, k, v, 1, 1, sub, 1, "token")
    kept = [sk.skiparse_checkpoint_save(t) for t in (q, k, v, o)]
    h = sk.skiparse_linear_fwd(flat(o), *p["o"], x, order="to_original", **grid)
    kh = sk.skiparse_checkpoint_save(h)
    u, pre = sk.skiparse_linear_fwd(h, *p["up"], act="gelu_tanh", keep="checkpoint")
    ku = sk.skiparse_checkpoint_save(u)
    y = sk.skiparse_linear_fwd(u, *p["down"], h)
    # backward
    g = {}
    du, *g["down"] = sk.skiparse_linear_bwd(dy, ku, p["down"][0])
    dh, *g["up"] = sk.skiparse_linear_bwd(du, kh, p["up"][0], pre=pre, act="gelu_tanh", dx_add=dy)
    q, k, v, o = (sk.skiparse_checkpoint_load(c) for c in kept)
    do, *g["o"] = sk.skiparse_linear_bwd(dh, flat(o), p["o"][0], order="to_original", **grid)
    dq, dk, dv = sk.skiparse_attn_bwd(q, k, v, o, heads(do), lse, 1, 1, sub, 1, "token")
    dq, dk = sk.skiparse_rope(dq, dk, table, T, H, W, S, PATTERN, "stay_sparse", inverse=True)
    dx = dh
    for n, t in (("q", dq), ("k", dk), ("v", dv)):
        dx, *g[n] = sk.skiparse_linear_bwd(flat(t.contiguous()), kx, p[n][0], order="to_sparse", dx_add=dx, **grid)
    return [y, dx] + [t for n in sorted(g) for t in g[n]]


def _reference(p, x, dy, t64):
    """The same block in float64 by autograd, without checkpoints."""
    leaf = {n: [t.double().requires_grad_() for t in wb] for n, wb in p.items()}
    x64 = x.double().requires_grad_()
    product = {}

    def lin(t, n):
        product[n] = t @ leaf[n][0].t() + leaf[n][1]
        product[n].retain_grad()
        return product[n]

    grid = (B, T, H, W)
    pairs = sum(AXES) // 2
    n = torch.arange(N, device="cuda")
    place, cs, first = (n // (H * W), n // W % H, n % W), [], 0
    for at, length, r in zip(place, (T, H, W), AXES):
        cs.append(t64.view(-1, 2)[first + at[:, None] * (r // 2) + torch.arange(r // 2, device="cuda")])
        first += length * (r // 2)
    cs = torch.cat(cs, 1)  # [N][pairs][2]

    def turned(t):
        z = torch.view_as_complex(t.reshape(B, N, HEADS, D)[..., : 2 * pairs].reshape(B, N, HEADS, pairs, 2).contiguous()) * torch.view_as_complex(cs.contiguous())[None, :, None]
        return torch.cat((torch.view_as_real(z).reshape(B, N, HEADS, 2 * pairs), t.reshape(B, N, HEADS, D)[..., 2 * pairs:]), -1)

    q, k, v = turned(lin(x64, "q")), turned(lin(x64, "k")), lin(x64, "v").reshape(B, N, HEADS, D)
    q, k, v = (ref.moved(t, "to_sparse", grid, S, PATTERN) for t in (q, k, v))
    s = torch.einsum("bihd,bjhd->bhij", q, k) * D ** -0.5
    o = torch.einsum("bhij,bjhd->bihd", s.softmax(-1), v)
    o = ref.moved(o.reshape(S * S * B, -1, C), "to_original", grid, S, PATTERN)
    h = x64 + lin(o, "o")
    y = h + lin(ref.act("gelu_tanh", lin(h, "up")), "down")
    (y * dy.double()).sum().backward()
    sizes = [None, None] + [s for m in sorted(p) for s in (None, float(product[m].grad.norm()))]
    return [y.detach(), x64.grad] + [t.grad for m in sorted(p) for t in leaf[m]], sizes


def test_training_step_of_a_block():
    """Against float64 autograd.  A checkpoint's values are off by 2^-4 of them at most, 2^-4 / sqrt(3) in the 2-norm; a gradient is a product of at most two such (weights: the kept
    input and, through the slope or the attention's probabilities, other kept values), so 2 * 2^-4 in the 2-norm bounds it; the result has none, only bf16 (8 roundings in a row).
    A bias's gradient is a sum over the rows of dZ, the gradient of its product, in which terms cancel: for k all but what the positions leave, since a softmax does not see a shift
    of all its logits.  Its error is the sum of dZ's, E: |sum of R rows of E| <= sqrt(R) |E|, by Cauchy and Schwarz, and |E| <= 2 * 2^-4 |dZ|."""
    import paper_2605_28691_amd as sk

    p, x, dy = _parameters(3)
    table = sk.skiparse_rope_table((T, H, W), AXES)
    got = _step(sk, p, x, dy, table)
    want, sizes = _reference(p, x, dy, table.data.double())
    for i, (a, b, dz) in enumerate(zip(got, want, sizes)):
        assert a.shape == b.shape and a.isfinite().all(), i
        off = float((a.double() - b).norm())
        if i == 0:
            assert off <= 8 * ref.BF16 * float(b.norm()), off
        elif dz is None:
            assert off <= 2 * ref.E4M3 * float(b.norm()), (i, off / float(b.norm()))
        else:
            assert off <= 2 * ref.E4M3 * (B * N) ** 0.5 * dz, (i, off, dz)


def test_block_captured_and_replayed():
    import paper_2605_28691_amd as sk

    p, x, dy = _parameters(5)
    table = sk.skiparse_rope_table((T, H, W), AXES)
    _step(sk, p, x, dy, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(sk, p, x, dy, table)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(sk, p, x, dy, table)
    for trial in range(3):
        np_, nx, ndy = _parameters(10 + trial)
        x.copy_(nx)
        dy.copy_(ndy)
        for n in p:
            for a, b in zip(p[n], np_[n]):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = _step(sk, np_, nx, ndy, table)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), trial
