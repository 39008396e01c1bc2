"""The norm in front of a block's products and the products in 8-bit integers, as cases that can be timed.

A case is one call sequence ("op") on one shape:

  norm       root-mean-square norm of x, or of x + residual (the sum is an output too), with weights for the channels
  norm_grad  its gradients: of the normalised tensor, with what comes along the residual stream added, and of the weights
  quant      rows as codes in 8-bit integers with a scale each
  linear8    act(x w^T + bias) + residual from such codes of tokens and of the weights' rows
  sublayer8  the two as a block calls them: the stream's sum, its norm in codes, and their product with the weights

Rows are the tokens of B grids of T x H x W.  Order "to_sparse" takes them from the original order to the sparse layout of `pattern` with ratio `s`, "to_original" the other way:
the norm's and the product's results, and the codes, are written in the other order than their rows are read in; sums stay where they are.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


def _case(name, op, B, T, H, W, s=1, pattern="token", order="same", **more):
    c = dict(op=op, B=B, T=T, H=H, W=W, s=s, pattern=pattern, order=order, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token's hidden state added to the stream and normalised: the call's latency
        _case("norm_one_token", "norm", 1, 1, 1, 1, cols=5120, dtype="bf16", residual=True),
        # every head of q of two short clips on a ragged grid, 16 heads of 64 channels, in float32
        _case("norm_heads_ragged", "norm", 2, 9, 17, 336, cols=64, dtype="fp32", residual=False),
        # the residual stream of an 81-frame 768x1280 video, normalised into the sparse layout
        _case("norm_video_768p", "norm", 1, 21, 48, 80, 2, "group", "to_sparse", cols=5120, dtype="bf16", residual=True),
        # two short clips in training, odd sizes, in float32
        _case("norm_grad_ragged", "norm_grad", 2, 9, 17, 21, cols=1000, dtype="fp32", add=False),
        # the gradients of an 81-frame 480x832 video, out of the sparse layout and into the stream's
        _case("norm_grad_video_480p", "norm_grad", 1, 21, 30, 52, 2, "token", "to_sparse", cols=1536, dtype="bf16", add=True),
        # a widened activation of two short clips in float32
        _case("quant_ragged", "quant", 2, 9, 17, 21, cols=4008, dtype="fp32"),
        # the attention's result of an 81-frame 768x1280 video, back from the sparse layout, in front of its output projection
        _case("quant_video_768p", "quant", 1, 21, 48, 80, 2, "token", "to_original", cols=5120, dtype="bf16"),
        # one token through the projection of a conditioning vector
        _case("linear8_one_token", "linear8", 1, 1, 1, 1, n_in=5120, n_out=5120, act="silu", bias=True, residual=False),
        # two short clips through the widening product, odd sizes
        _case("linear8_ragged", "linear8", 2, 9, 17, 21, n_in=1008, n_out=4008, act="gelu_tanh", bias=True, residual=False),
        # the output projection behind the last sparse block, 480x832: rows back in the original order, added to the residual stream
        _case("linear8_video_480p", "linear8", 1, 21, 30, 52, 2, "token", "to_original", n_in=1536, n_out=1536, act="none", bias=True, residual=True),
        # the widening product of an 81-frame 768x1280 video: the largest call
        _case("linear8_video_768p", "linear8", 1, 21, 48, 80, n_in=5120, n_out=20480, act="gelu_tanh", bias=True, residual=False),
        # the front of an attention block of an 81-frame 480x832 video: the stream's sum, its norm, and q, k and v in one product
        _case("sublayer8_video_480p", "sublayer8", 1, 21, 30, 52, 2, "token", "to_sparse", n_in=1536, n_out=4608),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(("norm", "norm", "norm", "norm_grad", "norm_grad", "quant", "quant", "linear8", "linear8", "linear8", "linear8", "sublayer8"))
        s = rng.choice((1, 1, 2, 2, 3, 4))
        pattern = rng.choice(("token", "group"))
        unit = s if pattern == "token" else s * s
        H, W = unit * max(1, _log_int(rng, 1, 64) // unit), unit * max(1, _log_int(rng, 1, 96) // unit)
        T, B = _log_int(rng, 1, 21), rng.choice((1, 1, 2, 3))
        if s == 1 and rng.random() < 0.3:  # a few tokens
            T, H, W, B = 1, 1, 1, _log_int(rng, 1, 64)
        order = "same" if s == 1 else "to_sparse" if op == "sublayer8" else rng.choice(("to_sparse", "to_original"))
        grid, rows = (B, T, H, W, s, pattern, order), B * T * H * W
        if op in ("norm", "norm_grad", "quant"):
            cols, dtype = 8 * _log_int(rng, 4, 2560), rng.choice(("bf16", "bf16", "fp32"))
            if order == "same" and cols <= 128 and rows * 16 < 1 << 21:  # the heads of a token are rows
                grid = (B, T, H, W * 16, s, pattern, order)
            if rows * cols > 5e8:
                continue
            if op == "quant":
                return _case(None, op, *grid, cols=cols, dtype=dtype)
            if op == "norm_grad":
                return _case(None, op, *grid, cols=cols, dtype=dtype, add=rng.random() < 0.7)
            return _case(None, op, *grid, cols=cols, dtype=dtype, residual=rng.random() < 0.6)
        n_in, n_out = 16 * _log_int(rng, 4, 560), 8 * _log_int(rng, 8, 1400)
        if op == "sublayer8":
            c = _case(None, op, *grid, n_in=n_in, n_out=n_out)
        else:
            c = _case(None, op, *grid, n_in=n_in, n_out=n_out, act=rng.choice(("none", "gelu_tanh", "silu")), bias=rng.random() < 0.8, residual=rng.random() < 0.5)
        if work(c)["flops"] <= 1.6e13:
            return c


def work(c):
    op, rows = c["op"], c["B"] * c["T"] * c["H"] * c["W"]
    if "cols" in c:
        n, e = rows * c["cols"], 2 if c["dtype"] == "bf16" else 4
        if op == "quant":
            return {"bytes": n * (e + 1) + 4 * rows, "flops": 3 * n}
        if op == "norm":  # x and the weights, and with a residual two more tensors
            return {"bytes": n * e * (4 if c["residual"] else 2) + c["cols"] * e, "flops": 4 * n}
        return {"bytes": n * e * (4 if c["add"] else 3) + 2 * c["cols"] * e, "flops": 9 * n}
    K, N = c["n_in"], c["n_out"]
    weights = N * K + 4 * N
    if op == "sublayer8":  # reads x and the stream, writes the stream and the product
        return {"bytes": rows * (6 * K + 2 * N) + weights + 2 * K + 2 * N, "flops": 2 * rows * K * N + 4 * rows * K}
    return {"bytes": rows * (K + 4 + 2 * N * (2 if c["residual"] else 1)) + weights + (2 * N if c["bias"] else 0), "flops": 2 * rows * K * N}


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * scale).to(dtype)


def _activation(gen, shape, dtype):
    """Channels of an activation differ in size by a few powers of two, and tokens by a factor."""
    x = torch.randn(shape, generator=gen, device=DEVICE)
    x *= torch.exp2(torch.randn(shape[-1], generator=gen, device=DEVICE))
    x *= torch.exp2(0.5 * torch.randn((*shape[:-1], 1), generator=gen, device=DEVICE))
    return x.to(dtype)


def _lead(c, sparse):
    """Leading dimensions of a tensor of tokens."""
    n, s2 = c["T"] * c["H"] * c["W"], c["s"] * c["s"]
    return (s2 * c["B"], n // s2) if sparse else (c["B"], n)


def prepare(c, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    op = c["op"]
    lead, lead_out = _lead(c, c["order"] == "to_original"), _lead(c, c["order"] == "to_sparse")
    if "cols" in c:
        dtype, cols = DTYPES[c["dtype"]], c["cols"]
        st = dict(c=c, x=_activation(gen, (*lead, cols), dtype))
        if op != "quant":
            st["weight"] = (1.0 + 0.25 * torch.randn(cols, generator=gen, device=DEVICE)).to(dtype)
        if op == "norm":
            st["residual"] = _activation(gen, (*lead, cols), dtype) if c["residual"] else None
        if op == "norm_grad":
            st["dy"] = _normal(gen, (*lead_out, cols), dtype)
            st["add"] = _normal(gen, (*lead, cols), dtype) if c["add"] else None
        return st
    K, N = c["n_in"], c["n_out"]
    # what a program keeps of the weights: codes and scales
    w, w_scales = _codes(torch.randn((N, K), generator=gen, device=DEVICE) * K ** -0.5)
    st = dict(c=c, w=w, w_scales=w_scales)
    if op == "sublayer8":
        st.update(x=_activation(gen, (*lead, K), torch.bfloat16), residual=_activation(gen, (*lead, K), torch.bfloat16), bias=_normal(gen, (N,), torch.bfloat16, 0.5),
                  weight=(1.0 + 0.25 * torch.randn(K, generator=gen, device=DEVICE)).bfloat16())
        return st
    st["x"], st["x_scales"] = _codes(_activation(gen, (*lead, K), torch.float32))
    st["bias"] = _normal(gen, (N,), torch.bfloat16, 0.5) if c["bias"] else None
    st["residual"] = _normal(gen, (*lead_out, N), torch.bfloat16) if c["residual"] else None
    return st


# ---- the plain forms


def _codes(v):
    """(int8 codes, a scale for each row) of float32 rows."""
    top = v.abs().amax(-1, keepdim=True)
    top = torch.where(top > 0, top.clamp(min=2.0 ** -118), torch.full_like(top, 127.0))
    most = torch.full_like(top, 127.0)
    return torch.round(v * (most / top)).to(torch.int8), (top / most)[..., 0]


def _reorder(x, c, order):
    """Rows from the original order to the sparse layout or back: a view's transposition and a copy."""
    if order == "same" or c["s"] == 1:
        return x.reshape(*_lead(c, False), *x.shape[2:])
    s, tail = c["s"], x.shape[2:]
    # an axis with its classes and the places in them taken apart: (classes of places, class, place) or (places, class)
    split = (lambda n: (n // (s * s), s, s)) if c["pattern"] == "group" else (lambda n: (n // s, s))
    h, w = split(c["H"]), split(c["W"])
    full = (c["B"], c["T"], *h, *w)
    at_h, at_w = 3, 3 + len(h)
    to_sparse = [at_h, at_w, 0, 1] + [d for d in range(2, len(full)) if d not in (at_h, at_w)]
    behind = range(len(full), len(full) + len(tail))
    if order == "to_sparse":
        return x.reshape(*full, *tail).permute(*to_sparse, *behind).reshape(*_lead(c, True), *tail)
    back = [to_sparse.index(d) for d in range(len(full))]
    return x.reshape(*(full[d] for d in to_sparse), *tail).permute(*back, *behind).reshape(*_lead(c, False), *tail)


BACK = {"same": "same", "to_sparse": "to_original", "to_original": "to_sparse"}


def _act(z, act):
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _inverse_size(h):
    return 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS)


def _product(x, x_scales, w, w_scales):
    return (x.float() @ w.float().t()) * x_scales[..., None] * w_scales


def _plain(st):
    c = st["c"]
    op, x = c["op"], st["x"]
    if op == "quant":
        codes, scales = _codes(_reorder(x.float(), c, c["order"]))
        return dict(codes=codes, scales=scales)
    if op == "norm":
        h = x.float() if st["residual"] is None else x.float() + st["residual"].float()
        got = dict(out=_reorder(h * _inverse_size(h) * st["weight"].float(), c, c["order"]).to(x.dtype))
        return got if st["residual"] is None else dict(got, sum=h.to(x.dtype))
    if op == "norm_grad":
        h = x.float()
        r = _inverse_size(h)
        dy, h = _reorder(st["dy"].float(), c, BACK[c["order"]]).reshape(h.shape), h * r
        g = dy * st["weight"].float()
        dx = r * (g - h * (g * h).mean(-1, keepdim=True))
        if st["add"] is not None:
            dx = dx + st["add"].float()
        return dict(dx=dx.to(x.dtype), dw=(dy * h).sum((0, 1)).to(x.dtype))
    if op == "sublayer8":
        h = x.float() + st["residual"].float()
        codes, scales = _codes(_reorder(h * _inverse_size(h) * st["weight"].float(), c, c["order"]))
        return dict(out=(_product(codes, scales, st["w"], st["w_scales"]) + st["bias"].float()).to(x.dtype), sum=h.to(x.dtype))
    z = _product(_reorder(x, c, c["order"]), _reorder(st["x_scales"], c, c["order"]), st["w"], st["w_scales"])
    if st["bias"] is not None:
        z = z + st["bias"].float()
    out = _act(z, c["act"])
    if st["residual"] is not None:
        out = out + st["residual"].float()
    return out.to(torch.bfloat16)


# ---- the framework's calls


def _own(st):
    import paper_2605_28691_amd as sk

    c = st["c"]
    op, x = c["op"], st["x"]
    rows = dict(order=c["order"], T=c["T"], H=c["H"], W=c["W"], s=c["s"], pattern=c["pattern"])
    if op == "quant":
        got = sk.skiparse_quantize_int8(x, **rows)
        return dict(codes=got.codes, scales=got.scales)
    if op == "norm":
        if st["residual"] is None:
            return dict(out=sk.skiparse_rmsnorm_fwd(x, st["weight"], eps=EPS, **rows))
        out, total = sk.skiparse_rmsnorm_fwd(x, st["weight"], st["residual"], eps=EPS, **rows)
        return dict(out=out, sum=total)
    if op == "norm_grad":
        dx, dw = sk.skiparse_rmsnorm_bwd(st["dy"], x, st["weight"], dx_add=st["add"], eps=EPS, **rows)
        return dict(dx=dx, dw=dw)
    w = sk.Quantized(st["w"], st["w_scales"])
    if op == "sublayer8":
        codes, total = sk.skiparse_rmsnorm_fwd(x, st["weight"], st["residual"], eps=EPS, quantize=True, **rows)
        return dict(out=sk.skiparse_linear_fwd_int8(codes, w, st["bias"]), sum=total)
    return sk.skiparse_linear_fwd_int8(sk.Quantized(x, st["x_scales"]), w, st["bias"], st["residual"], act=c["act"], **rows)


def run(st):
    if own:
        return _own(st)
    return _plain(st)


# ---- the definition in 64 bits, written from the index formulas and apart from the plain forms


def _exact_order(x, c, order):
    """x as [rows][...] in the order of the other side."""
    rows = x.reshape(-1, *x.shape[2:])
    if order == "same" or c["s"] == 1:
        return rows
    B, T, H, W, s = c["B"], c["T"], c["H"], c["W"], c["s"]
    # the row of the original order that row i of the sparse layout holds (Algorithm 1)
    i = torch.arange(B * T * H * W, device=DEVICE)
    ws, i = i % (W // s), i // (W // s)
    hs, i = i % (H // s), i // (H // s)
    t, i = i % T, i // T
    b, i = i % B, i // B
    q, p = i % s, i // s
    if c["pattern"] == "token":
        h, w = hs * s + p, ws * s + q
    else:
        h, w = (hs // s) * s * s + p * s + hs % s, (ws // s) * s * s + q * s + ws % s
    at = ((b * T + t) * H + h) * W + w
    if order == "to_sparse":
        return rows[at]
    out = torch.empty_like(rows)
    out[at] = rows
    return out


def _exact_product(x, x_scales, w, w_scales, bias):
    z = torch.mm(x.double() * x_scales.double()[:, None], (w.double() * w_scales.double()[:, None]).t())
    return z if bias is None else z.add_(bias.double())


def exact(c, seed):
    st = prepare(c, seed)
    op, order, x = c["op"], c["order"], st["x"]
    lead_out = _lead(c, order == "to_sparse")
    if op == "quant":
        top = torch.linalg.vector_norm(x.double(), float("inf"), -1)
        top = torch.where(top > 0, top, torch.full_like(top, 127.0))
        return dict(codes=None, scales=(_exact_order(top, c, order) / 127.0).view(lead_out))
    if op in ("norm", "sublayer8"):
        h = x.double()
        if st["residual"] is not None:
            h = h + st["residual"].double()
        n = h.shape[-1]
        y = h / torch.sqrt(torch.linalg.vector_norm(h, 2, -1, keepdim=True) ** 2 / n + EPS)
        y = _exact_order(y * st["weight"].double(), c, order)
        if op == "norm":
            y = y.view(*lead_out, n)
            return dict(out=y) if st["residual"] is None else dict(out=y, sum=h)
        steps = torch.linalg.vector_norm(y, float("inf"), -1, keepdim=True) / 127.0
        out = _exact_product(torch.round(y / steps), steps[:, 0], st["w"], st["w_scales"], st["bias"])
        return dict(out=out.view(*lead_out, -1), sum=h)
    if op == "norm_grad":
        h = x.double().reshape(-1, c["cols"])
        n = c["cols"]
        size = torch.sqrt(torch.linalg.vector_norm(h, 2, -1, keepdim=True) ** 2 / n + EPS)
        dy = _exact_order(st["dy"].double(), c, BACK[order])
        g = dy * st["weight"].double()
        dx = g / size - h * ((g * h).sum(-1, keepdim=True) / (n * size ** 3))
        dx = dx.view(x.shape)
        return dict(dx=dx if st["add"] is None else dx + st["add"].double(), dw=(dy * (h / size)).sum(0))
    z = _exact_product(_exact_order(x, c, order), _exact_order(st["x_scales"], c, order), st["w"], st["w_scales"], st["bias"])
    if c["act"] == "silu":
        z = z * torch.sigmoid(z)
    elif c["act"] == "gelu_tanh":
        z = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    z = z.view(*lead_out, c["n_out"])
    return z if st["residual"] is None else z + st["residual"].double()
