"""Plain float64 forms of the root-mean-square norm, rows in 8-bit integers and their products.  Written from the formulas in include/skiparse.h."""
import numpy as np
import torch

import _block_ref as ref

F32, BF16 = ref.F32, ref.BF16
ROUND = {torch.float32: F32, torch.bfloat16: BF16}
INVS = {"same": "same", "to_sparse": "to_original", "to_original": "to_sparse"}


def norm(x, weight, residual, eps):
    """(y, h) in float64."""
    h = x.double() + (0 if residual is None else residual.double())
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return (y if weight is None else y * weight.double()), h


# Relative error of what float32 makes of a row before its last rounding: squares and sums of up to 32 + 6 + 16 terms one after the other give 55 roundings in the sum, half of that in its root; h, the
# quotient, the root and two products one each.  64 covers it with room for longer runs of sums.
ROW = 64 * F32


def norm_bound(y, dtype):
    return (ROUND[dtype] + ROW) * y.abs() + (2.0 ** -149 if dtype is torch.float32 else 2.0 ** -134)


def norm_grads(dy, h, weight, add, eps):
    """(dx, dweight, bound of dx before its rounding, bound of dweight before its rounding): everything in h's rows."""
    dy, h = dy.double(), h.double()
    w = torch.ones(h.shape[-1], dtype=torch.float64, device=h.device) if weight is None else weight.double()
    r = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    g, u = dy * w, h * r
    dx = r * (g - u * (g * u).mean(-1, keepdim=True)) + (0 if add is None else add.double())
    slack = r * (g.abs() + u.abs() * (g * u).abs().mean(-1, keepdim=True)) * 2 * ROW + F32 * dx.abs()
    terms = (dy * u).reshape(-1, h.shape[-1])
    # a sum of `rows` terms in any order is off by rows * 2^-24 of the sum of their sizes at most, the terms themselves by ROW
    return dx, terms.sum(0), slack, terms.abs().sum(0) * (ROW + F32 * terms.shape[0])


def codes(v):
    """(codes, scales) of float32 rows as the definition has them, every decision in float32 (numpy rounds each of these operations correctly)."""
    v = v.cpu().numpy().astype(np.float32)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(-1, keepdims=True)
        finite = np.isfinite(v).all(-1, keepdims=True)
        m = np.maximum(top, np.float32(2.0 ** -118))
        c = np.where(finite, np.rint(v * (np.float32(127) / m)), 0)
        scale = np.where(finite, np.where(top > 0, m / np.float32(127), np.float32(1)), np.float32("nan")).astype(np.float32)
        return torch.from_numpy(np.nan_to_num(c).astype(np.int8)), torch.from_numpy(scale[..., 0])


def linear(x, xs, w, ws, bias, residual, act):
    """(result, bound of its error before rounding) in float64; x, w int8 rows in the result's order."""
    acc = x.double() @ w.double().t()
    prod = acc * xs.double()[..., None] * ws.double()
    z = prod + (0 if bias is None else bias.double())
    y = ref.act(act, z) + (0 if residual is None else residual.double())
    # int32 -> float32, two products and a sum: four roundings; an activation's slope is at most 1.13, its own arithmetic good to 2^-19 of z
    slack = 1.2 * 4 * F32 * (prod.abs() + z.abs()) + (2.0 ** -19 * z.abs() if act != "none" else 0) + 2 * F32 * y.abs()
    return y, slack


def close(got, want, bound, what):
    got = got.double()
    assert got.isfinite().all(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), f"{what}: {float(over.max()):.3e} over its bound, {int((over > 0).sum())} of {over.numel()}"
