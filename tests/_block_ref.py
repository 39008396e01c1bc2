"""Plain float64 forms of the operators round the attention: positions, checkpoints, the linear layer.  Written from the formulas in include/skiparse.h; row
orders by the oracle's index loops, not the library's."""
import functools
import math

import numpy as np
import torch

import oracle

BF16 = 2.0 ** -8    # largest relative rounding error
F32 = 2.0 ** -24
E4M3 = 2.0 ** -4


@functools.lru_cache(maxsize=64)
def _moved_rows(B, T, H, W, s, pattern, to_sparse):
    """For every destination row the source row: a tensor of row numbers through the oracle's rearrangement."""
    n = B * T * H * W
    rows = np.arange(n, dtype=np.int64).astype(np.float64)
    if to_sparse:
        x = oracle.permute(rows.reshape(B, T * H * W, 1, 1), T, H, W, s, pattern)
    else:
        x = oracle.unpermute(rows.reshape(s * s * B, T * H * W // (s * s), 1, 1), T, H, W, s, pattern)
    return torch.from_numpy(np.ascontiguousarray(x).reshape(-1).astype(np.int64))


def moved(x, order, grid, s, pattern):
    """Rows of x (any trailing shape), flattened to two leading dimensions, in the order they have on the other side."""
    B, T, H, W = grid
    rows = x.reshape(B * T * H * W, *x.shape[2:])
    if order in ("same", "stay_sparse"):
        return x
    at = _moved_rows(B, T, H, W, s, pattern, order == "to_sparse").to(x.device)
    lead = (s * s * B, T * H * W // (s * s)) if order == "to_sparse" else (B, T * H * W)
    return rows[at].reshape(*lead, *x.shape[2:])


# ---- positions

def frequencies(r, theta, scaling, factor, trained, fast=32.0, slow=1.0):
    out = []
    for j in range(r // 2):
        base = theta * factor ** (r / (r - 2)) if scaling == "ntk" and r > 2 else theta
        f = base ** (-2.0 * j / r)
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            n = trained * f / (2 * math.pi)
            g = min(1.0, max(0.0, (n - slow) / (fast - slow)))
            f = f * g + (1 - g) * f / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def table(lengths, axes, theta=10000.0, scaling="none", factor=(1.0,) * 3, trained=(0,) * 3, attention=1.0):
    parts = []
    for n, r, s, t in zip(lengths, axes, factor, trained):
        a = torch.arange(n, dtype=torch.float64)[:, None] * frequencies(r, theta, scaling, s, t)[None]
        parts.append(torch.stack((a.cos(), a.sin()), -1).reshape(-1) * attention)
    return torch.cat(parts)


def rope(x, table, lengths, axes, grid, at, layout, sign):
    """x [B][T*H*W][heads][D] float64 in the original order; table as the library lays it out, float64."""
    B, T, H, W = grid
    D, pairs = x.shape[-1], sum(axes) // 2
    y = x.clone()
    n = torch.arange(T * H * W, device=x.device)
    place = (n // (H * W) + at[0], n // W % H + at[1], n % W + at[2])
    first, i = 0, 0
    for p, length, r in zip(place, lengths, axes):
        for j in range(r // 2):
            c = table[2 * (first + p * (r // 2) + j)][None, :, None]
            s = sign * table[2 * (first + p * (r // 2) + j) + 1][None, :, None]
            a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + pairs)
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., a] * s + x[..., b] * c
            i += 1
        first += length * (r // 2)
    return y


# ---- checkpoints

def checkpoint(x):
    """(codes, scale bytes, values) of a float64 tensor [rows][cols] that holds values of bf16 or float32; a loop over nothing but blocks."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    p = torch.zeros(rows, blocks * 32, dtype=torch.float64, device=x.device)
    p[:, :cols] = x
    p = p.reshape(rows, blocks, 32)
    a = torch.where(p.isfinite(), p.abs(), 0.0).amax(-1)
    e = torch.ceil(torch.log2(torch.where(a > 0, a, 1.0) / 448.0))
    e = torch.where(448.0 * torch.exp2(e) < a, e + 1, e)
    e = torch.where((a > 0) & (448.0 * torch.exp2(e - 1) >= a), e - 1, e)
    e = torch.where(a > 0, e.clamp(-127, 127), 0.0)
    v = torch.where(p.isfinite(), p, float("nan")) * torch.exp2(-e)[..., None]
    # three bits behind the leading one, and steps of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    q = torch.round(v / step) * step
    codes = q.float().to(torch.float8_e4m3fn).view(torch.uint8)  # exact
    codes = torch.where(p.isfinite(), codes, torch.full_like(codes, 0x7f))
    values = (q * torch.exp2(e)[..., None]).reshape(rows, -1)[:, :cols]
    return codes.reshape(rows, -1)[:, :cols].contiguous(), (e + 127).to(torch.uint8), values


def values(codes, scales):
    """What a checkpoint stands for, in float64."""
    up = torch.exp2(scales.to(torch.float64) - 127).repeat_interleave(32, -1)[..., : codes.shape[-1]]
    return codes.view(torch.float8_e4m3fn).to(torch.float64) * up


# ---- linear layer

def act(name, z):
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if name == "silu" else z


def slope(name, z):
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)
