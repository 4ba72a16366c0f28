"""Plain implementations, in 64 bits on the CPU, of a cache in 4 bits and of norms and rotations of heads."""
import math

import numpy as np
import torch

from tests.serveref import EPS

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LIMITS = {torch.bfloat16: (2, 252), torch.float16: (104, 140)}


def scale_of(m, dtype):
    """The scale byte of a block whose largest magnitude is m."""
    if not math.isfinite(m):
        return 255
    lo, hi = LIMITS[dtype]
    if m == 0:
        return lo
    f, e = math.frexp(m)                                     # m = f 2^e, 0.5 <= f < 1
    e -= 1
    if 2 * f >= 1.75:                                        # two significant bits: 1, 1.5 or up to 2
        e += 1
    return min(max(e - 2 + 127, lo), hi)


def quantize(x, dtype):
    """[..., d] -> (codes [..., d], scales [..., d / 32]), bytes as numpy arrays; of a block of NaN the codes say nothing."""
    x = x.double().numpy()
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.where(np.isnan(y).any(-1), np.inf, np.abs(np.where(np.isnan(y), 0, y)).max(-1))
    s = np.vectorize(lambda m: scale_of(float(m), dtype), otypes=[np.uint8])(top) if top.size else top.astype(np.uint8)
    unit = np.ldexp(1.0, np.where(s == 255, 127, s).astype(int) - 127)[..., None]
    a = np.abs(np.where(np.isfinite(y), y, 0)) / unit
    off = np.abs(a[..., None] - GRID)
    off[..., 1::2] *= 1 + 1e-15                              # halfway: the even code
    code = off.argmin(-1).astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)
    return code.reshape(x.shape), s


def pack(x, dtype):
    code, s = quantize(x, dtype)
    return torch.from_numpy(code[..., 0::2] | code[..., 1::2] << 4), torch.from_numpy(s)


def unpack(p, s, dtype):
    """The numbers that packed bytes and scales stand for, in the rows' type."""
    p, s = p.numpy(), s.numpy()
    code = np.stack([p & 15, p >> 4], -1).reshape(*p.shape[:-1], -1)
    x = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    unit = np.where(s == 255, np.nan, np.ldexp(1.0, s.astype(int) - 127)).repeat(32, -1)
    return torch.from_numpy(x * unit).to(dtype)


def turned(x, pos, turns, pairs, weight, eps):
    """Heads x [..., heads, d] of rows at positions pos [...], in 64 bits: normed, rotated."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    if turns is None:
        return x
    half = turns.shape[1] // 2
    inside = (pos >= 0) & (pos < turns.shape[0])
    cs = turns[pos.clamp(0, turns.shape[0] - 1)].double()
    cs = torch.where(inside[..., None], cs, math.nan)[..., None, :]
    i = torch.arange(half)
    i, j = (i, i + half) if pairs == "halves" else (2 * i, 2 * i + 1)
    y = x.clone()
    y[..., i] = x[..., i] * cs[..., :half] - x[..., j] * cs[..., half:]
    y[..., j] = x[..., i] * cs[..., half:] + x[..., j] * cs[..., :half]
    return y


def turned_error(y, dtype):
    """What such values may be off by as numbers of a type: half a step of fp32 and half a step of the type; fp16's steps are not below 2^-24."""
    return y.abs() * (EPS[dtype] * (1 + 2.0 ** -20) + 2.0 ** -24) + (2.0 ** -25 * (1 + 2.0 ** -10) if dtype is torch.float16 else 2.0 ** -126)


def turns(positions, dims, base=10000.0):
    half = dims // 2
    a = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(half, dtype=torch.float64) / half)
    return torch.cat([a.cos(), a.sin()], 1).float()
