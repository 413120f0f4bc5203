"""The training step's operators in 64 bits on the CPU, from their definitions, and how far 32-bit sums may be from them.

Numbers that a kernel stores in T bits are rounded once, by at most half a unit of the last place: HALF_ULP of their size.  A 32-bit
sum of n terms, in whatever order, errs per addition by at most 2^-24 of the partial sum, which is at most the sum S of the terms'
sizes; the matrix units cut off where the vector units round, so 2^-23.  The errors of the additions are independent: sqrt(n) 2^-23 S is
one deviation of their sum, and tests allow four of them and eight roundings more (products, divisions, the joining of parts)."""
import numpy as np
import torch

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def sum_error(n, size):
    return (4.0 * np.sqrt(n) + 8.0) * 2.0 ** -23 * size


def stored(value, dtype):
    """What storing a number of this size as `dtype` may add to its error."""
    return HALF_ULP[dtype] * np.abs(value) + TINY[dtype]


def words(dim):
    groups = -(-dim // 32)
    return 4 * groups + -(-groups // 4)


def nearest_code(m):
    """Code of the nearest magnitude for m >= 0, halves to the even code."""
    distance = np.abs(m[..., None] - MAGNITUDES)
    best = distance.min(-1, keepdims=True)
    close = distance == best                               # one magnitude, or two neighbours
    first, last = close.argmax(-1), 7 - close[..., ::-1].argmax(-1)
    return np.where(first % 2 == 0, first, last)


def quantize(x):
    """(packed bytes uint8 [n, 4 * words], values float64 [n, dim]) of float64 rows."""
    n, dim = x.shape
    groups = -(-dim // 32)
    packed = np.zeros((n, 4 * words(dim)), dtype=np.uint8)
    values = np.zeros((n, groups * 32))
    for g in range(groups):
        v = np.zeros((n, 32))
        v[:, :min(32, dim - 32 * g)] = x[:, 32 * g:32 * g + 32]
        good = np.isfinite(v).all(1)
        top = np.where(good, np.abs(np.where(np.isfinite(v), v, 0.0)).max(1), 1.0)
        exponent = np.maximum(np.frexp(np.where(top > 0, top, 2.0 ** -200))[1] - 1 - 2, -127)
        scaled = np.where(good[:, None], np.ldexp(np.where(good[:, None], v, 0.0), -exponent[:, None]), 0.0)
        code = nearest_code(np.minimum(np.abs(scaled), 6.0)) + 8 * (np.signbit(v) & good[:, None])
        packed[:, 16 * g:16 * g + 16] = code[:, 0::2] + 16 * code[:, 1::2]
        packed[:, 16 * groups + g] = np.where(good, exponent + 127, 255)
        values[:, 32 * g:32 * g + 32] = np.where(good[:, None], np.ldexp(np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code % 8],
                                                                          exponent[:, None]), np.nan)
    return packed, values[:, :dim]


def dequantize(packed, dim):
    """float64 [n, dim] of packed bytes."""
    groups = -(-dim // 32)
    place = np.arange(dim)
    code = (packed[:, place // 2] >> (4 * (place % 2)).astype(np.uint8)) & 15
    scale = packed[:, 16 * groups + place // 32].astype(np.int64)
    value = np.ldexp(np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code % 8], scale - 127)
    return np.where(scale == 255, np.nan, value)


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def layer_norm_grad(dy, x, gamma, mean, rstd):
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def clip(tensors, max_norm):
    norm = np.sqrt(sum(float((t ** 2).sum()) for t in tensors))
    scale = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [t * scale for t in tensors]
