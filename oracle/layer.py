"""Plain definitions of a layer's operators (include/pat_ops.h), in 64 bits: 8-bit blocks, root-mean-square norm, the gated
block, and their gradients.

Written from the formats' and operators' definitions; shares no code with the
library under test.
"""

import math

import numpy as np
import torch

CODES = np.array([(1 if c < 128 else -1) * ((1 + c % 8 / 8) * 2.0**(c // 8 % 16 - 7) if c // 8 % 16 else c % 8 * 2.0**-9)
                  for c in range(256)])
CODES[127] = CODES[255] = math.nan


def scale_of(high):
    """The scale byte of blocks whose largest magnitudes are `high`: the least for which none is above 3.75 units."""
    finite = np.isfinite(high)
    f, e = np.frexp(np.where(finite, high, 1.0))  # high = f 2^e, f in [1/2, 1); 3.75 = 15/16 * 2^2
    s = np.where(high == 0, 0, np.clip(e - 2 + (f > 0.9375) + 127, 0, 254))
    return np.where(finite, s, 255)


def code_of(x, scale):
    """The nearest code, ties to the even one, of values x under scale bytes (no NaN, none above 448 units)."""
    a = np.abs(x) / np.exp2(scale.astype(np.float64) - 127)
    at = np.clip(np.searchsorted(CODES[:127], a), 1, 126)
    below, above = a - CODES[at - 1], CODES[at] - a
    code = np.where((below < above) | ((below == above) & (at % 2 == 1)), at - 1, at)
    return code + 128 * np.signbit(x)


def mxb_quantize(x):
    """x [rows, cols] -> codes [rows, 128 G] and scales [rows, 4 G], uint8, filled up to whole groups of 128."""
    rows, cols = x.shape
    groups = -(-cols // 128)
    full = np.zeros((rows, 4 * groups, 32))
    full.reshape(rows, -1)[:, :cols] = x
    scale = scale_of(np.abs(full).max(axis=2, initial=0.0))
    scale = np.where(np.isnan(full).any(axis=2), 255, scale)
    good = (scale < 255)[..., None]
    codes = np.where(good, code_of(np.where(good, full, 0.0), np.where(good, scale[..., None], 127)), 0)
    return codes.reshape(rows, -1).astype(np.uint8), scale.astype(np.uint8)


def mxb_values(codes, scales, cols):
    """What a stored form stands for: float64 [rows, cols]."""
    unit = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (CODES[codes] * np.repeat(unit, 32, axis=1))[:, :cols]


def _erf(x):
    return torch.erf(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64))).numpy()


def act(a, name):
    """The activation and its derivative."""
    if name == "silu":
        s = 0.5 * (1 + np.tanh(0.5 * a))
        return a * s, s * (1 + a * (1 - s))
    p = 0.5 * (1 + _erf(a / math.sqrt(2)))
    return a * p, p + a * np.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)


def gated(a, b, name):
    return act(a, name)[0] * b


def gated_grad(g, a, b, name):
    value, slope = act(a, name)
    return np.concatenate((g * b * slope, g * value), axis=1)


def rms_norm(t, weight, eps):
    return t * weight / np.sqrt(np.mean(t * t, axis=1, keepdims=True) + eps)


def rms_norm_grad(g, t, weight, eps, total_grad=None):
    """(dx, dweight)."""
    r = 1 / np.sqrt(np.mean(t * t, axis=1, keepdims=True) + eps)
    u = g * weight
    dx = r * (u - t * r**2 * np.mean(u * t, axis=1, keepdims=True))
    return dx if total_grad is None else dx + total_grad, np.sum(g * t * r, axis=0)
