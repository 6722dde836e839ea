"""TEST INFRASTRUCTURE -- plain CPU statement of the AdamW step and of its 8-bit states; shares nothing with the CUDA path.

Moments are NumPy FP32, operation by operation, as the definition has them (every operation rounded), so that they and the codes made
of them are compared bit for bit; the parameters are FP64.  The 8-bit formats are tables of their 127 non-negative values here, and a
rounding looks up the two neighbours; the random integer decides by where the value lies between them.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
F = np.float32


def table(mantissa: int):
    """Non-negative finite values of the 8-bit float with `mantissa` mantissa bits, code by code (code 127 is NaN)."""
    bias = 7 if mantissa == 3 else 15
    c = np.arange(127)
    e, m = c >> mantissa, c & ((1 << mantissa) - 1)
    return np.where(e == 0, m * 2.0 ** (1 - bias - mantissa), (1 + m / 2.0 ** mantissa) * 2.0 ** (e - bias))


def decode(codes, scale, mantissa: int):
    """uint8 codes [n], exponent bytes [ceil(n / 32)] -> FP32."""
    values = np.append(table(mantissa), np.nan)[codes & 127] * 2.0 ** (np.repeat(scale, GROUP)[:codes.size].astype(np.float64) - 127.0)
    values = np.where((codes & 127) == 0, 0.0, values)
    return np.where(codes & 128, -values, values).astype(F)


def encode(v, mantissa: int, noise):
    """FP32 [n] -> (codes, exponent bytes); noise: integers in [0, 2^16) or None (to nearest, ties to even)."""
    n = v.size
    top = 7 if mantissa == 3 else 14
    size = np.abs(np.append(v, np.zeros(-n % GROUP, F)).astype(np.float64)).reshape(-1, GROUP)
    most = np.where(np.isfinite(size), size, 0.0).max(axis=1)
    floor_log2 = np.where(most >= 2.0 ** -126, np.frexp(np.maximum(most, 2.0 ** -126))[1] - 1, -127)
    scale = np.maximum(floor_log2 + 127 - top, 1).astype(np.uint8)
    fine = np.isfinite(size)
    y = np.where(fine, size, 0.0) * 2.0 ** (127.0 - scale.astype(np.float64))[:, None]      # exact: at most 2^15
    t = table(mantissa)
    lo = np.searchsorted(t, y, side="right") - 1
    part = (y - t[lo]) / (t[np.minimum(lo + 1, 126)] - t[lo] + (lo == 126))
    if noise is None:
        up = (part > 0.5) | ((part == 0.5) & (lo % 2 == 1))
    else:
        r = np.append(noise, np.zeros(-n % GROUP, np.int64)).reshape(part.shape)
        # the value's place between its neighbours in 2^-(23 - mantissa) of their distance (exact but for subnormal codes) plus the
        # noise, which has 16 bits and stands in the middle of what they leave open
        low = np.rint(part * 2.0 ** (23 - mantissa))
        up = low + r * 2.0 ** (7 - mantissa) + 2.0 ** (6 - mantissa) >= 2.0 ** (23 - mantissa)
    code = np.where(fine, lo + up, 127).reshape(-1)[:n].astype(np.uint8) | (np.signbit(v).astype(np.uint8) << 7)
    return code, scale


def mix(x):
    """The published 32-bit mixer lowbias32 (C. Wellons' hash-prospector): two products, three shifts."""
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    w = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x7FEB352D)) & w
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x846CA68B)) & w
    return x ^ (x >> np.uint64(16))


def noise(seed: int, step: int, tensor: int, index):
    """32 random bits for each element `index` of a tensor."""
    h = np.uint64(0)
    for word in (seed & 0xFFFFFFFF, seed >> 32, step & 0xFFFFFFFF, step >> 32, tensor):
        h = mix(h ^ np.uint64((word + 0x9E3779B9) & 0xFFFFFFFF))
    index = np.asarray(index, np.uint64)
    high = index >> np.uint64(32)
    h = np.where(high > 0, mix(h ^ high), h)
    return mix(h ^ (index & np.uint64(0xFFFFFFFF))).astype(np.int64)


def moments(m, v, g, beta1: float, beta2: float):
    """FP32 arrays -> the new m, v, every operation rounded."""
    with np.errstate(invalid="ignore", over="ignore"):
        return m * F(beta1) + g * F(1.0 - beta1), v * F(beta2) + g * g * F(1.0 - beta2)


def parameters(p, m, v, t: int, lr, beta1, beta2, eps, decay):
    """FP64 -> (new p, size of the update's parts)."""
    denom = np.sqrt(v) / np.sqrt(1.0 - beta2 ** t) + eps
    step = lr / (1.0 - beta1 ** t) / denom
    return p * (1.0 - lr * decay) - step * m, np.abs(step)


def bf16_by_chance(p, bits):
    """FP32 -> BF16 as FP32, rounded by 16 random bits."""
    b = p.view(np.uint32).astype(np.uint64) + bits.astype(np.uint64)
    return (b >> np.uint64(16) << np.uint64(16)).astype(np.uint32).view(np.float32)
