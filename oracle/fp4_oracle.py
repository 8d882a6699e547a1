"""Plain CPU oracle of rows held in 4 bits and of rows on their way into the
pool (slow, obvious, 64-bit).

TEST INFRASTRUCTURE, as ``entmtp_oracle``: only the tests import it, and it
shares no code with the kernels.  Every function follows the definition that
``include/entmtp.h`` gives for the entry point of the same name.
"""
from __future__ import annotations

import math

import numpy as np

from oracle import entmtp_oracle as orc

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def quantize_group(x):
    """32 numbers (64-bit) -> their codes and scale byte."""
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    m = float(np.abs(x).max())
    e = -200
    if m > 0:
        e = math.frexp(m)[1] - 1          # floor(log2 m)
        e += m >= 1.75 * 2.0 ** e
    s = min(max(e - 2 + 127, 2), 252)
    codes = []
    for v in x:
        a = abs(float(v)) / 2.0 ** (s - 127)
        far = [abs(a - level) for level in LEVELS]
        near = [k for k in range(8) if far[k] == min(far)]
        k = near[0] if len(near) == 1 else [k for k in near if k % 2 == 0][0]
        codes.append(k + 8 * (math.copysign(1.0, v) < 0))
    return np.array(codes, np.uint8), s


def quantize(x):
    """x [..., n] (64-bit) -> codes [..., n / 2] and scales [..., n / 32] bytes."""
    flat = x.reshape(-1, 32)
    codes, scales = np.zeros(flat.shape, np.uint8), np.zeros(len(flat), np.uint8)
    for i, g in enumerate(flat):
        codes[i], scales[i] = quantize_group(g)
    codes = codes[:, 0::2] | codes[:, 1::2] << 4
    return codes.reshape(*x.shape[:-1], -1), scales.reshape(*x.shape[:-1], -1)


def values(codes, scales):
    """What codes and scale bytes stand for, in 64 bits."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.array(LEVELS)[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    step = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(step, 32, -1)


def planes(pool):
    """Codes [..., page, 64] and scale bytes [..., page, 4] of 4-bit pages [..., page * 68] (copies)."""
    page = pool.shape[-1] // 68
    return (pool[..., :64 * page].reshape(*pool.shape[:-1], page, 64),
            pool[..., 64 * page:].reshape(*pool.shape[:-1], page, 4))


def join(codes, scales):
    return np.concatenate([codes.reshape(*codes.shape[:-2], -1), scales.reshape(*scales.shape[:-2], -1)], -1)


def pool_values(pool):
    """4-bit pages [..., page * 68] as numbers [..., page, 128]."""
    return values(*planes(pool))


def norm_turn(x, pos, weight, eps, theta):
    """x [H, d] of one row normed per head and turned to pos, in 64 bits."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    return orc.rope(x, pos, theta) if theta > 0 else x


def logits(hidden, codes, scales):
    return hidden @ values(codes, scales).T
