"""The operators of the training step, stated in 64 bits with numpy.

Definitions only, on the CPU: nothing here is shared with the library, and nothing is arranged for speed.
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
ACTS = ("none", "gelu", "gelu_tanh", "silu")


# ---- checkpoints in 8 bits -----------------------------------------------------------------------------------

def mx8_encode(x: np.ndarray):
    """(codes int8 [rows, cols], scales uint8 [rows, ceil(cols / 32)]) of a matrix, one group after the other."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    codes = np.zeros((rows, cols), np.int8)
    scales = np.zeros((rows, -(-cols // GROUP)), np.uint8)
    for i in range(rows):
        for g in range(scales.shape[1]):
            part = x[i, g * GROUP:(g + 1) * GROUP]
            if not np.isfinite(part).all():
                scales[i, g] = 255
                continue
            top = np.abs(part).max()
            if top == 0:
                continue
            e = max(math.frexp(top)[1] - 1, -126)
            scales[i, g] = e + 127
            steps = np.array([math.ldexp(v, 6 - e) for v in part])
            codes[i, g * GROUP:(g + 1) * GROUP] = np.clip(np.rint(steps), -127, 127)
    return codes, scales


def mx8_steps(scales: np.ndarray, cols: int) -> np.ndarray:
    """The step of every column; NaN where a group has no values."""
    step = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 133))
    return np.repeat(step, GROUP, axis=1)[:, :cols]


def mx8_decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return codes.astype(np.float64) * mx8_steps(scales, codes.shape[1])


# ---- activations ---------------------------------------------------------------------------------------------

_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z: np.ndarray, name: str) -> np.ndarray:
    z = np.asarray(z, np.float64)
    if name == "gelu":
        return z * 0.5 * (1 + _erf(z / math.sqrt(2))) if z.size else z
    if name == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * 0.5 * (1 + np.tanh(z / 2))          # 1 / (1 + exp(-z)) without an overflow
    return z


def act_slope(z: np.ndarray, name: str) -> np.ndarray:
    z = np.asarray(z, np.float64)
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi) if z.size else z
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = np.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 0.5 * (1 + np.tanh(z / 2))
        return p + z * p * (1 - p)
    return np.ones_like(z)


def act_backward(dy, z, name: str):
    """(dz, dbias)"""
    dz = np.asarray(dy, np.float64) * act_slope(z, name)
    return dz, dz.sum(0)


# ---- layer norm ----------------------------------------------------------------------------------------------

def layernorm(x, gamma, beta, eps: float):
    """(y, mean, rstd)"""
    x = np.asarray(x, np.float64)
    mean = x.sum(1) / x.shape[1]
    centred = x - mean[:, None]
    rstd = 1 / np.sqrt((centred ** 2).sum(1) / x.shape[1] + eps)
    return centred * rstd[:, None] * gamma + beta, mean, rstd


def layernorm_backward(dy, x, mean, rstd, gamma, residual=0.0):
    """(dx, dgamma, dbeta)"""
    dy, cols = np.asarray(dy, np.float64), dy.shape[1]
    h = (np.asarray(x, np.float64) - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.sum(1, keepdims=True) / cols - h * (g * h).sum(1, keepdims=True) / cols) + residual
    return dx, (dy * h).sum(0), dy.sum(0)


# ---- products ------------------------------------------------------------------------------------------------

def matmul(a, b, bias=0.0, name: str = "none", residual=0.0):
    """(c, z)"""
    z = np.asarray(a, np.float64) @ np.asarray(b, np.float64) + bias
    return act(z, name) + residual, z
