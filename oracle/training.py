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


# ---- values from 0 on in 8 bits ------------------------------------------------------------------------------

def _bits(x: np.ndarray) -> np.ndarray:
    return np.asarray(x, np.float32).view(np.uint32).astype(np.int64)


def uf8_scale(top: float) -> int:
    """The byte of a group whose largest value, a 32-bit float, is `top`."""
    return max(0, (int(_bits(np.float32(top))) >> 23) - 30)


def uf8_encode(x: np.ndarray):
    """(codes uint8 [rows, cols], scales uint8 [rows, ceil(cols / 32)]), each value rounded to the nearest code."""
    x = np.asarray(x, np.float32) + np.float32(0)
    rows, cols = x.shape
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, -(-cols // GROUP)), np.uint8)
    for i in range(rows):
        for g in range(scales.shape[1]):
            part = x[i, g * GROUP:(g + 1) * GROUP]
            if not np.isfinite(part).all() or (part < 0).any():
                scales[i, g] = 255
                continue
            s = uf8_scale(part.max())
            bits = _bits(part)
            code = ((bits + 0x7ffff + (bits >> 20 & 1)) >> 20) - 8 * s
            scales[i, g] = s
            codes[i, g * GROUP:(g + 1) * GROUP] = np.where(bits == 0, 0, np.clip(code, 1, min(255, 2039 - 8 * s)))
    return codes, scales


def uf8_decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    s = np.repeat(scales.astype(np.int64), GROUP, axis=1)[:, :codes.shape[1]]
    c = codes.astype(np.int64)
    value = ((c + 8 * np.where(s == 255, 0, s)) << 20).astype(np.uint32).view(np.float32).astype(np.float64)
    return np.where(s == 255, np.nan, np.where(c == 0, 0.0, value))


# ---- the update ----------------------------------------------------------------------------------------------

def mix(x):
    x = np.asarray(x, np.uint64) & np.uint64(0xffffffff)
    for shift, factor in ((16, 0x9E3779B9), (15, 0xBB67AE85)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xffffffff)
    return x ^ (x >> np.uint64(16))


def adamw_random(rows: int, cols: int, tensor: int, t: int, seed: int) -> np.ndarray:
    """The random number of every element, as int64 of 32 bits."""
    u = lambda v: np.uint64(v & 0xffffffff)  # noqa: E731
    key = mix(u(tensor) + mix(u(t) + mix(u(seed) ^ mix(u(seed >> 32)))))
    return mix(np.arange(rows * cols, dtype=np.uint64) + key).astype(np.int64).reshape(rows, cols)


def adamw_factor(grad_scale: float, squares=None, most_norm: float = 0.0) -> float:
    if squares is None or not most_norm:
        return grad_scale
    norm = math.sqrt(squares) * abs(grad_scale)
    return grad_scale * (most_norm / norm if norm > most_norm else 1.0)


def adamw(param, grad, m, v, t, rate, beta1, beta2, eps, factor=1.0, decay=0.0):
    """(param, m, v) after step t."""
    param, g = np.asarray(param, np.float64), np.asarray(grad, np.float64) * factor
    m = beta1 * np.asarray(m, np.float64) + (1 - beta1) * g
    v = beta2 * np.asarray(v, np.float64) + (1 - beta2) * g * g
    step = m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return param - rate * decay * param - rate * step, m, v


# ---- log probabilities ---------------------------------------------------------------------------------------

def logprobs(x, scale: float, tokens, top: int = 0):
    """A dict of logprob, largest, logsum, entropy, top_tokens, top_logprobs, and logp of every column."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    out = {"logprob": np.zeros(rows), "largest": np.zeros(rows), "logsum": np.zeros(rows), "entropy": np.zeros(rows),
           "top_tokens": np.full((rows, top), -1, np.int64), "top_logprobs": np.full((rows, top), -np.inf), "logp": np.full((rows, cols), -np.inf)}
    for i in range(rows):
        given = 0 <= tokens[i] < cols
        if np.isnan(x[i]).any() or (x[i] == np.inf).any():
            for name in ("largest", "logsum", "entropy", "top_logprobs", "logp"):
                out[name][i] = np.nan
            out["logprob"][i] = np.nan if given else 0.0
            continue
        left = np.flatnonzero(x[i] > -np.inf)
        if not left.size:
            out["largest"][i] = out["logsum"][i] = -np.inf
            out["logprob"][i] = -np.inf if given else 0.0
            continue
        out["largest"][i] = x[i].max()
        z = scale * (x[i, left] - x[i].max())
        out["logsum"][i] = math.log(np.exp(z).sum())
        logp = z - out["logsum"][i]
        out["logp"][i, left] = logp
        out["entropy"][i] = -(np.exp(logp) * logp).sum()
        out["logprob"][i] = out["logp"][i, tokens[i]] if given else 0.0
        order = left[np.lexsort((left, -x[i, left]))][:top]
        out["top_tokens"][i, :order.size] = order
        out["top_logprobs"][i, :order.size] = out["logp"][i, order]
    return out


def logprobs_backward(forward: dict, scale: float, tokens, dlogprob, dentropy) -> np.ndarray:
    logp = forward["logp"]
    rows, cols = logp.shape
    grad = np.zeros((rows, cols))
    for i in range(rows):
        a = dlogprob[i] if 0 <= tokens[i] < cols else 0.0
        if (a == 0 and dentropy[i] == 0) or forward["largest"][i] == -np.inf:
            continue
        p = np.exp(logp[i])
        flow = p * np.where(p > 0, logp[i] + forward["entropy"][i], 0.0) if not np.isnan(p).any() else p
        grad[i] = -a * p - dentropy[i] * flow
        if a:
            grad[i, tokens[i]] += a
    return scale * grad


# ---- joints --------------------------------------------------------------------------------------------------

def rstd(x, eps: float) -> np.ndarray:
    x = np.asarray(x, np.float64)
    return 1 / np.sqrt((x * x).sum(1) / x.shape[1] + eps)


def join(u, x, after, gate, keep: float, scale: float, eps: float):
    """(out, rstd_after) with out as it is before it is stored; `after`: gamma of the norm behind the block, or None."""
    v, r = np.asarray(u, np.float64), None
    if after is not None:
        r = rstd(u, eps)
        v = v * r[:, None] * after
    return keep * np.asarray(x, np.float64) + scale * gate * v, r


def join_backward(dout, dy, u, out, rstd_after, rstd_before, after, gate, before, keep: float, scale: float):
    """(du, dx, dafter, dgate, dbefore); after, before: gamma, or None where there is no norm."""
    u, cols = np.asarray(u, np.float64), u.shape[1]
    d, dbefore = np.asarray(dout, np.float64), None
    if before is not None:
        r = np.asarray(rstd_before, np.float64)[:, None]
        h, g = np.asarray(out, np.float64) * r, dy * before
        d = d + r * (g - h * (g * h).sum(1, keepdims=True) / cols)
        dbefore = (dy * h).sum(0)
    dv = scale * gate * d
    if after is None:
        return dv, keep * d, None, (scale * d * u).sum(0), dbefore
    r = np.asarray(rstd_after, np.float64)[:, None]
    k, w = u * r, dv * after
    return r * (w - k * (w * k).sum(1, keepdims=True) / cols), keep * d, (dv * k).sum(0), (scale * d * k * after).sum(0), dbefore
