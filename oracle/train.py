"""The training step around the codec: embedding lookup and gradient, gradient
norm, AdamW with float32 and 8-bit moments.

Sums are float64.  AdamW's moments and codes round once per float32 operation,
as the step's contract has it, so they are comparable bit for bit;
:func:`adamw_formula` is the step in float64 throughout.

Pins (``tests/test_oracle_train.py``): the lookup's gradient against one-hot
products and finite differences, one AdamW step against the closed form of the
first step, the block rounding against enumeration of E4M3's grid and its mean
over all 2^16 random numbers.
"""

from __future__ import annotations

import numpy as np

from . import e4m3
from .subspace import philox4x32_10

BLOCK = 256
GROUP = 512
F = np.float32


def to_bf16(x: np.ndarray) -> np.ndarray:
    """float32 -> bfloat16 bit patterns (uint16), to nearest even."""
    u = np.ascontiguousarray(x, F).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), ((u >> 16) | 0x40).astype(np.uint16), r)


def lookup(table: np.ndarray, tokens: np.ndarray, scale: float = 1.0) -> np.ndarray:
    """float32 ``scale * table[tokens]``; zeros for ids outside the table."""
    V = table.shape[0]
    inside = (tokens >= 0) & (tokens < V)
    rows = table.astype(F)[np.where(inside, tokens, 0)] * F(scale)
    return np.where(inside[..., None], rows, F(0))


def lookup_grad(tokens: np.ndarray, dout: np.ndarray, V: int, scale: float = 1.0) -> np.ndarray:
    """float64 gradient ``[N, V, d]`` of the lookup of every rank."""
    N, T, d = dout.shape
    out = np.zeros((N, V, d))
    for j in range(N):
        inside = (tokens[j] >= 0) & (tokens[j] < V)
        np.add.at(out[j], tokens[j][inside], dout[j][inside].astype(np.float64))
    return out * float(scale)


def grad_norm(grads, max_norm: float = np.inf):
    """``(norm, clip coefficient)`` in float64."""
    norm = np.sqrt(sum((np.asarray(g, np.float64) ** 2).sum() for g in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else np.nan


def random_numbers(n: int, tensor: int, step: int, seed: int) -> np.ndarray:
    """The 16-bit number of each of a tensor's n elements in one step."""
    e = np.arange(n)
    u = e % GROUP
    call = (e // GROUP) * 64 + (u % BLOCK) // 4
    words = np.stack(philox4x32_10(call & 0xFFFFFFFF, call >> 32, np.full(n, tensor), np.full(n, step & 0xFFFFFFFF),
                                   seed & 0xFFFFFFFF, seed >> 32))
    word = words[2 * (u // BLOCK) + (u % 4) // 2, e].astype(np.uint32)
    return np.where(e % 2 == 0, word & 0xFFFF, word >> 16).astype(np.int64)


def block_maxima(x: np.ndarray) -> np.ndarray:
    """Largest magnitude of every 256 elements (NaN where one is)."""
    pad = np.zeros(-x.size % BLOCK, F)
    return np.abs(np.concatenate([x, pad])).reshape(-1, BLOCK).max(1)


def stochastic_codes(x: np.ndarray, r: np.ndarray, keep: bool):
    """E4M3 codes and block scales of float32 values x, rounded by the numbers r."""
    with np.errstate(all="ignore"):
        amax = block_maxima(x)
        mult = np.where(amax == 0, F(0), np.minimum(F(448) * (F(1) / amax), np.finfo(F).max)).astype(F)
        y = (x * np.repeat(mult, BLOCK)[:x.size]).astype(F)
        a = np.abs(y)
        # below 2^-6 (grid step 2^-9) y + 2^-6, rounded to float32, stands for y
        low = a < F(2.0 ** -6)
        t = np.where(low, a + F(2.0 ** -6), a).astype(np.float64)
        step = 2.0 ** (np.floor(np.log2(np.where(np.isfinite(t) & (t > 0), t, 1.0))) - 3)
        below = np.floor(t / step)
        q = (below + (t / step - below + (r + 0.5) / 65536 >= 1)) * step - np.where(low, 2.0 ** -6, 0.0)
        q = np.minimum(q, 448.0)
        if keep:
            q = np.where((q == 0) & (a > 0), 2.0 ** -9, q)
        q = np.where(np.isnan(y), np.nan, np.copysign(q, y))
    return e4m3.quantize(q.astype(F)), (amax * (F(1) / F(448))).astype(F)


def decode_moment(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """float32 values of codes under their blocks' scales."""
    with np.errstate(all="ignore"):
        return (e4m3.dequantize(codes).astype(F) * np.repeat(scales, BLOCK)[:codes.size]).astype(F)


def adamw_moments(m, v, g, beta1, beta2, grad_scale=1.0):
    """The new float32 moments."""
    with np.errstate(all="ignore"):
        g = g.astype(F) * F(grad_scale)
        m = m * F(beta1) + g * F(1 - beta1)
        v = v * F(beta2) + (g * g) * F(1 - beta2)
    return m, v


def adamw_param(p, m, v, lr, beta1, beta2, eps, weight_decay, step):
    """The new float32 parameters from the new moments."""
    c1, c2 = 1.0 - beta1 ** step, 1.0 - beta2 ** step
    with np.errstate(all="ignore"):
        update = m / (np.sqrt(v) * F(1 / np.sqrt(c2)) + F(eps))
        return p * F(1 - lr * weight_decay) - update * F(lr / c1)


def adamw_formula(p, m, v, g, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """One step in float64: ``(p, m, v)``."""
    p, m, v, g = (np.asarray(x, np.float64) for x in (p, m, v, g))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p * (1 - lr * weight_decay) - lr * mh / (np.sqrt(vh) + eps), m, v
