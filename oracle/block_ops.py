"""The steps around the linears of a block, in float64 from their definitions: 8-bit activation checkpoints, layer norm, SwiGLU."""
from __future__ import annotations

import numpy as np

GROUP = 32


def e4m3_magnitudes() -> np.ndarray:
    """The 127 non-negative E4M3 values, in order of their codes."""
    code = np.arange(127)
    field, mantissa = code >> 3, code & 7
    return np.where(field > 0, np.ldexp(1 + mantissa / 8, np.maximum(field, 1) - 7), np.ldexp(mantissa / 8, -6))


def _group_exponent(a: float) -> int:
    """The smallest integer e >= -117 with a <= 448 * 2^e, by trying."""
    e = -117
    while a > np.ldexp(448.0, e):
        e += 1
    return e


def ckpt8(x: np.ndarray):
    """(codes [R, ld], scale bytes [R, ld / 32], values [R, K]) of a matrix, every code by comparison with all E4M3 values."""
    x = np.asarray(x, dtype=np.float64)
    R, K = x.shape
    ld = -(-K // GROUP) * GROUP
    wide = np.zeros((R, ld))
    wide[:, :K] = x
    groups = wide.reshape(R, ld // GROUP, GROUP)
    finite = np.where(np.isfinite(groups), np.abs(groups), 0.0)
    e = np.vectorize(_group_exponent, otypes=[np.int64])(finite.max(2))
    y = finite / np.ldexp(1.0, e)[..., None]
    table = e4m3_magnitudes()
    hi = np.minimum(np.searchsorted(table, y, side="left"), 126)
    lo = np.maximum(hi - 1, 0)
    down, up = y - table[lo], table[hi] - y
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi))) | np.signbit(groups).astype(np.int64) << 7
    value = np.where(code < 128, 1.0, -1.0) * table[code & 127] * np.ldexp(1.0, e)[..., None]
    bad = ~np.isfinite(groups)
    value[bad] = np.nan
    code = np.where(bad, 0x7F, code)
    return code.reshape(R, ld).astype(np.uint8), (e + 127).astype(np.uint8), value.reshape(R, ld)[:, :K]


def layernorm(x, gamma, beta, eps):
    """(y, mean [T, 1], r [T, 1])."""
    mean = x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * r * gamma + (0.0 if beta is None else beta), mean, r


def layernorm_bwd(dy, x, mean, r, gamma):
    """(dx, dgamma, dbeta); x may be the checkpoint's values."""
    xh, h = (x - mean) * r, dy * gamma
    dx = r * (h - h.mean(1, keepdims=True) - xh * (h * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0, e) / (1 + e)


def swiglu(g, u):
    return g * _sigmoid(g) * u


def swiglu_bwd(dh, g, u):
    """(dg, du); 1 - sigmoid(g) is sigmoid(-g)."""
    s = _sigmoid(g)
    return dh * u * s * (1 + g * _sigmoid(-g)), dh * g * s
