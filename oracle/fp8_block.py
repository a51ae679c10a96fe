"""The linear layer in 8-bit floating point with a scale for each block of 128, its gradients, and the layer norm with its
gradient, from their formulas (numpy, 64 bits).  Test infrastructure only.
"""
from __future__ import annotations

import math

import numpy as np

from .linear_block import activation, epilogue  # noqa: F401  (the formulas are the int8 layer's)

G = 128


def e4m3_values():
    """The 127 numbers of either sign that an e4m3 code can stand for, by code 0..126."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))


def encode(v):
    """e4m3 codes (uint8) of fp64 values: the nearest number, ties to the even code; NaN, and what rounds beyond 448, is NaN."""
    v = np.asarray(v, np.float64)
    table = e4m3_values()
    mag = np.abs(v)
    hi = np.searchsorted(table, mag).clip(1, 126)
    lo = hi - 1
    down, up = mag - table[lo], table[hi] - mag
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(mag >= 464.0 + (mag == 464.0) * 1.0, 127, code)   # (464, the middle to the next step, is a tie to even: 448)
    code = np.where(np.isnan(v), 127, code)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def decode(codes):
    codes = np.asarray(codes, np.uint8)
    table = np.concatenate([e4m3_values(), [math.nan]])
    v = table[codes & 127]
    return np.where(codes & 128, -v, v)


def pow2_scale(top):
    """The smallest power of two s >= 2^-126 with top <= 448 s (an infinite top: that of the largest finite number)."""
    top = np.minimum(np.asarray(top, np.float64), np.float64(np.finfo(np.float32).max))
    s = np.full(top.shape, 2.0 ** -126)
    for e in range(-125, 121):
        s = np.where(top > 448.0 * s, 2.0 ** e, s)
    return s


def _top(v, axis):
    a = np.abs(np.asarray(v, np.float64))
    return np.where(np.isnan(a), 0.0, a).max(axis=axis)


def quantize_rows(v):
    """(codes uint8 [R][groups 128], scales fp64 [R][groups]) of rows, a last group filled up with zeros."""
    v = np.asarray(v, np.float64)
    R, C = v.shape
    p = np.zeros((R, -(-C // G) * G))
    p[:, :C] = v
    p = p.reshape(R, -1, G)
    s = pow2_scale(_top(p, 2))
    return encode(p / s[..., None]).reshape(R, -1), s


def row_values(codes, scales, C):
    """What codes and scales stand for, [R][C]."""
    R, groups = scales.shape
    return (decode(codes).reshape(R, groups, G) * np.asarray(scales, np.float64)[..., None]).reshape(R, -1)[:, :C]


def through(v):
    """v as the products see it."""
    return row_values(*quantize_rows(v), np.shape(v)[1])


def quantize_blocks(w):
    """(codes [Cout][Cin], scales [out blocks][in blocks]) of weights."""
    w = np.asarray(w, np.float64)
    O, C = w.shape
    s = np.empty((-(-O // G), -(-C // G)))
    codes = np.empty((O, C), np.uint8)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            b = w[i * G:(i + 1) * G, j * G:(j + 1) * G]
            s[i, j] = pow2_scale(_top(b, None))
            codes[i * G:(i + 1) * G, j * G:(j + 1) * G] = encode(b / s[i, j])
    return codes, s


def block_values(codes, scales):
    O, C = codes.shape
    return decode(codes) * np.repeat(np.repeat(np.asarray(scales, np.float64), G, 0)[:O], G, 1)[:, :C]


def product(rows, weights, bias):
    """(z, S): z = bias + rows weights^T, S = |bias| + the sum of the terms' magnitudes."""
    b = np.zeros(weights.shape[0]) if bias is None else np.asarray(bias, np.float64)
    return b + rows @ weights.T, np.abs(b) + np.abs(rows) @ np.abs(weights).T


def slope(z, act: str):
    """The activation's derivative; relu's at 0 is 0."""
    z = np.asarray(z, np.float64)
    if act == "none":
        return np.ones_like(z)
    if act == "relu":
        return (z > 0).astype(np.float64)
    with np.errstate(over="ignore"):
        if act == "gelu":
            return 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-z / math.sqrt(2.0)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        k = math.sqrt(2.0 / math.pi)
        u, du = (z, 1.0) if act == "silu" else (2 * k * (z + 0.044715 * z ** 3), 2 * k * (1 + 3 * 0.044715 * z * z))
        s, c = 1.0 / (1.0 + np.exp(-u)), 1.0 / (1.0 + np.exp(u))
        return s + z * s * c * du


def gate_grad(dy, z, act: str, gated: bool):
    """dz from the gradient of y and the values before the activation."""
    dy = np.asarray(dy, np.float64)
    if gated:
        F = np.shape(z)[1] // 2
        g, u = np.asarray(z[:, :F], np.float64), np.asarray(z[:, F:], np.float64)
        return np.concatenate([dy * u * slope(g, act), dy * activation(g, act)], axis=1)
    return dy if act == "none" else dy * slope(z, act)


def layer_norm(x, residual, gamma, beta, eps: float):
    """(h, v), both fp32: h = x + residual, v = fl(fl(fl(o r) gamma) + beta), o = fl(h - mean), r = fl(1 / sqrt(var + eps)), mean and
    variance exactly rounded to 64 bits."""
    h = np.asarray(x, np.float32) if residual is None else np.asarray(x, np.float32) + np.asarray(residual, np.float32)
    o, r = centred(h, eps)
    v = o * r
    if gamma is not None:
        v = v * np.asarray(gamma, np.float32)
    return h, (v if beta is None else v + np.asarray(beta, np.float32))


def centred(h, eps: float):
    """(o, r), fp32."""
    wide = np.asarray(h, np.float64)
    C = wide.shape[1]
    mean = np.array([math.fsum(row) / C for row in wide])
    off = wide - mean[:, None]
    var = np.array([math.fsum(row * row) / C for row in off])
    return off.astype(np.float32), (1.0 / np.sqrt(var + eps)).astype(np.float32)[:, None]


def layer_norm_grad(dy, h, gamma, residual_grad, eps: float):
    """(dx, dgamma, dbeta) in 64 bits."""
    dy, h = np.asarray(dy, np.float64), np.asarray(h, np.float64)
    off = h - h.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt((off * off).mean(axis=1, keepdims=True) + eps)
    n = off * r
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = r * (g - g.mean(axis=1, keepdims=True) - n * (g * n).mean(axis=1, keepdims=True))
    if residual_grad is not None:
        dx = dx + np.asarray(residual_grad, np.float64)
    return dx, (dy * n).sum(axis=0), dy.sum(axis=0)
