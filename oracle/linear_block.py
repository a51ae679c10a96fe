"""What stands around a quantized linear layer: the norm in front of it and the epilogue behind it, from
their formulas (numpy; the quantizer is the oracle's).  Test infrastructure only.
"""
from __future__ import annotations

import math

import numpy as np

from . import _f32, quantize_pixels


def rms_norm(x, residual, gamma, eps: float):
    """(h, v), both fp32: h = x + residual, v = fl(fl(h rho) gamma) with rho = fl(1 / sqrt(mean(h^2) + eps)), the mean in
    64 bits.  x, residual: fp32 arrays (values of a narrower type are fp32 numbers too)."""
    h = _f32(x) if residual is None else _f32(x) + _f32(residual)
    wide = h.astype(np.float64)
    squares = np.array([math.fsum(r * r) for r in wide])   # the exact products' exactly rounded sum
    rho = (1.0 / np.sqrt(squares / h.shape[1] + eps)).astype(np.float32)
    v = h * rho[:, None]
    return h, (v if gamma is None else v * _f32(gamma))


def rms_norm_quantize(x, residual, gamma, eps: float, g: int):
    """(h, codes [rows][C] int8, scales [rows][groups] fp32)"""
    h, v = rms_norm(x, residual, gamma, eps)
    return (h, *quantize_pixels(v, g))


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activation(z, act: str):
    z = np.asarray(z, np.float64)
    if act == "none":
        return z
    if act == "relu":
        return np.maximum(z, 0.0)
    if act == "gelu":
        return 0.5 * z * _erfc(-z / math.sqrt(2.0))
    u = z if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)
    with np.errstate(over="ignore"):
        return z / (1.0 + np.exp(-u))


def product(xq, sx, wq, sw, bias, g: int):
    """(z, S) in fp64: z = bias + sum over groups of sx sw P, S = |bias| + the sum of the terms' magnitudes.
    xq [R][C], sx [R][groups], wq [Cout][C], sw [groups][Cout]."""
    R, C = xq.shape
    b = np.zeros(wq.shape[0]) if bias is None else np.asarray(bias, np.float64)
    z, S = np.tile(b, (R, 1)), np.tile(np.abs(b), (R, 1))
    for k in range(C // g):
        P = xq[:, k * g:(k + 1) * g].astype(np.float64) @ wq[:, k * g:(k + 1) * g].astype(np.float64).T
        t = P * sx[:, k, None].astype(np.float64) * sw[None, k].astype(np.float64)
        z += t
        S += np.abs(t)
    return z, S


def epilogue(z, act: str, gated: bool, residual):
    if gated:
        F = z.shape[1] // 2
        y = activation(z[:, :F], act) * z[:, F:]
    else:
        y = activation(z, act)
    return y if residual is None else y + np.asarray(residual, np.float64)


def epilogue_bound(z, S, groups: int, act: str, gated: bool, residual, half_step: float):
    """How far an fp32 evaluation with `groups` terms, rounded once to a type with relative half step `half_step`, may be
    from epilogue().  u = 2^-24 is the half step of fp32.
      sums: a term is an exact integer times a rounded product of scales (1 u), added with one rounding each; up to 16 partial
        sums are added behind that, and the bias: (groups + 18) u S;
      activations: slopes are at most 1.13 (gelu); expf, erfcf and their arguments are off by a few u, and z times the
        change of 1 / (1 + e^-a) or erfc by a few u of its argument is at most a few u in absolute terms, because
        z^2 sigma (1 - sigma) < 0.5 and gelu_tanh's argument grows with z^3 only where sigma (1 - sigma) has vanished:
        16 u (|y| + 1);
      gate, residual, the result: one rounding each."""
    u = 2.0 ** -24
    e = (groups + 18) * u * S

    def through(t, et):
        return et if act in ("none", "relu") else 1.13 * et + 16 * u * (np.abs(activation(t, act)) + 1.0)

    if gated:
        F = z.shape[1] // 2
        a, up = activation(z[:, :F], act), z[:, F:]
        ea, eu = through(z[:, :F], e[:, :F]), e[:, F:]
        y = a * up
        ey = np.abs(a) * eu + np.abs(up) * ea + ea * eu + u * (np.abs(y))
    else:
        y = activation(z, act)
        ey = through(z, e)
    if residual is not None:
        y = y + np.asarray(residual, np.float64)
        ey = ey + u * np.abs(y)
    return ey * 1.01 + half_step * (np.abs(y) + ey)
