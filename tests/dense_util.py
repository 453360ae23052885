"""Helpers of the GPU tests of group norm and of the 4-bit operators: device arrays, and the error bounds.

u = 2^-24 is half a unit of fp32, h(T) half a unit of the output's type relative to the value (bf16 2^-8, fp16 2^-11).
Sums: a value is added at most 64 times on its way to a total (16 in a thread's registers, 5 + 5 across lanes, up to 16 rows of
shared memory per lane, 8 blocks of a cluster; chunks are united in fewer steps), so a sum is off by at most 64 u times the
sum of magnitudes."""
from __future__ import annotations

import numpy as np

U, D = 2.0 ** -24, 64
HALF = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}     # half the smallest number


def types(alcs):
    import torch
    return {"f32": (alcs.ALCS_F32, torch.float32), "f16": (alcs.ALCS_F16, torch.float16), "bf16": (alcs.ALCS_BF16, torch.bfloat16)}


def flags_of(alcs, act):
    return {"none": 0, "relu": alcs.ALCS_RELU, "silu": alcs.ALCS_SILU}[act]


def f64(t):
    return t.detach().double().cpu().numpy()


def _over_groups(v, groups, f):
    n, hw, c = v.shape
    r = f(v.reshape(n, hw, groups, c // groups), axis=(1, 3), keepdims=True)
    return np.broadcast_to(r, (n, hw, groups, c // groups)).reshape(n, hw, c)


def norm_bound(ref, x, gamma, beta, groups, dtype):
    """How far y may be off.  The mean is off by at most D u mean|x|, which moves xh by D u M, M = max|x| rstd; the variance, a
    sum of squares, by a relative 2 D u or so, rstd by half of that.  act has a slope of at most 1.1; exp and the quotient of SiLU are
    good to 8 u + 2 |z| u of the result."""
    m = _over_groups(np.abs(x), groups, np.max) * np.repeat(ref["rstd"], x.shape[2] // groups, axis=1)[:, None, :]
    z = D * U * (np.abs(gamma) * (np.abs(ref["xh"]) + m) + np.abs(beta))
    y = np.abs(ref["y"])
    return 1.1 * z + U * (8 + 2 * np.abs(ref["z"])) * y + HALF[dtype] * (y + 1.1 * z) + TINY[dtype]


def back_bounds(ref, x, dy, gamma, beta, groups, dtype):
    """dx, dgamma, dbeta.  With e = D u (1 + M) (1 + |gamma| + |beta|), more than xh and, through the slope of act' (at most 1/2) and exp, dz / dy are off by, every
    term of dx is off by e times itself with |dz| as |dy| and, for the product of xh and the second mean, the terms of its factors."""
    c = x.shape[2]
    r = np.repeat(ref["rstd"], c // groups, axis=1)[:, None, :]
    m = _over_groups(np.abs(x), groups, np.max) * r
    e = 2 * D * U * (1 + m) * (1 + np.abs(gamma) + np.abs(beta))
    s = np.abs(gamma * dy)
    h = np.abs(ref["xh"])
    terms = s + _over_groups(s, groups, np.mean) * (1 + h) + (1 + h) * _over_groups(s * h, groups, np.mean)
    dx = _over_groups(e, groups, np.max) * r * terms
    return (dx + HALF[dtype] * (np.abs(ref["dx"]) + dx) + TINY[dtype], (e * np.abs(dy) * (1 + h)).sum((0, 1)), (e * np.abs(dy)).sum((0, 1)))


def product_bound(scale, ref, cin, dtype):
    """Sums of 64 products at a time, exact in value, are added to fp32 sums: cin / 64 roundings, up to 8 parts of a cluster, bias and residual; a unit
    each (the hardware may cut instead of rounding), of the sum of magnitudes."""
    e = (cin / 64 + 12) * 2 * U * scale
    return e + HALF[dtype] * (np.abs(ref) + e) + TINY[dtype]
