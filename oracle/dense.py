"""Definitions, in 64 bits, of the dense operators next to the pruned layers: group norm with an activation on
channels-last activations and its gradients, and microscaled 4-bit floating point (OCP Microscaling Formats 1.0, MXFP4):
rounding of values, and the storage format of include/alcs.h.  Plain loops over groups and blocks."""
from __future__ import annotations

import numpy as np

MX4_VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def activation(z, act):
    if act == "relu":
        return np.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1 + np.exp(-z))
    return z


def activation_slope(z, act):
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        return s + z * s * (1 - s)
    return np.ones_like(z)


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act="none"):
    """x [n, hw, c].  dict(y, mean, rstd, xh, z)."""
    x = np.asarray(x, dtype=np.float64)
    n, hw, c = x.shape
    k = c // groups
    mean, rstd, xh = np.empty((n, groups)), np.empty((n, groups)), np.empty_like(x)
    for i in range(n):
        for g in range(groups):
            v = x[i, :, g * k:(g + 1) * k]
            mean[i, g] = v.sum() / v.size
            d = v - mean[i, g]
            rstd[i, g] = 1 / np.sqrt((d * d).sum() / v.size + eps)
            xh[i, :, g * k:(g + 1) * k] = d * rstd[i, g]
    z = xh * (1.0 if gamma is None else np.asarray(gamma, np.float64)) + (0.0 if beta is None else np.asarray(beta, np.float64))
    return dict(y=activation(z, act), mean=mean, rstd=rstd, xh=xh, z=z)


def group_norm_backward(x, dy, groups, gamma=None, beta=None, eps=1e-5, act="none"):
    """dict(dx, dgamma, dbeta), and scale = |dx|'s terms, for error bounds."""
    f = group_norm(x, groups, gamma, beta, eps, act)
    n, hw, c = f["xh"].shape
    k = c // groups
    dz = np.asarray(dy, np.float64) * activation_slope(f["z"], act)
    t = dz * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    dx, scale = np.empty_like(t), np.empty_like(t)
    for i in range(n):
        for g in range(groups):
            at = (i, slice(None), slice(g * k, (g + 1) * k))
            v, h = t[at], f["xh"][at]
            dx[at] = f["rstd"][i, g] * (v - v.mean() - h * (v * h).mean())
            scale[at] = f["rstd"][i, g] * (np.abs(v) + np.abs(v).mean() + np.abs(h) * np.abs(v * h).mean())
    return dict(dx=dx, dgamma=(dz * f["xh"]).sum((0, 1)), dbeta=dz.sum((0, 1)), scale=scale,
                dgamma_scale=np.abs(dz * f["xh"]).sum((0, 1)), dbeta_scale=np.abs(dz).sum((0, 1)), **f)


def mx4_round(q):
    """Codes (0 .. 15) of finite values already divided by their scale: nearest, ties to the even code, at most 6."""
    a = np.minimum(np.abs(q), 6.0)
    hi = np.searchsorted(MX4_VALUES, a)                 # first value that is not below
    lo = np.maximum(hi - 1, 0)
    up, down = MX4_VALUES[hi] - a, a - MX4_VALUES[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code + 8 * np.signbit(q)).astype(np.uint8)


def mx4_quantize(x):
    """x [rows, cols] -> codes [rows, 32 * blocks], scale bytes [rows, blocks]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    codes, scales = np.zeros((rows, nb * 32), np.uint8), np.zeros((rows, nb), np.uint8)
    for r in range(rows):
        for b in range(nb):
            v = x[r, b * 32:(b + 1) * 32]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            m = np.abs(v).max()
            e = -127 if m == 0 else max(int(np.frexp(m)[1]) - 1 - 2, -127)
            scales[r, b] = e + 127
            codes[r, b * 32:b * 32 + v.size] = mx4_round(v / 2.0 ** e)
    return codes, scales


def mx4_values(codes, scales):
    v = MX4_VALUES[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1)


def mx4_data_index(r, b, cols):
    """Where the 16 bytes of block b of row r start."""
    return ((r // 128 * (2 * -(-cols // 64)) + b) * 128 + r % 128) * 16


def mx4_scale_index(r, b, cols):
    return (r // 128 * -(-cols // 128) + b // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + b % 4


def mx4_store(codes, scales, cols, fill=0):
    """(data, scales) as bytes; `fill` where the format leaves a byte to anything."""
    rows, nb = codes.shape[0], codes.shape[1] // 32
    kb, kq, tiles = 2 * -(-cols // 64), -(-cols // 128), -(-rows // 128)
    data = np.full(tiles * kb * 2048, fill, np.uint8)
    sc = np.full(tiles * kq * 512, fill, np.uint8)
    r = np.arange(rows)
    for b in range(kb):
        v = codes[:, b * 32:(b + 1) * 32] if b < nb else np.zeros((rows, 32), np.uint8)
        at = mx4_data_index(r, b, cols)
        data[at[:, None] + np.arange(16)] = v[:, 0::2] | (v[:, 1::2] << 4)
    for b in range(kq * 4):
        sc[mx4_scale_index(r, b, cols)] = scales[:, b] if b < nb else 0
    return data, sc


def mx4_load(data, scales, rows, cols):
    nb = -(-cols // 32)
    codes, sc = np.empty((rows, nb * 32), np.uint8), np.empty((rows, nb), np.uint8)
    r = np.arange(rows)
    for b in range(nb):
        v = data[mx4_data_index(r, b, cols)[:, None] + np.arange(16)]
        codes[:, b * 32:(b + 1) * 32:2], codes[:, b * 32 + 1:(b + 1) * 32:2] = v & 15, v >> 4
        sc[:, b] = scales[mx4_scale_index(r, b, cols)]
    return codes, sc
