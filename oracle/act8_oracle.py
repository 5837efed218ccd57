"""Layers on 8-bit activations (include/act8.h) in numpy float64: packing, unpacking, group normalisation forward and backward.

Written from the definitions, with no code of the GPU path.  A matrix in 8 bits: one e4m3 code per value (sign, four bits of
exponent with bias 7, three of mantissa; 0x7f and 0xff are NaN, 448 the largest) and per row and block of 128 columns a power of
two 2^(byte - 127)."""
import math

import numpy as np

BLOCK = 128

# the value of every code
_c = np.arange(256)
_e, _m = (_c >> 3) & 15, _c & 7
CODE = np.where(_e > 0, (1 + _m / 8.0) * 2.0 ** (_e - 7.0), _m * 2.0 ** -9.0) * np.where(_c < 128, 1.0, -1.0)
CODE[[0x7f, 0xff]] = np.nan
_POS = CODE[:0x7f]      # ascending


def scale_byte(block):
    """Of one row's block: the smallest power of two that brings the largest finite magnitude to 448 or less."""
    f = np.abs(block[np.isfinite(block)])
    top = f.max() if f.size else 0.0
    if top == 0.0:
        return 127
    e = -127
    if top > 448.0 * 2.0 ** -127:
        e = math.ceil(math.log2(top / 448.0))
        while top > 448.0 * 2.0 ** e:
            e += 1
        while e > -127 and top <= 448.0 * 2.0 ** (e - 1):
            e -= 1
    return e + 127


def code_of(v):
    """Nearest code of each value (|v| <= 448), ties to the code with an even mantissa; NaN for what is not finite."""
    v = np.asarray(v, np.float64)
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, len(_POS) - 1)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    c = c + 128 * np.signbit(v)
    return np.where(np.isfinite(v), c, 0x7f).astype(np.uint8)


def pack(x):
    """codes [rows, columns rounded up to 16], scale bytes [rows, blocks]"""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    codes = np.zeros((rows, -(-cols // 16) * 16), np.uint8)
    scales = np.zeros((rows, nb), np.uint8)
    for r in range(rows):
        for b in range(nb):
            blk = x[r, b * BLOCK:(b + 1) * BLOCK]
            s = scale_byte(blk)
            scales[r, b] = s
            codes[r, b * BLOCK:b * BLOCK + blk.size] = code_of(blk * 2.0 ** (127 - s))
    return codes, scales


def unpack(codes, scales, cols):
    return CODE[codes[:, :cols]] * np.repeat(2.0 ** (scales.astype(np.float64) - 127), BLOCK, 1)[:, :cols]


def _erf(x):
    from scipy.special import erf
    return erf(x)


def act(u, kind):
    if kind == "relu":
        return np.where(u > 0, u, 0.0)
    if kind == "silu":
        return u / (1 + np.exp(-u))
    if kind == "gelu":
        return 0.5 * u * (1 + _erf(u / math.sqrt(2)))
    return u


def act_slope(u, kind):
    if kind == "relu":
        return (u > 0).astype(np.float64)
    if kind == "silu":
        s = 1 / (1 + np.exp(-u))
        return s + u * s * (1 - s)
    if kind == "gelu":
        return 0.5 * (1 + _erf(u / math.sqrt(2))) + u * np.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(u)


def _wide(v, per):
    return np.repeat(v, per, 1)[:, None, :]


def _means(v, groups):
    n, hw, c = v.shape
    return v.sum(1).reshape(n, groups, c // groups).sum(2) / (hw * (c // groups))


def statistics(x, groups, eps):
    per = x.shape[2] // groups
    mean = _means(x, groups)
    var = _means((x - _wide(mean, per)) ** 2, groups)
    return mean, 1 / np.sqrt(var + eps)


def before_act(x, gamma, beta, mean, rstd, residual=None):
    per = x.shape[2] // mean.shape[1]
    xhat = (x - _wide(mean, per)) * _wide(rstd, per)
    u = xhat * gamma + beta
    return xhat, u if residual is None else u + residual


def group_norm_bwd(dy, x, gamma, beta, mean, rstd, kind, residual=None):
    """dx, dresidual, dgamma, dbeta"""
    groups = mean.shape[1]
    per = x.shape[2] // groups
    xhat, u = before_act(x, gamma, beta, mean, rstd, residual)
    du = dy * act_slope(u, kind)
    t = du * gamma
    dx = _wide(rstd, per) * (t - _wide(_means(t, groups), per) - xhat * _wide(_means(t * xhat, groups), per))
    return dx, du, (du * xhat).sum((0, 1)), du.sum((0, 1))
