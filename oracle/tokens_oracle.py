"""Transformers over the tiles of slides in 64 bits (numpy): norm and rotation of heads, attention over packed slides, their
gradients, and how far the gradients of operands rounded on the way may be off.  Written from the formulas of include/tokens.h."""
from __future__ import annotations

import numpy as np


# ---- norm and rotation of heads ------------------------------------------------------------------

def rotation(pos, pairs, head_dim, theta):
    """cos, sin [rows, 1, head_dim / 2]; the phase is taken modulo a turn in extended precision."""
    rows, half = pos.shape[0], head_dim // 2
    phi = np.zeros((rows, half), dtype=np.longdouble)
    at = 0
    for a, n in enumerate(pairs):
        for j in range(n):
            phi[:, at + j] = pos[:, a].astype(np.longdouble) * np.longdouble(theta) ** (-np.longdouble(j) / n)
        at += n
    turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
    phi = (phi - np.floor(phi / turn) * turn).astype(np.float64)
    return np.cos(phi)[:, None], np.sin(phi)[:, None]


def columns(head_dim, pairing):
    p = np.arange(head_dim // 2)
    return (p, p + head_dim // 2) if pairing == "halves" else (2 * p, 2 * p + 1)


def turned(x, cos, sin, pairing):
    a, b = columns(x.shape[-1], pairing)
    y = np.empty_like(x)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def rope_fwd(x, gain, cos, sin, pairing, eps):
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    return turned(x, cos, sin, pairing)


def rope_bwd(dy, x, gain, cos, sin, pairing, eps):
    """dx, dgain."""
    dn = turned(dy, cos, -sin, pairing)
    if gain is None:
        return dn, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = x * r
    u = dn * gain
    return r * (u - h * (u * h).mean(-1, keepdims=True)), (dn * h).sum((0, 1))


# ---- attention ------------------------------------------------------------------------------------

def slides(q_start, k_start):
    return [(slice(q_start[i], q_start[i + 1]), slice(k_start[i], k_start[i + 1])) for i in range(len(q_start) - 1)]


def _scores(q, k, scale, cap, dist, slope):
    """Scores, and their derivative by scale q.k: 1 / cosh^2, as 1 - tanh^2 would be 0 from 19 on."""
    x = scale * (q @ k.T)
    s = cap * np.tanh(x / cap) if cap else x
    by = np.cosh(np.minimum(np.abs(x / cap), 300)) ** -2 if cap else 1.0
    return s - slope * dist if dist is not None else s, by


def _distance(pos_q, pos_k, lead_q, lead_k):
    d = np.hypot(pos_q[:, None, 0] - pos_k[None, :, 0], pos_q[:, None, 1] - pos_k[None, :, 1])
    d[:lead_q] = 0
    d[:, :lead_k] = 0
    return d


def attn(q, k, v, q_start, k_start, scale, cap=0.0, pos_q=None, pos_k=None, slopes=None, lead_q=0, lead_k=0, do=None,
         half_step=0.0, operand=0.0):
    """Outputs of the forward and, where `do` is given, the gradients; behind each name `name_off`: the bound on what comes out where
    results are rounded with `half_step` and probabilities and score gradients are rounded with `operand` before a product, both relative,
    beside float32 arithmetic.  Rows of no slide are NaN."""
    hq, hk = q.shape[1], k.shape[1]
    group = hq // hk
    out = {"o": np.full_like(q, np.nan), "lse": np.full((hq, q.shape[0]), np.nan)}
    if do is not None:
        out.update(dq=np.full_like(q, np.nan), dk=np.full_like(k, np.nan), dv=np.full_like(v, np.nan))
    out.update({n + "_off": np.full_like(a, np.nan) for n, a in list(out.items())})
    for rq, rk in slides(q_start, k_start):
        if do is not None:
            for n in ("dk", "dv", "dk_off", "dv_off"):
                out[n][rk] = 0
        dist = _distance(pos_q[rq], pos_k[rk], lead_q, lead_k) if slopes is not None else None
        for h in range(hq):
            _one(out, q[rq, h], k[rk, h // group], v[rk, h // group], None if do is None else do[rq, h], scale, cap, dist,
                 0.0 if slopes is None else slopes[h], rq, rk, h, h // group, half_step, operand)
    for n in ("dk", "dv"):
        if do is not None:
            out[n + "_off"] += half_step * np.abs(out[n])
    return out


def _one(out, q, k, v, do, scale, cap, dist, slope, rq, rk, h, hk, half_step, operand):
    n, m, dim = q.shape[0], k.shape[0], q.shape[1]
    if n == 0:
        return
    if m == 0:
        out["o"][rq, h], out["lse"][h, rq] = 0, -np.inf
        out["o_off"][rq, h] = out["lse_off"][h, rq] = 0
        if do is not None:
            out["dq"][rq, h] = out["dq_off"][rq, h] = 0
        return
    s, slope_t = _scores(q, k, scale, cap, dist, slope)
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    z = e.sum(1, keepdims=True)
    p = e / z
    lse = (top + np.log(z))[:, 0]
    o = p @ v
    # float32: a score is off by a unit (2^-24) for every product in it and a few for cap, bias, exponent and the maximum; sums of m terms
    u = 2.0 ** -24
    size = scale * (np.abs(q) @ np.abs(k).T)
    far = np.abs(slope) * dist if dist is not None else 0.0
    # tanh is right to some units of itself, but in bfloat16 up to a cap of 64, where 1 - 2 / (1 + exp 2u) is: six units of one
    one = cap if operand and cap <= 64 else 0.0
    off = u * ((dim + 8) * size + 8 * (one + np.abs(s) + far + np.abs(lse)[:, None]) + 16)     # of a score, so relative of exp(score)
    worst = off.max(1, keepdims=True)
    rel = 2 * worst + (m + 8) * u                                                             # of a probability
    # below 2^-126 there are no normal floats: a probability, a score's gradient, a product of either, a sum and a result may each be zero instead
    tiny = 2.0 ** -126
    a = p @ np.abs(v)
    o_off = half_step * np.abs(o) + (operand + rel) * a + tiny * (np.abs(v).sum(0) + m + 1)
    out["o"][rq, h], out["lse"][h, rq] = o, lse
    out["o_off"][rq, h] = o_off
    out["lse_off"][h, rq] = worst[:, 0] + u * (m + 8 + 4 * np.abs(lse))
    if do is None:
        return
    dp = do @ v.T
    delta = (do * o).sum(1, keepdims=True)
    ds = p * (dp - delta) * slope_t
    delta_off = (np.abs(do) * o_off).sum(1, keepdims=True) + dim * u * (np.abs(do) * np.abs(o)).sum(1, keepdims=True)
    dp_off = (dim + 8) * u * (np.abs(do) @ np.abs(v).T)
    # 1 - tanh^2 is off by twice the tanh's error where it is not small, relative else
    ds_off = operand * np.abs(ds) + p * ((delta_off + dp_off) * np.abs(slope_t) + (rel + 16 * u + (2 * off / cap if cap else 0.0)) * np.abs(dp - delta)) \
        + tiny * (np.abs(dp - delta) + 2)
    terms = (m + 8) * u
    out["dq"][rq, h] = scale * (ds @ k)
    out["dq_off"][rq, h] = scale * ((ds_off + terms * np.abs(ds)) @ np.abs(k)) + half_step * np.abs(out["dq"][rq, h]) \
        + tiny * (m + 1)
    terms = (n + 8) * u
    out["dk"][rk, hk] += scale * (ds.T @ q)
    out["dk_off"][rk, hk] += scale * ((ds_off + terms * np.abs(ds)).T @ np.abs(q)) + tiny * (n + 1)
    out["dv"][rk, hk] += p.T @ do
    out["dv_off"][rk, hk] += ((operand + rel + terms) * p + tiny).T @ np.abs(do) + tiny * (n + 1)


# ---- the size of bfloat16's roundings ---------------------------------------------------------------

def step_variance(x):
    """Of the error of x rounded to bfloat16: even over a step of 2^-7 of the power of two below |x|, so a twelfth of its square."""
    _, e = np.frexp(x)
    return np.where(x == 0, 0.0, np.ldexp(1.0, 2 * (e - 8)) / 12)


def attn_spread(q, k, v, do, q_start, k_start, scale, cap=0.0, pos_q=None, pos_k=None, slopes=None, lead_q=0, lead_k=0, operand=True):
    """Variances of o, dq, dk and dv in bfloat16 where nothing is rounded but the results and (`operand`) the probabilities and scores' gradients that are
    multiplied, each by itself.  Rows of no slide are 0."""
    group = q.shape[1] // k.shape[1]
    val = {"o": np.zeros_like(q), "dq": np.zeros_like(q), "dk": np.zeros_like(k), "dv": np.zeros_like(k)}
    var = {n: np.zeros_like(x) for n, x in val.items()}
    for rq, rk in slides(q_start, k_start):
        if rq.stop == rq.start or rk.stop == rk.start:
            continue
        dist = _distance(pos_q[rq], pos_k[rk], lead_q, lead_k) if slopes is not None else None
        for h in range(q.shape[1]):
            a, b, c, g = q[rq, h], k[rk, h // group], v[rk, h // group], do[rq, h]
            s, by = _scores(a, b, scale, cap, dist, 0.0 if slopes is None else slopes[h])
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o = p @ c
            ds = p * (g @ c.T - (g * o).sum(1, keepdims=True)) * by
            vp, vd = (step_variance(p), step_variance(ds)) if operand else (0 * p, 0 * p)
            val["o"][rq, h], var["o"][rq, h] = o, vp @ c ** 2
            val["dq"][rq, h], var["dq"][rq, h] = scale * ds @ b, scale ** 2 * vd @ b ** 2
            val["dk"][rk, h // group] += scale * ds.T @ a
            var["dk"][rk, h // group] += scale ** 2 * vd.T @ a ** 2
            val["dv"][rk, h // group] += p.T @ g
            var["dv"][rk, h // group] += vp.T @ g ** 2
    return {n: x + step_variance(val[n]) for n, x in var.items()}


def spread_ratios(off, var, groups):
    """For every group of rows: the norm of the errors `off` [rows, heads, dim] relative to what the variances say, and the limit of that ratio.  The square of an
    error that is even over a step is its twelfth with a relative standard deviation of 0.9; counted as one rounding a row and head, their weights being
    `var`, the group's is 0.9 / sqrt(n), n the sum's square over the sum of squares.  Five of those, and a hundredth for float32."""
    out = []
    for rows in groups:
        w = var[rows].sum(-1).ravel()
        n = w.sum() ** 2 / (w * w).sum()
        out.append((np.sqrt((off[rows] ** 2).sum() / w.sum()), np.sqrt(1 + 5 * 0.9 / np.sqrt(n)) + 0.01))
    return out
