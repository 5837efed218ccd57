"""What the error bounds of the oracle of include/tokens.h tell apart: mistakes planted here in numpy are outside of them (no GPU)."""
import numpy as np
import pytest

from oracle import tokens_oracle as to


@pytest.mark.parametrize("cap", [1e4, 2.0 ** 20, 2.0 ** 25])
def test_a_cap_whose_scores_lose_their_bits_is_seen(cap):
    """tanh as 1 - 2 / (1 + exp 2u) in float32 is off by units of one, so scores by units of the cap."""
    rng = np.random.default_rng(3)
    f = np.float32
    q, k, v, do = (rng.standard_normal((60, 1, 32)) for _ in range(4))
    kw = dict(scale=32 ** -0.5, cap=cap, do=do)
    half = 2.0 ** -8
    got = to.attn(q, k, v, [0, 60], [0, 60], half_step=half, operand=half, **kw)
    free = to.attn(q, k, v, [0, 60], [0, 60], half_step=half, operand=half, scale=kw["scale"], do=do)
    u = (kw["scale"] * q[:, 0] @ k[:, 0].T / cap).astype(f)
    r = f(1) / (f(1) + np.exp(f(2) * u))
    lost = cap * (1 - 2 * r.astype(np.float64))

    def outside(s):
        lse = np.log(np.exp(s).sum(1))
        return np.any(np.abs(lse - got["lse"][0]) > got["lse_off"][0])
    assert outside(lost)
    # a right one is inside, also in float32, and from some cap on it is that without a cap
    assert not outside(cap * np.tanh(u.astype(np.float64)))
    if cap >= 2.0 ** 20:
        for n in ("o", "dq", "dk", "dv"):
            assert np.all(np.abs(got[n] - free[n]) <= got[n + "_off"]), n


def _bf16(x):
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 256) / 256, e)


def _passes(q, k, v, do, starts, scale, times_q, times_k, two_terms=False):
    """The gradients as the kernels make them: delta out of an o that has been rounded, the error that this leaves taken off `times_q` times in the queries' pass
    and `times_k` times in the keys'."""
    operand = (lambda x: x) if two_terms else _bf16
    group = q.shape[1] // k.shape[1]
    o, dq, dk, dv = np.zeros_like(q), np.zeros_like(q), np.zeros_like(k), np.zeros_like(k)
    for rows, _ in to.slides(starts, starts):
        for h in range(q.shape[1]):
            a, b, c, g = q[rows, h], k[rows, h // group], v[rows, h // group], do[rows, h]
            p = np.exp(scale * a @ b.T)
            p /= p.sum(1, keepdims=True)
            o[rows, h] = _bf16(operand(p) @ c)
            ds = p * (g @ c.T - (g * o[rows, h]).sum(1, keepdims=True))
            e = ds.sum(1, keepdims=True)
            dq[rows, h] = _bf16(scale * (operand(ds) @ b - times_q * e * (_bf16(p) @ b)))
            dk[rows, h // group] += scale * operand(ds - times_k * e * p).T @ a
            dv[rows, h // group] += operand(p).T @ g
    return {"o": o, "dq": dq, "dk": _bf16(dk), "dv": _bf16(dv)}


@pytest.mark.parametrize("length,slides", [(2, 200), (7, 60)])
def test_the_size_of_roundings_tells_a_mended_gradient_from_others(length, slides):
    rng = np.random.default_rng(length)
    rows = length * slides
    starts = np.arange(0, rows + 1, length)
    q, do = (_bf16(rng.standard_normal((rows, 4, 64))) for _ in range(2))
    k, v = (_bf16(rng.standard_normal((rows, 2, 64))) for _ in range(2))
    want = to.attn(q, k, v, starts, starts, 0.125, do=do)
    every = [slice(0, rows)]

    def outside(times_q, times_k, operand=True, two_terms=False):
        got = _passes(q, k, v, do, starts, 0.125, times_q, times_k, two_terms)
        var = to.attn_spread(q, k, v, do, starts, starts, 0.125, operand=operand)
        return {n for n in got for ratio, limit in to.spread_ratios(got[n] - want[n], var[n], every) if ratio > limit}
    assert outside(1, 1) == set()
    assert outside(1, 1, operand=False, two_terms=True) == set()
    assert {"dq", "dk", "dv"} <= outside(1, 1, operand=False)         # operands of one term
    for times in (0, -1, 3):
        assert outside(times, 1) == {"dq"} and outside(1, times) == {"dk"}, times
