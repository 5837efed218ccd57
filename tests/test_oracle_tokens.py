"""The oracle of include/tokens.h: its gradients against differences of its own forward, and what its rotation and masks keep (no GPU)."""
import numpy as np
import pytest

from oracle import tokens_oracle as to


def _difference(f, x, at, h=1e-5):
    x = x.copy()
    old = x[at]
    x[at] = old + h
    a = f(x)
    x[at] = old - h
    return (a - f(x)) / (2 * h)


@pytest.mark.parametrize("cap,bias,lead", [(0.0, False, 0), (3.0, True, 1), (0.0, True, 2), (1.0, False, 0)])
def test_attention_gradients_are_the_forwards_differences(cap, bias, lead):
    rng = np.random.default_rng(5)
    qs, ks = [0, 3, 3, 8], [1, 6, 8, 8]     # one slide without queries, one without keys, a row of no slide in front
    q, do = rng.standard_normal((8, 4, 6)), rng.standard_normal((8, 4, 6))
    k, v = rng.standard_normal((8, 2, 6)), rng.standard_normal((8, 2, 6))
    kw = dict(scale=0.4, cap=cap, lead_q=lead, lead_k=lead)
    if bias:
        kw.update(pos_q=rng.uniform(0, 9, (8, 2)), pos_k=rng.uniform(0, 9, (8, 2)), slopes=np.array([0.5, 0.1, 0.3, 0.0]))
    got = to.attn(q, k, v, qs, ks, do=do, **kw)
    assert np.all(got["o"][3:] == 0) and np.all(got["lse"][:, 3:] == -np.inf) and np.all(got["dq"][3:] == 0)
    assert np.all(np.isnan(got["dk"][0])) and np.all(got["dk"][6:] == 0) and np.all(got["dv"][6:] == 0)

    def loss(q, k, v):
        return float((to.attn(q, k, v, qs, ks, **kw)["o"] * do).sum())
    for i in range(30):
        r, c = rng.integers(0, 3), rng.integers(0, 6)
        at = (r, rng.integers(0, 4), c)
        assert abs(_difference(lambda x: loss(x, k, v), q, at) - got["dq"][at]) < 1e-8
        at = (1 + rng.integers(0, 5), rng.integers(0, 2), c)
        assert abs(_difference(lambda x: loss(q, x, v), k, at) - got["dk"][at]) < 1e-8
        assert abs(_difference(lambda x: loss(q, k, x), v, at) - got["dv"][at]) < 1e-8


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_rope_gradients_are_the_forwards_differences(pairing):
    rng = np.random.default_rng(6)
    x, dy, gain = rng.standard_normal((4, 3, 16)), rng.standard_normal((4, 3, 16)), rng.standard_normal(16)
    c, s = to.rotation(rng.integers(-50, 50, (4, 2)), (3, 4), 16, 100.0)
    dx, dg = to.rope_bwd(dy, x, gain, c, s, pairing, 1e-6)
    for i in range(30):
        at = tuple(rng.integers(0, n) for n in x.shape)
        assert abs(_difference(lambda v: float((to.rope_fwd(v, gain, c, s, pairing, 1e-6) * dy).sum()), x, at) - dx[at]) < 1e-8
        assert abs(_difference(lambda v: float((to.rope_fwd(x, v, c, s, pairing, 1e-6) * dy).sum()), gain, at[2]) - dg[at[2]]) < 1e-8


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_rotated_products_depend_on_the_difference_of_positions(pairing):
    rng = np.random.default_rng(7)
    a, b = rng.standard_normal((1, 1, 32)), rng.standard_normal((1, 1, 32))
    pos = np.array([[3, -7], [40, 2]])

    def product(shift):
        c, s = to.rotation(pos + shift, (8, 6), 32, 50.0)
        return float((to.turned(a, c[:1], s[:1], pairing) * to.turned(b, c[1:], s[1:], pairing)).sum())
    assert abs(product(np.array([100000, -23456])) - product(0)) < 1e-9
    c, s = to.rotation(pos, (8, 6), 32, 50.0)
    first, second = to.columns(32, pairing)
    y = to.turned(a, c[:1], s[:1], pairing)
    assert np.array_equal(y[..., first[14:]], a[..., first[14:]]) and np.array_equal(y[..., second[14:]], a[..., second[14:]])


def test_bounds_hold_for_rounded_operands():
    """Probabilities and score gradients rounded to 8 bits of mantissa, as the kernels' operands are, stay within the bounds."""
    rng = np.random.default_rng(8)

    def rounded(x):
        m, e = np.frexp(x)
        return np.ldexp(np.round(m * 256) / 256, e)
    q, k, v, do = (rng.standard_normal((40, 1, 16)) for _ in range(4))
    got = to.attn(q, k, v, [0, 40], [0, 40], 0.25, do=do, half_step=2.0 ** -8, operand=2.0 ** -8)
    s = 0.25 * q[:, 0] @ k[:, 0].T
    e = np.exp(s - s.max(1, keepdims=True))
    o = rounded(rounded(e) @ v[:, 0] / e.sum(1, keepdims=True))
    p = e / e.sum(1, keepdims=True)
    ds = rounded(p * (do[:, 0] @ v[:, 0].T - (do[:, 0] * o).sum(1, keepdims=True)))
    for name, x in (("o", o), ("dq", rounded(0.25 * ds @ k[:, 0])), ("dk", rounded(0.25 * ds.T @ q[:, 0])), ("dv", rounded(rounded(p).T @ do[:, 0]))):
        off = np.abs(x - got[name][:, 0])
        assert np.all(off <= got[name + "_off"][:, 0]), name
        assert off.max() > 0
