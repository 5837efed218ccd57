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
