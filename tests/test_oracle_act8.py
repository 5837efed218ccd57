"""Pins of the 8-bit layers' oracle: codes against torch's e4m3 type, the scale rule, gradients against differences."""
import numpy as np
import pytest

from oracle import act8_oracle as ao


def test_codes_are_those_of_the_e4m3_type():
    import torch
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(v, ao.CODE, equal_nan=True)
    rng = np.random.Generator(np.random.PCG64(1))
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 2, 4000),
                        (ao.CODE[:0x7e] + ao.CODE[1:0x7f]) / 2, [0.0, -0.0, 448.0, -448.0]]).astype(np.float32)   # ties among them
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ao.code_of(x), t)
    assert np.array_equal(ao.code_of([np.inf, -np.inf, np.nan]), [0x7f] * 3)


@pytest.mark.parametrize("top,byte", [(448.0, 127), (448.001, 128), (224.0, 126), (1.75, 119), (1.7501, 120), (1.0, 119),
                                      (0.0, 127), (2.0 ** -149, 0), (3.4e38, 247), (448 * 2.0 ** -127, 0)])
def test_scale_is_the_smallest_power_that_holds_the_largest(top, byte):
    assert ao.scale_byte(np.array([top / 3, -top, 0.0, np.nan, np.inf])) == byte


def test_packing_rounds_to_the_nearest_within_half_a_step():
    rng = np.random.Generator(np.random.PCG64(2))
    x = rng.standard_normal((5, 300)) * np.exp(rng.standard_normal((5, 300)))
    codes, scales = ao.pack(x)
    assert codes.shape == (5, 304) and scales.shape == (5, 3) and not codes[:, 300:].any()
    v = ao.unpack(codes, scales, 300)
    top = np.repeat(np.stack([np.abs(x[:, b * 128:(b + 1) * 128]).max(1) for b in range(3)], 1), 128, 1)[:, :300]
    # half a step: 2^-4 of the value, or of the smallest normal code, 2^-6 of at most 2 top / 448
    assert np.all(np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * 2 * top / 448))
    c2, s2 = ao.pack(v)     # what 8 bits hold packs to itself
    assert np.array_equal(ao.unpack(c2, s2, 300), v)


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
def test_group_norm_gradients_against_differences(kind):
    rng = np.random.Generator(np.random.PCG64(3))
    n, hw, c, groups, eps, h = 2, 5, 6, 3, 1e-3, 1e-5
    x, res, dy = (rng.standard_normal((n, hw, c)) for _ in range(3))
    gamma, beta = 1 + 0.3 * rng.standard_normal(c), 0.3 * rng.standard_normal(c)

    def loss(x, gamma, beta, res):
        mean, rstd = ao.statistics(x, groups, eps)
        return (dy * ao.act(ao.before_act(x, gamma, beta, mean, rstd, res)[1], kind)).sum()

    mean, rstd = ao.statistics(x, groups, eps)
    dx, dres, dgamma, dbeta = ao.group_norm_bwd(dy, x, gamma, beta, mean, rstd, kind, res)
    for k, (a, grad) in enumerate(((x, dx), (gamma, dgamma), (beta, dbeta), (res, dres))):
        for i in range(0, a.size, 3):
            args = [x, gamma, beta, res]
            d = np.zeros(a.size)
            d[i] = h
            up, down = list(args), list(args)
            up[k], down[k] = a + d.reshape(a.shape), a - d.reshape(a.shape)
            # central difference: h^2 third derivatives (of order ten here) and rounding 1e-15 / h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad.ravel()[i]) <= 1e-7
