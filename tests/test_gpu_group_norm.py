"""Group norm with its activation (include/act8.h) against float64 (needs an MI355X).

Bounds, per value, from float32 arithmetic: a statistic or sum of a group adds its terms with fewer than 256 roundings on the way of
any term (rows of a thread, threads of a workgroup, channels of a group, pieces of a tile), so it is off by at most
D = 256 * 2^-24 of the mean magnitude of its terms.  The activations' slopes are at most 1.13 and change by at most 0.8 per unit; the
activations are approximated to 2^-20 of their argument or 5e-7, whichever is larger.  A result is rounded once: 2^-24 or, in bfloat16,
2^-8 of half a step's width."""
import numpy as np
import pytest

from oracle import act8_oracle as ao

pytestmark = pytest.mark.gpu

D = 256 * 2.0 ** -24


def _types():
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16}


def _lib():
    from paper_2403_04865_amd import Act8Lib
    return Act8Lib()


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _strided(t, extra, offset=0):
    import torch
    n, hw, c = t.shape
    full = torch.full((n * hw * (c + extra) + offset,), 7.0, dtype=t.dtype, device=t.device)
    v = full[offset:].view(n, hw, c + extra)[:, :, :c]
    v.copy_(t)
    return v


def _untouched(v, extra, offset=0):
    n, hw, c = v.shape
    return not extra or bool((v._base.view(-1)[offset:].view(n, hw, c + extra)[:, :, c:] == 7).all())


def _np(t):
    return t.double().cpu().numpy()


def _wide(v, per):
    return np.repeat(v, per, 1)[:, None, :]


def _inputs(n, hw, c, groups, dtype, residual, seed, shift=1.0):
    rng = np.random.Generator(np.random.PCG64(seed))
    t = _types()[dtype]
    size = np.exp(0.5 * rng.standard_normal(c))
    x = _dev((rng.standard_normal((n, hw, c)) * size + shift * rng.standard_normal(c)).astype(np.float32), t)
    res = _dev(rng.standard_normal((n, hw, c)).astype(np.float32), t) if residual else None
    dy = _dev((rng.standard_normal((n, hw, c)) * 1e-2).astype(np.float32), t)
    gamma = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32)
    beta = (0.2 * rng.standard_normal(c)).astype(np.float32)
    return x, res, dy, gamma, beta


def _half_step(dtype):
    return 2.0 ** -24 if dtype == "fp32" else 2.0 ** -8


def _check(name, got, want, bound):
    worst = float((np.abs(got - want) / bound).max())
    print(f"  {name}: worst share of its bound {worst:.3f}", flush=True)
    assert worst <= 1.0, name


def _run(n, hw, c, groups, dtype, act, residual=False, extra=0, offset=0, checkpoint=False, in_place=False, accumulate=False,
         shift=1.0, eps=1e-5):
    import torch
    from paper_2403_04865_amd import Act8
    print("case", n, hw, c, groups, dtype, act, residual, extra, offset, checkpoint, in_place, accumulate, shift, flush=True)
    t, per = _types()[dtype], c // groups
    x, res, dy, gamma, beta = _inputs(n, hw, c, groups, dtype, residual, n + 7 * hw + 31 * c + groups, shift)
    L = _lib()
    work = torch.full((L.slide_group_norm_workspace_bytes(n, hw, c, groups, t) // 4,), float("nan"), device="cuda")
    put = lambda v: None if v is None else _strided(v, extra, offset)   # noqa: E731
    xs, rs, g, b = put(x), put(res), _dev(gamma), _dev(beta)
    y = xs if in_place else put(torch.zeros_like(x))
    mean, rstd = (torch.full((n, groups), float("nan"), device="cuda") for _ in range(2))
    x8 = Act8.empty(n * hw, c) if checkpoint else None
    L.slide_group_norm_fwd(xs, g, b, groups, y, mean, rstd, eps=eps, act=act, residual=rs, x8=x8, workspace=work)

    X, R = _np(x), None if res is None else _np(res)
    m, r = ao.statistics(X, groups, eps)
    xhat, u = ao.before_act(X, gamma, beta, m, r, R)
    want = ao.act(u, act)
    mag = ao._means(np.abs(X), groups)
    e_mean = D * mag + 2.0 ** -24 * np.abs(m)
    # of the variance: the terms are squares of distances from a mean that is e_mean off; of rstd: half of it
    e_rstd = r * (0.5 * (D + 2.0 ** -22) + e_mean ** 2 * r ** 2 + 2.0 ** -22)
    _check("mean", _np(mean), m, e_mean + 1e-30)
    _check("rstd", _np(rstd), r, e_rstd)
    e_u = np.abs(gamma) * (_wide(e_mean * r, per) + np.abs(xhat) * (_wide(e_rstd / r, per) + 2.0 ** -22))
    e_u = e_u + 2.0 ** -22 * (np.abs(xhat * gamma) + np.abs(beta) + (0 if R is None else np.abs(R)))
    e_act = 0 if act in ("none", "relu") else np.maximum(2.0 ** -20 * np.abs(u), 5e-7)
    _check("y", _np(y), want, 1.13 * e_u + e_act + _half_step(dtype) * 1.01 * np.abs(want) + 1e-30)
    assert _untouched(y, extra, offset)

    if checkpoint:
        codes, scales = ao.pack(X.reshape(n * hw, c))
        assert np.array_equal(x8.codes.cpu().numpy(), codes) and np.array_equal(x8.scales.cpu().numpy(), scales)
        X = ao.unpack(codes, scales, c).reshape(n, hw, c)
    if in_place:
        xs = put(x)
    ds = put(dy)
    dx = ds if in_place else put(torch.zeros_like(x))
    dres = put(torch.zeros_like(x)) if residual else None
    g0, b0 = (np.random.Generator(np.random.PCG64(k)).standard_normal(c).astype(np.float32) for k in (1, 2))
    dg, db = _dev(g0), _dev(b0)
    L.slide_group_norm_bwd(ds, x8 if checkpoint else xs, g, b, mean, rstd, groups, dx, dg, db, act=act, residual=rs, dresidual=dres,
                           accumulate=accumulate, workspace=work)
    # from the statistics that the call was given
    m, r, DY = _np(mean), _np(rstd), _np(dy)
    w_dx, w_du, w_dg, w_db = ao.group_norm_bwd(DY, X, gamma, beta, m, r, act, R)
    xhat, u = ao.before_act(X, gamma, beta, m, r, R)
    if act == "relu":
        assert not (np.abs(u) < 1e-13).any()    # which side these are on is not settled in 64 bits either
    e_xhat = 2.0 ** -22 * np.abs(xhat)
    e_u = 2.0 ** -22 * (np.abs(xhat * gamma) + np.abs(beta) + (0 if R is None else np.abs(R)))
    e_du = np.abs(DY) * ((0.8 * e_u + 1e-6) if act in ("silu", "gelu") else 0.0) + 2.0 ** -23 * np.abs(w_du)
    if residual:
        _check("dresidual", _np(dres), w_du, e_du + _half_step(dtype) * 1.01 * np.abs(w_du) + 1e-30)
        assert _untouched(dres, extra, offset)
    depth = max(D, 2.0 ** -24 * 300)
    e_dg = (e_du * np.abs(xhat) + np.abs(w_du) * e_xhat).sum((0, 1)) + depth * np.abs(w_du * xhat).sum((0, 1)) + 2.0 ** -23 * np.abs(w_dg)
    e_db = e_du.sum((0, 1)) + depth * np.abs(w_du).sum((0, 1)) + 2.0 ** -23 * np.abs(w_db)
    if accumulate:
        w_dg, w_db = w_dg + g0, w_db + b0
        e_dg, e_db = e_dg + 2.0 ** -23 * np.abs(w_dg), e_db + 2.0 ** -23 * np.abs(w_db)
    _check("dgamma", _np(dg), w_dg, e_dg + 1e-30)
    _check("dbeta", _np(db), w_db, e_db + 1e-30)
    tg = np.abs(w_du * gamma)
    e_t = e_du * np.abs(gamma) + 2.0 ** -22 * tg
    e_m1 = ao._means(e_t, groups) + D * ao._means(tg, groups)
    th = tg * np.abs(xhat)
    e_m2 = ao._means(e_t * np.abs(xhat) + tg * e_xhat, groups) + D * ao._means(th, groups)
    m1, m2 = ao._means(tg, groups), ao._means(th, groups)
    e_dx = _wide(r, per) * (e_t + _wide(e_m1, per) + np.abs(xhat) * _wide(e_m2, per) + e_xhat * _wide(m2, per)
                            + 2.0 ** -22 * (tg + _wide(m1, per) + np.abs(xhat) * _wide(m2, per)))
    _check("dx", _np(dx), w_dx, e_dx + _half_step(dtype) * 1.01 * np.abs(w_dx) + 1e-30)
    assert _untouched(dx, extra, offset)


SMALL = [(1, 1, 8, 1), (1, 1, 2, 1), (2, 1, 16, 16), (3, 2, 30, 5), (2, 49, 64, 32), (1, 7, 1, 1), (5, 16, 96, 8), (2, 64, 320, 32),
         (3, 49, 2048, 32), (2, 9, 2048, 1), (7, 33, 24, 3), (1, 100, 40, 20), (2, 784, 128, 32), (1, 50, 4096, 4)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,hw,c,groups", SMALL)
def test_sizes(n, hw, c, groups, dtype):
    _run(n, hw, c, groups, dtype, "silu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("n,hw,c,groups", [(3, 196, 64, 8), (2, 50, 36, 6), (1, 9000, 64, 16)])
def test_activations_and_residuals(n, hw, c, groups, act, dtype):
    _run(n, hw, c, groups, dtype, act, residual=True)
    _run(n, hw, c, groups, dtype, act, checkpoint=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,hw,c,groups", [(1, 5003, 64, 32), (2, 4000, 72, 9), (1, 30001, 24, 1), (1, 3000, 2056, 8), (1, 20011, 6, 3), (3, 3136, 64, 32),
                                           (1, 700, 65536, 64)])
def test_tiles_that_are_split_over_rows(n, hw, c, groups, dtype):
    if c * hw * n > 10_000_000 and dtype == "bf16":
        hw = 60          # (the oracle's time)
    if c == 65536:
        hw = min(hw, 60)
    _run(n, hw, c, groups, dtype, "gelu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("extra,offset", [(8, 0), (3, 0), (8, 1), (0, 4), (16, 8)])
def test_strides_and_alignment(extra, offset, dtype):
    _run(3, 81, 48, 6, dtype, "relu", residual=True, extra=extra, offset=offset, checkpoint=True)
    _run(1, 9001, 64, 4, dtype, "silu", residual=True, extra=extra, offset=offset, checkpoint=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,hw,c,groups", [(4, 100, 64, 8), (1, 9001, 64, 4), (3, 20, 33, 11)])
def test_in_place_and_accumulated(n, hw, c, groups, dtype):
    _run(n, hw, c, groups, dtype, "silu", in_place=True, accumulate=True)
    _run(n, hw, c, groups, dtype, "none", residual=True, in_place=True, accumulate=True)


def test_more_tiles_than_workgroups():
    _run(9001, 4, 8, 4, "fp32", "gelu")
    _run(5000, 2, 64, 8, "bf16", "none")


@pytest.mark.parametrize("n,hw,c,groups", [(2, 100, 32, 4), (1, 9001, 64, 4)])
def test_a_mean_far_from_zero(n, hw, c, groups):
    """Values around 300 with a deviation of one: squares of distances, not differences of squares."""
    _run(n, hw, c, groups, "fp32", "none", shift=300.0)


def test_constant_groups_and_their_gradient():
    """No variance: xhat is 0, rstd is 1 / sqrt(eps), and y is act(beta)."""
    import torch
    L = _lib()
    for hw in (5, 9001):
        x = torch.full((2, hw, 64), 3.0, device="cuda")
        g, b = torch.ones(64, device="cuda"), torch.linspace(-1, 1, 64, device="cuda")
        y, mean, rstd = torch.empty_like(x), torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda")
        work = torch.empty(L.slide_group_norm_workspace_bytes(2, hw, 64, 4, torch.float32), dtype=torch.uint8, device="cuda")
        L.slide_group_norm_fwd(x, g, b, 4, y, mean, rstd, eps=1e-4, act="relu", workspace=work)
        assert (mean == 3).all() and (rstd - 100).abs().max() < 1e-4 and torch.equal(y, b.clamp(min=0).expand_as(y))
        dx, dg, db = torch.empty_like(x), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
        L.slide_group_norm_bwd(torch.ones_like(x), x, g, b, mean, rstd, 4, dx, dg, db, act="none", workspace=work)
        assert (dg == 0).all() and (db - 2 * hw).abs().max() == 0 and dx.abs().max() <= 100 * D


def test_what_is_not_finite_stays_in_its_group():
    import torch
    L = _lib()
    for n, hw, c in ((3, 40, 64), (2, 9001, 64)):
        x = torch.randn(n, hw, c, device="cuda")
        ref = x.clone()
        x[1, 3, 20] = float("nan")
        x[0, 5, 40] = float("inf")
        g, b = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
        work = torch.empty(L.slide_group_norm_workspace_bytes(n, hw, c, 4, torch.float32), dtype=torch.uint8, device="cuda")
        outs = []
        for v in (x, ref):
            y, mean, rstd = torch.empty_like(x), torch.empty(n, 4, device="cuda"), torch.empty(n, 4, device="cuda")
            L.slide_group_norm_fwd(v, g, b, 4, y, mean, rstd, workspace=work)
            outs.append(y)
        got, want = outs
        assert got[1, :, 16:32].isnan().all()
        assert not got[0, :, 32:48].isfinite().any()
        got[1, :, 16:32] = want[1, :, 16:32]
        got[0, :, 32:48] = want[0, :, 32:48]
        assert torch.equal(got, want)


def test_a_rectifier_at_zero():
    """Sums that cancel to zero, or to the last bit next to it: the sides of zero are those of 64 bits."""
    import torch
    L = _lib()
    n, hw, c, groups = 2, 64, 64, 8
    rng = np.random.Generator(np.random.PCG64(8))
    x = rng.standard_normal((n, hw, c)).astype(np.float32)
    gamma = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32)
    beta = (0.2 * rng.standard_normal(c)).astype(np.float32)
    mean = rng.standard_normal((n, groups)).astype(np.float32)
    rstd = (1 + rng.random((n, groups))).astype(np.float32)
    u = ao.before_act(x.astype(np.float64), gamma.astype(np.float64), beta.astype(np.float64), mean.astype(np.float64), rstd.astype(np.float64))[1]
    res = (-u).astype(np.float32)      # the nearest float to what takes the sum to zero
    sign = u + res.astype(np.float64)
    dy = np.ones_like(x)
    dx, dres = torch.empty(n, hw, c, device="cuda"), torch.empty(n, hw, c, device="cuda")
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    work = torch.empty(L.slide_group_norm_workspace_bytes(n, hw, c, groups, torch.float32), dtype=torch.uint8, device="cuda")
    L.slide_group_norm_bwd(_dev(dy), _dev(x), _dev(gamma), _dev(beta), _dev(mean), _dev(rstd), groups, dx, dg, db, act="relu",
                           residual=_dev(res), dresidual=dres, workspace=work)
    sure = np.abs(sign) > 1e-14
    assert sure.mean() > 0.9 and np.array_equal(dres.cpu().numpy()[sure], (sign > 0).astype(np.float32)[sure])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_value_of_many_tiles(dtype):
    """All values of a hundred megabytes of output, five times over, against the formula on the device: a store whose data the next
    instruction overwrote was wrong in one value of some thousands."""
    import torch
    L = _lib()
    t = _types()[dtype]
    for n, hw, c, groups in ((600, 784, 64, 32), (200, 196, 320, 32)):
        g = torch.Generator(device="cuda").manual_seed(n)
        x = torch.randn(n, hw, c, device="cuda", generator=g).to(t)
        dy = torch.randn(n, hw, c, device="cuda", generator=g).to(t)
        gamma, beta = 1 + 0.1 * torch.randn(c, device="cuda", generator=g), 0.1 * torch.randn(c, device="cuda", generator=g)
        work = torch.empty(L.slide_group_norm_workspace_bytes(n, hw, c, groups, t), dtype=torch.uint8, device="cuda")
        v = x.double().view(n, hw, groups, -1)
        m = v.mean((1, 3), keepdim=True)
        r = 1 / torch.sqrt(v.var((1, 3), unbiased=False, keepdim=True) + 1e-5)
        xhat = ((v - m) * r).view(n, hw, c)
        want = xhat * gamma + beta
        du = dy.double()
        q = (du * gamma).view(n, hw, groups, -1)
        h = xhat.view(n, hw, groups, -1)
        want_dx = (r * (q - q.mean((1, 3), keepdim=True) - h * (q * h).mean((1, 3), keepdim=True))).view(n, hw, c)
        for _ in range(5):
            y, dx, dres = (torch.full_like(x, float("nan")) for _ in range(3))
            mean, rstd = torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda")
            dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            L.slide_group_norm_fwd(x, gamma, beta, groups, y, mean, rstd, workspace=work)
            L.slide_group_norm_bwd(dy, x, gamma, beta, mean, rstd, groups, dx, dg, db, dresidual=dres, workspace=work)
            # statistics to D (above) of values of size one, gains up to 1.5, |xhat| up to 6
            tol = 20 * D + _half_step(dtype) * 1.01 * want.abs()
            assert ((y.double() - want).abs() <= tol).all()
            assert ((dx.double() - want_dx).abs() <= 20 * D + _half_step(dtype) * 1.01 * want_dx.abs()).all()
            assert torch.equal(dres, dy)
