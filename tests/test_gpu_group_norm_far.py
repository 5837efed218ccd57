"""Group norm over a tile of 2^31 - 1 rows and over rows whose offsets pass 32 bits (needs an MI355X)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2403_04865_amd import Act8Lib
    return Act8Lib()


def test_the_longest_tile():
    """One channel, 2^31 - 1 rows, 1024 chunks of 2^21 rows, the last one a row short.  A thread merges 1024 groups of eight rows and a channel
    256 threads, each a rounding of the mean: off by 1288 * 2^-24 of the mean magnitude at most.  A thread's sums of the backward have 8192
    terms, a channel's 256 of those, a few more roundings in a term: 8456 * 2^-24 of the mean magnitude of their terms."""
    import torch
    hw, piece = 2 ** 31 - 1, 1 << 27
    L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda: torch.empty(hw, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    x, dy = new(), new()
    parts = [slice(lo, min(lo + piece, hw)) for lo in range(0, hw, piece)]
    for p in parts:
        x[p].normal_(1.0, 1.0, generator=gen)
        dy[p].normal_(0.5, 1.0, generator=gen)
    x[-2048:] += 4     # what a row too many or too few at the end would show
    y, dx = new().fill_(float("nan")), new().fill_(float("nan"))
    f = lambda v: torch.tensor(v, device="cuda")   # noqa: E731
    gamma, beta = f([1.25]), f([-0.5])
    mean, rstd, dg, db = (torch.full((1,), float("nan"), device="cuda") for _ in range(4))
    work = torch.empty(L.slide_group_norm_workspace_bytes(1, hw, 1, 1, torch.bfloat16), dtype=torch.uint8, device="cuda")
    t = lambda v: v.view(1, hw, 1)   # noqa: E731
    print("case longest tile, forward", flush=True)
    L.slide_group_norm_fwd(t(x), gamma, beta, 1, t(y), mean.view(1, 1), rstd.view(1, 1), workspace=work)
    m = sum(x[p].double().sum() for p in parts) / hw
    mag = sum(x[p].double().abs().sum() for p in parts) / hw
    r = 1 / torch.sqrt(sum((x[p].double() - m).square().sum() for p in parts) / hw + 1e-5)
    U = 2.0 ** -24
    e_mean = 1290 * U * mag
    assert (mean[0] - m).abs() <= e_mean
    assert (rstd[0] - r).abs() <= r * (1290 * U + (e_mean * r) ** 2)
    for p in parts:
        xhat = (x[p].double() - m) * r
        tol = 1.25 * (e_mean * r + xhat.abs() * 2000 * U) + U * 8 + 1.01 * 2.0 ** -8 * (1.25 * xhat - 0.5).abs()
        assert ((y[p].double() - (1.25 * xhat - 0.5)).abs() <= tol).all()
    print("case longest tile, backward", flush=True)
    L.slide_group_norm_bwd(t(dy), t(x), gamma, beta, mean.view(1, 1), rstd.view(1, 1), 1, t(dx), dg, db, workspace=work)
    m, r = mean[0].double(), rstd[0].double()
    s = {k: 0.0 for k in ("b", "g", "|b|", "|g|")}
    for p in parts:
        d = dy[p].double()
        h = d * (x[p].double() - m) * r
        for k, v in (("b", d), ("g", h), ("|b|", d.abs()), ("|g|", h.abs())):
            s[k] = s[k] + v.sum()
    eps = 8460 * U
    assert (db[0] - s["b"]).abs() <= eps * s["|b|"] and (dg[0] - s["g"]).abs() <= eps * s["|g|"]
    for p in parts:
        xhat = (x[p].double() - m) * r
        want = r * 1.25 * (dy[p].double() - s["b"] / hw - xhat * s["g"] / hw)
        tol = r * 1.25 * (eps * (s["|b|"] + xhat.abs() * s["|g|"]) / hw + 8 * U * (dy[p].double().abs() + 1 + xhat.abs())) + 1.01 * 2.0 ** -8 * want.abs()
        assert ((dx[p].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hw", [(1, 5), (2, 3)])
def test_rows_beyond_32_bit_offsets(n, hw, dtype):
    """The same bits as from rows that lie together, all in the kernels that take 64-bit offsets; and what is between the rows stays."""
    import torch
    from paper_2403_04865_amd import Act8
    print("case rows beyond 32-bit offsets", n, hw, dtype, flush=True)
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    rows, c, groups, ld = n * hw, 96, 12, (1 << 30) + 64
    rng = np.random.Generator(np.random.PCG64(rows))
    put = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().to(t)   # noqa: E731
    x, dy, res = put(n, hw, c), put(n, hw, c), put(n, hw, c)
    gamma, beta = put(c).float(), put(c).float()
    L = _lib()
    memory = [torch.empty((rows - 1) * ld + c + 1, dtype=t, device="cuda") for _ in range(4)]

    def run(ld, x, dy, res, memory):
        far = lambda i: torch.as_strided(memory[i], (n, hw, c), (hw * ld, ld, 1))   # noqa: E731
        a, b, r, d = (far(i) for i in range(4))
        a.copy_(x)
        b.copy_(dy)
        r.copy_(res)
        for m in memory:
            m[c] = 7.0          # behind the first row
            m[(rows - 1) * ld + c] = 7.0
        mean, rstd = (torch.empty(n, groups, device="cuda") for _ in range(2))
        dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        work = torch.empty(L.slide_group_norm_workspace_bytes(n, hw, c, groups, t), dtype=torch.uint8, device="cuda")
        x8 = Act8.empty(rows, c)
        L.slide_group_norm_fwd(a, gamma, beta, groups, d, mean, rstd, act="silu", residual=r, x8=x8, workspace=work)
        y = d.contiguous().clone()
        L.slide_group_norm_bwd(b, a, gamma, beta, mean, rstd, groups, b, dg, db, act="silu", residual=r, dresidual=d, workspace=work)
        assert all(bool((m[c] == 7) & (m[(rows - 1) * ld + c] == 7)) for m in memory)
        return y, b.contiguous().clone(), d.contiguous().clone(), mean, rstd, dg, db, x8.codes, x8.scales
    got = run(ld, x, dy, res, memory)
    del memory
    # together, but still too far apart for 32 bits: a row stride of 2^19 bytes with 4096 rows behind the last passes them
    near = 1 << 19
    want = run(near, x, dy, res, [torch.empty((rows - 1) * near + c + 1, dtype=t, device="cuda") for _ in range(4)])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # and near to what adjacent rows give, in whichever kernels they take
    mean, rstd, y = torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda"), torch.empty_like(x)
    work = torch.empty(L.slide_group_norm_workspace_bytes(n, hw, c, groups, t), dtype=torch.uint8, device="cuda")
    L.slide_group_norm_fwd(x, gamma, beta, groups, y, mean, rstd, act="silu", residual=res, workspace=work)
    assert torch.allclose(got[3], mean, rtol=0, atol=2e-5) and torch.allclose(got[4], rstd, rtol=2e-5, atol=0)
    assert torch.allclose(got[0].float(), y.float(), rtol=2.0 ** -7 if dtype == "bf16" else 1e-5, atol=1e-4)
