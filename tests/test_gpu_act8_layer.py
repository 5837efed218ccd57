"""The 8-bit operators as a user runs them together: group norm with its activation and checkpoint, a linear layer on 8-bit
activations with a residual, its input gradient through the packed transpose, its weight gradient out of the checkpoint, the norm's backward out of its own;
on other streams, in captured graphs, and two of them at once (needs an MI355X)."""
import numpy as np
import pytest

from oracle import act8_oracle as ao

pytestmark = pytest.mark.gpu


class Layer:
    """z = pack(silu(groupnorm(x))) pack(W)^T + b + residual, on tiles [n, hw, c]; buffers of its own, nothing shared."""

    def __init__(self, n, hw, c, out, groups, dtype, seed):
        import torch
        from paper_2403_04865_amd import Act8, Act8Lib
        rng = np.random.Generator(np.random.PCG64(seed))
        t = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
        put = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()   # noqa: E731
        self.n, self.hw, self.c, self.out, self.groups, self.t = n, hw, c, out, groups, t
        rows = n * hw
        self.x, self.res, self.dz = put(n, hw, c).to(t), put(rows, out).to(t), put(rows, out).to(t)
        self.gamma, self.beta, self.bias = 1 + 0.2 * put(c), 0.2 * put(c), put(out)
        self.W = (put(out, c) / c ** 0.5).to(t)
        self.lib = L = Act8Lib()
        self.x8, self.h8, self.dz8 = Act8.empty(rows, c), Act8.empty(rows, c), Act8.empty(rows, out)
        self.w8, self.wt8 = Act8.empty(out, c), Act8.empty(c, out)
        L.slide_act8_pack(self.W, self.w8)
        L.slide_act8_pack(self.W, self.wt8, transpose=True)
        e = lambda *s, d=t: torch.empty(s, dtype=d, device="cuda")   # noqa: E731
        f = torch.float32
        self.y, self.dh, self.dx, self.z = e(n, hw, c), e(n, hw, c), e(n, hw, c), e(rows, out)
        self.mean, self.rstd = e(n, groups, d=f), e(n, groups, d=f)
        self.dW, self.db, self.dgamma, self.dbeta = e(out, c, d=f), e(out, d=f), e(c, d=f), e(c, d=f)
        self.gn_work = e(max(L.slide_group_norm_workspace_bytes(n, hw, c, groups, t), 4) // 4, d=f)
        self.w_work = e(max(L.slide_act8_wgrad_workspace_bytes(rows, out, c), 4) // 4, d=f)

    def run(self):
        L, rows = self.lib, self.n * self.hw
        L.slide_group_norm_fwd(self.x, self.gamma, self.beta, self.groups, self.y, self.mean, self.rstd, act="silu", x8=self.x8,
                               workspace=self.gn_work)
        L.slide_act8_linear(self.y.view(rows, self.c), self.h8, self.w8, self.z, bias=self.bias, residual=self.res)
        L.slide_act8_wgrad(self.dz, self.h8, self.dW, db=self.db, workspace=self.w_work)
        L.slide_act8_linear(self.dz, self.dz8, self.wt8, self.dh.view(rows, self.c))
        L.slide_group_norm_bwd(self.dh, self.x8, self.gamma, self.beta, self.mean, self.rstd, self.groups, self.dx, self.dgamma,
                               self.dbeta, act="silu", workspace=self.gn_work)

    RESULTS = ("mean", "rstd", "y", "z", "dh", "dx", "dW", "db", "dgamma", "dbeta")

    def results(self):
        out = {k: getattr(self, k).clone() for k in self.RESULTS}
        out.update({k: v for k in ("x8", "h8", "dz8") for k, v in ((k, getattr(self, k).codes.clone()), (k + "s", getattr(self, k).scales.clone()))})
        return out

    def forget(self):
        for k in self.RESULTS:
            getattr(self, k).fill_(float("nan"))
        for k in ("x8", "h8", "dz8"):
            getattr(self, k).codes.fill_(0x55)
            getattr(self, k).scales.fill_(0x7f)
        self.gn_work.fill_(float("nan"))
        self.w_work.fill_(float("nan"))


def _same(a, b):
    import torch
    return [k for k in a if not torch.equal(a[k], b[k])]


def _np(t):
    return t.double().cpu().numpy()


def _rel(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


SHAPES = [(3, 49, 64, 96, 8), (2, 200, 384, 130, 32), (1, 1, 16, 8, 2), (1, 9001, 32, 40, 4)]


# Float32 sums and one rounding of each result: 2^-24 sqrt(terms) at most for what is summed, and at most 2^-8, 1.7e-3 in the mean square, where a result is stored in
# bfloat16 (the matrix core adds 8e-5).  What a step takes in is taken from the library as it stored it, so limits do not add up
# over the steps; the norm's backward subtracts means, which leaves at least a tenth of its terms here.
@pytest.mark.parametrize("dtype,limit", [("fp32", 1e-5), ("bf16", 3e-3)])
@pytest.mark.parametrize("n,hw,c,out,groups", SHAPES)
def test_against_float64(n, hw, c, out, groups, dtype, limit):
    print("case", n, hw, c, out, groups, dtype, flush=True)
    a = Layer(n, hw, c, out, groups, dtype, 5)
    a.run()
    X, W, dz, gamma, beta = _np(a.x), _np(a.W), _np(a.dz), _np(a.gamma), _np(a.beta)
    val = lambda m: ao.unpack(*ao.pack(m), m.shape[1])   # noqa: E731
    m, r = ao.statistics(X, groups, 1e-5)
    want = {"mean": m, "rstd": r, "y": ao.act(ao.before_act(X, gamma, beta, m, r)[1], "silu")}
    h = val(_np(a.y).reshape(n * hw, c))
    want["z"] = h @ val(W).T + _np(a.bias) + _np(a.res)
    want["dW"], want["db"] = dz.T @ h, dz.sum(0)
    want["dh"] = (val(dz) @ val(np.ascontiguousarray(W.T)).T).reshape(n, hw, c)
    kept = val(X.reshape(n * hw, c)).reshape(X.shape)
    want["dx"], _, want["dgamma"], want["dbeta"] = ao.group_norm_bwd(_np(a.dh), kept, gamma, beta, _np(a.mean), _np(a.rstd), "silu")
    errs = {k: _rel(_np(getattr(a, k)), v) for k, v in want.items() if np.linalg.norm(v)}
    print(errs, flush=True)
    assert max(errs.values()) <= limit, errs


def test_gradients_are_differences():
    """On whole numbers every sum is exact, and the loss sum(z dz) is linear in the weights, in the inputs and in the bias: a step in each
    changes it by exactly the gradient's product with the step."""
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    L, rng = Act8Lib(), np.random.default_rng(11)
    rows, cin, out = 150, 200, 72
    whole = lambda top, *s: torch.from_numpy(rng.integers(-top, top + 1, s).astype(np.float32)).cuda()   # noqa: E731
    x, w, b, dz = whole(4, rows, cin), whole(4, out, cin), whole(9, out), whole(4, rows, out)
    step = {"x": whole(4, rows, cin), "w": whole(4, out, cin), "b": whole(9, out)}

    def z(x, w, b):
        x8, w8, y = Act8.empty(rows, cin), Act8.empty(out, cin), torch.empty(rows, out, device="cuda")
        L.slide_act8_pack(w, w8)
        L.slide_act8_linear(x, x8, w8, y, bias=b)
        return y, x8
    y, x8 = z(x, w, b)
    loss = lambda y: float((y.double() * dz.double()).sum())   # noqa: E731
    dW, db, dx = torch.empty(out, cin, device="cuda"), torch.empty(out, device="cuda"), torch.empty(rows, cin, device="cuda")
    work = torch.empty(L.slide_act8_wgrad_workspace_bytes(rows, out, cin) // 4 + 1, device="cuda")
    L.slide_act8_wgrad(dz, x8, dW, db=db, workspace=work)
    wt8 = Act8.empty(cin, out)
    L.slide_act8_pack(w, wt8, transpose=True)
    L.slide_act8_linear(dz, Act8.empty(rows, out), wt8, dx)
    for k, g, moved in (("x", dx, (x + step["x"], w, b)), ("w", dW, (x, w + step["w"], b)), ("b", db, (x, w, b + step["b"]))):
        assert loss(z(*moved)[0]) - loss(y) == float((g.double() * step[k].double()).sum()), k


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_on_another_stream(dtype):
    import torch
    a = Layer(2, 200, 384, 130, 32, dtype, 6)
    a.run()
    want = a.results()
    a.forget()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a.run()
    s.synchronize()
    assert not _same(a.results(), want)


@pytest.mark.parametrize("n,hw,c,out,groups", SHAPES)
def test_two_captured_graphs(n, hw, c, out, groups):
    """Two layers captured, each with buffers of its own, replayed several times on other inputs with eager work in between."""
    import torch
    print("case", n, hw, c, out, groups, flush=True)
    pair = [Layer(n, hw, c, out, groups, "bf16", 7 + i) for i in range(2)]
    graphs = []
    for a in pair:
        a.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            a.run()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in pair]
    for turn in range(4):
        want = []
        for a in pair:
            a.x.normal_(turn, 1 + turn)
            a.dz.normal_()
            a.run()
            want.append(a.results())
            a.forget()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):      # both at once
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i, a in enumerate(pair):
            assert not _same(a.results(), want[i]), (turn, i)


def test_two_at_once():
    import torch
    pair = [Layer(2, 784, 128, 512, 32, "bf16", 20 + i) for i in range(2)]
    want = []
    for a in pair:
        a.run()
        want.append(a.results())
        a.forget()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pair]
    for _ in range(10):
        for a, s in zip(pair, streams):
            with torch.cuda.stream(s):
                a.run()
    torch.cuda.synchronize()
    for a, w in zip(pair, want):
        assert not _same(a.results(), w)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,width", [(1, 4096), (5, 272), (16, 1040), (17, 1040), (300, 384), (33000, 384)])
def test_a_residual_stream_updated_in_place(rows, width, dtype):
    """x, residual and y the same matrix: the same bits as apart, and the checkpoint of what x was."""
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    print("case", rows, width, dtype, flush=True)
    t = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rng = np.random.default_rng(rows + width)
    x = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).cuda().to(t)
    w = torch.from_numpy((rng.standard_normal((width, width)) / width ** 0.5).astype(np.float32)).cuda().to(t)
    L, w8 = Act8Lib(), Act8.empty(width, width)
    L.slide_act8_pack(w, w8)
    y, a, b = torch.empty_like(x), Act8.empty(rows, width), Act8.empty(rows, width)
    L.slide_act8_pack(x, a)
    L.slide_act8_linear(None, a, w8, y, act="silu", residual=x)
    L.slide_act8_linear(x, b, w8, x, act="silu", residual=x)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    assert torch.equal(x, y)


@pytest.mark.parametrize("rows,cin,cout,extra", [(17, 2048, 40, 0), (32, 2040, 4096, 8), (33, 1024, 72, 0), (64, 136, 333, 8), (200, 384, 1024, 0),
                                                 (257, 8, 64, 8), (1000, 640, 64, 0), (7, 384, 40, 0), (16, 333, 64, 5), (33000, 384, 384, 0), (40000, 333, 64, 0), (33001, 200, 100, 8),
                                                 (32768, 128, 8, 3), (32770, 1, 384, 0), (50000, 256, 129, 16), (32999, 384, 385, 0)])
def test_packing_inside_the_product(rows, cin, cout, extra):
    """As packing first does: the checkpoint bit for bit, with its zeros behind the last column and nothing else touched, and y."""
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    print("case", rows, cin, cout, extra, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + cin)
    x = torch.randn(rows, cin + extra, generator=gen, device="cuda").bfloat16()[:, :cin]
    x[rows // 2, cin // 2] = float("nan")
    x[rows - 1] = 0
    w = torch.randn(cout, cin, generator=gen, device="cuda").bfloat16()
    bias = torch.randn(cout, generator=gen, device="cuda")
    L, w8 = Act8Lib(), Act8.empty(cout, cin)
    L.slide_act8_pack(w, w8)
    k16, nb = -(-cin // 16) * 16, -(-cin // 128)

    def guarded():
        codes, scales = torch.full((rows + 1, k16 + 16), 0x5a, dtype=torch.uint8, device="cuda"), torch.full((rows + 1, nb + 1), 0x5a, dtype=torch.uint8, device="cuda")
        return Act8(rows, cin, codes[:rows, :k16], scales[:rows, :nb]), codes, scales
    (a, ac, as_), (b, bc, bs) = guarded(), guarded()
    y, z = (torch.full((rows + 1, cout), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    L.slide_act8_pack(x, a)
    L.slide_act8_linear(None, a, w8, y[:rows], bias=bias, act="relu")
    L.slide_act8_linear(x, b, w8, z[:rows], bias=bias, act="relu")
    assert torch.equal(ac, bc) and torch.equal(as_, bs)
    same = (y == z) | (y.isnan() & z.isnan())
    # with another kernel the 8-bit products may be added in another order: half a step's rounding of results, nothing more
    assert same.float().mean() > 0.99 and torch.allclose(y.float(), z.float(), rtol=2.0 ** -7, atol=1e-2, equal_nan=True)
    assert bool((z[rows] == 7).all()) and bool(z[rows // 2].isnan().all()) and int(z.isnan().sum()) == cout
