"""Attention over packed slides through the C ABI against the 64-bit oracle and its error bounds (needs an MI355X)."""
import math

import numpy as np
import pytest

from oracle import tokens_oracle as to

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
OPERAND = {"bf16": 2.0 ** -8, "fp32": 0.0}


def _starts(lengths, first):
    return np.concatenate(([first], first + np.cumsum(lengths))).astype(np.int32)


class Case:
    """Inputs on the GPU: queries, keys and values are views of one matrix where the slides' rows are the same; `front` and `behind`
    rows of no slide hold NaN."""

    def __init__(self, lq, lk, hq, hk, dim, dtype, cap=0.0, bias=False, lead_q=0, lead_k=0, front=0, behind=0, size=1.0, seed=11, backward=True):
        import torch
        from paper_2403_04865_amd import TokensLib
        self.L = TokensLib()
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.t = dtype, torch.float32 if dtype == "fp32" else torch.bfloat16
        self.qs, self.ks = _starts(lq, front), _starts(lk, front)
        nq, nk = int(self.qs[-1]) + behind, int(self.ks[-1]) + behind

        def rand(*shape):
            return torch.randn(shape, generator=g)
        if list(lq) == list(lk):
            m = (rand(nq, hq + 2 * hk, dim) * size).to(self.t)
            q, k, v = m[:, :hq], m[:, hq:hq + hk], m[:, hq + hk:]
        else:
            m = (rand(nk, 2 * hk, dim) * size).to(self.t)
            q, k, v = (rand(nq, hq, dim) * size).to(self.t), m[:, :hk], m[:, hk:]
        do = rand(nq, hq, dim).to(self.t)
        for x, s in ((q, self.qs), (k, self.ks), (v, self.ks), (do, self.qs)):
            x[:s[0]] = float("nan")
            x[s[-1]:] = float("nan")
        self.host = dict(q=q, k=k, v=v, do=do)
        dev = m.cuda()
        if list(lq) == list(lk):
            self.q, self.k, self.v = dev[:, :hq], dev[:, hq:hq + hk], dev[:, hq + hk:]
        else:
            self.q, self.k, self.v = q.cuda(), dev[:, :hk], dev[:, hk:]
        self.do = do.cuda()
        self.how = dict(scale=1 / math.sqrt(dim), cap=cap, lead_q=lead_q, lead_k=lead_k)
        self.places = {}
        if bias:
            pk = torch.randint(0, 40, (nk, 2), generator=g).float()
            pq = pk.clone() if list(lq) == list(lk) else torch.randint(0, 40, (nq, 2), generator=g).float()
            self.places = dict(pos_q=pq, pos_k=pk, slopes=torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]))
        self.dev_places = {n: x.cuda() for n, x in self.places.items()}
        self.q_start, self.k_start = torch.from_numpy(self.qs).cuda(), torch.from_numpy(self.ks).cuda()
        need = self.L.slide_tokens_attn_workspace_bytes(nq, nk, len(lq), hq, hk, dim, self.t, backward=backward)
        self.work = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")     # NaN wherever it is read before it is written

    def outputs(self, fill=7.0):
        import torch
        full = lambda x: torch.full(x.shape, fill, dtype=x.dtype, device="cuda")   # noqa: E731
        return dict(o=full(self.q), lse=torch.full((self.q.shape[1], self.q.shape[0]), fill, device="cuda"), dq=full(self.q), dk=full(self.k), dv=full(self.v))

    def forward(self, out, stream=None):
        self.L.slide_tokens_attn_fwd(self.q, self.k, self.v, self.q_start, self.k_start, out["o"], out["lse"], **self.how, **self.dev_places,
                                     workspace=self.work, stream=stream)

    def backward(self, out, stream=None):
        self.L.slide_tokens_attn_bwd(self.do, self.q, self.k, self.v, out["o"], out["lse"], self.q_start, self.k_start, out["dq"], out["dk"], out["dv"],
                                     **self.how, **self.dev_places, workspace=self.work, stream=stream)

    def oracle(self):
        n = {k: x.double().numpy() for k, x in {**self.host, **self.places}.items()}
        return to.attn(n.pop("q"), n.pop("k"), n.pop("v"), self.qs, self.ks, **self.how, **n, half_step=HALF[self.dtype], operand=OPERAND[self.dtype])


def _check(case, out, names=("o", "lse", "dq", "dk", "dv")):
    want = case.oracle()
    for n in names:
        got, w, off = out[n].double().cpu().numpy(), want[n], want[n + "_off"]
        nowhere = np.isnan(w)
        assert np.all(got[nowhere] == 7.0), (n, "rows of no slide were written")
        assert np.array_equal(np.isinf(got), np.isinf(np.where(nowhere, 0, w))), n
        there = ~nowhere & np.isfinite(w)
        with np.errstate(invalid="ignore"):
            d = np.where(there, np.abs(got - w) - off, -1)
        assert not np.any(np.isnan(got[there])), (n, "not a number")
        assert np.all(d <= 0), (n, float(d.max()), np.unravel_index(d.argmax(), d.shape), float(np.abs(np.where(there, got - w, 0)).max()))


SELF = [
    # lengths, heads, key heads, head_dim, type, cap, bias, lead
    ([1], 1, 1, 16, "bf16", 0.0, False, 0),
    ([1], 4, 2, 64, "fp32", 0.0, True, 1),
    ([2, 1, 31, 32, 33], 4, 2, 64, "bf16", 0.0, True, 1),
    ([63, 64, 65, 0, 127, 128, 129], 3, 1, 48, "bf16", 15.0, True, 1),
    ([0, 5, 0], 2, 2, 32, "bf16", 0.0, False, 0),
    ([300], 6, 6, 64, "bf16", 0.0, True, 1),
    ([257, 40], 5, 1, 128, "bf16", 20.0, False, 0),
    ([190, 17], 8, 2, 80, "bf16", 0.0, True, 2),
    ([129, 31], 4, 4, 96, "bf16", 5.0, True, 0),
    ([2, 1, 31, 32, 33], 4, 2, 64, "fp32", 3.0, True, 1),
    ([63, 64, 65, 0, 127], 3, 1, 48, "fp32", 0.0, True, 0),
    ([200], 2, 2, 128, "fp32", 20.0, False, 0),
    ([97, 30], 4, 2, 80, "fp32", 0.0, False, 0),
    ([130], 2, 1, 112, "fp32", 1.0, True, 100),
    ([700, 900], 2, 1, 64, "bf16", 0.0, True, 1),
    ([1] * 70 + [3] * 5, 3, 3, 32, "bf16", 0.0, True, 1),
    # two heads at a time: of one key head and of two, one slide after the other in a table
    ([150, 33, 0, 257], 8, 2, 64, "bf16", 0.0, True, 3),
    ([140, 161], 4, 4, 48, "bf16", 7.0, True, 1),
    ([3, 90, 41] * 30, 4, 2, 64, "bf16", 0.0, True, 1),
    ([3, 90, 41] * 30, 3, 1, 48, "fp32", 9.0, False, 0),
    ([1, 200, 0] * 25, 2, 2, 128, "bf16", 9.0, True, 200),
    ([1] * 5000, 1, 1, 16, "fp32", 0.0, False, 0),
]


@pytest.mark.parametrize("lengths,hq,hk,dim,dtype,cap,bias,lead", SELF)
def test_inside_slides(lengths, hq, hk, dim, dtype, cap, bias, lead):
    print(f"case attn {str(lengths)[:60]} ({hq},{hk})x{dim} {dtype} cap={cap} bias={bias} lead={lead}", flush=True)
    c = Case(lengths, lengths, hq, hk, dim, dtype, cap, bias, lead, lead, front=3, behind=2)
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)


CROSS = [
    # queries, keys of each slide
    ([1], [5000], 12, 12, 64, "bf16", 0.0, True, 1),
    ([1], [5000], 4, 1, 64, "fp32", 0.0, True, 1),
    ([1, 1, 1, 0, 1], [3000, 1, 0, 77, 640], 12, 4, 64, "bf16", 9.0, True, 8),
    ([8], [4000], 6, 6, 48, "fp32", 0.0, True, 8),
    ([4, 0, 9, 33], [900, 20, 0, 1300], 4, 2, 128, "bf16", 0.0, False, 0),
    ([3000], [5], 2, 2, 64, "bf16", 0.0, True, 0),
    ([2500, 100], [40, 0], 4, 1, 80, "fp32", 4.0, True, 1),
    ([1], [1], 1, 1, 128, "bf16", 0.0, False, 0),
    ([40], [9000], 2, 1, 32, "bf16", 0.0, False, 0),
]


@pytest.mark.parametrize("lq,lk,hq,hk,dim,dtype,cap,bias,lead", CROSS)
def test_few_queries_or_few_keys(lq, lk, hq, hk, dim, dtype, cap, bias, lead):
    print(f"case cross {lq} x {lk} ({hq},{hk})x{dim} {dtype} cap={cap} bias={bias}", flush=True)
    c = Case(lq, lk, hq, hk, dim, dtype, cap, bias, lead, 0, front=1, behind=1)
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)


@pytest.mark.parametrize("heads,dim,dtype", [((4, 4), 64, "bf16"), ((3, 1), 64, "bf16"), ((2, 1), 128, "bf16"), ((2, 2), 48, "fp32")])
def test_far_places_with_fractions(heads, dim, dtype):
    """Distances are those of the float32 positions however far from the origin they lie."""
    import torch
    print(f"case far places {heads} {dim} {dtype}", flush=True)
    c = Case([170, 61], [170, 61], *heads, dim, dtype, bias=True, lead_q=1, lead_k=1)
    g = torch.Generator().manual_seed(9)
    place = 123456.0 + 60 * torch.rand((231, 2), generator=g)
    c.places.update(pos_q=place, pos_k=place)
    c.dev_places = {n: x.cuda() for n, x in c.places.items()}
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)


def test_scores_that_fall_and_rise_along_the_keys():
    """A row's maximum far below and far above that of its first keys: sums are kept relative to it."""
    import torch
    print("case falling and rising scores", flush=True)
    for order in (1, -1):
        c = Case([96], [1200], 2, 2, 64, "fp32", backward=True)
        ramp = torch.linspace(-6 * order, 6 * order, 1200)
        c.host["k"].mul_(0.2).add_(ramp[:, None, None] * 0.5)
        c.host["q"].mul_(0.2).add_(3.0)
        c.k.copy_(c.host["k"].cuda())
        c.q.copy_(c.host["q"].cuda())
        out = c.outputs()
        c.forward(out)
        c.backward(out)
        _check(c, out)


@pytest.mark.parametrize("lengths,dim", [([50, 7], 16), ([9, 30], 64)])
def test_many_heads_share_a_key_head(lengths, dim):
    print(f"case group 128 {lengths} {dim}", flush=True)
    c = Case(lengths, lengths, 128, 1, dim, "bf16", bias=True, lead_q=1, lead_k=1)
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)


@pytest.mark.parametrize("dtype,heads,dim", [("bf16", 2, 64), ("bf16", 3, 48), ("fp32", 2, 32)])
def test_places_of_leading_rows_are_not_used(dtype, heads, dim):
    print(f"case lead places {dtype} {heads} {dim}", flush=True)
    import torch
    lengths = [140, 1, 2, 33]
    c = Case(lengths, lengths, heads, heads, dim, dtype, bias=True, lead_q=2, lead_k=2, front=3, behind=5)
    want, got = c.outputs(), c.outputs()
    c.forward(want)
    c.backward(want)
    _check(c, want)
    unused = [r for a, n in zip(c.qs[:-1], lengths) for r in range(a, a + min(2, n))] + [0, 1, 2] + list(range(c.qs[-1], c.qs[-1] + 5))
    for name, x in (("pos_q", float("nan")), ("pos_k", float("inf"))):
        c.dev_places[name][unused] = x
    c.forward(got)
    c.backward(got)
    for n in want:
        assert torch.equal(want[n], got[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores(dtype):
    """Scores of some hundreds: all but one or two probabilities of a row are nothing; behind a cap every one counts."""
    print(f"case large scores {dtype}", flush=True)
    for cap in (0.0, 2.0):
        c = Case([150], [150], 2, 2, 64, dtype, cap=cap, bias=True, size=8.0)
        out = c.outputs()
        c.forward(out)
        c.backward(out)
        _check(c, out)


def test_an_infinite_value_stays_in_its_slide():
    import torch
    print("case infinite value", flush=True)
    c = Case([70, 70, 70], [70, 70, 70], 2, 2, 64, "bf16", bias=True)
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    bad = c.outputs()
    c.k[75] = float("inf")
    c.v[80] = float("nan")
    c.forward(bad)
    c.backward(bad)
    for n in ("o", "dq", "dk", "dv"):
        for rows in (slice(0, 70), slice(140, 210)):
            assert torch.equal(out[n][rows], bad[n][rows]), n
    assert torch.isnan(bad["o"][70:140]).any()


@pytest.mark.parametrize("starts", [[0, 40, 20, 60], [0, 60, 0, 60], [-5, 10, 30, 1000], [60, 40, 20, 0], [70, 80, 90, 100]])
def test_starts_that_do_not_fit_stay_inside(starts):
    """What a wrong table gives is unspecified; rows behind the matrices are never touched (outputs lie inside larger ones)."""
    import torch
    print(f"case starts {starts}", flush=True)
    c = Case([20, 20, 20], [20, 20, 20], 2, 1, 32, "bf16")
    c.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
    c.k_start.copy_(torch.tensor(starts, dtype=torch.int32))
    big = {n: torch.full((x.shape[0] + 40, *x.shape[1:]), 7.0, dtype=x.dtype, device="cuda") for n, x in c.outputs().items() if n != "lse"}
    out = {n: x[20:-20] for n, x in big.items()}
    lse = torch.full((4, 60), 7.0, device="cuda")
    out["lse"] = lse[1:3]
    c.forward(out)
    c.backward(out)
    torch.cuda.synchronize()
    for n, x in big.items():
        assert torch.all(x[:20] == 7) and torch.all(x[-20:] == 7), n
    assert torch.all(lse[0] == 7) and torch.all(lse[3] == 7)


@pytest.mark.parametrize("lq,lk", [([400, 77], [400, 77]), ([1, 2], [2000, 900]), ([1500], [9])])
def test_same_bits_on_another_stream_and_captured(lq, lk):
    import torch
    print(f"case captured {lq} {lk}", flush=True)
    c = Case(lq, lk, 4, 2, 64, "bf16", cap=10.0, bias=True, lead_q=1)
    want, got = c.outputs(), c.outputs()
    c.forward(want)
    c.backward(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.forward(got, stream=side)
    c.backward(got, stream=side)
    side.synchronize()
    for n in want:
        assert torch.equal(want[n], got[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(got)
        c.backward(got)
    for i in range(3):
        c.q.mul_(1.1)
        c.do.mul_(0.9)
        c.forward(want)
        c.backward(want)
        torch.cuda.synchronize()
        for t in got.values():
            t.fill_(7.0)
        c.work.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(want[n], got[n]), (n, i)


def test_offsets_past_32_bits():
    """Keys and values 2^31 elements from their matrix's start on: a slide in a matrix of wide rows."""
    import torch
    from paper_2403_04865_amd import TokensLib
    print("case far offsets", flush=True)
    L = TokensLib()
    rows, wide = 1100, 1 << 21           # a row every 2^21 - 8 elements: 4.6 GB
    m = torch.zeros(rows * (wide - 8), dtype=torch.bfloat16, device="cuda")
    kv = m.as_strided((rows, 2, 64), (wide - 8, 64, 1))
    g = torch.Generator().manual_seed(2)
    kv.copy_(torch.randn((rows, 2, 64), generator=g).bfloat16().cuda())
    q = torch.randn((rows, 1, 64), generator=g).bfloat16().cuda()
    do = torch.randn((rows, 1, 64), generator=g).bfloat16().cuda()
    start = torch.tensor([0, 1000, 1100], dtype=torch.int32, device="cuda")
    far = {"k": kv[:, :1], "v": kv[:, 1:]}
    near = {n: x.contiguous() for n, x in far.items()}
    work = torch.empty(L.slide_tokens_attn_workspace_bytes(rows, rows, 2, 1, 1, 64, q.dtype, backward=True), dtype=torch.uint8, device="cuda")
    res = []
    for x in (far, near):
        o, lse = torch.empty_like(q), torch.empty(1, rows, device="cuda")
        L.slide_tokens_attn_fwd(q, x["k"], x["v"], start, start, o, lse, 0.125, workspace=work)
        d = [torch.empty_like(q) for _ in range(3)]
        L.slide_tokens_attn_bwd(do, q, x["k"], x["v"], o, lse, start, start, *d, 0.125, workspace=work)
        res.append([o, lse, *d])
    for a, b in zip(*res):
        assert torch.equal(a, b)
    # and the gradients written there
    out = kv.clone()
    dk, dv = kv[:, :1], kv[:, 1:]
    o, lse = res[1][0], res[1][1]
    dq = torch.empty_like(q)
    L.slide_tokens_attn_bwd(do, q, near["k"], near["v"], o, lse, start, start, dq, dk, dv, 0.125, workspace=work)
    assert torch.equal(dk.contiguous(), res[1][3]) and torch.equal(dv.contiguous(), res[1][4]) and out.shape == kv.shape


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_block_of_a_slide_encoder(dtype):
    """Rotated, normalised queries and keys out of one matrix, attention over a batch of slides, and back to that matrix' gradient."""
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print(f"case block {dtype}", flush=True)
    L = TokensLib()
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    lengths, hq, hk, dim = [90, 1, 143], 4, 2, 64
    starts = _starts(lengths, 0)
    rows = int(starts[-1])
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn((rows, hq + 2 * hk, dim), generator=g).to(t)
    do = torch.randn((rows, hq, dim), generator=g).to(t)
    gq, gk = 1 + 0.2 * torch.randn(dim, generator=g), 1 + 0.2 * torch.randn(dim, generator=g)
    place = torch.randint(0, 30, (rows, 2), generator=g, dtype=torch.int32)
    place[torch.from_numpy(starts[:-1]).long()] = 0
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0625])
    how = dict(scale=dim ** -0.5, cap=30.0, lead_q=1, lead_k=1)

    rope = HeadRope(dim, (16, 16), theta=100.0)
    x, dev = qkv.cuda(), {n: v.cuda() for n, v in dict(do=do, gq=gq, gk=gk, pos=place, slopes=slopes, start=torch.from_numpy(starts)).items()}
    v = x[:, hq + hk:]
    qk = torch.empty((rows, hq + hk, dim), dtype=t, device="cuda")
    q, k = qk[:, :hq], qk[:, hq:]
    L.slide_head_rope_fwd(rope, x[:, :hq], x[:, hq:hq + hk], dev["pos"], q, k, gq=dev["gq"], gk=dev["gk"])
    work = torch.empty(max(L.slide_tokens_attn_workspace_bytes(rows, rows, 3, hq, hk, dim, t, backward=True),
                           L.slide_head_rope_workspace_bytes(rope, rows, hq, hk)), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty((rows, hq, dim), dtype=t, device="cuda"), torch.empty((hq, rows), device="cuda")
    where = dict(pos_q=dev["pos"].float(), pos_k=dev["pos"].float(), slopes=dev["slopes"], workspace=work)
    L.slide_tokens_attn_fwd(q, k, v, dev["start"], dev["start"], o, lse, **how, **where)
    dx = torch.empty_like(x)
    dq, dk, dv = dx[:, :hq], dx[:, hq:hq + hk], dx[:, hq + hk:]
    L.slide_tokens_attn_bwd(dev["do"], q, k, v, o, lse, dev["start"], dev["start"], dq, dk, dv, **how, **where)
    dgq, dgk = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    L.slide_head_rope_bwd(rope, dq, dk, x[:, :hq], x[:, hq:hq + hk], dev["pos"], dq, dk, gq=dev["gq"], gk=dev["gk"], dgq=dgq, dgk=dgk, workspace=work)

    n = lambda a: a.double().numpy()   # noqa: E731
    xn = n(qkv)
    c, s = to.rotation(place.numpy(), (16, 16), dim, 100.0)
    qn = to.rope_fwd(xn[:, :hq], n(gq), c, s, "halves", 1e-6)
    kn = to.rope_fwd(xn[:, hq:hq + hk], n(gk), c, s, "halves", 1e-6)
    want = to.attn(qn, kn, xn[:, hq + hk:], starts, starts, **how, pos_q=n(place), pos_k=n(place), slopes=n(slopes), do=n(do))
    wq, wgq = to.rope_bwd(want["dq"], xn[:, :hq], n(gq), c, s, "halves", 1e-6)
    wk, wgk = to.rope_bwd(want["dk"], xn[:, hq:hq + hk], n(gk), c, s, "halves", 1e-6)
    # Of the whole run, relative to a tensor's norm: at most ten roundings of 2^-8 in a row for bfloat16 (q, k, p, o, ds, dq, dx and the
    # scores' size of a few units), each of either sign; 2^-24 and sums of some hundred terms for float32
    limit = 10 * 2.0 ** -8 if dtype == "bf16" else 400 * 2.0 ** -24
    for name, a, b in (("o", o, want["o"]), ("dq", dq, wq), ("dk", dk, wk), ("dv", dv, want["dv"]), ("dgq", dgq, wgq), ("dgk", dgk, wgk)):
        a = a.double().cpu().numpy()
        assert np.linalg.norm(a - b) <= limit * np.linalg.norm(b), (name, np.linalg.norm(a - b) / np.linalg.norm(b))
