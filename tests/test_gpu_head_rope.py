"""Norm and rotation of heads through the C ABI against the 64-bit oracle (needs an MI355X)."""
import numpy as np
import pytest

from oracle import tokens_oracle as to

pytestmark = pytest.mark.gpu

EPS, THETA = 1e-6, 100.0


def _make(rows, hq, hk, dim, pairs, dtype, norm, seed=3, far=1 << 12):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    qkv = torch.randn((rows, hq + 2 * hk, dim), generator=g).to(t)
    pos = torch.randint(-far, far, (rows, len(pairs)), generator=g, dtype=torch.int32)
    gains = [1 + 0.3 * torch.randn(dim, generator=g) if norm else None for _ in range(2)]
    dy = torch.randn((rows, hq + hk, dim), generator=g).to(t)
    return qkv, pos, gains, dy


def _np(t):
    return t.double().cpu().numpy()


def _tolerance(dtype):
    # float32: sum of squares, root, gain, angle (2^-31 turns: 3e-9; a series and the phase's rounding to 24 bits: 3 units) and two products
    # of a rotation: 12 units of 2^-24 of the pair's size; bfloat16: the same and half a step, 2^-8
    return 12 * 2.0 ** -24, 0.0 if dtype == "fp32" else 2.0 ** -8


def _close(got, want, size, dtype, what):
    unit, half = _tolerance(dtype)
    off = np.abs(got - want) - half * np.abs(want) - unit * size
    assert np.all(off <= 0), (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


CASES = [(1, 12, 12, 64, (16, 16), "halves", "bf16", True), (37, 6, 6, 64, (16, 16), "neighbours", "bf16", True),
         (5, 3, 1, 16, (8,), "halves", "fp32", True), (130, 4, 2, 48, (9, 5), "neighbours", "fp32", True),
         (257, 8, 2, 80, (14, 14, 6), "halves", "fp32", True), (64, 2, 2, 96, (16, 16, 16), "halves", "bf16", True),
         (19, 5, 5, 112, (0, 20), "neighbours", "bf16", True), (41, 3, 3, 128, (64,), "halves", "fp32", False),
         (12, 1, 1, 256, (50, 50, 28), "neighbours", "bf16", True), (33, 7, 0, 32, (), "halves", "fp32", True),
         (70001, 3, 1, 32, (8, 8), "halves", "bf16", True), (1003, 2, 1, 240, (30, 30, 30), "halves", "fp32", True)]


@pytest.mark.parametrize("rows,hq,hk,dim,pairs,pairing,dtype,norm", CASES)
def test_forward_and_backward(rows, hq, hk, dim, pairs, pairing, dtype, norm):
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print(f"case rope {rows}x({hq},{hk})x{dim} {pairs} {pairing} {dtype} norm={norm}", flush=True)
    L, rope = TokensLib(), HeadRope(dim, pairs, THETA, pairing, EPS)
    qkv, pos, (gq, gk), dy = _make(rows, hq, hk, dim, pairs, dtype, norm)
    if not hk:
        gk = None
    d = lambda t: None if t is None else t.cuda()   # noqa: E731
    x = d(qkv)
    q, k = x[:, :hq], x[:, hq:hq + hk] if hk else None
    # outputs inside a larger matrix, whose other columns stay
    y = torch.full((rows, hq + hk + 2, dim), 7.0, dtype=x.dtype, device="cuda")
    L.slide_head_rope_fwd(rope, q, k, d(pos) if pairs else None, y[:, 1:1 + hq], y[:, 1 + hq:-1] if hk else None, gq=d(gq), gk=d(gk))
    c, s = to.rotation(pos.numpy(), pairs, dim, THETA)
    a, b = to.columns(dim, pairing)

    def pair_size(v):
        w = np.abs(v).copy()
        w[..., a] = w[..., b] = np.hypot(v[..., a], v[..., b])
        return w
    parts = [("q", q, gq, y[:, 1:1 + hq], dy[:, :hq])] + ([("k", k, gk, y[:, 1 + hq:-1], dy[:, hq:])] if hk else [])
    for name, xin, gain, got, _ in parts:
        want = to.rope_fwd(_np(xin), None if gain is None else _np(gain), c, s, pairing, EPS)
        _close(_np(got), want, pair_size(want), dtype, name)
    assert torch.all(y[:, 0] == 7) and torch.all(y[:, -1] == 7)

    # backward, with the gains' gradients written and then added to
    work = torch.empty(L.slide_head_rope_workspace_bytes(rope, rows, hq, hk), dtype=torch.uint8, device="cuda")
    dyg = d(dy)
    dx = torch.full((rows, hq + hk + 1, dim), 7.0, dtype=x.dtype, device="cuda")
    dg = [torch.full((dim,), 5.0, device="cuda") if n is not None else None for n in (gq, gk)]
    for accumulate in (False, True):
        L.slide_head_rope_bwd(rope, dyg[:, :hq], dyg[:, hq:] if hk else None, q if norm else None, k if norm and hk else None, d(pos) if pairs else None,
                              dx[:, :hq], dx[:, hq:hq + hk] if hk else None, gq=d(gq), gk=d(gk), dgq=dg[0], dgk=dg[1], accumulate=accumulate, workspace=work)
    assert torch.all(dx[:, -1] == 7)
    for (name, xin, gain, _, g), got, dgain in zip(parts, (dx[:, :hq], dx[:, hq:hq + hk]), dg):
        v = _np(xin)
        want, want_gain = to.rope_bwd(_np(g), v, None if gain is None else _np(gain), c, s, pairing, EPS)
        size = pair_size(_np(g))
        if gain is not None:
            # the difference in dx: its terms' sizes, and the mean's sum over the columns
            w, r = _np(gain), 1 / np.sqrt((v * v).mean(-1, keepdims=True) + EPS)
            u = size * np.abs(w)
            size = r * (u + 2 * np.abs(v * r) * (u * np.abs(v * r)).mean(-1, keepdims=True))
            terms = (pair_size(_np(g)) * np.abs(v * r)).sum((0, 1))
            # float32 sums over n terms in parts: 12 units a term and sqrt-free worst case of 40 additions in a row + log2 of the rest
            off = np.abs(_np(dgain) - 2 * want_gain)
            assert np.all(off <= 2 * (12 + 64 + rows * hq / 4096) * 2.0 ** -24 * terms), (name, off.max())
        _close(_np(got), want, 2 * size, dtype, "d" + name)


@pytest.mark.parametrize("which", [0, 1])
def test_one_of_the_gains(which):
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print(f"case rope one gain {which}", flush=True)
    L, rope = TokensLib(), HeadRope(48, (10, 8), THETA, "neighbours", EPS)
    qkv, pos, gains, dy = _make(301, 3, 3, 48, (10, 8), "fp32", True)
    gains[1 - which] = None
    x, g = qkv.cuda(), dy.cuda()
    gq, gk = (None if v is None else v.cuda() for v in gains)
    y, d = torch.empty_like(g), torch.empty_like(g)
    L.slide_head_rope_fwd(rope, x[:, :3], x[:, 3:6], pos.cuda(), y[:, :3], y[:, 3:], gq=gq, gk=gk)
    dg = [None if v is None else torch.empty(48, device="cuda") for v in gains]
    work = torch.empty(L.slide_head_rope_workspace_bytes(rope, 301, 3, 3), dtype=torch.uint8, device="cuda")
    L.slide_head_rope_bwd(rope, g[:, :3], g[:, 3:], x[:, :3] if which == 0 else None, x[:, 3:6] if which else None, pos.cuda(), d[:, :3], d[:, 3:], gq=gq, gk=gk,
                          dgq=dg[0], dgk=dg[1], workspace=work)
    c, s = to.rotation(pos.numpy(), (10, 8), 48, THETA)
    for i in (0, 1):
        v, w = _np(qkv[:, 3 * i:3 * i + 3]), _np(dy[:, 3 * i:3 * i + 3])
        gain = None if gains[i] is None else _np(gains[i])
        want, (wx, wg) = to.rope_fwd(v, gain, c, s, "neighbours", EPS), to.rope_bwd(w, v, gain, c, s, "neighbours", EPS)
        # float32 as above, of the whole tensors' norms: 12 roundings, four times that where differences are taken, sums of 903 terms in parts
        for got, ref, units in ((y, want, 12), (d, wx, 48)):
            assert np.linalg.norm(_np(got[:, 3 * i:3 * i + 3]) - ref) <= units * 2.0 ** -24 * np.linalg.norm(ref)
        if gain is not None:
            assert np.linalg.norm(_np(dg[i]) - wg) <= 76 * 2.0 ** -24 * np.linalg.norm(np.abs(w).sum((0, 1)) + np.abs(wg))


def test_in_place_and_bits_again():
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print("case rope in place", flush=True)
    L, rope = TokensLib(), HeadRope(64, (16, 16), THETA)
    qkv, pos, (gq, gk), dy = _make(999, 6, 2, 64, (16, 16), "bf16", True)
    x, p, gq, gk = qkv.cuda(), pos.cuda(), gq.cuda(), gk.cuda()
    y = torch.empty_like(x)
    L.slide_head_rope_fwd(rope, x[:, :6], x[:, 6:8], p, y[:, :6], y[:, 6:8], gq=gq, gk=gk)
    z = x.clone()
    L.slide_head_rope_fwd(rope, z[:, :6], z[:, 6:8], p, z[:, :6], z[:, 6:8], gq=gq, gk=gk)
    assert torch.equal(y[:, :8], z[:, :8]) and torch.equal(z[:, 8:], x[:, 8:])
    work = torch.empty(L.slide_head_rope_workspace_bytes(rope, 999, 6, 2), dtype=torch.uint8, device="cuda")
    out = []
    for place in (False, True, False):
        g = dy.cuda()
        d = g if place else torch.empty_like(g)
        dgq, dgk = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
        L.slide_head_rope_bwd(rope, g[:, :6], g[:, 6:], x[:, :6], x[:, 6:8], p, d[:, :6], d[:, 6:], gq=gq, gk=gk, dgq=dgq, dgk=dgk, workspace=work)
        out.append((d, dgq, dgk))
    for a, b in zip(out[0], out[1]):
        assert torch.equal(a, b)
    for a, b in zip(out[0], out[2]):
        assert torch.equal(a, b)


def test_far_positions_and_large_values():
    """Positions to the ends of 32 bits; values whose squares float32 does not hold; a row of zeros."""
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print("case rope far", flush=True)
    L, rope = TokensLib(), HeadRope(32, (8, 8), 3.0)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31], [0, 0], [123456789, -987654321], [1, 1]], dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    x = torch.randn((4, 2, 32), generator=g)
    c, s = to.rotation(pos.numpy(), (8, 8), 32, 3.0)
    y = torch.empty_like(x, device="cuda")
    L.slide_head_rope_fwd(rope, x.cuda(), None, pos.cuda(), y, None)
    want = to.rope_fwd(_np(x), None, c, s, "halves", EPS)
    # a phase is right to 2^-31 of a turn, 2^-33 of one a rounding of its frequency: 4e-9 in all
    assert np.abs(_np(y) - want).max() <= (12 * 2.0 ** -24 + 4e-9) * 1.5 * np.abs(_np(x)).max()
    x[0] *= 1e25
    x[1] = 0
    x[2] *= 1e-30
    gain = torch.ones(32)
    L.slide_head_rope_fwd(rope, x.cuda(), None, pos.cuda(), y, None, gq=gain.cuda())
    want = to.rope_fwd(_np(x), np.ones(32), c, s, "halves", EPS)
    assert np.all(_np(y)[1] == 0)
    for r in (0, 2, 3):
        assert np.abs(_np(y)[r] - want[r]).max() <= (12 * 2.0 ** -24 + 4e-9) * 1.5 * np.abs(want[r]).max()


def test_captured_and_on_another_stream():
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print("case rope captured", flush=True)
    L, rope = TokensLib(), HeadRope(64, (16, 16), THETA)
    qkv, pos, (gq, gk), dy = _make(513, 6, 6, 64, (16, 16), "bf16", True)
    x, p, gq, gk, g = qkv.cuda(), pos.cuda(), gq.cuda(), gk.cuda(), dy.cuda()
    work = torch.empty(L.slide_head_rope_workspace_bytes(rope, 513, 6, 6), dtype=torch.uint8, device="cuda")

    def run(y, d, dgq, dgk):
        L.slide_head_rope_fwd(rope, x[:, :6], x[:, 6:12], p, y[:, :6], y[:, 6:], gq=gq, gk=gk)
        L.slide_head_rope_bwd(rope, g[:, :6], g[:, 6:], x[:, :6], x[:, 6:12], p, d[:, :6], d[:, 6:], gq=gq, gk=gk, dgq=dgq, dgk=dgk, workspace=work)

    def outputs():
        return torch.zeros_like(g), torch.zeros_like(g), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    want, got = outputs(), outputs()
    run(*want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run(*got)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*got)
    for i in range(3):
        x.mul_(1.25)
        g.mul_(0.5)
        run(*want)
        torch.cuda.synchronize()
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b), i
