"""Operators of a transformer over the tiles of slides, as cases that can be timed: what include/tokens.h offers.

A case is a dict of plain values.  `op` names what a pass goes through:
  rope       slide_head_rope_fwd: queries and keys of every head normalised and rotated by their row's position
  rope_bwd   slide_head_rope_bwd: gradients of both, and of the norms' weights
  attn       slide_tokens_attn_fwd: attention inside every slide of a packed batch, as inference runs it
  attn_step  slide_tokens_attn_fwd and slide_tokens_attn_bwd: training
`own` false: elementary torch operations in 32 bits (angles in 64); true: the calls of this package.

Rows are tokens.  Queries, keys and values are [rows, heads, head_dim], mostly views of one matrix that a linear layer wrote; query head h
reads key head h // (heads_q // heads_k).  A pair of a head's columns belongs to one axis of the positions and turns by
position * theta^(-j / n), j counting the axis' n pairs; pair p is columns p and p + head_dim / 2 ("halves") or 2 p and 2 p + 1
("neighbours"), and the pairs behind the last axis' stay.  A score is cap * tanh(scale q.k / cap) (scale q.k where cap is 0) less slope[head] times the
distance of the two tokens' positions, which is 0 where either is one of the first `lead` rows of its slide (class tokens, which
have no place).  `lengths_q` and `lengths_k` count the rows of each slide.
"""
import math

import torch

own = False

TOKENS = 197       # tokens of a 224-pixel tile in patches of 16, class token included
EPS = 1e-6
THETA = 100.0


def _rope(op, rows, heads_q, heads_k, head_dim, pairs="16,16", pairing="halves", norm=True, dtype="bf16"):
    return dict(op=op, rows=rows, heads_q=heads_q, heads_k=heads_k, head_dim=head_dim, pairs=pairs, pairing=pairing, norm=norm, dtype=dtype)


def _attn(op, lengths_q, heads_q, heads_k, head_dim, lengths_k=None, cap=0.0, bias=True, lead_q=1, lead_k=1, dtype="bf16"):
    text = lambda n: ",".join(str(v) for v in n)   # noqa: E731
    return dict(op=op, lengths_q=text(lengths_q), lengths_k=text(lengths_q if lengths_k is None else lengths_k), heads_q=heads_q,
                heads_k=heads_k, head_dim=head_dim, cap=cap, bias=bias, lead_q=lead_q, lead_k=lead_k, dtype=dtype)


def listed():
    return [
        # one slide token put in front of a stored slide: latency
        dict(_rope("rope", 1, 12, 12, 64), name="rope_one_row"),
        # a needle biopsy's tiles in the ViT-S encoder
        dict(_rope("rope", 37 * TOKENS, 6, 6, 64), name="rope_vit_s_37"),
        # a slide of 2048 tiles in the ViT-S encoder, training
        dict(_rope("rope_bwd", 2048 * TOKENS, 6, 6, 64), name="rope_bwd_vit_s_2048"),
        # float32, rows, columns and a level, shared key heads of an odd width, some columns not rotated
        dict(_rope("rope_bwd", 1001, 8, 2, 80, pairs="14,14,6", pairing="neighbours", dtype="fp32"), name="rope_bwd_fp32_1001"),
        # the 8192-tile slide through a slide encoder of 768 columns
        dict(_attn("attn", [8193], 12, 12, 64), name="attn_slide_8192"),
        # inference on a batch of slides of all sizes, capped scores, shared key heads
        dict(_attn("attn", [1901, 37, 700, 1, 264, 1288, 65, 451, 128, 990, 2047, 5, 333, 1536, 18, 806], 8, 2, 128, cap=30.0),
             name="attn_batch_16_capped"),
        # float32 check of a few biopsies
        dict(_attn("attn", [197, 64, 33], 6, 6, 48, dtype="fp32"), name="attn_fp32_294"),
        # one slide token asks the largest slide of the paper's census: the stored keys and values are all there is to read
        dict(_attn("attn", [1], 12, 12, 64, lengths_k=[50578], lead_k=0), name="attn_token_50578"),
        # a token each of a batch of slides, shared key heads
        dict(_attn("attn", [1] * 12, 12, 4, 64, lengths_k=[4096, 1, 900, 2500, 333, 8192, 47, 1800, 64, 5000, 129, 700], lead_k=0),
             name="attn_token_12_slides"),
        # training on the 8192-tile slide, 384 columns
        dict(_attn("attn_step", [8193], 6, 6, 64), name="attn_step_slide_8192"),
        # training on a batch of small slides, capped scores without a bias
        dict(_attn("attn_step", [520, 1033, 77, 256, 1999, 3, 610], 12, 4, 64, cap=20.0, bias=False), name="attn_step_batch_7"),
        # training where eight tokens pool a slide of 20000 tiles, float32
        dict(_attn("attn_step", [8], 6, 6, 64, lengths_k=[20000], lead_q=8, lead_k=0, dtype="fp32"), name="attn_step_pool_fp32_20000"),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    heads_k = rng.choice((1, 2, 4, 6, 8, 12))
    return heads_k * (rng.choice((1, 1, 2, 3, 4)) if heads_k < 6 else 1), heads_k


def draw(rng):
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    heads_q, heads_k = _heads(rng)
    family = rng.randrange(5)
    if family < 2:
        dim = rng.choice((32, 48, 64, 64, 80, 96, 128))
        axes = rng.randint(1, 3)
        room = dim // 2 - rng.choice((0, 0, 4))
        pairs = [room // axes] * axes
        pairs[0] += room - sum(pairs)
        most = 2048 * TOKENS * 6 * 64 * 2 // ((heads_q + heads_k) * dim * (2 if dtype == "fp32" else 1))
        return _rope("rope" if family == 0 else "rope_bwd", _spread(rng, 1, most), heads_q, heads_k, dim, ",".join(map(str, pairs)),
                     rng.choice(("halves", "neighbours")), rng.random() < 0.7, dtype)
    dim = rng.choice((32, 48, 64, 64, 80, 96, 128))
    cap = rng.choice((0.0, 0.0, 20.0, 50.0))
    bias = rng.random() < 0.7
    if family == 4:      # few queries over long slides
        docs = rng.choice((1, 1, 3, 16))
        most = 50578 * 12 * 64 // (heads_q * dim * docs)
        lengths_k = [_spread(rng, 1 if docs > 2 else 16, most) for _ in range(docs)]
        queries = [rng.choice((1, 1, 1, 4, 8)) for _ in range(docs)]
        return _attn(rng.choice(("attn", "attn", "attn_step")), queries, heads_q, heads_k, dim, lengths_k, cap, bias, 8, 0, dtype)
    step = family == 3
    docs = rng.choice((1, 2, 5, 12, 24))
    budget = 8193 ** 2 * (6 if step else 12) * 64 // (heads_q * dim * (8 if dtype == "fp32" else 1))   # squares of lengths times heads and width
    most = int(math.sqrt(budget / docs))
    lengths = [_spread(rng, 1 if docs > 2 else 16, min(9000, most)) for _ in range(docs)]
    return _attn("attn_step" if step else "attn", lengths, heads_q, heads_k, dim, None, cap, bias, rng.choice((0, 1, 1)), 1, dtype)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _numbers(text):
    return [int(v) for v in text.split(",")]


def _randn(shape, dtype, g, size=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        hi = min(flat.numel(), lo + (1 << 26))
        flat[lo:hi] = torch.randn(hi - lo, device="cuda", generator=g) * size
    return out


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def _places(lengths, g):
    """[rows, 2]: every slide's tiles at places of a grid that they fill to three quarters, row by row."""
    out = []
    for n in lengths:
        side = max(1, math.ceil(math.sqrt(n / 0.75)))
        keep = torch.randperm(side * side, device="cuda", generator=g)[:n].sort().values
        out.append(torch.stack((keep // side, keep % side), 1).float())
    return torch.cat(out).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _type(case)
    hq, hk, dim = case["heads_q"], case["heads_k"], case["head_dim"]
    s = {"case": case, "kept": {}}
    if case["op"].startswith("rope"):
        rows = case["rows"]
        qkv = _randn((rows, hq + 2 * hk, dim), t, g)                 # as a linear layer leaves them
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        axes = len(_numbers(case["pairs"]))
        s["pos"] = torch.randint(0, 1 << 12, (rows, axes), device="cuda", generator=g, dtype=torch.int32)
        s["gq"] = 1 + 0.1 * torch.randn(dim, device="cuda", generator=g) if case["norm"] else None
        s["gk"] = 1 + 0.1 * torch.randn(dim, device="cuda", generator=g) if case["norm"] else None
        if case["op"] == "rope_bwd":
            s["dyq"], s["dyk"] = _randn((rows, hq, dim), t, g, 1e-2), _randn((rows, hk, dim), t, g, 1e-2)
        return s
    lq, lk = _numbers(case["lengths_q"]), _numbers(case["lengths_k"])
    s["lengths"] = (lq, lk)
    s["same"] = case["lengths_q"] == case["lengths_k"]
    if s["same"]:
        qkv = _randn((sum(lq), hq + 2 * hk, dim), t, g)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        kv = _randn((sum(lk), 2 * hk, dim), t, g)
        s["q"], s["k"], s["v"] = _randn((sum(lq), hq, dim), t, g), kv[:, :hk], kv[:, hk:]
    s["q_start"] = _starts(lq)
    s["k_start"] = s["q_start"] if s["same"] else _starts(lk)
    s["pos_q"] = s["pos_k"] = s["slopes"] = None
    if case["bias"]:
        s["pos_k"] = _places(lk, g)
        s["pos_q"] = s["pos_k"] if s["same"] else _places(lq, g)
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device="cuda")
    s["scale"] = 1.0 / math.sqrt(dim)
    if case["op"] == "attn_step":
        s["do"] = _randn((sum(lq), hq, dim), t, g, 1e-2)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _turns(s):
    """cos and sin of every row's pairs, [rows, 1, head_dim / 2], angles in 64 bits."""
    half = s["case"]["head_dim"] // 2
    rows = s["pos"].shape[0]
    phi = torch.zeros((rows, half), dtype=torch.float64, device="cuda")
    at = 0
    for a, n in enumerate(_numbers(s["case"]["pairs"])):
        freq = THETA ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
        phi[:, at:at + n] = s["pos"][:, a, None].double() * freq
        at += n
    return torch.cos(phi).float()[:, None], torch.sin(phi).float()[:, None]


def _halves(x, s):
    if s["case"]["pairing"] == "halves":
        half = x.shape[-1] // 2
        return x[..., :half], x[..., half:]
    return x[..., 0::2], x[..., 1::2]


def _joined(a, b, s):
    return torch.cat((a, b), -1) if s["case"]["pairing"] == "halves" else torch.stack((a, b), -1).flatten(-2)


def _rope_plain(x, gain, cos, sin, s):
    n = x.float()
    if gain is not None:
        n = n * torch.rsqrt(n.square().mean(-1, keepdim=True) + EPS) * gain
    a, b = _halves(n, s)
    return _joined(a * cos - b * sin, b * cos + a * sin, s).to(x.dtype)


def _rope_bwd_plain(dy, x, gain, cos, sin, s):
    a, b = _halves(dy.float(), s)
    dn = _joined(a * cos + b * sin, b * cos - a * sin, s)
    if gain is None:
        return dn.to(x.dtype), None
    v = x.float()
    r = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
    h = v * r
    dgain = (dn * h).sum((0, 1))
    u = dn * gain
    return ((u - h * (u * h).mean(-1, keepdim=True)) * r).to(x.dtype), dgain


def _blocks(s):
    """Slides and runs of key heads: (query rows, key rows, key heads) as slices, whose scores are 2^28 at most where a head's are."""
    group = s["case"]["heads_q"] // s["case"]["heads_k"]
    q0 = k0 = 0
    for nq, nk in zip(*s["lengths"]):
        step = max(1, (1 << 28) // max(1, group * nq * nk))
        for h in range(0, s["case"]["heads_k"], step):
            yield slice(q0, q0 + nq), slice(k0, k0 + nk), slice(h, min(s["case"]["heads_k"], h + step))
        q0, k0 = q0 + nq, k0 + nk


def _heads_first(x, heads, group):
    """[rows, heads * group, dim] -> [heads, group * rows, dim] of the key heads `heads`, 32 bits."""
    rows, _, dim = x.shape
    x = x[:, heads.start * group:heads.stop * group].float()
    return x.reshape(rows, -1, group, dim).permute(1, 2, 0, 3).reshape(-1, group * rows, dim)


def _rows_first(x, group):
    heads, rows, dim = x.shape
    return x.reshape(heads, group, rows // group, dim).permute(2, 0, 1, 3).reshape(rows // group, heads * group, dim)


def _scores(q, k, rq, rk, heads, s):
    """Scores [heads, group * rows, keys] and the cap's tanh, or None."""
    case = s["case"]
    group = case["heads_q"] // case["heads_k"]
    x = torch.matmul(q, k.transpose(1, 2)) * s["scale"]
    t = None
    if case["cap"]:
        t = torch.tanh(x / case["cap"])
        x = t * case["cap"]
    if case["bias"]:
        d = (s["pos_q"][rq, None] - s["pos_k"][None, rk]).square().sum(-1).sqrt()
        d[:case["lead_q"]] = 0
        d[:, :case["lead_k"]] = 0
        slope = s["slopes"][heads.start * group:heads.stop * group].view(-1, group, 1, 1)
        x = (x.view(-1, group, *d.shape) - slope * d).view(x.shape)
    return x, t


def _attn_plain(s):
    case = s["case"]
    group = case["heads_q"] // case["heads_k"]
    o = torch.empty_like(s["q"], dtype=torch.float32)
    lse = torch.empty((case["heads_q"], s["q"].shape[0]), device="cuda")
    for rq, rk, heads in _blocks(s):
        q, k, v = _heads_first(s["q"][rq], heads, group), _heads_first(s["k"][rk], heads, 1), _heads_first(s["v"][rk], heads, 1)
        x, _ = _scores(q, k, rq, rk, heads, s)
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - m)
        z = p.sum(-1, keepdim=True)
        hq = slice(heads.start * group, heads.stop * group)
        o[rq, hq] = _rows_first(torch.matmul(p, v) / z, group)
        lse[hq, rq] = (m + torch.log(z)).view(-1, rq.stop - rq.start)
    return o, lse


def _attn_bwd_plain(s, o, lse):
    case = s["case"]
    group = case["heads_q"] // case["heads_k"]
    dq = torch.empty_like(s["q"], dtype=torch.float32)
    dk, dv = torch.empty_like(s["k"], dtype=torch.float32), torch.empty_like(s["v"], dtype=torch.float32)
    for rq, rk, heads in _blocks(s):
        hq = slice(heads.start * group, heads.stop * group)
        q, k, v = _heads_first(s["q"][rq], heads, group), _heads_first(s["k"][rk], heads, 1), _heads_first(s["v"][rk], heads, 1)
        do = _heads_first(s["do"][rq], heads, group)
        x, t = _scores(q, k, rq, rk, heads, s)
        p = torch.exp(x - lse[hq, rq].reshape(heads.stop - heads.start, -1, 1))
        dv[rk, heads] = _rows_first(torch.matmul(p.transpose(1, 2), do), 1)
        dx = torch.matmul(do, v.transpose(1, 2))
        dx = p * (dx - (do * _heads_first(o[rq], heads, group)).sum(-1, keepdim=True))
        if t is not None:
            dx = dx * (1 - t * t)
        dq[rq, hq] = _rows_first(torch.matmul(dx, k), group) * s["scale"]
        dk[rk, heads] = _rows_first(torch.matmul(dx.transpose(1, 2), q), 1) * s["scale"]
    return dq, dk, dv


def _plain(s):
    case, t = s["case"], _type(s["case"])
    if case["op"] == "rope":
        c = _turns(s)
        return {"q": _rope_plain(s["q"], s["gq"], *c, s), "k": _rope_plain(s["k"], s["gk"], *c, s)}
    if case["op"] == "rope_bwd":
        c = _turns(s)
        dq, dgq = _rope_bwd_plain(s["dyq"], s["q"], s["gq"], *c, s)
        dk, dgk = _rope_bwd_plain(s["dyk"], s["k"], s["gk"], *c, s)
        return {"dq": dq, "dk": dk, "dgq": dgq, "dgk": dgk} if case["norm"] else {"dq": dq, "dk": dk}
    o, lse = _attn_plain(s)
    out = {"o": o.to(t), "lse": lse}
    if case["op"] == "attn_step":
        dq, dk, dv = _attn_bwd_plain(s, o, lse)
        out.update(dq=dq.to(t), dk=dk.to(t), dv=dv.to(t))
    return out


# ---- the package's calls ---------------------------------------------------------------------------------------------

def _buffers(s):
    """Outputs and work space, which a program makes once."""
    from paper_2403_04865_amd import HeadRope, TokensLib
    case, lib = s["case"], TokensLib()
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")   # noqa: E731
    like = lambda x: torch.empty(x.shape, dtype=x.dtype, device="cuda")                        # noqa: E731
    k = {"lib": lib}
    hq, hk, dim = case["heads_q"], case["heads_k"], case["head_dim"]
    if case["op"].startswith("rope"):
        k["rope"] = HeadRope(dim, tuple(_numbers(case["pairs"])), theta=THETA, pairing=case["pairing"], eps=EPS)
        k["q"], k["k"] = like(s["q"]), like(s["k"])
        if case["op"] == "rope_bwd":
            k["dgq"], k["dgk"] = (new(dim), new(dim)) if case["norm"] else (None, None)
            k["work"] = new(lib.slide_head_rope_workspace_bytes(k["rope"], case["rows"], hq, hk), dtype=torch.uint8)
        return k
    rows_q, rows_k = s["q"].shape[0], s["k"].shape[0]
    docs = len(s["lengths"][0])
    step = case["op"] == "attn_step"
    k["o"], k["lse"] = like(s["q"]), new(hq, rows_q)
    k["work"] = new(lib.slide_tokens_attn_workspace_bytes(rows_q, rows_k, docs, hq, hk, dim, s["q"].dtype, backward=step), dtype=torch.uint8)
    if step:
        k["dq"], k["dk"], k["dv"] = like(s["q"]), like(s["k"]), like(s["v"])
    return k


def _own(s):
    if not s["kept"]:
        s["kept"] = _buffers(s)
    case, k = s["case"], s["kept"]
    lib = k["lib"]
    if case["op"] == "rope":
        lib.slide_head_rope_fwd(k["rope"], s["q"], s["k"], s["pos"], k["q"], k["k"], gq=s["gq"], gk=s["gk"])
        return {"q": k["q"], "k": k["k"]}
    if case["op"] == "rope_bwd":
        lib.slide_head_rope_bwd(k["rope"], s["dyq"], s["dyk"], s["q"], s["k"], s["pos"], k["q"], k["k"], gq=s["gq"], gk=s["gk"],
                                dgq=k["dgq"], dgk=k["dgk"], workspace=k["work"])
        out = {"dq": k["q"], "dk": k["k"]}
        if case["norm"]:
            out.update(dgq=k["dgq"], dgk=k["dgk"])
        return out
    how = dict(scale=s["scale"], cap=case["cap"], pos_q=s["pos_q"], pos_k=s["pos_k"], slopes=s["slopes"], lead_q=case["lead_q"],
               lead_k=case["lead_k"], workspace=k["work"])
    lib.slide_tokens_attn_fwd(s["q"], s["k"], s["v"], s["q_start"], s["k_start"], k["o"], k["lse"], **how)
    out = {"o": k["o"], "lse": k["lse"]}
    if case["op"] == "attn_step":
        lib.slide_tokens_attn_bwd(s["do"], s["q"], s["k"], s["v"], k["o"], k["lse"], s["q_start"], s["k_start"], k["dq"], k["dk"], k["dv"], **how)
        out.update(dq=k["dq"], dk=k["dk"], dv=k["dv"])
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    hq, hk, dim = case["heads_q"], case["heads_k"], case["head_dim"]
    if case["op"].startswith("rope"):
        values = case["rows"] * (hq + hk) * dim
        places = 4 * case["rows"] * len(_numbers(case["pairs"]))
        if case["op"] == "rope":
            return {"bytes": 2 * values * size + places, "flops": values * (7 if case["norm"] else 3)}
        return {"bytes": (3 if case["norm"] else 2) * values * size + places, "flops": values * (14 if case["norm"] else 3)}
    lq, lk = _numbers(case["lengths_q"]), _numbers(case["lengths_k"])
    products = hq * dim * sum(a * b for a, b in zip(lq, lk))
    queries, keys = sum(lq) * hq * dim * size, sum(lk) * hk * dim * size
    rest = 4 * sum(lq) * hq + (8 * (sum(lq) + sum(lk)) if case["bias"] else 0)
    if case["op"] == "attn":
        return {"bytes": 2 * queries + 2 * keys + rest, "flops": 4 * products}
    # the step: queries, keys, values and the gradient in, output and three gradients out
    return {"bytes": 4 * queries + 4 * keys + rest, "flops": 14 * products}


# ---- in 64 bits, from the definitions --------------------------------------------------------------------------------

def _turned(x, gain, s):
    """Every pair as a complex number times e^(i phi)."""
    case = s["case"]
    n = x
    if gain is not None:
        n = n / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
    half = case["head_dim"] // 2
    first = torch.arange(half, device="cuda")
    first, second = (first, first + half) if case["pairing"] == "halves" else (2 * first, 2 * first + 1)
    phi = [s["pos"][:, a, None].double() * torch.tensor([THETA ** (-j / c) for j in range(c)], dtype=torch.float64, device="cuda")
           for a, c in enumerate(_numbers(case["pairs"]))]
    phi = torch.cat(phi, 1)
    phi = torch.nn.functional.pad(phi, (0, half - phi.shape[1]))[:, None]
    z = torch.complex(n[..., first], n[..., second]) * torch.polar(torch.ones_like(phi), phi)
    y = torch.empty_like(x)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _rope_exact(x, gain, dy, s):
    """The rotated values, or the gradients of both inputs."""
    if dy is None:
        return _turned(x.double(), None if gain is None else gain.double(), s), None
    v = x.double().requires_grad_()
    w = None if gain is None else gain.double().requires_grad_()
    wanted = [v] if w is None else [v, w]
    with torch.enable_grad():
        got = torch.autograd.grad(_turned(v, w, s), wanted, dy.double())
    return got if w is not None else (got[0], None)


def _one_head(q, k, v, d, slope, s):
    x = (q @ k.t()) * s["scale"]
    if s["case"]["cap"]:
        x = s["case"]["cap"] * torch.tanh(x / s["case"]["cap"])
    if d is not None:
        x = x - slope * d
    return torch.softmax(x, 1) @ v, torch.logsumexp(x, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return {"q": _rope_exact(s["q"], s["gq"], None, s)[0], "k": _rope_exact(s["k"], s["gk"], None, s)[0]}
    if case["op"] == "rope_bwd":
        dq, dgq = _rope_exact(s["q"], s["gq"], s["dyq"], s)
        dk, dgk = _rope_exact(s["k"], s["gk"], s["dyk"], s)
        return {"dq": dq, "dk": dk, "dgq": dgq, "dgk": dgk} if case["norm"] else {"dq": dq, "dk": dk}
    step = case["op"] == "attn_step"
    like = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")   # noqa: E731
    out = {"o": like(s["q"]), "lse": torch.zeros((case["heads_q"], s["q"].shape[0]), dtype=torch.float64, device="cuda")}
    if step:
        out.update(dq=like(s["q"]), dk=like(s["k"]), dv=like(s["v"]))
    q1 = k1 = 0
    for nq, nk in zip(*s["lengths"]):
        q0, k0, q1, k1 = q1, k1, q1 + nq, k1 + nk
        d = None
        if case["bias"]:
            a, b = s["pos_q"][q0:q1].double(), s["pos_k"][k0:k1].double()
            d = torch.hypot(a[:, None, 0] - b[None, :, 0], a[:, None, 1] - b[None, :, 1])
            placed_q, placed_k = torch.arange(nq, device="cuda") >= case["lead_q"], torch.arange(nk, device="cuda") >= case["lead_k"]
            d = torch.where(placed_q[:, None] & placed_k[None], d, 0.0)
        for h in range(case["heads_q"]):
            hk = h * case["heads_k"] // case["heads_q"]
            q, k, v = (x.double().requires_grad_(step) for x in (s["q"][q0:q1, h], s["k"][k0:k1, hk], s["v"][k0:k1, hk]))
            with torch.set_grad_enabled(step):
                o, lse = _one_head(q, k, v, d, None if d is None else s["slopes"][h].double(), s)
                if step:
                    dq, dk, dv = torch.autograd.grad(o, (q, k, v), s["do"][q0:q1, h].double())
                    out["dq"][q0:q1, h] = dq
                    out["dk"][k0:k1, hk] += dk
                    out["dv"][k0:k1, hk] += dv
            out["o"][q0:q1, h] = o.detach()
            out["lse"][h, q0:q1] = lse.detach()
    return out
