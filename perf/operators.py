"""Layers on activations that are kept in 8 bits, as cases that can be timed: what include/act8.h offers.

A case is a dict of plain values.  `op` names what a pass goes through:
  checkpoint  slide_act8_pack + slide_act8_unpack: an activation is put away in 8 bits and taken back for the backward
  linear      slide_act8_linear: activations packed and multiplied by packed weights, bias, activation, residual
  wgrad       slide_act8_wgrad: a linear layer's weight and bias gradients out of the packed activations
  norm        slide_group_norm_fwd: group norm with its activation, channels last, as inference runs it
  norm_bwd    slide_group_norm_bwd on the statistics that the forward left
  norm_step   slide_group_norm_fwd, which puts its input away in 8 bits, and slide_group_norm_bwd out of that
`own` false: elementary torch operations in 32 bits; true: the calls of this package.

A matrix in 8 bits is one e4m3 code a value and one power of two (a byte: its exponent plus 127) for each row's block of 128
columns, the smallest that brings the block's largest magnitude to 448 or less.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
ACTS = ("none", "relu", "silu", "gelu")
TOKENS = 197       # tokens of a 224-pixel tile in patches of 16, class token included
EPS = 1e-5


def _checkpoint(rows, cols, dtype="bf16"):
    return dict(op="checkpoint", rows=rows, cols=cols, dtype=dtype)


def _linear(rows, cin, cout, dtype="bf16", bias=True, act="none", residual=False):
    return dict(op="linear", rows=rows, cin=cin, cout=cout, dtype=dtype, bias=bias, act=act, residual=residual)


def _wgrad(rows, cin, cout, dtype="bf16"):
    return dict(op="wgrad", rows=rows, cin=cin, cout=cout, dtype=dtype)


def _norm(op, n, hw, channels, groups, dtype="bf16", act="relu", residual=False):
    return dict(op=op, n=n, hw=hw, channels=channels, groups=groups, dtype=dtype, act=act, residual=residual)


def listed():
    return [
        # block inputs of the ViT-S encoder over a slide of 2048 tiles: what the recompute policy keeps per block
        dict(_checkpoint(2048 * TOKENS, 384), name="checkpoint_vit_s_2048"),
        # a float32 matrix of odd width, a few tiles: latency
        dict(_checkpoint(3 * 65, 100, dtype="fp32"), name="checkpoint_fp32_195x100"),
        # serving one row (a slide embedding, a token) through a wide layer: the weights are all there is to read
        dict(_linear(1, 4096, 4096, act="gelu"), name="linear_one_row"),
        # a needle biopsy's tiles: queries, keys and values of ViT-S
        dict(_linear(37 * TOKENS, 384, 1152), name="linear_qkv_37"),
        # a whole slide's first MLP layer of ViT-S: little contraction, many rows, the output is most of the bytes
        dict(_linear(2048 * TOKENS, 384, 1536, act="gelu"), name="linear_fc1_2048"),
        # a wide square layer with its residual: bound by the products
        dict(_linear(8192, 4096, 4096, residual=True), name="linear_square_8192"),
        # weight gradients of the same slide's first MLP layer
        dict(_wgrad(2048 * TOKENS, 384, 1536), name="wgrad_fc1_2048"),
        # float32 gradients of an odd little layer
        dict(_wgrad(1001, 333, 200, dtype="fp32"), name="wgrad_fp32_1001"),
        # training: first stage of a residual encoder over 1024 tiles of 224 pixels, forward and backward
        dict(_norm("norm_step", 1024, 56 * 56, 64, 32, act="silu"), name="norm_step_56x56x64_1024"),
        # inference on a few tiles in float32, last stage
        dict(_norm("norm", 3, 7 * 7, 512, 32, dtype="fp32", act="silu"), name="norm_fp32_7x7x512_3"),
        # the backward at a residual block's end: rectifier behind the sum with the shortcut
        dict(_norm("norm_bwd", 1024, 28 * 28, 128, 32, residual=True), name="norm_bwd_28x28x128_1024"),
        # two large maps of odd sides: one group's values are spread over many compute units
        dict(_norm("norm_step", 2, 300 * 301, 320, 32, act="gelu"), name="norm_step_300x301x320_2"),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: mostly a multiple of 32, now and then any number."""
    w = _spread(rng, lo, hi)
    return w if rng.random() < 0.2 else max(lo, w // 32 * 32)


def draw(rng):
    family = rng.randrange(6)
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    act = rng.choice(ACTS)
    if family == 0:
        cols = _width(rng, 32, 4096)
        return _checkpoint(_spread(rng, 1, min(400000, 75_000_000 // cols)), cols, dtype)
    if family in (1, 2, 3):
        cin, cout = _width(rng, 32, 4096), _width(rng, 32, 4096)
        most = min(400000, 200_000_000_000 // (cin * cout), 700_000_000 // (cin + cout))
        if family == 3:
            return _wgrad(_spread(rng, 1, most), cin, cout, dtype)
        rows = _spread(rng, 1, 64) if family == 1 else _spread(rng, 65, most)
        return _linear(rows, cin, cout, dtype, bias=rng.random() < 0.7, act=act, residual=rng.random() < 0.3)
    op = rng.choice(("norm", "norm_bwd", "norm_step"))
    if op == "norm_step":
        act = rng.choice(("none", "silu", "gelu"))
    per = rng.choice((1, 2, 4, 6, 8, 10, 16, 32, 64))
    groups = rng.choice((1, 4, 8, 16, 32, 32))
    channels = per * groups
    if family == 4:     # many small maps
        hw = rng.randint(2, 56) ** 2
        n = _spread(rng, 1, max(1, min(4096, 100_000_000 // (hw * channels))))
    else:               # few large ones
        hw = rng.randint(57, 400) * rng.randint(57, 400)
        n = rng.randint(1, max(1, min(8, 100_000_000 // (hw * channels))))
        hw = min(hw, 100_000_000 // channels)
    return _norm(op, n, hw, channels, groups, dtype, act, residual=rng.random() < 0.3 and op != "norm_step")


# ---- 8 bits in elementary operations ---------------------------------------------------------------------------------

def _blocks(x):
    """[rows, cols] -> [rows, blocks, 128], zeros behind the last column."""
    rows, cols = x.shape
    pad = -cols % BLOCK
    if pad:
        x = torch.nn.functional.pad(x, (0, pad))
    return x.reshape(rows, -1, BLOCK)


def _pack(x):
    """Codes (bytes) [rows, columns rounded up to 16] and scales (bytes) [rows, blocks] of x."""
    rows, cols = x.shape
    b = _blocks(x.float())
    m, e = torch.frexp(b.abs().amax(2))                 # amax = m 2^e, 1/2 <= m < 1
    e = torch.where(m > 0.875, e - 8, e - 9)            # 1.75 2^8 = 448
    e = torch.where(m == 0, 0, e).clamp(-127, 127)
    codes = torch.ldexp(b, -e[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(rows, -1)
    return codes[:, :-(-cols // 16) * 16].contiguous(), (e + 127).to(torch.uint8)


def _unpack(codes, scales, cols):
    v = codes.view(torch.float8_e4m3fn).float()
    s = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    return (_blocks(v) * s[:, :, None]).reshape(v.shape[0], -1)[:, :cols]


def _act(u, act):
    if act == "relu":
        return torch.clamp(u, min=0)
    if act == "silu":
        return u / (1 + torch.exp(-u))
    if act == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u


def _act_slope(u, act):
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-u))
        return s * (1 + u * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(u)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _activations(rows, cols, dtype, g):
    """Rows of a residual stream: every channel has a size of its own, a few are much larger than the rest."""
    size = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    size = torch.where(torch.rand(cols, device="cuda", generator=g) < 0.01, 20 * size, size)
    x = torch.empty((rows, cols), dtype=dtype, device="cuda")
    for lo in range(0, rows, 65536):
        hi = min(rows, lo + 65536)
        x[lo:hi] = torch.randn((hi - lo, cols), device="cuda", generator=g) * size
    return x


def _gradients(shape, dtype, g):
    """Gradients of a mean over many positions: small."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        hi = min(flat.numel(), lo + (1 << 26))
        flat[lo:hi] = torch.randn(hi - lo, device="cuda", generator=g) * 1e-3
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, op = _type(case), case["op"]
    s = {"case": case, "kept": {}}
    if op == "checkpoint":
        s["x"] = _activations(case["rows"], case["cols"], t, g)
    elif op == "linear":
        s["x"] = _activations(case["rows"], case["cin"], t, g)
        s["codes"], s["scales"] = _pack(torch.randn((case["cout"], case["cin"]), device="cuda", generator=g) / math.sqrt(case["cin"]))
        s["bias"] = 0.1 * torch.randn(case["cout"], device="cuda", generator=g) if case["bias"] else None
        s["residual"] = _activations(case["rows"], case["cout"], t, g) if case["residual"] else None
    elif op == "wgrad":
        s["codes"], s["scales"] = _pack(_activations(case["rows"], case["cin"], t, g))
        s["dy"] = _gradients((case["rows"], case["cout"]), t, g)
    else:
        n, hw, c = case["n"], case["hw"], case["channels"]
        x = _activations(n * hw, c, t, g)
        s["x"] = x.add_(torch.randn(c, device="cuda", generator=g).to(t)).view(n, hw, c)
        s["gamma"] = 1 + 0.1 * torch.randn(c, device="cuda", generator=g)
        s["beta"] = 0.1 * torch.randn(c, device="cuda", generator=g)
        s["residual"] = _activations(n * hw, c, t, g).view(n, hw, c) if case["residual"] else None
        if op != "norm":
            s["dy"] = _gradients((n, hw, c), t, g)
        if op == "norm_bwd":
            s["mean"], s["rstd"] = _statistics(s["x"], case)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _grouped(x, case):
    return x.view(case["n"], case["hw"], case["groups"], -1)


def _statistics(x, case):
    v = _grouped(x, case).float()
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, 1 / torch.sqrt(var + EPS)


def _normalised(x, mean, rstd, case, t=torch.float32):
    v = _grouped(x, case).to(t)
    return ((v - mean.to(t)[:, None, :, None]) * rstd.to(t)[:, None, :, None]).view(x.shape)


def _before_act(xhat, s):
    u = xhat * s["gamma"].to(xhat.dtype) + s["beta"].to(xhat.dtype)
    return u if s["residual"] is None else u + s["residual"].to(xhat.dtype)


def _norm_gradients(x, mean, rstd, s):
    """dx, residual's gradient, dgamma, dbeta in 32 bits."""
    case = s["case"]
    xhat = _normalised(x, mean, rstd, case)
    # which side of zero a value is on: next to zero 32 bits do not tell
    u = _before_act(_normalised(x, mean, rstd, case, torch.float64) if case["act"] == "relu" else xhat, s)
    du = s["dy"].float() * _act_slope(u, case["act"]).float()
    dgamma, dbeta = (du * xhat).sum((0, 1)), du.sum((0, 1))
    t = _grouped(du * s["gamma"], case)
    h = _grouped(xhat, case)
    dx = (t - t.mean((1, 3), keepdim=True) - h * (t * h).mean((1, 3), keepdim=True)) * rstd[:, None, :, None]
    return dx.view(x.shape), du, dgamma, dbeta


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    t = _type(case)
    if op == "checkpoint":
        return {"x": _unpack(*_pack(s["x"]), case["cols"]).to(t)}
    if op == "linear":
        x = _unpack(*_pack(s["x"]), case["cin"])
        y = x @ _unpack(s["codes"], s["scales"], case["cin"]).t()
        if s["bias"] is not None:
            y += s["bias"]
        y = _act(y, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(t)}
    if op == "wgrad":
        dy = s["dy"].float()
        return {"dW": dy.t() @ _unpack(s["codes"], s["scales"], case["cin"]), "db": dy.sum(0)}
    if op == "norm_bwd":
        mean, rstd, x = s["mean"], s["rstd"], s["x"]
        out = {}
    else:
        mean, rstd = _statistics(s["x"], case)
        y = _act(_before_act(_normalised(s["x"], mean, rstd, case), s), case["act"])
        out = {"y": y.to(t), "mean": mean, "rstd": rstd}
        if op == "norm":
            return out
        x = _unpack(*_pack(s["x"].view(-1, case["channels"])), case["channels"]).view(s["x"].shape)
    dx, dres, dgamma, dbeta = _norm_gradients(x, mean, rstd, s)
    out.update(dx=dx.to(t), dgamma=dgamma, dbeta=dbeta)
    if s["residual"] is not None:
        out["dresidual"] = dres.to(t)
    return out


# ---- the package's calls ---------------------------------------------------------------------------------------------

def _buffers(s):
    """Outputs, checkpoints and work space, which a program makes once."""
    from paper_2403_04865_amd import Act8, Act8Lib
    case, op = s["case"], s["case"]["op"]
    t = _type(case)
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")   # noqa: E731
    lib = Act8Lib()
    k = {"lib": lib}
    if op == "checkpoint":
        k["x8"] = Act8.empty(case["rows"], case["cols"], "cuda")
        k["x"] = torch.empty_like(s["x"])
    elif op == "linear":
        k["x8"] = Act8.empty(case["rows"], case["cin"], "cuda")
        k["w8"] = Act8(case["cout"], case["cin"], s["codes"], s["scales"])
        k["y"] = new(case["rows"], case["cout"], dtype=t)
    elif op == "wgrad":
        k["x8"] = Act8(case["rows"], case["cin"], s["codes"], s["scales"])
        k["dW"], k["db"] = new(case["cout"], case["cin"]), new(case["cout"])
        k["work"] = new(lib.slide_act8_wgrad_workspace_bytes(case["rows"], case["cout"], case["cin"]), dtype=torch.uint8)
    else:
        n, hw, c, groups = case["n"], case["hw"], case["channels"], case["groups"]
        need = lib.slide_group_norm_workspace_bytes(n, hw, c, groups, t)
        k["work"] = new(need, dtype=torch.uint8)
        if op != "norm_bwd":
            k["y"], k["mean"], k["rstd"] = torch.empty_like(s["x"]), new(n, groups), new(n, groups)
        if op == "norm_step":
            k["x8"] = Act8.empty(n * hw, c, "cuda")
        if op != "norm":
            k["dx"], k["dgamma"], k["dbeta"] = torch.empty_like(s["x"]), new(c), new(c)
            k["dresidual"] = torch.empty_like(s["x"]) if s["residual"] is not None else None
    return k


def _own(s):
    if not s["kept"]:
        s["kept"] = _buffers(s)
    case, k = s["case"], s["kept"]
    op, lib = case["op"], k["lib"]
    if op == "checkpoint":
        lib.slide_act8_pack(s["x"], k["x8"])
        lib.slide_act8_unpack(k["x8"], k["x"])
        return {"x": k["x"]}
    if op == "linear":
        lib.slide_act8_linear(s["x"], k["x8"], k["w8"], k["y"], bias=s["bias"], act=case["act"], residual=s["residual"])
        return {"y": k["y"]}
    if op == "wgrad":
        lib.slide_act8_wgrad(s["dy"], k["x8"], k["dW"], k["db"], workspace=k["work"])
        return {"dW": k["dW"], "db": k["db"]}
    groups, act = case["groups"], case["act"]
    out = {}
    if op != "norm_bwd":
        lib.slide_group_norm_fwd(s["x"], s["gamma"], s["beta"], groups, k["y"], k["mean"], k["rstd"], eps=EPS, act=act,
                                 residual=s["residual"], x8=k.get("x8"), workspace=k["work"])
        out = {"y": k["y"], "mean": k["mean"], "rstd": k["rstd"]}
        if op == "norm":
            return out
    mean, rstd = (k["mean"], k["rstd"]) if op == "norm_step" else (s["mean"], s["rstd"])
    x = k["x8"] if op == "norm_step" else s["x"]
    lib.slide_group_norm_bwd(s["dy"], x, s["gamma"], s["beta"], mean, rstd, groups, k["dx"], k["dgamma"], k["dbeta"], act=act,
                             residual=s["residual"], dresidual=k["dresidual"], workspace=k["work"])
    out.update(dx=k["dx"], dgamma=k["dgamma"], dbeta=k["dbeta"])
    if s["residual"] is not None:
        out["dresidual"] = k["dresidual"]
    return out


def run(s):
    return _own(s) if own else _plain(s)


# ---- work ------------------------------------------------------------------------------------------------------------

def work(case):
    e, op = (2 if case["dtype"] == "bf16" else 4), case["op"]
    in8 = lambda rows, cols: rows * (cols + -(-cols // BLOCK))   # noqa: E731
    if op == "checkpoint":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": 2.0 * (rows * cols * e + in8(rows, cols)), "flops": 2.0 * rows * cols}
    if op in ("linear", "wgrad"):
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        flops = 2.0 * rows * cin * cout
        if op == "wgrad":
            return {"bytes": in8(rows, cin) + rows * cout * e + 4.0 * cout * (cin + 1), "flops": flops}
        return {"bytes": rows * (cin + cout * (2 if case["residual"] else 1)) * float(e) + in8(cout, cin) + 4.0 * cout * case["bias"],
                "flops": flops}
    values = float(case["n"] * case["hw"] * case["channels"])
    res = 1 if case["residual"] else 0
    kept = in8(case["n"] * case["hw"], case["channels"])
    fwd, bwd = values * e * (2 + res), values * e * (3 + 2 * res)
    if op == "norm":
        return {"bytes": fwd, "flops": 10 * values}
    if op == "norm_bwd":
        return {"bytes": bwd, "flops": 20 * values}
    return {"bytes": fwd + bwd - values * e + 2 * kept, "flops": 30 * values}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _held(x):
    """What 8 bits keep of the rows of x, from the definition: per block the power of two, then the nearest number of four
    significant bits that is a multiple of 2^-9, ties to the even one."""
    x = x.double()
    rows, cols = x.shape
    for lo in range(0, cols, 128):
        b = x[:, lo:lo + 128]
        top = b.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 448.0))
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)          # what log2 rounded away
        e = torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(-127, 127)
        v = b * torch.exp2(-e)
        fine = torch.exp2(torch.clamp(torch.floor(torch.log2(v.abs().clamp(min=1e-30))), min=-6) - 3)
        x[:, lo:lo + 128] = torch.round(v / fine) * fine * torch.exp2(e)
    return x


def _stands_for(s, cols):
    """The values of the packed matrix in hand, bit by bit of the code: sign, four of exponent, three of mantissa."""
    c = s["codes"][:, :cols].int()
    power, frac = (c >> 3) & 15, (c & 7).double()
    v = torch.where(power > 0, (1 + frac / 8) * torch.exp2(power.double() - 7), frac * 2.0 ** -9)
    v = torch.where(c >= 128, -v, v)
    e = s["scales"].double() - 127
    return v * torch.exp2(e.repeat_interleave(128, 1)[:, :cols])


def _phi(u):
    return 0.5 * torch.special.erfc(-u / math.sqrt(2))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "checkpoint":
        return {"x": _held(s["x"])}
    if op == "wgrad":
        dy = s["dy"].double()
        return {"dW": dy.t() @ _stands_for(s, case["cin"]), "db": dy.sum(0)}
    curve = {"none": lambda u: u, "relu": lambda u: u * (u > 0), "silu": lambda u: u * torch.sigmoid(u), "gelu": lambda u: u * _phi(u)}
    if op == "linear":
        y = _held(s["x"]) @ _stands_for(s, case["cin"]).t()
        y = curve[case["act"]](y if s["bias"] is None else y + s["bias"].double())
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    n, hw, c, groups = case["n"], case["hw"], case["channels"], case["groups"]
    per = c // groups
    wide = lambda v: v.repeat_interleave(per, 1)[:, None, :]            # noqa: E731  [n, groups] -> [n, 1, channels]
    means = lambda v: v.sum(1).view(n, groups, per).sum(2) / (hw * per)  # noqa: E731  [n, hw, channels] -> [n, groups]
    x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
    shift = 0.0 if s["residual"] is None else s["residual"].double()
    out = {}
    if op == "norm_bwd":
        mean, rstd = s["mean"].double(), s["rstd"].double()
    else:
        mean = means(x)
        rstd = (means((x - wide(mean)) ** 2) + EPS) ** -0.5
        u = (x - wide(mean)) * wide(rstd) * gamma + beta + shift
        out = {"y": curve[case["act"]](u), "mean": mean, "rstd": rstd}
        if op == "norm":
            return out
        x = _held(x.view(-1, c)).view(n, hw, c)
    h = (x - wide(mean)) * wide(rstd)
    u = h * gamma + beta + shift
    du = s["dy"].double()
    if case["act"] == "relu":
        du = du * (u > 0)
    elif case["act"] == "silu":
        du = du * torch.sigmoid(u) * (1 + u * torch.sigmoid(-u))
    elif case["act"] == "gelu":
        du = du * (_phi(u) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi))
    out["dgamma"], out["dbeta"] = (du * h).sum((0, 1)), du.sum((0, 1))
    t = du * gamma
    out["dx"] = wide(rstd) * (t - wide(means(t)) - h * wide(means(t * h)))
    if s["residual"] is not None:
        out["dresidual"] = du
    return out
