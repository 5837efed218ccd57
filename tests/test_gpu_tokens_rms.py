"""Attention over packed slides in bfloat16: errors no larger than the roundings that are left, slide length by slide length (needs an MI355X)."""
import numpy as np
import pytest

from oracle import tokens_oracle as to

pytestmark = pytest.mark.gpu

SHORT = [2] * 120 + [7] * 40 + [40] * 6
CASES = [
    # queries, keys of each slide, heads, key heads, head_dim, cap, slopes are times, lead, rows behind the last slide, operands of two terms in the queries' and
    # in the keys' passes (of a single wavefront: up to 32 columns a slide on average)
    (SHORT, SHORT, 4, 2, 64, 0.0, 0, 0, 0, True, True),
    (SHORT, SHORT, 4, 2, 64, 0.0, 0, 0, 50000, False, False),
    (SHORT, SHORT, 3, 1, 48, 2.0, 0, 0, 50000, False, False),
    (SHORT, SHORT, 3, 1, 48, 100.0, 0, 0, 50000, False, False),
    (SHORT, SHORT, 4, 2, 128, 0.0, 1, 1, 50000, False, False),
    ([2] * 8 + [700] * 6, [2] * 8 + [700] * 6, 16, 16, 32, 0.0, 0, 0, 0, False, False),
    ([250] * 3, [250] * 3, 2, 2, 64, 0.0, 64, 0, 0, False, False),     # tiles of several workgroups
    ([257] * 3, [257] * 3, 2, 2, 64, 0.0, 1, 0, 0, False, False),
    ([1] * 64, [100] * 64, 4, 4, 64, 0.0, 0, 0, 0, True, False),
    ([4] * 6, [1500] * 6, 4, 1, 128, 0.0, 0, 0, 0, True, False),
    ([300] * 4, [3] * 4, 4, 4, 96, 0.0, 0, 0, 0, False, True),
]


@pytest.mark.parametrize("lq,lk,hq,hk,dim,cap,slopes,lead,behind,two_q,two_k", CASES)
def test_errors_are_those_of_the_roundings(lq, lk, hq, hk, dim, cap, slopes, lead, behind, two_q, two_k):
    from test_gpu_tokens_attn import Case, _check
    print(f"case rms {str(lq)[:30]} x {str(lk)[:30]} ({hq},{hk})x{dim} cap={cap} slopes={slopes} behind={behind}", flush=True)
    c = Case(lq, lk, hq, hk, dim, "bf16", cap, slopes > 0, lead, lead, behind=behind)
    if slopes:
        c.places["slopes"] *= slopes
        c.dev_places = {n: x.cuda() for n, x in c.places.items()}
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)
    # without the rows of no slide
    ends = {"q": c.qs[-1], "k": c.ks[-1]}
    n = {k: x[:ends["q" if k in ("q", "do", "pos_q") else "k"]].double().numpy() for k, x in {**c.host, **c.places}.items() if k != "slopes"}
    if slopes:
        n["slopes"] = c.places["slopes"].double().numpy()
    q, k, v, do = (n.pop(x) for x in ("q", "k", "v", "do"))
    want = to.attn(q, k, v, c.qs, c.ks, do=do, **c.how, **n)
    var = {two: to.attn_spread(q, k, v, do, c.qs, c.ks, operand=not two, **c.how, **n) for two in {two_q, two_k}}
    for name, starts, lengths, two in (("o", c.qs, lq, two_q), ("dq", c.qs, lq, two_q), ("dk", c.ks, lk, two_k), ("dv", c.ks, lk, two_k)):
        off = out[name][:starts[-1]].double().cpu().numpy() - want[name]
        groups = {m: np.concatenate([np.arange(a, a + m) for a, b in zip(starts[:-1], lengths) if b == m]) for m in sorted(set(lengths))}
        for (ratio, limit), m in zip(to.spread_ratios(off, var[two][name], groups.values()), groups):
            print(f"  {name} of slides of {m}: {ratio:.3f} ({limit:.3f})", flush=True)
            assert ratio <= limit, (name, m, ratio, limit)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("behind", [0, 9000])
def test_slides_of_one_key_move_nothing(dtype, behind):
    """Their only probability is one, whatever the query: its gradient and the key's are what float32 leaves of do . v - do . v."""
    import torch
    from test_gpu_tokens_attn import Case
    print(f"case one key {dtype} {behind}", flush=True)
    lq, dim = [1, 3, 1, 70, 2] * 4, 64
    c = Case(lq, [1] * 20, 2, 2, dim, dtype, behind=behind)
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    h = {n: x.double() for n, x in c.host.items()}
    doc = torch.repeat_interleave(torch.arange(20), torch.tensor(lq))
    rows = len(doc)
    size = (h["do"][:rows].abs() * h["v"][doc].abs()).sum(-1, keepdim=True)         # [rows, heads, 1]
    # each of both sums of 64 products is off by 64 units of 2^-24 of their size; probability, e and the products' own: below as many again
    unit = 3 * dim * 2.0 ** -24 * c.how["scale"]
    assert torch.all(out["dq"][:rows].double().cpu().abs() <= unit * size * h["k"][doc].abs())
    most = torch.zeros_like(h["k"][:20]).index_add_(0, doc, size * h["q"][:rows].abs())
    assert torch.all(out["dk"][:20].double().cpu().abs() <= unit * most)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert torch.all((out["o"][:rows].double().cpu() - h["v"][doc]).abs() <= (half + 64 * 2.0 ** -24) * h["v"][doc].abs())
