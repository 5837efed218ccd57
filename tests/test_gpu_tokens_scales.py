"""Attention over packed slides with scales and slopes of every accepted size, through the C ABI against the 64-bit oracle (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu

CASES = [
    # scale, size of queries, keys and values, cap, slopes times
    (2.0 ** -40, 1.0, 0.0, 1.0),            # only the distances count
    (2.0 ** -40, 2.0 ** 19, 0.0, 0.0),
    (2.0 ** -40, 2.0 ** 19, 5.0, 4.0),
    (2.0 ** 40, 2.0 ** -21, 0.0, 0.0),
    (2.0 ** 40, 2.0 ** -21, 3.0, 1.0),
    (2.0 ** 40, 2.0 ** -40, 0.0, 1.0),      # products of 2^-40 and distances
    (1.0, 1.0, 0.0, -1.0),                  # the farthest keys count
    (0.125, 1.0, 0.0, 2.0 ** 8),            # a row's own place, and those that share it
    (0.125, 1.0, 2.0 ** 40, 2.0 ** 8),
    (3.0, 1.0, 1.0, -0.01),
]


@pytest.mark.parametrize("scale,size,cap,slopes", CASES)
@pytest.mark.parametrize("lq,lk,hq,hk,dim", [([150, 33, 1], [150, 33, 1], 4, 2, 64), ([61, 20], [61, 20], 3, 1, 48), ([2, 1], [500, 90], 2, 2, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scales_and_slopes(scale, size, cap, slopes, lq, lk, hq, hk, dim, dtype):
    from test_gpu_tokens_attn import Case, _check
    print(f"case scale {scale} size {size} cap {cap} slopes {slopes} {lq} x {lk} ({hq},{hk})x{dim} {dtype}", flush=True)
    c = Case(lq, lk, hq, hk, dim, dtype, cap, slopes != 0, 0, 0, front=1, behind=1, size=size)
    c.how["scale"] = scale
    if slopes:
        c.places["slopes"] *= slopes
        c.dev_places = {n: x.cuda() for n, x in c.places.items()}
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)


@pytest.mark.parametrize("heads,dim", [((2, 2), 64), ((2, 1), 48), ((2, 2), 128)])
@pytest.mark.parametrize("rows", [[40, 3], [400, 90]])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_key_far(heads, dim, rows, dtype):
    """Rows whose largest score is some -30000: the nearest of far keys share them; other keys, 2^40 away, have nothing."""
    from test_gpu_tokens_attn import Case, _check
    print(f"case far keys {heads} {dim} {rows} {dtype}", flush=True)
    c = Case(rows, [300, 70], *heads, dim, dtype, bias=True)
    c.places["pos_q"] += 30000.0
    c.places["pos_k"][::3] -= 2.0 ** 39
    c.places["slopes"].fill_(0.75)
    c.dev_places = {n: x.cuda() for n, x in c.places.items()}
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)
