"""Attention over packed slides with caps of every accepted size, through the C ABI against the 64-bit oracle (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu

SHAPES = [
    # queries, keys of each slide, heads, key heads, head_dim, bias
    ([150, 33, 1], [150, 33, 1], 4, 2, 64, True),      # two heads at a time
    ([130, 61], [130, 61], 3, 1, 48, False),
    ([90, 40], [90, 40], 2, 2, 128, True),
    ([3, 1], [700, 90], 4, 1, 80, True),               # a wavefront a workgroup
]


@pytest.mark.parametrize("cap", [2.0 ** -40, 0.5, 63.5, 64.0, 65.0, 1e4, 2.0 ** 20, 1e9, 2.0 ** 40])
@pytest.mark.parametrize("lq,lk,hq,hk,dim,bias", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_caps_of_every_size(lq, lk, hq, hk, dim, bias, dtype, cap):
    from test_gpu_tokens_attn import Case, _check
    print(f"case cap {cap} {lq} x {lk} ({hq},{hk})x{dim} {dtype} bias={bias}", flush=True)
    c = Case(lq, lk, hq, hk, dim, dtype, cap, bias, 1, 1, front=1, behind=2)
    out = c.outputs()
    c.forward(out)
    c.backward(out)
    _check(c, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_far_cap_is_none(dtype):
    """Scores far below the cap are those without one, to the rounding of a tanh's few units."""
    import torch
    from test_gpu_tokens_attn import Case
    print(f"case far cap {dtype}", flush=True)
    res = []
    for cap in (0.0, 2.0 ** 30):
        c = Case([120, 77], [120, 77], 4, 2, 64, dtype, cap, True, 1, 1)
        out = c.outputs()
        c.forward(out)
        c.backward(out)
        res.append({n: x.double().cpu() for n, x in out.items()})
    for n in res[0]:
        a, b = res[0][n], res[1][n]
        # scores up to 14 that differ by twelve units of 2^-24 of themselves, in a probability and in the sum: 2e-5.  Where that moves a rounding of
        # bfloat16 the result moves by a step, few of them: half a step of each in the norm at most
        limit = 2e-5 if dtype == "fp32" or n == "lse" else 2.0 ** -9
        assert torch.linalg.norm(a - b) <= limit * torch.linalg.norm(a), n

