"""Float32 linear layers on 8-bit activations: positive operands, whose products' errors a bias would line up (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu


# One row, a few, tiles of 128.  Limit of the mean error: what float32 products elsewhere keep to, 3e-8 of the result.  Each result: its products are
# exact, its additions round by 2^-24 of a partial sum each, of either sign, 2 sqrt(K) 2^-24 of the result at most.
@pytest.mark.parametrize("rows,cin,cout", [(1, 4096, 4096), (40, 768, 1000), (300, 4096, 512), (4096, 384, 768), (2048, 768, 1024), (1100, 10000, 1000)])
def test_positive_operands_have_no_bias(rows, cin, cout):
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    print("case", rows, cin, cout, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    L = Act8Lib()
    # over some decades: of one size, all sums of such short numbers would be exact
    x, w = (torch.exp(2 * torch.randn(r, cin, device="cuda", generator=gen)) for r in (rows, cout))
    x8, w8, y = Act8.empty(rows, cin), Act8.empty(cout, cin), torch.empty(rows, cout, device="cuda")
    L.slide_act8_pack(w, w8)
    L.slide_act8_linear(x, x8, w8, y)
    L.slide_act8_unpack(x8, x)
    L.slide_act8_unpack(w8, w)
    want = x.double() @ w.double().t()
    bias = float((y.double() - want).sum() / want.sum())
    worst = float(((y.double() - want).abs() / want).max())
    print("bias", bias, "worst", worst, flush=True)
    assert abs(bias) < 3e-8
    assert worst <= 2 * cin ** 0.5 * 2.0 ** -24 + 2.0 ** -24
