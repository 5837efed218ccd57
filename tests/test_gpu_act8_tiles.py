"""Linear layers on 8-bit activations: the tile size, chosen by rows and columns, leaves a result's bits as they are (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu


# Rounds of small and large tiles: 1 1 (small), 2 1 (large), 2 2 (small), 3 2 (large), 4 3 (small); wide layers of few rows (small)
@pytest.mark.parametrize("rows,cin,cout", [(6000, 520, 1152), (7289, 520, 1152), (14000, 520, 1152), (20000, 520, 1152), (28000, 520, 1152), (600, 520, 20000),
                                           (600, 4096, 2000)])
def test_rows_do_not_depend_on_how_many_there_are(rows, cin, cout):
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    print("case", rows, cin, cout, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    L = Act8Lib()
    x = torch.randn(rows, cin, device="cuda", generator=gen).bfloat16()
    w8 = Act8.empty(cout, cin)
    L.slide_act8_pack(torch.randn(cout, cin, device="cuda", generator=gen), w8)

    def run(x):
        y = torch.full((x.shape[0], cout), float("nan"), dtype=torch.bfloat16, device="cuda")
        L.slide_act8_linear(x, Act8.empty(*x.shape), w8, y, act="silu")
        return y
    y = run(x)
    assert not y.isnan().any()
    part = max(128, rows // 5 // 128 * 128)       # by the small tiles
    assert torch.equal(run(x[:part]), y[:part]) and torch.equal(run(x[-part:]), y[-part:])
