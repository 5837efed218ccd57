"""Linear layers on 8-bit activations whose operands lie far from one, as do their powers of two (needs an MI355X).  Bounds are those of
test_gpu_act8.py, without their floor."""
import numpy as np
import pytest

from oracle import act8_oracle as ao
from test_gpu_act8 import _dev, _eights, _heavy, _packed, _rng, _types

pytestmark = pytest.mark.gpu


# Powers of the operands' sizes; results of 2^-110 to 2^100
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("xp,wp", [(100, -95), (-95, 100), (-60, -50), (60, 40), (110, -120), (-110, 120)])
@pytest.mark.parametrize("rows,cin,cout", [(3, 300, 40), (64, 384, 384), (300, 300, 260), (9000, 256, 520), (600, 1040, 4608)])
def test_sizes_far_from_one(rows, cin, cout, xp, wp, dtype):
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    print("case", rows, cin, cout, xp, wp, dtype, flush=True)
    rng = _rng(rows + cin)
    n = min(rows, 300)      # the oracle's rows; the others repeat them
    small = _dev(np.ldexp(rng.standard_normal((n, cin)) * np.exp(0.5 * rng.standard_normal((n, cin))), xp).astype(np.float32), _types()[dtype])
    x = small.repeat(rows // n, 1)
    w8, w = _packed(np.ldexp(rng.standard_normal((cout, cin)), wp))
    y, x8 = torch.full((rows, cout), float("nan"), dtype=x.dtype, device="cuda"), Act8.empty(rows, cin)
    Act8Lib().slide_act8_linear(x, x8, w8, y)
    assert torch.equal(y, y[:n].repeat(rows // n, 1))
    xv = ao.unpack(*ao.pack(small.double().cpu().numpy()), cin)
    want, S = xv @ w.T, np.abs(xv) @ np.abs(w).T
    err = cin * 2.0 ** -24 * S + 2.0 ** -22 * np.abs(want)
    if dtype == "bf16":
        err = err + 7 * 2.0 ** -13 * (_eights(xv) @ _eights(w).T) + 1.01 * 2.0 ** -8 * np.abs(want)
    got = y[:n].double().cpu().numpy()
    share = float((np.abs(got - want) / err).max())
    print("worst share of the bound", share, flush=True)
    assert share <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,cout", [(3, 300, 40), (64, 384, 384), (300, 300, 260), (9000, 256, 520)])
def test_results_beyond_the_largest_number(rows, cin, cout, dtype):
    """Rows of one sign: infinite, of that sign; beside them rows that stay in the range."""
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    t = _types()[dtype]
    x = torch.full((rows, cin), 2.0 ** 90, dtype=t, device="cuda")
    x[::3] *= -1
    x[1::3] = 1.0
    w8, _ = _packed(np.full((cout, cin), 2.0 ** 60))
    y = torch.empty(rows, cout, dtype=t, device="cuda")
    Act8Lib().slide_act8_linear(x, Act8.empty(rows, cin), w8, y)
    assert (y[::3] == -float("inf")).all() and (y[2::3] == float("inf")).all()
    assert (y[1::3] == torch.tensor(cin * 2.0 ** 60, device="cuda").to(t)).all()
