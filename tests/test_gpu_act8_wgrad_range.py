"""Float32 weight gradients out of 8-bit checkpoints at the ends of the range, and without a bias (needs an MI355X).

Products of a column are off by 2^-24 each and its `rows` additions by as much of a partial sum, of either sign: 2 sqrt(rows) 2^-24 of the terms' norm
is what their worst element of some ten thousand stays below, where the rows are added in one chain."""
import numpy as np
import pytest

from test_gpu_act8 import _dev, _heavy, _packed, _rng, _strided

pytestmark = pytest.mark.gpu

SIZES = [(70, 40, 5), (300, 136, 152), (1001, 333, 200), (9000, 136, 152)]


def _wgrad(dy, x8, accumulate=None, extra=0):
    import torch
    from paper_2403_04865_amd import Act8Lib
    L, out = Act8Lib(), dy.shape[1]
    dW = torch.full((out, x8.cols), float("nan"), device="cuda") if accumulate is None else accumulate[0].clone()
    db = torch.full((out,), float("nan"), device="cuda") if accumulate is None else accumulate[1].clone()
    work = torch.full((L.slide_act8_wgrad_workspace_bytes(x8.rows, out, x8.cols) // 4,), float("nan"), device="cuda")
    L.slide_act8_wgrad(_strided(dy, extra), x8, dW, db, accumulate=accumulate is not None, workspace=work)
    return dW.double().cpu().numpy(), db.double().cpu().numpy()


def _check(got, want, norm, rows, what):
    share = float((np.abs(got - want) / (2 * np.sqrt(rows) * 2.0 ** -24 * norm + 2.0 ** -24 * np.abs(want))).max())
    print(what, "worst share of its bound", share, flush=True)
    assert share <= 1.0, what


# Gradients of about 2^-120, whose trailing bits no bfloat16 holds, subnormal ones, and such of 2^84 and 2^120, with checkpoints that take the results
# back into the range.
@pytest.mark.parametrize("power,xpower", [(-120, 0), (-120, 20), (-140, 60), (84, 0), (120, -40)])
@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_gradients_at_the_ends_of_the_range(rows, cin, cout, power, xpower):
    print("case", rows, cin, cout, power, xpower, flush=True)
    rng = _rng(rows + cin)
    x8, xv = _packed(np.ldexp(_heavy(rng, rows, cin), xpower))
    dy = _dev(np.ldexp(rng.standard_normal((rows, cout)), power).astype(np.float32))
    d = dy.double().cpu().numpy()
    W, b = _wgrad(dy, x8, extra=3 if cout == 152 else 0)
    _check(W, d.T @ xv, np.sqrt((d ** 2).T @ xv ** 2), rows, "dW")
    # (rounding of a subnormal result is a step of 2^-149)
    tiny = 2.0 ** -150 if power == -140 else 0.0
    wb, nb = d.sum(0), np.sqrt((d ** 2).sum(0))
    # (9000 gradients of 2^120 add up to 95 * 2^120 in the mean square, past 2^128 in the largest of 152 columns, where float32 has no number)
    over = ~np.isfinite(b) & (np.abs(wb) + 4 * nb >= 2.0 ** 128)
    assert power == 120 or not over.any()
    assert np.all(over | (np.abs(b - wb) <= 2 * np.sqrt(rows) * 2.0 ** -24 * nb + 2.0 ** -24 * np.abs(wb) + tiny))


@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_gradients_next_to_the_largest_float(rows, cin, cout):
    """They round up to a bfloat16's infinity, and are finite all the same: nothing where the input is zero, themselves where it is one."""
    x = np.zeros((rows, cin))
    x[:, 1::2] = 1.0
    x8, xv = _packed(x)
    d = np.zeros((rows, cout), np.float32)
    d[rows // 2, :] = 3.4e38 * (-1.0) ** np.arange(cout)
    d[rows // 3, 1] = 1.0
    W, b = _wgrad(_dev(d), x8)
    want = d.astype(np.float64).T @ xv
    assert np.array_equal(W, want.astype(np.float32)) and np.array_equal(b, d[rows // 2].astype(np.float64))


@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_what_is_not_finite_stays_in_its_rows(rows, cin, cout):
    """Beside an infinity and a NaN every other row of dW has what it has without them, to the last bits of float32 sums."""
    import torch
    rng = _rng(rows)
    x8, xv = _packed(_heavy(rng, rows, cin))
    d = rng.standard_normal((rows, cout)).astype(np.float32)
    bad = [0, cout // 2]
    d[1, bad[0]], d[rows - 1, bad[1]] = np.nan, np.inf
    before = (torch.from_numpy(rng.standard_normal((cout, cin)).astype(np.float32)).cuda(), torch.from_numpy(rng.standard_normal(cout).astype(np.float32)).cuda())
    W, b = _wgrad(_dev(d), x8, accumulate=before)
    assert np.isnan(W[bad[0]]).all() and np.isnan(b[bad[0]]) and b[bad[1]] == np.inf
    assert not np.isfinite(W[bad[1]]).any()
    keep = np.setdiff1d(np.arange(cout), bad)
    D, w0, b0 = d.astype(np.float64)[:, keep], before[0].double().cpu().numpy()[keep], before[1].double().cpu().numpy()[keep]
    _check(W[keep], D.T @ xv + w0, np.sqrt((D ** 2).T @ xv ** 2) + np.abs(w0), rows, "dW")
    _check(b[keep], D.sum(0) + b0, np.sqrt((D ** 2).sum(0)) + np.abs(b0), rows, "db")


# Positive operands, whose products' errors a bias would line up.  In a chain of 96 additions or more (each of sixteen rows) that the matrix core pulls downwards by 2e-8
# over 48, slabs of either sign cancel it; one and a half times that is the limit.
@pytest.mark.parametrize("rows,cin,cout", [(1600, 333, 200), (9000, 136, 152), (100000, 128, 128)])
def test_positive_operands_have_no_bias(rows, cin, cout):
    import torch
    print("case positive operands", rows, cin, cout, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    from paper_2403_04865_amd import Act8, Act8Lib
    L = Act8Lib()
    x8 = Act8.empty(rows, cin)
    L.slide_act8_pack(torch.rand(rows, cin, device="cuda", generator=gen) + 0.5, x8)
    x = torch.empty(rows, cin, device="cuda")
    L.slide_act8_unpack(x8, x)
    dy = torch.rand(rows, cout, device="cuda", generator=gen) + 0.5
    W, b = _wgrad(dy, x8)
    want = (dy.double().t() @ x.double()).cpu().numpy()
    wb = dy.double().sum(0).cpu().numpy()
    bias = float((W - want).sum() / want.sum()), float((b - wb).sum() / wb.sum())
    print("bias", bias, "worst", float((np.abs(W - want) / want).max()), flush=True)
    assert abs(bias[0]) < 3e-8 and abs(bias[1]) < 3e-8
