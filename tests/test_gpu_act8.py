"""Checkpoints in 8 bits and the linear layers that multiply out of them (include/act8.h) against float64 (needs an MI355X).

Packing and unpacking are compared bit by bit.  Bounds of the products, per element, with S = sum |x w| over the contraction:
  float32:   K 2^-24 S for any order of float32 sums, 2^-23 of the parts that the epilogue adds and rounds, 2^-20 of the activation's
             argument for its approximations (erf 1.5e-7, exponential and reciprocal of a few units in the last place)
  bfloat16:  the matrix core's cut: of eight neighbouring products the seven smaller ones lose up to 2^-13 of the largest, which is at
             most the product of the eights' largest operands; and half a step, 2^-8, of the result
An activation's slope is at most 1.13, so it passes an error of its argument on with that."""
import numpy as np
import pytest

from oracle import act8_oracle as ao

pytestmark = pytest.mark.gpu


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _types():
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16}


def _lib():
    from paper_2403_04865_amd import Act8Lib
    return Act8Lib()


def _strided(t, extra, offset=0):
    """t's values in a matrix whose rows are `extra` elements longer, starting `offset` elements into its memory"""
    import torch
    rows, cols = t.shape
    full = torch.full((rows * (cols + extra) + offset,), 7.0, dtype=t.dtype, device=t.device)
    v = full[offset:].view(rows, cols + extra)[:, :cols]
    v.copy_(t)
    return v


def _heavy(rng, rows, cols):
    return rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, cols)))


def _packed(x, guard=False):
    """x (numpy) as an Act8 made by the oracle; guard: rows further apart, surrounded by other bytes"""
    import torch
    from paper_2403_04865_amd import Act8
    codes, scales = ao.pack(x)
    if guard:
        c = torch.full((x.shape[0], codes.shape[1] + 48), 0x7f, dtype=torch.uint8, device="cuda")
        s = torch.full((x.shape[0], scales.shape[1] + 3), 0xff, dtype=torch.uint8, device="cuda")
        c[:, :codes.shape[1]] = _dev(codes)
        s[:, :scales.shape[1]] = _dev(scales)
        return Act8(*x.shape, c[:, :codes.shape[1]], s[:, :scales.shape[1]]), ao.unpack(codes, scales, x.shape[1])
    return Act8(*x.shape, _dev(codes), _dev(scales)), ao.unpack(codes, scales, x.shape[1])


# ---- pack, unpack -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,extra,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 128, 0, 0), (2, 129, 0, 0), (17, 100, 4, 0), (4, 384, 8, 0),
                                                    (33, 257, 3, 1), (9, 640, 0, 8), (700, 16, 0, 0), (1, 4099, 0, 0)])
def test_pack_and_unpack_bit_by_bit(rows, cols, extra, offset, dtype):
    import torch
    from paper_2403_04865_amd import Act8
    print("case", rows, cols, extra, offset, dtype, flush=True)
    rng = _rng(rows * 1000 + cols)
    t = _dev(_heavy(rng, rows, cols).astype(np.float32), _types()[dtype])
    if rows > 2:
        t[1] = 0.0
        t[2, cols // 2:] = 0.0
    x = _strided(t, extra, offset)
    want_c, want_s = ao.pack(t.double().cpu().numpy())
    # the packed rows stand apart, and what is between them stays as it is
    codes = torch.full((rows, want_c.shape[1] + 16), 0xaa, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, want_s.shape[1] + 1), 0xaa, dtype=torch.uint8, device="cuda")
    a = Act8(rows, cols, codes[:, :want_c.shape[1]] if rows > 1 else codes, scales[:, :want_s.shape[1]] if rows > 1 else scales)
    L = _lib()
    L.slide_act8_pack(x, a)
    assert np.array_equal(codes[:, :want_c.shape[1]].cpu().numpy(), want_c)
    assert np.array_equal(scales[:, :want_s.shape[1]].cpu().numpy(), want_s)
    assert (codes[:, want_c.shape[1]:] == 0xaa).all() and (scales[:, want_s.shape[1]:] == 0xaa).all()
    v = torch.from_numpy(ao.unpack(want_c, want_s, cols))
    for out in ("fp32", "bf16"):
        y = _strided(torch.zeros(rows, cols, dtype=_types()[out], device="cuda"), extra, offset)
        L.slide_act8_unpack(a, y)
        assert torch.equal(y.cpu(), v.to(_types()[out]))
        if extra:
            assert (y._base.view(-1)[offset:].view(rows, cols + extra)[:, cols:] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,extra", [(1, 1, 0), (40, 300, 0), (128, 128, 8), (33, 77, 5), (300, 1, 0)])
def test_pack_of_the_transpose(rows, cols, extra, dtype):
    from paper_2403_04865_amd import Act8
    t = _dev(_heavy(_rng(rows), rows, cols).astype(np.float32), _types()[dtype])
    a = Act8.empty(cols, rows)
    _lib().slide_act8_pack(_strided(t, extra), a, transpose=True)
    want_c, want_s = ao.pack(t.double().cpu().numpy().T)
    assert np.array_equal(a.codes.cpu().numpy(), want_c) and np.array_equal(a.scales.cpu().numpy(), want_s)


def test_values_at_the_ends_of_the_range():
    """Subnormal, largest and infinite numbers, NaN, every tie between two codes, and every code under every scale."""
    import torch
    from paper_2403_04865_amd import Act8
    ties = (ao.CODE[:0x7e] + ao.CODE[1:0x7f]) / 2
    rows = [np.full(128, 2.0 ** -149), np.full(128, 2.0 ** -126), np.full(128, 3.4028234e38), np.zeros(128), -np.zeros(128),
            np.r_[np.inf, -np.inf, np.nan, np.linspace(-2, 2, 125)], np.full(128, np.nan), np.full(128, -np.inf),
            np.r_[448.0, ties, 0.0], np.r_[448.0, -ties, 0.0], np.r_[3e38, np.full(127, 1e-38)], np.r_[1e-38, np.full(127, 1e-45)],
            np.r_[448 * 2.0 ** -127, np.full(127, 2.0 ** -130)], np.r_[449 * 2.0 ** -127, np.full(127, 2.0 ** -130)]]
    x = np.array(rows).astype(np.float32)
    a = Act8.empty(*x.shape)
    L = _lib()
    L.slide_act8_pack(_dev(x), a)
    want_c, want_s = ao.pack(x)
    got = a.codes.cpu().numpy()
    assert np.array_equal(a.scales.cpu().numpy(), want_s)
    nan = (want_c & 0x7f) == 0x7f      # a NaN's sign says nothing
    assert np.array_equal((got & 0x7f) == 0x7f, nan) and np.array_equal(got[~nan], want_c[~nan])
    codes = np.tile(np.arange(256, dtype=np.uint8), (255, 1))
    scales = np.repeat(np.arange(255, dtype=np.uint8)[:, None], 2, 1)
    v = torch.from_numpy(ao.unpack(codes, scales, 256))
    a = Act8(255, 256, _dev(codes), _dev(scales))
    for out in ("fp32", "bf16"):
        y = torch.empty(255, 256, dtype=_types()[out], device="cuda")
        L.slide_act8_unpack(a, y)
        assert torch.equal(torch.nan_to_num(y.cpu(), nan=1.25), torch.nan_to_num(v.to(_types()[out]), nan=1.25))


def test_pack_beyond_32_bit_offsets():
    """Rows whose last values lie more than 2^32 bytes behind the first."""
    import torch
    from paper_2403_04865_amd import Act8
    rows, cols, ld = 5, 200, 1 << 29
    x = torch.empty(4 * ld + cols, device="cuda")
    v = torch.as_strided(x, (rows, cols), (ld, 1))
    src = _dev(_heavy(_rng(9), rows, cols).astype(np.float32))
    v.copy_(src)
    codes, scales = torch.empty((rows, 1 << 30), dtype=torch.uint8, device="cuda"), torch.empty((rows, 1 << 20), dtype=torch.uint8, device="cuda")
    a = Act8(rows, cols, codes, scales)
    L = _lib()
    L.slide_act8_pack(v, a)
    want_c, want_s = ao.pack(src.cpu().numpy())
    assert np.array_equal(codes[:, :208].cpu().numpy(), want_c) and np.array_equal(scales[:, :2].cpu().numpy(), want_s)
    v.zero_()
    L.slide_act8_unpack(a, v)
    assert np.array_equal(v.cpu().numpy(), ao.unpack(want_c, want_s, cols))
    # and a layer over those rows
    w, wv = _packed(_heavy(_rng(10), 24, cols))
    y = torch.empty(rows, 24, device="cuda")
    L.slide_act8_linear(None, a, w, y)
    xv = ao.unpack(want_c, want_s, cols)
    assert np.all(np.abs(y.cpu().numpy() - xv @ wv.T) <= (cols + 2) * 2.0 ** -24 * (np.abs(xv) @ np.abs(wv).T))


# ---- linear -----------------------------------------------------------------------------------------------------------

def _eights(v):
    pad = -v.shape[1] % 8
    v = np.pad(np.abs(v), ((0, 0), (0, pad)))
    return v.reshape(v.shape[0], -1, 8).max(2)


def _linear_case(rows, cin, cout, dtype, bias, act, residual, extra=0, guard=False, given=False, in_place=False):
    import torch
    from paper_2403_04865_amd import Act8
    print("case", rows, cin, cout, dtype, bias, act, residual, extra, guard, given, in_place, flush=True)
    t = _types()[dtype]
    rng = _rng(rows * 7919 + cin * 31 + cout)
    x = _dev(_heavy(rng, rows, cin).astype(np.float32), t)
    w8, w = _packed(rng.standard_normal((cout, cin)) / np.sqrt(cin), guard)
    b = rng.standard_normal(cout).astype(np.float32) if bias else None
    res = _dev(rng.standard_normal((rows, cout)).astype(np.float32), t) if residual else None
    L = _lib()
    codes, scales = ao.pack(x.double().cpu().numpy())
    xv = ao.unpack(codes, scales, cin)
    if given:
        x8, _ = _packed(x.double().cpu().numpy(), guard)
    else:
        x8 = Act8.empty(rows, cin)
    y = _strided(torch.zeros(rows, cout, dtype=t, device="cuda"), extra)
    r = None if res is None else _strided(res, extra)
    if in_place:
        y = r
    L.slide_act8_linear(None if given else _strided(x, extra), x8, w8, y, bias=None if b is None else _dev(b), act=act, residual=r)
    if not given:
        assert np.array_equal(x8.codes.cpu().numpy(), codes) and np.array_equal(x8.scales.cpu().numpy(), scales)
    u = xv @ w.T
    S = np.abs(xv) @ np.abs(w).T
    arg = u if b is None else u + b
    h = ao.act(arg, act)
    want = h if res is None else h + res.double().cpu().numpy()
    err = cin * 2.0 ** -24 * S + 2.0 ** -23 * (np.abs(u) + np.abs(arg))
    if dtype == "bf16":
        err += 7 * 2.0 ** -13 * (_eights(xv) @ _eights(w).T)
    if act != "none":
        err = 1.13 * err + 2.0 ** -20 * np.abs(arg)
    err += (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * (np.abs(want) + np.abs(h)) * (1.0 if dtype == "fp32" else 1.01) + 1e-30
    got = y.double().cpu().numpy()
    worst = (np.abs(got - want) / err).max()
    print("worst share of the bound", worst, flush=True)
    assert worst <= 1.0
    if extra and rows > 1:
        assert (y._base.view(rows, cout + extra)[:, cout:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,cout", [(1, 1, 1), (1, 384, 1152), (2, 130, 17), (16, 1024, 64), (17, 100, 33), (64, 16, 1000), (65, 257, 129),
                                           (200, 384, 384), (257, 640, 520), (1000, 96, 72), (3, 5000, 40)])
def test_linear_sizes(rows, cin, cout, dtype):
    _linear_case(rows, cin, cout, dtype, True, "none", False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows,bias,residual", [(5, True, True), (300, False, True), (300, True, False), (700, True, True)])
def test_linear_epilogues(rows, act, bias, residual, dtype):
    _linear_case(rows, 256, 264, dtype, bias, act, residual)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,cout,extra", [(9, 72, 40, 3), (300, 333, 259, 1), (520, 384, 384, 16), (2100, 208, 272, 8)])
def test_linear_strides_in_place_and_packed_before(rows, cin, cout, extra, dtype):
    _linear_case(rows, cin, cout, dtype, True, "gelu", True, extra=extra)
    _linear_case(rows, cin, cout, dtype, True, "none", True, extra=extra, in_place=True)
    _linear_case(rows, cin, cout, dtype, False, "none", False, extra=extra, guard=True, given=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,cout", [(9001, 520, 1160), (8200, 1040, 1500), (70000, 384, 520), (140000, 104, 264), (131100, 256, 256), (60000, 384, 1000)])
def test_linear_many_tiles(rows, cin, cout, dtype):
    """As many output tiles as compute units and more, against float64 products on the device."""
    import torch
    from paper_2403_04865_amd import Act8
    t = _types()[dtype]
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(rows, cin, device="cuda", generator=g).to(t)
    w = torch.randn(cout, cin, device="cuda", generator=g)
    L = _lib()
    x8, w8 = Act8.empty(rows, cin), Act8.empty(cout, cin)
    L.slide_act8_pack(w, w8)
    y = torch.full((rows, cout), float("nan"), dtype=t, device="cuda")
    L.slide_act8_linear(x, x8, w8, y)
    xv, wv = torch.empty(rows, cin, device="cuda"), torch.empty(cout, cin, device="cuda")
    L.slide_act8_unpack(x8, xv)
    L.slide_act8_unpack(w8, wv)
    ref = xv.double() @ wv.double().t()
    S = xv.double().abs() @ wv.double().abs().t()
    err = cin * 2.0 ** -24 * S + 2.0 ** -23 * ref.abs()
    if dtype == "bf16":
        e8 = lambda v: v.double().abs().view(v.shape[0], -1, 8).amax(2)   # noqa: E731
        err = err + 7 * 2.0 ** -13 * (e8(xv) @ e8(wv).t()) + 1.01 * 2.0 ** -8 * ref.abs()
    assert ((y.double() - ref).abs() <= err).all()
    # the whole product is much nearer than the worst case of each element
    assert (y.double() - ref).norm() / ref.norm() <= (2.0 ** -8 if dtype == "bf16" else 1e-6)


def test_linear_keeps_what_is_not_finite_to_its_rows():
    import torch
    from paper_2403_04865_amd import Act8
    L = _lib()
    for rows in (20, 400):
        x = torch.ones(rows, 300, device="cuda", dtype=torch.bfloat16)
        x[3, 299] = float("nan")
        x[7, 0] = float("inf")
        w8, w = _packed(np.ones((50, 300)))
        y = torch.empty(rows, 50, device="cuda", dtype=torch.bfloat16)
        L.slide_act8_linear(x, Act8.empty(rows, 300), w8, y, act="relu")
        bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
        bad[3] = bad[7] = True
        assert y[bad].isnan().all() and (y[~bad] == 300).all()


# ---- weight gradient --------------------------------------------------------------------------------------------------

def _wgrad_case(rows, cin, cout, dtype, db=True, accumulate=False, extra=0, guard=False):
    import torch
    print("case", rows, cin, cout, dtype, db, accumulate, extra, guard, flush=True)
    t = _types()[dtype]
    rng = _rng(rows * 131 + cin * 7 + cout)
    x8, xv = _packed(_heavy(rng, rows, cin), guard)
    dy = _dev((_heavy(rng, rows, cout) * 1e-3).astype(np.float32), t)
    L = _lib()
    w0 = rng.standard_normal((cout, cin)).astype(np.float32) * 1e-2
    b0 = rng.standard_normal(cout).astype(np.float32) * 1e-2
    dW, b = _strided(_dev(w0), extra), _dev(b0)
    work = torch.full((L.slide_act8_wgrad_workspace_bytes(rows, cout, cin) // 4,), float("nan"), device="cuda")
    L.slide_act8_wgrad(_strided(dy, extra), x8, dW, b if db else None, accumulate=accumulate, workspace=work)
    d = dy.double().cpu().numpy()
    want, S = d.T @ xv, np.abs(d).T @ np.abs(xv)
    wb, Sb = d.sum(0), np.abs(d).sum(0)
    if accumulate:
        want, wb = want + w0, wb + b0
    assert np.all(np.abs(dW.double().cpu().numpy() - want) <= rows * 2.0 ** -24 * S + 2.0 ** -23 * np.abs(want) + 1e-30)
    if db:
        assert np.all(np.abs(b.double().cpu().numpy() - wb) <= rows * 2.0 ** -24 * Sb + 2.0 ** -23 * np.abs(wb) + 1e-30)
    else:
        assert np.array_equal(b.cpu().numpy(), b0)
    if extra and cout > 1:
        assert (dW._base.view(cout, cin + extra)[:, cin:] == 7).all()
    if rows >= 64:   # far from the worst case
        got = dW.double().cpu().numpy()
        assert np.linalg.norm(got - want) <= 2e-6 * np.linalg.norm(want) + 1e-30


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,cout", [(1, 1, 1), (1, 384, 64), (3, 100, 7), (64, 128, 128), (65, 130, 129), (200, 384, 384), (1000, 500, 40),
                                           (4099, 200, 300), (20000, 96, 72)])
def test_wgrad_sizes(rows, cin, cout, dtype):
    _wgrad_case(rows, cin, cout, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("accumulate,db,extra", [(True, True, 0), (False, False, 0), (True, False, 3), (False, True, 8)])
def test_wgrad_options(accumulate, db, extra, dtype):
    _wgrad_case(300, 136, 152, dtype, db=db, accumulate=accumulate, extra=extra, guard=True)
    _wgrad_case(9000, 136, 152, dtype, db=db, accumulate=accumulate, extra=extra, guard=True)


def test_wgrad_runs_give_the_same_bits():
    import torch
    rng = _rng(4)
    x8, _ = _packed(_heavy(rng, 6000, 256))
    dy = _dev(rng.standard_normal((6000, 384)).astype(np.float32), torch.bfloat16)
    L = _lib()
    work = torch.empty(L.slide_act8_wgrad_workspace_bytes(6000, 384, 256), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(2):
        dW, db = torch.empty(384, 256, device="cuda"), torch.empty(384, device="cuda")
        L.slide_act8_wgrad(dy, x8, dW, db, workspace=work)
        outs.append((dW, db))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_wgrad_of_gradients_that_are_not_finite():
    import torch
    x8, _ = _packed(np.ones((100, 64)))
    L = _lib()
    for dtype in ("fp32", "bf16"):
        dy = torch.ones(100, 40, device="cuda", dtype=_types()[dtype])
        dy[5, 3], dy[6, 4], dy[7, 9] = float("nan"), float("inf"), -3.4e38
        dW, db = torch.empty(40, 64, device="cuda"), torch.empty(40, device="cuda")
        L.slide_act8_wgrad(dy, x8, dW, db, workspace=torch.empty(L.slide_act8_wgrad_workspace_bytes(100, 40, 64), dtype=torch.uint8, device="cuda"))
        assert dW[3].isnan().all() and (dW[4] == float("inf")).all() and (dW[9] < -3e38).all()
        keep = [i for i in range(40) if i not in (3, 4, 9)]
        assert (dW[keep] == 100).all() and (db[keep] == 100).all()
