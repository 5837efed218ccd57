"""What include/act8.h refuses, on the host: no call gets as far as the device.  Addresses are host memory that nothing reads."""
import ctypes as C

import pytest

EINVAL, EARENA, EUNSUPPORTED, EHIP = -1, -2, -3, -5


@pytest.fixture(scope="module")
def lib():
    import torch
    from paper_2403_04865_amd.binding import load_cdll
    if torch.cuda.is_available():
        pytest.skip("passes addresses that no kernel may read; accepted calls would launch")
    return load_cdll()


BUF = C.create_string_buffer(4096)
AT = (C.addressof(BUF) + 255) // 256 * 256


def a8(rows=4, cols=200, **kw):
    from paper_2403_04865_amd.binding import _CAct8
    d = dict(codes=AT, ldc=208, scales=AT, lds=2, rows=rows, cols=cols)
    d.update(kw)
    return _CAct8(**d)


BAD_ACT8 = [dict(codes=None), dict(scales=None), dict(rows=0), dict(cols=0), dict(rows=-1), dict(cols=1 << 24, ldc=1 << 25, lds=1 << 20),
            dict(rows=1 << 31), dict(codes=AT + 8), dict(ldc=200), dict(ldc=192), dict(lds=1), dict(ldc=1 << 41)]


@pytest.mark.parametrize("bad", BAD_ACT8)
def test_bad_matrices_in_8_bits(lib, bad):
    b, ok = a8(**bad), a8()
    r = C.byref
    assert lib.slide_act8_pack(AT, 0, 200, 0, r(b), None) == EINVAL
    assert lib.slide_act8_unpack(r(b), AT, 0, 200, None) == EINVAL
    assert lib.slide_act8_linear(None, 0, 0, r(b), r(ok), None, 0, None, 0, AT, 8, None) == EINVAL
    assert lib.slide_act8_linear(None, 0, 0, r(ok), r(b), None, 0, None, 0, AT, 8, None) == EINVAL
    assert lib.slide_act8_wgrad(AT, 0, 8, 8, r(b), AT, 200, None, 0, AT, 1 << 40, None) == EINVAL


def test_pack_and_unpack(lib):
    r = C.byref(a8())
    for call in (lambda x, dt, ld: lib.slide_act8_pack(x, dt, ld, 0, r, None), lambda x, dt, ld: lib.slide_act8_unpack(r, x, dt, ld, None)):
        assert call(AT, 0, 200) == EHIP          # accepted; there is no device here
        assert call(None, 0, 200) == EINVAL
        assert call(AT, 2, 200) == EINVAL
        assert call(AT, 0, 199) == EINVAL
        assert call(AT + 2, 0, 200) == EINVAL    # not an address of a float
        assert call(AT + 2, 1, 200) == EHIP      # but one of a bfloat16
        assert call(AT + 1, 1, 200) == EINVAL
    assert lib.slide_act8_pack(AT, 0, 4, 1, r, None) == EHIP        # x is [200][4]
    assert lib.slide_act8_pack(AT, 0, 3, 1, r, None) == EINVAL


def test_linear(lib):
    r = C.byref
    x8, w8 = a8(4, 200), a8(7, 200)
    ok = dict(x=AT, dt=1, ldx=200, w=w8, bias=AT, act=3, res=AT, ldr=7, y=AT, ldy=7)

    def call(**kw):
        d = {**ok, **kw}
        return lib.slide_act8_linear(d["x"], d["dt"], d["ldx"], r(x8), r(d["w"]), d["bias"], d["act"], d["res"], d["ldr"], d["y"],
                                     d["ldy"], None)
    for good in (dict(), dict(x=None, ldx=0), dict(bias=None), dict(res=None, ldr=0), dict(dt=0), dict(ldr=9, ldy=9)):
        assert call(**good) == EHIP, good
    for bad in (dict(dt=-1), dict(dt=2), dict(ldx=199), dict(act=-1), dict(act=4), dict(y=None), dict(ldy=6), dict(ldr=6),
                dict(ldr=9), dict(bias=AT + 2), dict(w=a8(7, 199)), dict(y=AT + 1), dict(x=AT + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(w=a8(1 << 24, 200), ldr=1 << 24, ldy=1 << 24) == EUNSUPPORTED


def test_wgrad(lib):
    x8 = a8(1000, 200)
    need = lib.slide_act8_wgrad_workspace_bytes(1000, 7, 200)
    assert need > 0 and need % 256 == 0
    for bad in ((0, 7, 200), (1000, 0, 200), (1000, 7, 0), (1 << 31, 7, 200), (1000, 1 << 24, 200), (1000, 7, 1 << 24),
                (1000, (1 << 24) - 1, (1 << 24) - 1)):
        assert lib.slide_act8_wgrad_workspace_bytes(*bad) == 0, bad
    ok = dict(dy=AT, dt=1, ld=7, out=7, dW=AT, ldw=200, db=AT, work=AT, bytes=need)

    def call(**kw):
        d = {**ok, **kw}
        return lib.slide_act8_wgrad(d["dy"], d["dt"], d["ld"], d["out"], C.byref(x8), d["dW"], d["ldw"], d["db"], 0, d["work"], d["bytes"], None)
    for good in (dict(), dict(db=None), dict(dt=0), dict(ldw=300)):
        assert call(**good) == EHIP, good
    for bad in (dict(dy=None), dict(dt=2), dict(ld=6), dict(out=0), dict(dW=None), dict(ldw=199), dict(db=AT + 1), dict(work=AT + 64),
                dict(dW=AT + 2)):
        assert call(**bad) == EINVAL, bad
    assert call(work=None) == EARENA and call(bytes=need - 1) == EARENA
    assert call(out=1 << 24, ld=1 << 24) == EUNSUPPORTED
    x8 = a8(1000, 200, ldc=(1 << 24) + 16)
    assert call() == EUNSUPPORTED


def _shape(**kw):
    from paper_2403_04865_amd.binding import _CGroupNorm
    d = dict(n=2, hw=9, channels=24, groups=4, dtype=1, act=1, eps=1e-5, reserved=0)
    d.update(kw)
    return _CGroupNorm(**d)


BAD_SHAPES = [dict(n=0), dict(hw=0), dict(n=1 << 20, hw=1 << 20), dict(channels=0), dict(channels=65537, groups=1), dict(groups=0),
              dict(groups=5), dict(dtype=2), dict(act=4), dict(act=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
              dict(eps=float("inf")), dict(reserved=1), dict(n=(1 << 62), hw=4)]


def test_group_norm(lib):
    r = C.byref
    sh = _shape()
    need = lib.slide_group_norm_workspace_bytes(r(sh))
    assert need > 0 and need % 256 == 0
    kept, wrong = a8(18, 24, ldc=32), a8(17, 24, ldc=32)

    def fwd(s=sh, **kw):
        d = {**dict(x=AT, ldx=24, gam=AT, bet=AT, res=AT + 512, ldr=24, y=AT + 1024, ldy=24, x8=kept, mean=AT, rstd=AT, work=AT, bytes=need), **kw}
        return lib.slide_group_norm_fwd(r(s), d["x"], d["ldx"], d["gam"], d["bet"], d["res"], d["ldr"], d["y"], d["ldy"],
                                        None if d["x8"] is None else r(d["x8"]), d["mean"], d["rstd"], d["work"], d["bytes"], None)

    def bwd(s=sh, **kw):
        d = {**dict(dy=AT + 2048, lddy=24, x=AT, ldx=24, x8=None, gam=AT, bet=AT, res=AT + 512, ldr=24, mean=AT, rstd=AT, dx=AT + 1024,
                    lddx=24, dres=AT + 1536, lddr=24, dg=AT, db=AT, work=AT, bytes=need), **kw}
        return lib.slide_group_norm_bwd(r(s), d["dy"], d["lddy"], d["x"], d["ldx"], None if d["x8"] is None else r(d["x8"]), d["gam"], d["bet"],
                                        d["res"], d["ldr"], d["mean"], d["rstd"], d["dx"], d["lddx"], d["dres"], d["lddr"], d["dg"],
                                        d["db"], 0, d["work"], d["bytes"], None)
    for bad in BAD_SHAPES:
        assert lib.slide_group_norm_workspace_bytes(r(_shape(**bad))) == 0, bad
        assert fwd(_shape(**bad)) == EINVAL and bwd(_shape(**bad)) == EINVAL, bad
    for good in (dict(), dict(res=None), dict(x8=None), dict(y=AT), dict(y=AT + 512), dict(ldx=40)):
        assert fwd(**good) == EHIP, good
    for bad in (dict(x=None), dict(ldx=23), dict(gam=None), dict(bet=None), dict(ldr=23), dict(y=None), dict(ldy=23), dict(x8=wrong),
                dict(mean=None), dict(rstd=None), dict(y=AT, ldy=32), dict(y=AT + 512, ldy=32), dict(work=AT + 128), dict(x=AT + 1)):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(work=None) == EARENA and fwd(bytes=need - 1) == EARENA
    for good in (dict(), dict(x=None, x8=kept), dict(res=None), dict(dres=None), dict(dx=AT + 2048), dict(dres=AT + 2048)):
        assert bwd(**good) == EHIP, good
    for bad in (dict(x=None), dict(x8=kept), dict(x=None, x8=wrong), dict(dy=None), dict(dx=None), dict(mean=None), dict(dg=None), dict(db=None),
                dict(dx=AT), dict(dx=AT + 512), dict(dx=AT + 1536), dict(dres=AT), dict(dres=AT + 512), dict(dx=AT + 2048, lddx=32),
                dict(dres=AT + 2048, lddr=32), dict(lddy=23), dict(lddx=23), dict(lddr=23)):
        assert bwd(**bad) == EINVAL, bad
    assert bwd(work=None) == EARENA and bwd(bytes=need - 1) == EARENA


def test_binding_refuses_what_it_cannot_pass_on():
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    L = Act8Lib()
    x, ok = torch.zeros(4, 40), Act8.empty(4, 40, "cpu")
    with pytest.raises(ValueError, match="GPU"):
        L.slide_act8_pack(x, ok)
    with pytest.raises(ValueError, match="expected 4 rows of 40"):
        L.slide_act8_pack(torch.zeros(4, 39), ok)
    with pytest.raises(ValueError, match="contiguous"):
        L.slide_act8_pack(torch.zeros(40, 4).t(), ok)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        L.slide_act8_pack(x.half(), ok)
    for codes, scales in ((torch.zeros(4, 39, dtype=torch.uint8), ok.scales), (ok.codes, torch.zeros(3, 1, dtype=torch.uint8)),
                          (ok.codes.float(), ok.scales), (torch.zeros(48, 4, dtype=torch.uint8).t(), ok.scales)):
        with pytest.raises(ValueError):
            Act8(4, 40, codes, scales)
    with pytest.raises(ValueError, match="activation"):
        L.slide_act8_linear(x, ok, Act8.empty(8, 40, "cpu"), torch.zeros(4, 8), act="tanh")
    with pytest.raises(ValueError, match="bias"):
        L.slide_act8_linear(x, ok, Act8.empty(8, 40, "cpu"), torch.zeros(4, 8), bias=torch.zeros(7))
    t = torch.zeros(2, 9, 24)
    with pytest.raises(ValueError, match="tiles"):
        L.slide_group_norm_fwd(torch.zeros(2, 10, 24)[:, :9], torch.ones(24), torch.zeros(24), 4, t, torch.zeros(2, 4), torch.zeros(2, 4))
