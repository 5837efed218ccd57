"""What include/tokens.h and its binding refuse, on the host: no call gets as far as the device.  Addresses are host memory that nothing reads."""
import ctypes as C

import pytest

EINVAL, EARENA, EUNSUPPORTED, EHIP = -1, -2, -3, -5
BUF = C.create_string_buffer(4096)
AT = (C.addressof(BUF) + 255) // 256 * 256
BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    import torch
    from paper_2403_04865_amd.binding import load_cdll
    if torch.cuda.is_available():
        pytest.skip("passes addresses that no kernel may read; accepted calls would launch")
    return load_cdll()


def rope(**kw):
    from paper_2403_04865_amd.binding import _CHeadRope
    d = dict(rows=5, heads_q=4, heads_k=2, head_dim=64, dtype=1, axes=2, pairing=0, pairs=(16, 16, 0), eps=1e-6, theta=100.0)
    d.update(kw)
    d["pairs"] = (C.c_int32 * 3)(*d["pairs"])
    return _CHeadRope(**d)


def rope_fwd(lib, s=None, **kw):
    d = dict(q=AT, ldq=256, k=AT + 1024, ldk=128, gq=AT, gk=AT, pos=AT, yq=AT + 256, ldyq=256, yk=AT + 512, ldyk=128)
    d.update(kw)
    return lib.slide_head_rope_fwd(C.byref(s or rope()), *d.values(), None)


def rope_bwd(lib, s=None, **kw):
    d = dict(dyq=AT, lddyq=256, dyk=AT + 16, lddyk=128, q=AT + 32, ldq=256, k=AT + 48, ldk=128, gq=AT, gk=AT, pos=AT, dq=AT + 64, lddq=256,
             dk=AT + 80, lddk=128, dgq=AT + 96, dgk=AT + 112, accumulate=0, work=AT, bytes=BIG)
    d.update(kw)
    return lib.slide_head_rope_bwd(C.byref(s or rope()), *d.values(), None)


BAD_ROPE = [dict(rows=0), dict(rows=-1), dict(rows=1 << 31), dict(heads_q=0), dict(heads_q=4097), dict(heads_k=-1), dict(head_dim=0), dict(dtype=2),
            dict(dtype=-1), dict(axes=-1), dict(axes=4), dict(pairing=2), dict(pairs=(17, 16, 0)), dict(pairs=(-1, 16, 0)), dict(eps=0.0),
            dict(eps=float("nan")), dict(eps=float("inf")), dict(theta=0.0), dict(theta=0.99), dict(theta=float("nan")), dict(theta=-1.0), dict(theta=float("inf"))]


@pytest.mark.parametrize("bad", BAD_ROPE)
def test_bad_rotations(lib, bad):
    s = rope(**bad)
    assert rope_fwd(lib, s) == EINVAL and rope_bwd(lib, s) == EINVAL
    assert lib.slide_head_rope_workspace_bytes(C.byref(s)) == 0


def test_rotation_arguments(lib):
    assert lib.slide_head_rope_fwd(None, AT, 256, AT, 128, None, None, AT, AT, 256, AT, 128, None) == EINVAL
    for good in (dict(), dict(gq=None), dict(gk=None), dict(yq=AT, yk=AT + 1024), dict(ldq=264), dict(ldyk=2097144)):
        assert rope_fwd(lib, **good) == EHIP, good          # accepted; there is no device here
    for bad in (dict(q=None), dict(yq=None), dict(k=None), dict(yk=None), dict(q=AT + 2), dict(yq=AT + 8), dict(ldq=255), dict(ldq=248), dict(ldq=257),
                dict(ldq=1 << 21), dict(ldk=120), dict(yq=AT, ldyq=264), dict(yk=AT + 1024, ldyk=136), dict(gq=AT + 4), dict(gk=AT + 8), dict(pos=None),
                dict(pos=AT + 2), dict(yk=AT + 256)):
        assert rope_fwd(lib, **bad) == EINVAL, bad
    one = dict(k=None, yk=None, gk=None, ldk=0, ldyk=0)
    assert rope_fwd(lib, rope(heads_k=0), **one) == EHIP
    assert rope_fwd(lib, rope(heads_k=0), **{**one, "k": AT}) == EINVAL
    assert rope_fwd(lib, rope(axes=0), pos=None) == EHIP
    assert rope_fwd(lib, rope(axes=0)) == EINVAL
    for dim in (8, 24, 272):
        assert rope_fwd(lib, rope(head_dim=dim, pairs=(4, 0, 0)), ldq=2048, ldk=2048, ldyq=2048, ldyk=2048) == EUNSUPPORTED


def test_rotation_backward_arguments(lib):
    need = lib.slide_head_rope_workspace_bytes(C.byref(rope()))
    assert need > 0 and need % 256 == 0
    for good in (dict(), dict(bytes=need), dict(gq=None, dgq=None, q=None), dict(gk=None, dgk=None, k=None), dict(dq=AT), dict(accumulate=1)):
        assert rope_bwd(lib, **good) == EHIP, good
    for bad in (dict(dyq=None), dict(dyk=None), dict(q=None), dict(k=None), dict(dgq=None), dict(dgk=None), dict(gq=None), dict(gk=None), dict(dq=AT + 32),
                dict(dk=AT + 48), dict(dk=AT + 64), dict(dgk=AT + 96), dict(dq=AT, lddq=264), dict(work=AT + 16), dict(pos=None), dict(lddyq=260)):
        assert rope_bwd(lib, **bad) == EINVAL, bad
    assert rope_bwd(lib, work=None) == EARENA and rope_bwd(lib, bytes=need - 1) == EARENA


def attn(**kw):
    from paper_2403_04865_amd.binding import _CTokensAttn
    d = dict(rows_q=50, rows_k=60, docs=2, heads_q=4, heads_k=2, head_dim=64, dtype=1, lead_q=1, lead_k=0, scale=0.125, cap=0.0, reserved=0)
    d.update(kw)
    return _CTokensAttn(**d)


def fwd(lib, s=None, **kw):
    d = dict(q=AT, ldq=256, k=AT + 16, ldk=128, v=AT + 32, ldv=128, qs=AT, ks=AT, pq=AT, pk=AT, sl=AT, o=AT + 48, ldo=256, lse=AT, work=AT, bytes=BIG)
    d.update(kw)
    return lib.slide_tokens_attn_fwd(C.byref(s or attn()), *d.values(), None)


def bwd(lib, s=None, **kw):
    d = dict(do=AT, lddo=256, q=AT + 16, ldq=256, k=AT + 32, ldk=128, v=AT + 48, ldv=128, o=AT + 64, ldo=256, lse=AT, qs=AT, ks=AT, pq=AT, pk=AT, sl=AT,
             dq=AT + 80, lddq=256, dk=AT + 96, lddk=128, dv=AT + 112, lddv=128, work=AT, bytes=BIG)
    d.update(kw)
    return lib.slide_tokens_attn_bwd(C.byref(s or attn()), *d.values(), None)


INF, NAN = float("inf"), float("nan")
BAD_ATTN = [dict(rows_q=0), dict(rows_k=0), dict(rows_q=1 << 31), dict(rows_k=(1 << 31) - 1), dict(docs=0), dict(docs=(1 << 20) + 1), dict(heads_q=0), dict(heads_k=0),
            dict(heads_k=3), dict(heads_q=5000, heads_k=50), dict(head_dim=0), dict(dtype=2), dict(lead_q=-1), dict(lead_k=-1), dict(scale=INF), dict(scale=NAN), dict(scale=0.0), dict(scale=-0.1), dict(scale=2.0 ** -41), dict(scale=2.0 ** 41), dict(cap=2.0 ** -41), dict(cap=2.0 ** 41),
            dict(cap=-1.0), dict(cap=INF), dict(cap=NAN), dict(reserved=1)]


@pytest.mark.parametrize("bad", BAD_ATTN)
def test_bad_attentions(lib, bad):
    s = attn(**bad)
    assert fwd(lib, s) == EINVAL and bwd(lib, s) == EINVAL
    assert lib.slide_tokens_attn_workspace_bytes(C.byref(s), 1) == 0


def test_unsupported_attentions(lib):
    wide = {n: 1 << 14 for n in ("ldq", "ldk", "ldv", "ldo")}
    for bad in (dict(head_dim=8), dict(head_dim=72), dict(head_dim=144), dict(heads_q=129, heads_k=1, head_dim=16), dict(rows_q=1 << 30)):
        assert fwd(lib, attn(**bad), **wide) == EUNSUPPORTED, bad
        assert lib.slide_tokens_attn_workspace_bytes(C.byref(attn(**bad)), 0) == 0


def test_attention_arguments(lib):
    for good in (dict(), dict(pq=None, pk=None, sl=None), dict(ldq=264, ldo=512)):
        assert fwd(lib, **good) == EHIP, good
        assert bwd(lib, **good) == EHIP, good
    both = [dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(lse=None), dict(lse=AT + 2), dict(qs=None), dict(ks=None), dict(qs=AT + 2), dict(ks=AT + 1),
            dict(pq=None), dict(pk=None), dict(sl=None), dict(pq=AT + 4), dict(pk=AT + 4), dict(sl=AT + 2), dict(ldq=255), dict(ldq=252), dict(ldk=64), dict(ldv=130),
            dict(ldo=1 << 21), dict(q=AT + 2), dict(v=AT + 8)]
    for bad in both:
        assert fwd(lib, **bad) == EINVAL, bad
        assert bwd(lib, **bad) == EINVAL, bad
    for same in ("q", "k", "v"):
        assert fwd(lib, o=dict(q=AT, k=AT + 16, v=AT + 32)[same]) == EINVAL
    for out in ("dq", "dk", "dv"):
        for i in range(5):
            assert bwd(lib, **{out: AT + 16 * i}) == EINVAL
        assert bwd(lib, **{out: None}) == EINVAL
    assert bwd(lib, dk=AT + 80) == EINVAL and bwd(lib, dv=AT + 96) == EINVAL and bwd(lib, do=None) == EINVAL


def test_attention_work_space(lib):
    for kw in (dict(), dict(rows_q=2, rows_k=50000), dict(rows_q=50000, rows_k=3), dict(dtype=0, rows_q=1, docs=1, rows_k=9000)):
        s = attn(**kw)
        f, b = (lib.slide_tokens_attn_workspace_bytes(C.byref(s), i) for i in (0, 1))
        assert b >= f and b > 0 and f % 256 == 0 and b % 256 == 0
        assert bwd(lib, s, bytes=b) == EHIP and bwd(lib, s, bytes=255) == EARENA and bwd(lib, s, work=None) == EARENA
        if b > f:
            assert bwd(lib, s, bytes=b - 1) == EARENA
        assert bwd(lib, s, work=AT + 64) == EINVAL
        assert fwd(lib, s, bytes=f) == EHIP and fwd(lib, s, bytes=f - 1) == EARENA and fwd(lib, s, work=None, bytes=0) == EARENA
        assert fwd(lib, s, work=AT + 64) == EINVAL
    # what a workgroup may leave is bounded, whatever the sizes
    assert lib.slide_tokens_attn_workspace_bytes(C.byref(attn(rows_q=1 << 24, rows_k=1 << 24, docs=1)), 0) < 1 << 27
    assert lib.slide_tokens_attn_workspace_bytes(C.byref(attn(rows_q=10, rows_k=10, docs=1)), 0) < 1 << 20


def test_binding():
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    L = TokensLib()
    for bad in (dict(pairs=(1, 1, 1, 1)), dict(pairs=(33,)), dict(pairs=(-1,)), dict(pairing="odd")):
        with pytest.raises(ValueError):
            HeadRope(64, **{"pairs": (16, 16), **bad})
    r = HeadRope(64, (16, 16))
    q, k, pos = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64), torch.zeros(3, 2, dtype=torch.int32)
    for bad in (dict(q=q[:, :, :32]), dict(q=q.view(3, 256)), dict(q=q.half()), dict(k=k[:2]), dict(k=k.bfloat16()), dict(pos=pos.long()), dict(pos=pos[:, :1]),
                dict(pos=pos[:2]), dict(gq=torch.ones(63)), dict(gq=torch.ones(64).double()), dict(q=torch.zeros(3, 64, 4).transpose(1, 2)),
                dict(q=torch.zeros(3, 8, 64)[:, ::2]), dict(q_out=torch.zeros(3, 4, 128)[:, :, ::2]), dict()):   # the last: not on a GPU
        d = {**dict(q=q, k=k, pos=pos, q_out=q.clone(), k_out=k.clone()), **bad}
        with pytest.raises(ValueError):
            L.slide_head_rope_fwd(r, **d)
    s, lse, o = torch.tensor([0, 3], dtype=torch.int32), torch.zeros(4, 3), torch.zeros(3, 4, 64)
    ok = dict(q=q, k=k, v=k.clone(), q_start=s, k_start=s, o=o, lse=lse, scale=0.1)
    for bad in (dict(v=torch.zeros(2, 2, 64)), dict(k=torch.zeros(3, 2, 32)), dict(q_start=s.long()), dict(k_start=torch.zeros(3, dtype=torch.int32)), dict(o=q[:2]),
                dict(lse=torch.zeros(3, 4)), dict(lse=torch.zeros(4, 6)[:, ::2]), dict(lead_q=-1), dict(lead_k=1 << 32), dict(pos_q=torch.zeros(3, 3)),
                dict(pos_k=torch.zeros(6)), dict(slopes=torch.zeros(2)), dict()):
        with pytest.raises(ValueError):
            L.slide_tokens_attn_fwd(**{**ok, **bad})
    assert L.slide_tokens_attn_workspace_bytes(3, 3, 1, 4, 2, 64, torch.float16) == 0
