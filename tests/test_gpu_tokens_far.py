"""Operators over tokens on matrices of more than 2^31 elements: the same bits as on rows beside each other (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu

ROWS, WIDE = 1100, (1 << 21) - 8      # 2.3e9 elements


class Columns:
    """[rows, heads, 64] views, one behind the other in the columns of one wide matrix or of a dense one."""

    def __init__(self, dtype, wide):
        import torch
        self.m = torch.zeros(ROWS * WIDE if wide else ROWS * 64 * 16, dtype=dtype, device="cuda")
        self.ld, self.at = WIDE if wide else 64 * 16, 0

    def take(self, heads):
        v = self.m.as_strided((ROWS, heads, 64), (self.ld, 64, 1), self.at)
        self.at += heads * 64
        return v


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_every_matrix_far(dtype):
    import torch
    from paper_2403_04865_amd import TokensLib
    print(f"case every matrix far {dtype}", flush=True)
    L, t = TokensLib(), torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(2)
    values = [torch.randn((ROWS, h, 64), generator=g).to(t) for h in (2, 1, 1, 2)]
    start = torch.tensor([0, 1000, 1100], dtype=torch.int32, device="cuda")
    work = torch.empty(L.slide_tokens_attn_workspace_bytes(ROWS, ROWS, 2, 2, 1, 64, t, backward=True), dtype=torch.uint8, device="cuda")
    res = []
    for wide in (True, False):
        c = Columns(t, wide)
        q, k, v, do = (c.take(x.shape[1]) for x in values)
        for a, b in zip((q, k, v, do), values):
            a.copy_(b.cuda())
        o, dq, dk, dv = (c.take(h) for h in (2, 2, 1, 1))
        lse = torch.empty(2, ROWS, device="cuda")
        L.slide_tokens_attn_fwd(q, k, v, start, start, o, lse, 0.125, workspace=work)
        L.slide_tokens_attn_bwd(do, q, k, v, o, lse, start, start, dq, dk, dv, 0.125, workspace=work)
        res.append([x.contiguous().clone() for x in (q, k, v, do, o, lse, dq, dk, dv)])
        del c, q, k, v, do, o, dq, dk, dv
    for name, a, b in zip(("q", "k", "v", "do", "o", "lse", "dq", "dk", "dv"), *res):
        assert torch.equal(a, b), name
        assert torch.isfinite(a).all() and a.abs().max() > 0, name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_rotation_every_matrix_far(dtype, pairing):
    import torch
    from paper_2403_04865_amd import HeadRope, TokensLib
    print(f"case rotation far {dtype} {pairing}", flush=True)
    L, rope, t = TokensLib(), HeadRope(64, (16, 16), 100.0, pairing), torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(5)
    values = [torch.randn((ROWS, h, 64), generator=g).to(t) for h in (2, 1, 2, 1)]
    pos = torch.randint(0, 4096, (ROWS, 2), generator=g, dtype=torch.int32).cuda()
    gq, gk = 1 + 0.1 * torch.randn(64, generator=g).cuda(), 1 + 0.1 * torch.randn(64, generator=g).cuda()
    work = torch.empty(L.slide_head_rope_workspace_bytes(rope, ROWS, 2, 1), dtype=torch.uint8, device="cuda")
    res = []
    for wide in (True, False):
        c = Columns(t, wide)
        q, k, dyq, dyk = (c.take(x.shape[1]) for x in values)
        for a, b in zip((q, k, dyq, dyk), values):
            a.copy_(b.cuda())
        yq, yk, dq, dk = (c.take(h) for h in (2, 1, 2, 1))
        dgq, dgk = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
        L.slide_head_rope_fwd(rope, q, k, pos, yq, yk, gq=gq, gk=gk)
        L.slide_head_rope_bwd(rope, dyq, dyk, q, k, pos, dq, dk, gq=gq, gk=gk, dgq=dgq, dgk=dgk, workspace=work)
        res.append([x.contiguous().clone() for x in (q, k, dyq, dyk, yq, yk, dq, dk, dgq, dgk)])
        del c, q, k, dyq, dyk, yq, yk, dq, dk
    for name, a, b in zip(("q", "k", "dyq", "dyk", "yq", "yk", "dq", "dk", "dgq", "dgk"), *res):
        assert torch.equal(a, b), name
        assert torch.isfinite(a).all() and a.abs().max() > 0, name
