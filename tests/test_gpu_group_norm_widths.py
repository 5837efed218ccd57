"""Group norm at widths where lanes or threads are left over: checkpoints of rows that end inside sixteen lanes, more groups than threads
(needs an MI355X).  Bounds are those of test_gpu_group_norm.py; checkpoints are compared bit by bit."""
import pytest

from test_gpu_group_norm import _run

pytestmark = pytest.mark.gpu


# A block of a checkpoint's columns is held by sixteen lanes, eight columns each.  Here rows are split, and the last block has 2, 6, 10, 12,
# 14 lanes' worth of columns behind no, one or sixteen whole blocks.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hw,c,groups", [(2, 3600, 96, 16), (1, 3001, 48, 6), (1, 3001, 80, 5), (1, 3001, 112, 14), (1, 2000, 144, 9), (1, 2000, 176, 11),
                                           (1, 2000, 208, 13), (1, 2000, 224, 28), (1, 2000, 240, 30), (1, 300, 2144, 4), (1, 200, 4080, 8)])
def test_checkpoints_of_split_rows(n, hw, c, groups, dtype):
    _run(n, hw, c, groups, dtype, "silu", checkpoint=True)

# Every channel a group of its own, on maps so small that a workgroup of 256 threads takes 320 to 512 of them
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hw,c,groups", [(300, 4, 512, 512), (300, 9, 384, 384), (600, 1, 320, 320), (300, 4, 512, 256)])
def test_more_groups_than_threads(n, hw, c, groups, dtype):
    _run(n, hw, c, groups, dtype, "silu")
    _run(n, hw, c, groups, dtype, "gelu", checkpoint=True)


# 4099 slices of one channel (a prime number of groups) of 4104 tiles: more than 2^32 threads as a workgroup each
def test_more_units_than_a_launch_has_workgroups():
    import torch
    from paper_2403_04865_amd import Act8Lib
    n, c = 4104, 4099
    L = Act8Lib()
    x, dy = torch.randn(n, 2, c, device="cuda"), torch.randn(n, 2, c, device="cuda")
    gamma, beta = torch.rand(c, device="cuda") + 0.5, torch.randn(c, device="cuda")
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd, dg, db = torch.empty(n, c, device="cuda"), torch.empty(n, c, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    work = torch.empty(L.slide_group_norm_workspace_bytes(n, 2, c, c, torch.float32), dtype=torch.uint8, device="cuda")
    L.slide_group_norm_fwd(x, gamma, beta, c, y, mean, rstd, eps=0.1, workspace=work)
    L.slide_group_norm_bwd(dy, x, gamma, beta, mean, rstd, c, dx, dg, db, workspace=work)
    X, DY, G = x.double(), dy.double(), gamma.double()
    m = X.mean(1, keepdim=True)
    r = 1 / torch.sqrt((X - m).square().mean(1, keepdim=True) + 0.1)     # <= 3.2, xhat <= 1
    h = (X - m) * r
    U = 2.0 ** -24      # a dozen roundings of parts that are |x|, |xhat|, |dy|, the gain and shift in size, times rstd
    assert ((y - (h * G + beta)).abs() <= 16 * U * (4 * X.abs().amax(1, keepdim=True) + 2 + beta.abs())).all()
    assert ((mean - m[:, 0]).abs() <= 4 * U * X.abs().amax(1)).all()
    t = DY * G
    want = r * (t - t.mean(1, keepdim=True) - h * (t * h).mean(1, keepdim=True))
    top = DY.abs().amax(1, keepdim=True)
    assert ((dx - want).abs() <= 16 * U * r * 1.5 * 3 * top * (1 + 4 * r * X.abs().amax(1, keepdim=True))).all()
    # a thread adds the four to eight tiles that it takes, 4104 partial sums go together in 64 bits
    assert ((db - DY.sum((0, 1))).abs() <= 32 * U * DY.abs().sum((0, 1))).all()
    assert ((dg - (DY * h).sum((0, 1))).abs() <= (32 * U * (DY.abs() * (1 + 4 * r * X.abs().amax(1, keepdim=True)))).sum((0, 1))).all()


# A checkpoint is written on the way: where a row's lanes need no padding (2, 4, 8 or a multiple of 16 of them, rows of up to 2048 channels or a multiple of
# that) the results keep their bits
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hw,c,groups", [(1, 9001, 16, 4), (1, 9001, 32, 8), (3, 12544, 64, 32), (2, 5000, 128, 32), (1, 3000, 384, 32), (1, 700, 2048, 32),
                                           (1, 90, 4096, 64), (40, 784, 64, 32), (30, 49, 96, 8)])
def test_a_checkpoint_leaves_the_results_as_they_are(n, hw, c, groups, dtype):
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    print("case", n, hw, c, groups, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(c)
    x = (torch.randn(n, hw, c, device="cuda", generator=gen) * torch.exp(torch.randn(c, device="cuda", generator=gen)) + 1).to(t)
    gamma, beta = torch.randn(c, device="cuda", generator=gen), torch.randn(c, device="cuda", generator=gen)
    L = Act8Lib()
    work = torch.empty(L.slide_group_norm_workspace_bytes(n, hw, c, groups, t), dtype=torch.uint8, device="cuda")
    outs = []
    for x8 in (None, Act8.empty(n * hw, c)):
        y, mean, rstd = torch.full_like(x, float("nan")), torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda")
        L.slide_group_norm_fwd(x, gamma, beta, groups, y, mean, rstd, act="silu", x8=x8, workspace=work)
        outs.append((y, mean, rstd))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    alone = Act8.empty(n * hw, c)
    L.slide_act8_pack(x.view(n * hw, c), alone)
    assert torch.equal(alone.codes, x8.codes) and torch.equal(alone.scales, x8.scales)
