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
