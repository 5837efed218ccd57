"""Rotation of heads: queries and keys run beside each other, so neither's output may be what the other still reads (host only, as test_tokens_refusals.py)."""
import pytest

from test_tokens_refusals import AT, EHIP, EINVAL, lib, rope, rope_bwd, rope_fwd  # noqa: F401


@pytest.mark.parametrize("crossed", [dict(yk=AT), dict(yq=AT + 1024), dict(yq=AT + 1024, yk=AT)])
def test_forward_outputs_on_the_other_input(lib, crossed):  # noqa: F811
    # the strides of both, so that nothing else is wrong: as many key heads as query heads
    same = dict(ldq=256, ldk=256, ldyq=256, ldyk=256)
    assert rope_fwd(lib, rope(heads_k=4), **same) == EHIP
    assert rope_fwd(lib, rope(heads_k=4), **same, yq=AT, yk=AT + 1024) == EHIP      # each in its own place
    assert rope_fwd(lib, rope(heads_k=4), **{**same, **crossed}) == EINVAL


@pytest.mark.parametrize("crossed", [dict(dk=AT), dict(dq=AT + 16), dict(dq=AT + 48), dict(dk=AT + 32)])
def test_backward_outputs_on_the_other_input(lib, crossed):  # noqa: F811
    same = dict(lddyq=256, lddyk=256, ldq=256, ldk=256, lddq=256, lddk=256)
    assert rope_bwd(lib, rope(heads_k=4), **same) == EHIP
    assert rope_bwd(lib, rope(heads_k=4), **same, dq=AT, dk=AT + 16) == EHIP
    assert rope_bwd(lib, rope(heads_k=4), **{**same, **crossed}) == EINVAL


def test_inputs_that_are_not_read_may_be_written(lib):  # noqa: F811
    """Without a gain the forward's inputs are not the backward's."""
    same = dict(lddyq=256, lddyk=256, ldq=256, ldk=256, lddq=256, lddk=256)
    assert rope_bwd(lib, rope(heads_k=4), **same, gk=None, dgk=None, dq=AT + 48) == EHIP
    assert rope_bwd(lib, rope(heads_k=4), **same, gq=None, dgq=None, dk=AT + 32) == EHIP
