"""ResNet configurations whose normalisation fields do not fit their 16 bits (no GPU)."""
import pytest


@pytest.mark.parametrize("bad", [dict(norm_groups=1 << 16), dict(norm_groups=(1 << 16) + 32), dict(norm_groups=-(1 << 16) + 32), dict(norm_groups=1 << 40),
                                 dict(norm_groups=32, checkpoint8=1 << 16), dict(norm_groups=32, checkpoint8=(1 << 16) + 1), dict(checkpoint8=-(1 << 16))])
def test_numbers_that_16_bits_do_not_hold_are_refused(bad):
    from paper_2403_04865_amd import ResNetConfig, ResNetLib, SlideError
    with pytest.raises(SlideError) as e:
        ResNetLib(ResNetConfig(tile=64, block=0, depths=(1, 1, 1, 1), width=64, mil_hidden=32, n_classes=1, **bad))
    assert e.value.code == -1
