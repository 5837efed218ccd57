"""ResNet encoder with group normalisation: the oracle against an autograd graph of library routines, and the host side of the
configuration."""
from dataclasses import replace

import numpy as np
import pytest

import gen


@pytest.mark.parametrize("block", ["basic", "bottleneck"])
def test_oracle_against_autograd(block):
    import torch
    import torch.nn.functional as F
    from oracle import resnet_oracle as ro
    cfg, n = gen.RESNET_CONFIGS["rn_probe"]
    cfg = replace(cfg, block=block, norm_groups=4)
    prm = {k: v.astype(np.float64) for k, v in gen.make_resnet_params(cfg, 7).items()}
    X = gen.make_pixels(cfg, n, 8, kind="blur").astype(np.float64)
    G = np.random.default_rng(9).standard_normal((n, cfg.dim))
    H, cache = ro.encoder_fwd(prm, X, cfg)
    g = ro.encoder_bwd(cache, G)
    P = {k: torch.tensor(v, requires_grad=True) for k, v in prm.items()}

    def cn(x, conv, bn, stride, pad):
        return F.group_norm(F.conv2d(x, P[conv + ".W"], stride=stride, padding=pad), cfg.norm_groups, P[bn + ".g"], P[bn + ".b"], cfg.bn_eps)
    x = F.max_pool2d(torch.relu(cn(torch.tensor(X), "stem.conv", "stem.bn", 2, 3)), 3, 2, 1)
    for name, stride, down in ro._blocks(cfg):
        p = name + "."
        if block == "basic":
            y = cn(torch.relu(cn(x, p + "conv1", p + "bn1", stride, 1)), p + "conv2", p + "bn2", 1, 1)
        else:
            y = torch.relu(cn(x, p + "conv1", p + "bn1", 1, 0))
            y = cn(torch.relu(cn(y, p + "conv2", p + "bn2", stride, 1)), p + "conv3", p + "bn3", 1, 0)
        x = torch.relu(y + (cn(x, p + "down.conv", p + "down.bn", stride, 0) if down else x))
    Ht = x.mean((2, 3))
    (Ht * torch.tensor(G)).sum().backward()
    assert np.allclose(H, Ht.detach().numpy(), rtol=1e-9, atol=1e-11)
    for k, v in g.items():
        assert np.allclose(v, P[k].grad.numpy(), rtol=1e-7, atol=1e-9), k


def test_oracle_on_checkpoints():
    # the forward is the one without; the backward sees values that are off by a 16th at most
    from oracle import resnet_oracle as ro
    cfg, n = gen.RESNET_CONFIGS["rn_probe"]
    prm = {k: v.astype(np.float64) for k, v in gen.make_resnet_params(cfg, 7).items()}
    X = gen.make_pixels(cfg, n, 8, kind="blur").astype(np.float64)
    H0, _ = ro.encoder_fwd(prm, X, replace(cfg, norm_groups=4))
    H1, c1 = ro.encoder_fwd(prm, X, replace(cfg, norm_groups=4, checkpoint8=1))
    assert np.array_equal(H0, H1)
    x = np.random.default_rng(3).standard_normal((2, 160, 3, 5))
    v = ro.checkpoint_values(x)
    assert v.shape == x.shape and np.all(np.abs(v - x) <= np.abs(x) / 16 + 2.0 ** -9 * 2.0 ** -6 * 4)


def test_configuration():
    from paper_2403_04865_amd import ResNetConfig, ResNetLib, SlideError, resnet_config_from
    ok = dict(tile=64, block=0, depths=(1, 1, 1, 1), width=64, mil_hidden=32, n_classes=1)
    for good in (dict(), dict(norm_groups=1), dict(norm_groups=32), dict(norm_groups=64, checkpoint8=1)):
        ResNetLib(ResNetConfig(**ok, **good))
    for bad in (dict(norm_groups=-1), dict(norm_groups=3), dict(norm_groups=128), dict(checkpoint8=1), dict(norm_groups=32, checkpoint8=2),
                dict(norm_groups=32, checkpoint8=-1)):
        with pytest.raises(SlideError) as e:
            ResNetLib(ResNetConfig(**ok, **bad))
        assert e.value.code == -1, bad
    cfg, _ = gen.RESNET_CONFIGS["rn18"]
    mk = lambda **k: ResNetLib(resnet_config_from(replace(cfg, **k)))   # noqa: E731
    plain, gn, c8 = mk(), mk(norm_groups=32), mk(norm_groups=32, checkpoint8=1)
    assert plain.param_layout() == gn.param_layout() == c8.param_layout()
    n = 512
    a, b = gn.resnet_arena_bytes(n), c8.resnet_arena_bytes(n)
    outs = sum((224 // s) ** 2 * w * k for s, w, k in ((2, 64, 1), (4, 64, 4), (8, 128, 5), (16, 256, 5), (32, 512, 5)))
    # two bytes a value of every convolution output become one and a scale byte per 128
    scales = sum((224 // s) ** 2 * max(1, w // 128) * k for s, w, k in ((2, 64, 1), (4, 64, 4), (8, 128, 5), (16, 256, 5), (32, 512, 5)))
    assert abs((a - b) - n * (outs - scales)) < 256 * 3 * 25
    for lib in (gn, c8):
        sizes = [lib.resnet_arena_bytes(k) for k in (1, 2, 7, 100, n)]
        assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
