"""The oracle of a ResNet whose group norms read 8-bit checkpoints in their backward: decisions the forward's, gradients near those without."""
from dataclasses import replace

import numpy as np
import pytest

import gen


# Of weights and shifts.  A norm adds 0.0325 of the gradient at most, 1.25 times the 2.6e-2 that four significant bits leave in the mean square, independently
# of the others; a gain's own gradient is a sum of du xhat, which may cancel to anything.
@pytest.mark.parametrize("block", ["basic", "bottleneck"])
@pytest.mark.parametrize("groups", [1, 4, 8])
def test_decisions_and_gradients(block, groups):
    from oracle import resnet_oracle as ro
    cfg, n = gen.RESNET_CONFIGS["rn_probe"]
    cfg = replace(cfg, block=block, norm_groups=groups)
    prm = {k: v.astype(np.float64) for k, v in gen.make_resnet_params(cfg, 7).items()}
    X = gen.make_pixels(cfg, n, 8, kind="blur").astype(np.float64)
    G = np.random.default_rng(9).standard_normal((n, cfg.dim))
    _, a = ro.encoder_fwd(prm, X, cfg)
    _, b = ro.encoder_fwd(prm, X, replace(cfg, checkpoint8=1))
    assert np.array_equal(a["stem"][1], b["stem"][1])
    for (_, on, _, out), (_, on8, _, out8) in zip(a["blocks"], b["blocks"]):
        assert all(np.array_equal(u, v) for u, v in zip(on, on8)) and np.array_equal(out, out8)
    want, got = ro.encoder_bwd(a, G), ro.encoder_bwd(b, G)
    norms = 1 + sum(cfg.depths) * (2 if block == "basic" else 3)
    errs = {k: float(np.linalg.norm(got[k] - v) / np.linalg.norm(v)) for k, v in want.items() if not k.endswith(".g")}
    print(sorted(errs.items(), key=lambda kv: -kv[1])[:5])
    assert max(errs.values()) <= 0.0325 * norms ** 0.5
