"""Slide steps with a ResNet encoder under group normalisation, with and without 8-bit checkpoints of the convolutions' outputs
(needs an MI355X).  Limits are those of the batch-normalised step: the same number of bfloat16 storage roundings on every path, one
more per projected shortcut, and the same replay of stored activations for the ReLU decisions (tests/test_gpu_resnet.py)."""
from dataclasses import replace

import numpy as np
import pytest

from resnet_harness import GpuResNet, bf16_store, compare_resnet_step, replay_reference, resnet_inputs
from slide_harness import rel_l2

pytestmark = pytest.mark.gpu

TOL, STORE_TOL = 2e-2, 3e-3


@pytest.mark.timeout(300)
@pytest.mark.parametrize("name,n,tile,groups", [("rn_tiny", 6, None, 32), ("rn_tiny_bneck", 5, None, 8), ("rn_tiny", 7, 96, 1),
                                                ("rn_tiny", 3, None, 64)])
def test_step(name, n, tile, groups):
    cfg, prm, X, label = resnet_inputs(name, n, None, tile)
    cfg = replace(cfg, norm_groups=groups)
    print(f"case {name} cfg={cfg} n={n} label={label}", flush=True)
    g = GpuResNet(cfg, prm, n)
    out = g.step(X, label)
    ref, links, (pooled, pooled_ref) = replay_reference(g, prm, X, label)
    assert max(links) <= STORE_TOL, links
    assert np.array_equal(pooled, pooled_ref)
    errs, bad = compare_resnet_step(out, ref, TOL)
    print("worst:", sorted(errs.items(), key=lambda kv: -kv[1])[:6], flush=True)
    assert not bad, bad
    assert errs["H"] <= 1e-5
    again = g.step(X, label)
    assert all(np.array_equal(again["grads"][k], v) for k, v in out["grads"].items())

    # convolution outputs in 8 bits: the same forward, and a backward at the checkpoints' values
    c8 = replace(cfg, checkpoint8=1)
    k = GpuResNet(c8, prm, n)
    out8 = k.step(X, label)
    for q in ("loss", "logits", "alpha", "H", "G"):
        assert np.array_equal(out8[q], out[q]), q
    g.cfg = c8      # the same stored activations, the oracle's backward at their checkpoints
    ref8, _, _ = replay_reference(g, prm, X, label)
    errs, bad = compare_resnet_step(out8, ref8, TOL)
    print("checkpoints, worst:", sorted(errs.items(), key=lambda kv: -kv[1])[:6], flush=True)
    assert not bad, bad
    print("checkpoints against none:", max(rel_l2(out8["grads"][q], v) for q, v in out["grads"].items()), flush=True)


@pytest.mark.timeout(300)
def test_forward_at_224px():
    from oracle import resnet_oracle as ro
    cfg, prm, X, label = resnet_inputs("rn18_small", 2)
    cfg = replace(cfg, norm_groups=32, checkpoint8=1)
    print(f"case rn18_small cfg={cfg} n=2", flush=True)
    out = GpuResNet(cfg, prm, 2).step(X, label)
    prm = {k: v.astype(np.float64) for k, v in prm.items()}
    H, _ = ro.encoder_fwd(prm, X.astype(np.float64), replace(cfg, checkpoint8=0), store=bf16_store)
    assert rel_l2(out["H"], H) <= 1.1e-3 * 43          # one storage rounding per stored tensor: 20 convolutions, 20 normalised outputs, 3 for the sums
    assert all(np.isfinite(v).all() for v in out["grads"].values())


@pytest.mark.timeout(300)
@pytest.mark.parametrize("checkpoint8", [0, 1])
def test_parts_of_a_slide(checkpoint8):
    # no tile depends on another: two calls over parts, gradients accumulated, against one over all.  The same numbers up to
    # the order of float32 sums (statistics; weight gradients) and the storage roundings that it turns
    import torch
    cfg, prm, X, label = resnet_inputs("rn_tiny", 9)
    cfg = replace(cfg, norm_groups=16, checkpoint8=checkpoint8)
    g = GpuResNet(cfg, prm, 9)
    px, dev = g.to_dev(X), g.dev
    G = torch.from_numpy(np.random.default_rng(5).standard_normal((9, cfg.dim)).astype(np.float32)).to(dev)
    H = torch.zeros(9, cfg.dim, device=dev)
    g.lib.resnet_encoder_fwd_tiles(px, 9, H)
    g.lib.resnet_encoder_bwd_tiles(G, 9, 0)
    torch.cuda.synchronize()
    whole, Hw = g.grads_dict(), H.cpu().numpy().copy()
    H.zero_()
    for lo, hi in ((0, 4), (4, 9)):
        g.lib.resnet_encoder_fwd_tiles(px[lo:hi], hi - lo, H[lo:hi])
        g.lib.resnet_encoder_bwd_tiles(G[lo:hi], hi - lo, int(lo > 0))
    torch.cuda.synchronize()
    assert rel_l2(H.cpu().numpy(), Hw) <= 5e-3
    parts = g.grads_dict()
    errs = {k: rel_l2(parts[k], v) for k, v in whole.items() if not k.startswith(("mil.", "head."))}
    print("parts, worst:", sorted(errs.items(), key=lambda kv: -kv[1])[:4], flush=True)
    assert max(errs.values()) <= TOL


def test_saved_activations():
    from paper_2403_04865_amd import SlideError
    cfg, prm, X, label = resnet_inputs("rn_tiny", 2)
    g = GpuResNet(replace(cfg, norm_groups=16, checkpoint8=1), prm, 2)
    g.step(X, label)
    refused = 0
    for i in range(g.lib.resnet_saved_activations()):
        try:
            g.lib.resnet_saved_activation(i)
        except SlideError as e:
            assert e.code == -3
            refused += 1
    assert refused == 12        # the convolutions: stem, two a block, three projections, and the first stage has none
