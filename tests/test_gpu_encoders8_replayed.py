"""Slide steps with 8-bit checkpoints, captured and replayed, and a second backward of one forward (needs an MI355X)."""
from dataclasses import replace

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _vit(n):
    import slide_harness
    from paper_2403_04865_amd import SlideConfig
    from test_gpu_parity import _inputs
    cfg, prm, X, label = _inputs("tiny", n=n, bf16=True)
    keep, slide_harness.lib_config = slide_harness.lib_config, lambda cfg, dtype, recompute=0: SlideConfig(
        cfg.tile, cfg.patch, cfg.dim, cfg.layers, cfg.heads, cfg.mlp_ratio, cfg.mil_hidden, cfg.n_classes, dtype=1, recompute=1, ln_eps=cfg.ln_eps,
        checkpoint8=1)
    try:
        g = slide_harness.GpuSlide(cfg, prm, 1, n, 1)
    finally:
        slide_harness.lib_config = keep
    return g, g.to_dev(X), label, g.lib.slide_step_fwd, g.lib.slide_step_bwd


def _resnet(n):
    from resnet_harness import GpuResNet, resnet_inputs
    cfg, prm, X, label = resnet_inputs("rn_tiny", n)
    g = GpuResNet(replace(cfg, norm_groups=16, checkpoint8=1), prm, n)
    return g, g.to_dev(X), label, g.lib.resnet_slide_step_fwd, g.lib.resnet_slide_step_bwd


@pytest.mark.timeout(200)
@pytest.mark.parametrize("make,n", [(_vit, 13), (_resnet, 7)])
def test_a_captured_step(make, n):
    import torch
    print("case", make.__name__, n, flush=True)
    g, px, label, fwd, bwd = make(n)
    loss, logits, alpha = torch.zeros(1, device="cuda"), torch.zeros(g.cfg.n_classes, device="cuda"), torch.zeros(n, device="cuda")

    def step():
        fwd(px, n, label, loss, logits, alpha)
        bwd(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    first = px.clone()
    for turn in range(4):
        px.copy_(first.roll(turn, 0) * (1 + turn))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (loss, logits, alpha, g.grads)]
        for t in (loss, logits, alpha, g.grads):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (loss, logits, alpha, g.grads))), turn
        assert bool(torch.isfinite(g.grads).all())


def test_a_second_backward_of_a_resnet():
    import torch
    g, px, label, _, _ = _resnet(5)
    H, G = torch.zeros(5, g.cfg.dim, device="cuda"), torch.randn(5, g.cfg.dim, device="cuda")
    g.lib.resnet_encoder_fwd_tiles(px, 5, H)
    out = []
    for _ in range(2):
        g.grads.fill_(0)
        g.lib.resnet_encoder_bwd_tiles(G, 5, 0)
        out.append(g.grads.clone())
    assert torch.equal(*out) and bool(out[0].any())
    g.lib.resnet_encoder_bwd_tiles(G, 5, 1)     # added to what is there: twice as much, to the roundings of float32 sums
    assert float((g.grads - 2 * out[0]).norm() / out[0].norm()) < 1e-5
    assert np.isfinite(H.cpu().numpy()).all()
