"""Block inputs kept in 8 bits where 8 bits hold them: not a bit of a gradient may change (needs an MI355X).

The patch embedding picks a pixel of two significant bits and a sign per column, times a power of two, so the first block's input has its values
exactly in 8 bits; a block whose projections are zero hands its input on as it is.  With every block but one such a block, and the last, which does not run
again, the one runs again on exactly its input: what it and the blocks in front of it give must be what they give from block inputs in bfloat16."""
from dataclasses import replace

import numpy as np
import pytest

import gen

pytestmark = pytest.mark.gpu


def _setup(name, layers, live, n):
    cfg = replace(gen.CONFIGS[name][0], layers=layers)
    ds, ws, ls = gen.SEEDS[name]
    prm = {k: gen.to_bf16_grid(v) for k, v in gen.make_params(cfg, ws, perturbed=True).items()}
    rng = np.random.default_rng(10 * layers + live)
    K = prm["pe.W"].shape[1]
    W = np.zeros_like(prm["pe.W"])
    W[np.arange(cfg.dim), rng.integers(0, K, cfg.dim)] = rng.choice([0.5, 1.0, -1.0, 2.0], cfg.dim)
    prm["pe.W"], prm["pe.b"], prm["pos"] = W, np.zeros_like(prm["pe.b"]), np.zeros_like(prm["pos"])
    prm["cls"] = (rng.integers(-3, 4, prm["cls"].shape) / 2).astype(prm["cls"].dtype)
    for l in range(layers - 1):
        if l != live:
            for k in ("proj.W", "proj.b", "fc2.W", "fc2.b"):
                prm[f"l{l}.{k}"] = np.zeros_like(prm[f"l{l}.{k}"])
    X = (rng.integers(-3, 4, (n, 3, cfg.tile, cfg.tile)) / 2).astype(np.float32)
    return cfg, prm, X, gen.make_label(cfg, ls)


def _step(monkeypatch, cfg, prm, X, lab, c8):
    import slide_harness
    from paper_2403_04865_amd import SlideConfig
    monkeypatch.setattr(slide_harness, "lib_config", lambda cfg, dtype, recompute=0: SlideConfig(
        cfg.tile, cfg.patch, cfg.dim, cfg.layers, cfg.heads, cfg.mlp_ratio, cfg.mil_hidden, cfg.n_classes, dtype=dtype, recompute=1,
        ln_eps=cfg.ln_eps, checkpoint8=c8))
    return slide_harness.GpuSlide(cfg, prm, 1, X.shape[0], 1).step(X, lab)


@pytest.mark.parametrize("name,layers,live,n", [("tiny", 2, 0, 13), ("tiny", 4, 0, 13), ("tiny", 4, 1, 6), ("tiny", 5, 3, 9), ("small", 3, 0, 5), ("small", 3, 1, 21),
                                                ("small", 4, 2, 7)])
def test_gradients_keep_their_bits(monkeypatch, name, layers, live, n):
    cfg, prm, X, lab = _setup(name, layers, live, n)
    print(f"case {name} layers={layers} live={live} n={n}", flush=True)
    want, got = (_step(monkeypatch, cfg, prm, X, lab, c8) for c8 in (0, 1))
    for k in ("loss", "logits", "alpha", "H", "G", "dX"):
        assert np.array_equal(got[k], want[k]), k
    assert np.abs(want["dX"]).max() > 0
    behind = tuple(f"l{l}." for l in range(live + 1, layers - 1))     # these run again on inputs that 8 bits do not hold
    for k, v in want["grads"].items():
        if not k.startswith(behind):
            assert np.array_equal(got["grads"][k], v), k
        if k.startswith(f"l{live}.") and k.endswith(".W"):
            assert np.abs(v).max() > 0, k
