"""Block inputs kept in 8 bits (slide_config.checkpoint8) through the C ABI (needs an MI355X).

The forward is the one without: features, logits, loss, attention weights and feature gradients are the same bits, and so are the gradients of
the aggregator, the final LayerNorm and the last block, which does not run again.  The other blocks run again on inputs whose values are
rounded to four significant bits, at most 2^-4 and in the mean square 2.6e-2 of themselves; their activations, and with them
their weight gradients and the gradient they hand on, are a few hundredths off per block, independently from block to block:
0.026 sqrt(2) sqrt(blocks), 0.13 over twelve blocks, is what to expect, and the limit is three times the mean square error's share."""
import numpy as np
import pytest

from test_gpu_parity import _inputs

pytestmark = pytest.mark.gpu


def _gpu(monkeypatch, cfg, prm, n, c8, arena=None):
    import slide_harness
    from paper_2403_04865_amd import SlideConfig

    def config(cfg, dtype, recompute=0):
        return SlideConfig(cfg.tile, cfg.patch, cfg.dim, cfg.layers, cfg.heads, cfg.mlp_ratio, cfg.mil_hidden, cfg.n_classes, dtype=dtype,
                           recompute=1, ln_eps=cfg.ln_eps, checkpoint8=c8)
    monkeypatch.setattr(slide_harness, "lib_config", config)
    return slide_harness.GpuSlide(cfg, prm, 1, n, 1, arena_bytes=arena)


@pytest.mark.parametrize("name,n", [("tiny", 13), ("small", 21)])
def test_against_block_inputs_in_bfloat16(monkeypatch, name, n):
    from slide_harness import rel_l2
    cfg, prm, X, lab = _inputs(name, n=n, bf16=True)
    print(f"case checkpoint8 {name} n={n}", flush=True)
    g = _gpu(monkeypatch, cfg, prm, n, 1)
    out = g.step(X, lab)
    ref = _gpu(monkeypatch, cfg, prm, n, 0).step(X, lab)
    for k in ("loss", "logits", "alpha", "H", "G"):
        assert np.array_equal(out[k], ref[k]), k
    last = f"l{cfg.layers - 1}."
    handed = f"l{cfg.layers - 2}.fc2.b"       # the column sums of the gradient that the last block hands on
    limit = 3 * 0.026 * np.sqrt(2) * np.sqrt(cfg.layers)
    worst = {}
    for k, v in ref["grads"].items():
        if k.startswith((last, "mil.", "head.", "lnf.")) or k == handed:
            assert np.array_equal(out["grads"][k], v), k
        elif k.endswith("qkv.b"):     # the key third is zero but for rounding
            D = cfg.dim
            worst[k] = rel_l2(np.delete(out["grads"][k], np.s_[D:2 * D]), np.delete(v, np.s_[D:2 * D]))
        else:
            worst[k] = rel_l2(out["grads"][k], v)
    worst["dX"] = rel_l2(out["dX"], ref["dX"])
    print("worst:", sorted(worst.items(), key=lambda kv: -kv[1])[:6], flush=True)
    assert max(worst.values()) <= limit and min(worst.values()) > 0.0
    # the slots of the inputs have been written over: no second backward
    from paper_2403_04865_amd import SlideError
    with pytest.raises(SlideError) as e:
        g.lib.slide_step_bwd(0)
    assert e.value.code == -4
    # and the next step is as the first
    again = g.step(X, lab)
    assert all(np.array_equal(again["grads"][k], v) for k, v in out["grads"].items()) and np.array_equal(again["dX"], out["dX"])


def test_chunked(monkeypatch):
    from slide_harness import rel_l2
    cfg, prm, X, lab = _inputs("small", n=21, bf16=True)
    out = _gpu(monkeypatch, cfg, prm, 21, 1, arena=lambda lib: lib.slide_chunked_arena_bytes(21, 8)).step_chunked(X, lab, 8)
    ref = _gpu(monkeypatch, cfg, prm, 21, 0).step(X, lab)
    limit = 3 * 0.026 * np.sqrt(2) * np.sqrt(cfg.layers)
    assert rel_l2(out["H"], ref["H"]) <= 2e-2 and abs(out["loss"] - ref["loss"]) <= 2e-2 * abs(ref["loss"])
    bad = {k: rel_l2(out["grads"][k], v) for k, v in ref["grads"].items() if k.startswith("l") and k.endswith(".W")}
    print("worst:", sorted(bad.items(), key=lambda kv: -kv[1])[:4], flush=True)
    assert max(bad.values()) <= limit
