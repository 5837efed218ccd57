"""Block inputs kept in 8 bits (slide_config.checkpoint8): host side."""
import pytest

import gen


def _lib(**kw):
    from paper_2403_04865_amd import SlideConfig, SlideLib
    ok = dict(tile=32, patch=8, dim=64, layers=2, heads=2, mlp_ratio=4, mil_hidden=32, n_classes=1, dtype=1, recompute=1)
    return SlideLib(SlideConfig(**{**ok, **kw}))


def test_only_with_recompute_and_bfloat16():
    from paper_2403_04865_amd import SlideError
    _lib(checkpoint8=1)
    _lib(checkpoint8=0, dtype=0, recompute=0)
    for bad in (dict(checkpoint8=1, recompute=0), dict(checkpoint8=1, dtype=0), dict(checkpoint8=2), dict(checkpoint8=-1)):
        with pytest.raises(SlideError) as e:
            _lib(**bad)
        assert e.value.code == -1, bad


def test_arena_holds_half_the_block_inputs():
    from paper_2403_04865_amd import SlideConfig, SlideLib
    cfg, n = gen.CONFIGS["full"]
    mk = lambda c8: SlideLib(SlideConfig(cfg.tile, cfg.patch, cfg.dim, cfg.layers, cfg.heads, cfg.mlp_ratio, cfg.mil_hidden,   # noqa: E731
                                         cfg.n_classes, dtype=1, recompute=1, checkpoint8=c8))
    tokens = (cfg.tile // cfg.patch) ** 2 + 1
    plain, kept = mk(0).slide_arena_bytes(n), mk(1).slide_arena_bytes(n)
    row = tokens * cfg.dim * n
    # L + 1 slots of two bytes a value become two of them and L - 1 of one byte and a 128th
    want = (cfg.layers + 1) * 2 * row - (2 * 2 * row + (cfg.layers - 1) * (row + row // 128))
    assert abs((plain - kept) - want) <= 256 * 4 * cfg.layers
    sizes = [mk(1).slide_arena_bytes(k) for k in (1, 2, 100, n)]
    assert sizes == sorted(sizes) and all(b % 256 == 0 for b in sizes)
