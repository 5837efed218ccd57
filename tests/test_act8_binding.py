"""What the binding of include/act8.h takes and refuses before a call reaches the library (no GPU)."""
import pytest


def test_rows_of_codes_reach_a_multiple_of_16():
    import torch
    from paper_2403_04865_amd import Act8
    new = lambda *s: torch.zeros(s, dtype=torch.uint8)   # noqa: E731
    one = new(1, 1)
    for codes in (new(1, 100), new(1, 111), new(400)[:100].view(1, 100), new(1, 112)[:, :100]):
        with pytest.raises(ValueError, match="112 bytes"):      # what lies behind 100 is not the row's to write
            Act8(1, 100, codes, one)
    assert Act8(1, 100, new(1, 112), one)._c.ldc == 112
    assert Act8(1, 100, new(1, 128), one)._c.ldc == 112
    assert Act8(1, 96, new(1, 96), one)._c.ldc == 96
    # between rows the bytes are the matrix's, behind the last row they have to be there
    assert Act8(3, 100, new(3, 112)[:, :100], new(3, 1))._c.ldc == 112
    assert Act8(2, 100, new(3, 112)[1:, :100], new(2, 1))._c.ldc == 112
    assert Act8(3, 100, new(2 * 112 + 112).as_strided((3, 100), (112, 1)), new(3, 1))._c.ldc == 112
    for short in (100, 111):
        with pytest.raises(ValueError, match="112 bytes"):
            Act8(3, 100, new(2 * 112 + short).as_strided((3, 100), (112, 1)), new(3, 1))
        with pytest.raises(ValueError, match="112 bytes"):
            Act8(3, 100, new(5 + 2 * 112 + short).as_strided((3, 100), (112, 1), 5), new(3, 1))


def test_the_library_is_declared_once():
    from paper_2403_04865_amd import Act8Lib
    from paper_2403_04865_amd.binding import load_cdll
    assert load_cdll() is load_cdll() and Act8Lib().lib is Act8Lib().lib


def test_a_library_built_again_is_loaded_again(monkeypatch, tmp_path):
    import shutil

    from paper_2403_04865_amd import binding
    at = tmp_path / "libslide.so"
    shutil.copy(binding.lib_path(), at)
    monkeypatch.setattr(binding, "lib_path", lambda: str(at))
    first = binding.load_cdll()
    again = tmp_path / "new"
    shutil.copy(at, again)
    again.rename(at)
    assert binding.load_cdll() is not first


def test_work_space_is_as_large_as_it_says():
    import torch
    from paper_2403_04865_amd import Act8, Act8Lib
    L = Act8Lib()
    need = L.slide_act8_wgrad_workspace_bytes(1000, 8, 32)
    with pytest.raises(ValueError, match="contiguous"):      # one byte of memory
        L.slide_act8_wgrad(torch.zeros(1000, 8), Act8.empty(1000, 32, "cpu"), torch.zeros(8, 32), workspace=torch.zeros(1, dtype=torch.uint8).expand(need))
    t, f = torch.zeros(2, 9, 24), torch.zeros(2, 4)
    need = L.slide_group_norm_workspace_bytes(2, 9, 24, 4, torch.float32)
    with pytest.raises(ValueError, match="contiguous"):
        L.slide_group_norm_fwd(t, torch.ones(24), torch.zeros(24), 4, t, f, f, workspace=torch.zeros(1).expand(need // 4))
