"""Arguments that the binding refuses before the library is called (CPU only: nothing here can reach a GPU)."""
import pytest
import torch

from paper_2607_25852_amd import binding as B


@pytest.mark.parametrize("inv_freq", [
    torch.ones(64), torch.ones(64, dtype=torch.bfloat16), torch.ones(128), torch.ones(63, dtype=torch.float64),
    torch.ones(64, dtype=torch.int64), torch.ones(128, dtype=torch.float64)[::2]])
def test_frequencies_are_doubles(inv_freq, monkeypatch):
    """Anything but rot_dim / 2 dense doubles would be read past its end, or as other numbers."""
    def called(*a):
        raise AssertionError("the call went on")
    monkeypatch.setattr(B, "_run", called)
    desc = B.rope_desc(2, 4, 8, 2, 128, (24, 20, 20), 16, 4, 8, B.SV_F32)
    z = torch.zeros
    args = lambda f: (desc, z(4, 8, 128), z(4, 2, 128), z(4, 2, 128), z((3, 4), dtype=torch.int32), f,
                      z((2, 4), dtype=torch.int32), z(3, dtype=torch.int32), z(2, dtype=torch.int32), z(4, 8, 128),
                      z(8, 2, 16, 128), z(8, 2, 16, 128))
    monkeypatch.setattr(B, "load", lambda: type("lib", (), {"sv_rope_append": None}))
    with pytest.raises(ValueError):
        B.rope_append(*args(inv_freq))
    with pytest.raises(AssertionError, match="went on"):
        B.rope_append(*args(torch.ones(64, dtype=torch.float64)))
