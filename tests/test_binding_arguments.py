"""Arguments that the binding refuses before the library is called (CPU only: nothing here can reach a GPU)."""
import inspect

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


class _Tensor:
    """What the binding asks of a tensor, on device 1."""
    dtype, itemsize, shape = torch.float64, 8, (4, 8, 128)

    def get_device(self):
        return 1

    def data_ptr(self):
        return 4096

    def numel(self):
        return 4096

    def element_size(self):
        return 8

    def is_contiguous(self):
        return True

    def is_floating_point(self):
        return True

    def stride(self):
        return (1024, 128, 1)


CALLS = ("alloc_budget", "verify_attn", "verify_attn_plan", "verify_attn_run", "prepare_round", "pack_verify", "append_kv",
         "spec_accept", "spec_accept_noalloc", "spec_accept_debug", "spec_accept_stats", "draft_stats", "rope_append",
         "window_attn", "fork_pages", "reserve_pages", "release_pages", "compact_pages", "copy_pages")


def arguments(name):
    out = []
    for a in inspect.signature(getattr(B, name)).parameters.values():
        if a.name == "stream":
            continue
        desc = {"bdesc": B.BudgetDesc, "pdesc": B.PackDesc, "adesc": B.AttnDesc}.get(a.name)
        if a.name == "desc":
            desc = B.RopeDesc if name == "rope_append" else B.AttnDesc
        out.append(desc() if desc else 1 if a.name in ("rows_in", "max_moves", "window", "sinks") else _Tensor())
    return out


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("raw", [True, False])
def test_calls_run_on_their_tensors_device(name, raw, monkeypatch):
    """With device 0 current and tensors on device 1: device 1 is current during the call, which gets its stream; with torch's
    own look-up of the handle and without."""
    state = {"device": 0}

    class device:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            self.was, state["device"] = state["device"], self.d

        def __exit__(self, *a):
            state["device"] = self.was

    class library:
        def __getattr__(self, fn):
            def call(*args):
                state["seen"] = (fn, state["device"], args[-1])
                return B.SV_OK
            return call

    monkeypatch.setattr(torch.cuda, "current_device", lambda: state["device"])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda d=None: type("s", (), {"cuda_stream": 100 + (state["device"] if d is None else d)}))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 100 + d, raising=False)
    if not raw:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(B, "_current_stream", None, raising=False)
    monkeypatch.setattr(B, "load", library)
    getattr(B, name)(*arguments(name))
    assert state["seen"] == ("sv_" + name, 1, 101) and state["device"] == 0
    getattr(B, name)(*arguments(name), stream=7)
    assert state["seen"] == ("sv_" + name, 1, 7) and state["device"] == 0
    assert set(CALLS) == {n[3:] for n in B.EXPORTED} - {"spec_accept_workspace_size", "verify_attn_workspace_size",
                                                       "draft_stats_workspace_size", "window_attn_workspace_size",
                                                       "reserve_pages_workspace_size", "compact_pages_workspace_size",
                                                       "status_string", "last_error", "abi_version"}
