"""How the binding finds the current stream, with and without torch's short way to its handle (no GPU needed)."""
import types

import torch

from paper_2601_21896_amd import binding as B


def test_current_stream_by_the_public_interface_where_the_short_way_is_missing(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=1000 + device))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 2000 + device, raising=False)
    assert B._stream(None) == 2003
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert B._stream(None) == 1003
    assert B._stream(7) == 7 and B._stream(types.SimpleNamespace(cuda_stream=8)) == 8


def test_the_paged_module_binds_without_the_short_ways(monkeypatch):
    monkeypatch.setattr(B, "_PAGED", None)
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    call = B._paged()
    monkeypatch.undo()
    B._PAGED = None
    assert B._paged() is call                       # bound again, to what this torch has
