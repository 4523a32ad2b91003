"""CPU-only: which attention workspace the binding uses (the device calls are replaced; nothing is launched)."""
import ctypes

import torch

from paper_2607_27090_b200 import memstore as M


class Machine:
    """Two devices with a current stream each, any of which may be capturing."""

    def __init__(self, monkeypatch):
        self.device, self.capturing = 0, set()
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.device, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: self.device in self.capturing, raising=False)
        outer = self

        class Guard:
            def __init__(self, index):
                self.index = index

            def __enter__(self):
                self.before, outer.device = outer.device, self.index

            def __exit__(self, *exc):
                outer.device = self.before

        monkeypatch.setattr(torch.cuda, "device", Guard)


def bare_store(index=0):
    s = object.__new__(M.MemStore)
    s.device, s._index, s._workspace_bytes, s._workspaces = torch.device("cuda", index), index, 64, {}
    s._empty = lambda stream, *specs: [torch.empty(shape, dtype=dtype) for shape, dtype in specs]
    return s


def test_a_capture_on_the_stores_device_gets_a_workspace_of_its_own_whichever_device_is_current(monkeypatch):
    m, s = Machine(monkeypatch), bare_store(index=1)
    kept = s._workspace(0, None)
    assert s._workspace(0, None) is kept
    m.capturing = {1}
    assert s._workspace(0, None) is not kept and m.device == 0
    m.device = 1
    assert s._workspace(0, None) is not kept
    m.capturing, m.device = {0}, 0  # a capture on another device has nothing to do with this store
    assert s._workspace(0, None) is kept


def test_workspaces_are_kept_for_the_streams_that_stay(monkeypatch):
    m, s = Machine(monkeypatch), bare_store()
    ids = {0: 0, 0x7F00AA10: 3, 0x7F00BB20: 0x7F00BB20}  # handle -> id: the default stream, one of torch's pool, an external one
    current = {}
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current["stream"])
    for handle, stays in ((0, True), (0x7F00AA10, True), (0x7F00BB20, False)):
        current["stream"] = type("Stream", (), {"stream_id": ids[handle]})
        first = s._workspace(handle, None)
        assert (s._workspace(handle, None) is first) == stays and (handle in s._workspaces) == stays
    assert m.device == 0


def test_close_gives_the_workspaces_back(monkeypatch):
    m, s = Machine(monkeypatch), bare_store()
    destroyed = []
    s._h, s._lib = ctypes.c_void_p(1), type("Lib", (), {"memstore_destroy": staticmethod(lambda h: destroyed.append(h.value))})
    s._workspace(0, None)
    assert s._workspaces
    s.close()
    assert destroyed == [1] and not s._workspaces
    s.close()
    assert destroyed == [1] and m.device == 0
