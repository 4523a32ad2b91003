"""CPU-only: the binding's marshalling and refusals of the calls for drafted trees and selected blocks (the library is replaced; nothing is launched)."""
import ctypes
import re
from pathlib import Path

import pytest
import torch

from paper_2607_27090_b200 import memstore as M

HEADER = (Path(__file__).resolve().parent.parent / "include" / "memstore.h").read_text()
NEW = ("memstore_plan_tree", "memstore_attend_tree", "memstore_accept", "memstore_summarize_blocks", "memstore_select_blocks", "memstore_attend_blocks")


def declared_parameters(name):
    text = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
    inside = re.search(r"\b%s\s*\(([^)]*)\)" % name, text).group(1)
    return [p.strip() for p in inside.split(",")]


@pytest.mark.parametrize("name", NEW)
def test_argument_types_follow_the_header(name):
    """One ctypes entry per declared parameter, of its kind: pointers and handles, 32-bit integers, floats, sizes."""
    kinds = []
    for p in declared_parameters(name):
        kinds.append("ptr" if "*" in p or p.startswith("ms_stream") else "f32" if p.startswith("float") else "size" if p.startswith("size_t") else "i32")
    args = getattr(M.load_library(), name).argtypes
    names = {ctypes.c_void_p: "ptr", ctypes.c_int32: "i32", ctypes.c_float: "f32", ctypes.c_size_t: "size"}
    assert [names.get(a, "ptr") for a in args] == kinds


class Recorder:
    """Stands in for the library: keeps the arguments of each call."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            assert len(args) == len(declared_parameters(name)), name
            self.calls.append((name, args))
            return 0

        return call


def bare_store(monkeypatch):
    s = object.__new__(M.MemStore)
    s._h, s._lib = ctypes.c_void_p(1), Recorder()
    s.device, s._index, s._workspace_bytes, s._workspaces = torch.device("cpu"), -1, 64, {}
    s.n_layers, s.n_kv_heads, s.head_dim = 2, 2, 64
    monkeypatch.setattr(M.MemStore, "_raw_stream", lambda self, stream: 77)
    monkeypatch.setattr(M.MemStore, "_workspace", lambda self, raw, stream: torch.empty(64, dtype=torch.uint8))
    monkeypatch.setattr(M.MemStore, "_paged", lambda self, cache: "cache")

    def heads(self, t, n_tokens, n_heads, name):
        assert t.shape == (n_tokens, n_heads, self.head_dim), name
        return name

    monkeypatch.setattr(M.MemStore, "_heads", heads)
    return s


def cache_of(n_layers=2, num_blocks=8, bs=16, h=2, d=64):
    k = torch.zeros((n_layers, num_blocks, bs, h, d), dtype=torch.bfloat16)
    return M.PagedCache(k, k.clone(), num_blocks * bs * h * d, bs * h * d, h * d, d, num_blocks, bs)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_calls_reach_the_library_with_their_arguments_in_place(monkeypatch):
    s = bare_store(monkeypatch)
    q, q_start, lens, tables, cache = torch.zeros((5, 8, 64), dtype=torch.bfloat16), ints(3), ints(2), ints(2, 9), cache_of()
    parents, tokens, choices, positions, free, taken = (ints(5) for _ in range(6))
    pos, mask, _ = s.plan_tree(parents, q_start, positions, 3)
    assert pos.shape == (5,) and (pos == -1).all() and mask.shape == (5, 3) and not mask.any()
    name, a = s._lib.calls[-1]
    assert name == "memstore_plan_tree" and a[1:9] == (parents.data_ptr(), 5, q_start.data_ptr(), 2, positions.data_ptr(), 3, pos.data_ptr(), mask.data_ptr())
    s.attend_tree(1, q, mask, cache, q_start, lens, tables, max_q_len=4)
    name, a = s._lib.calls[-1]
    assert name == "memstore_attend_tree" and a[1:5] == (1, "q", 8, 5) and a[7:12] == (2, mask.data_ptr(), 3, tables.data_ptr(), 9) and a[14] == 4 and a[-1] == 77
    got = s.accept(parents, tokens, choices, positions, q_start, lens, tables, cache, free, taken[:1])
    name, a = s._lib.calls[-1]
    assert name == "memstore_accept" and a[1:6] == (parents.data_ptr(), tokens.data_ptr(), choices.data_ptr(), positions.data_ptr(), 5)
    assert a[12:14] == (free.data_ptr(), 5) and a[15:21] == tuple(t.data_ptr() for t in (got.path, got.n_accepted, got.next_tokens, got.seq_lens, got.n_taken, got.status))
    assert got.path.shape == (5,) and got.n_accepted.shape == got.status.shape == (2,) and got.n_taken.shape == (1,)
    kept = s.accept(parents, tokens, choices, positions, q_start, lens, tables, cache)
    assert kept.n_taken is None and s._lib.calls[-1][1][12:15] == (None, 0, None) and s._lib.calls[-1][1][19] is None
    box = s.allocate_summaries(cache)
    assert box.shape == (2, 8, 2, 2, 64)
    s.summarize_blocks(1, cache, box[1], lens, tables, q_start=q_start, n_tokens=5)
    assert s._lib.calls[-1][1][1:9] == (1, q_start.data_ptr(), 5, lens.data_ptr(), 2, tables.data_ptr(), 9, "cache")
    s.summarize_blocks(0, cache, box[0], lens, tables)
    assert s._lib.calls[-1][1][2] is None
    blocks, scores = s.select_blocks(q, cache, box[0], q_start, lens, tables, 4, n_first=1, n_last=2)
    name, a = s._lib.calls[-1]
    assert blocks.shape == (5, 2, 4) and scores is None and a[10:14] == ("cache", 4, 1, 2) and a[14] == blocks.data_ptr()
    out, lse, status = s.attend_blocks(0, q, blocks, cache, q_start, lens, tables, want_lse=True)
    name, a = s._lib.calls[-1]
    assert name == "memstore_attend_blocks" and a[8:12] == (blocks.data_ptr(), 4, tables.data_ptr(), 9) and out.shape == q.shape and lse.shape == (5, 8)


def test_refusals_before_the_library_is_called(monkeypatch):
    s = bare_store(monkeypatch)
    q, q_start, lens, tables, cache = torch.zeros((5, 8, 64), dtype=torch.bfloat16), ints(3), ints(2), ints(2, 9), cache_of()
    five = ints(5)
    for call in (
        lambda: s.plan_tree(five, q_start, five),  # neither mask_words nor a mask
        lambda: s.plan_tree(five, q_start, five, 2, out_mask=ints(5, 3)),
        lambda: s.plan_tree(five, q_start, five, out_mask=five),
        lambda: s.attend_tree(0, q, five, cache, q_start, lens, tables),
        lambda: s.attend_tree(0, q, ints(5, 1), cache, q_start, lens, tables[0]),
        lambda: s.accept(five, five, five, five, q_start, lens, tables, cache, free_blocks=five),
        lambda: s.accept(five, five, five, five, q_start, lens, tables[0], cache),
        lambda: s.accept(five, five, five, five, q_start, lens, tables, cache_of(n_layers=1)),  # the call reaches every layer
        lambda: s.summarize_blocks(0, cache, s.allocate_summaries(cache)[0], lens, tables[:1]),
        lambda: s.select_blocks(q, cache, s.allocate_summaries(cache)[0], q_start, lens, tables[:1], 4),
        lambda: s.attend_blocks(0, q, ints(5, 2), cache, q_start, lens, tables),
    ):
        with pytest.raises(ValueError):
            call()
    for call in (
        lambda: s.plan_tree(five, q_start, five.float(), 2),
        lambda: s.attend_tree(0, q, ints(5, 1).long(), cache, q_start, lens, tables),
        lambda: s.select_blocks(q, cache, torch.zeros((8, 2, 2, 64)), q_start, lens, tables, 4),
        lambda: s.attend_blocks(0, q, ints(5, 2, 4).long(), cache, q_start, lens, tables),
    ):
        with pytest.raises(TypeError):
            call()
    assert not s._lib.calls


def test_a_null_store_is_refused():
    lib = M.load_library()
    for name in NEW:
        zeros = [None if t is ctypes.c_void_p or not isinstance(t(), (ctypes.c_int32, ctypes.c_float, ctypes.c_size_t)) else 0 for t in getattr(lib, name).argtypes]
        assert getattr(lib, name)(*zeros) == 1
