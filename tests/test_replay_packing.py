"""The binding's packed arguments against the structures of include/c3_replay.h."""
import ctypes

import pytest

replay = pytest.importorskip("paper_2608_11034_amd.replay")


def test_heads():
    raw = replay._HEADS.pack(1, 2, 3, 4, 5, 6, 7, 8, 9)
    assert len(raw) == ctypes.sizeof(replay.Heads)
    h = replay.Heads.from_buffer_copy(raw)
    assert (h.in_, h.out, list(h.in_stride), list(h.out_stride), h.heads) == (1, 2, [3, 4, 5], [6, 7, 8], 9)


def test_attention():
    raw = replay._ATTENTION.pack(1, 2, 3, 4, 5, 6, 0.5, 8, 9, 10, 11, 12, 13, 14)
    assert len(raw) == ctypes.sizeof(replay.Attention)
    a = replay.Attention.from_buffer_copy(raw)
    assert [getattr(a, n) for n, _ in replay.Attention._fields_] == [1, 2, 3, 4, 5, 6, 0.5, 8, 9, 10, 11, 12, 13, 14]
    raw = replay._ATTN_TENSOR.pack(1, 2, 3, 4)
    assert len(raw) == ctypes.sizeof(replay.AttnTensor)
    t = replay.AttnTensor.from_buffer_copy(raw)
    assert (t.ptr, list(t.stride)) == (1, [2, 3, 4])


def test_expert_rows():
    raw = replay._EXPERT_ROWS.pack(1, 2, 3, 4, 5, 6, 7, 8)
    assert len(raw) == ctypes.sizeof(replay.ExpertRows)
    r = replay.ExpertRows.from_buffer_copy(raw)
    assert [getattr(r, n) for n, _ in replay.ExpertRows._fields_] == [1, 2, 3, 4, 5, 6, 7, 8]
