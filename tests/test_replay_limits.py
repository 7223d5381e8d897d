"""Limits of the replay operators that stand in more than one place, without a GPU."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_11034_amd", "csrc")

replay = pytest.importorskip("paper_2608_11034_amd.replay")


def _read(*path):
    return open(os.path.join(ROOT, *path)).read()


def test_captured_sequences():
    """One number says how many sequences go along as an argument."""
    n = replay.MAX_CAPTURED_SEQUENCES
    assert f"#define C3_ATTENTION_CAPTURE_SEQUENCES {n}\n" in _read("include", "c3_replay.h")
    assert "kAttnArgSeqs = C3_ATTENTION_CAPTURE_SEQUENCES;" in _read("paper_2608_11034_amd", "csrc", "c3_attention.h")
    assert f"up to {n} sequences" in re.sub(r"\s+", " ", replay.attention.__doc__)


def test_nothing_is_staged_unasked():
    """Every list that attention stages goes through the check of the stream."""
    uses = []
    for name in sorted(os.listdir(CSRC)):
        if name.startswith("c3_attention"):
            uses += [name] * len(re.findall(r"\bstage_bytes\(", _read("paper_2608_11034_amd", "csrc", name)))
    assert uses == ["c3_attention.hip"]
    body = _read("paper_2608_11034_amd", "csrc", "c3_attention.hip")
    at = body.index("int attn_stage(")
    assert at < body.index("hipStreamIsCapturing", at) < body.index("stage_bytes(", at) < body.index("\n}", at)


def _attention(batch, kv_heads, grad=False):
    """Workspace bytes of one token a sequence on one key (0: refused)."""
    a = replay.Attention(dtype=replay.BF16, heads=kv_heads, kv_heads=kv_heads, dim=8, causal=1, window=0, scale=1.0,
                         batch=batch, q_tokens=1, k_tokens=1)
    f = replay._lib().c3_attention_grad_workspace_size if grad else replay._lib().c3_attention_workspace_size
    return f(ctypes.byref(a))


@pytest.mark.parametrize("grad", [False, True])
def test_workgroups_of_attention(grad):
    """A launch holds fewer than 2^32 threads, 256 to a workgroup: more are refused
    before anything is launched."""
    assert _attention(2 ** 14 - 1, 2 ** 10, grad) > 0
    assert _attention(2 ** 14, 2 ** 10, grad) == 0 and _attention(2 ** 16, 2 ** 12, grad) == 0
