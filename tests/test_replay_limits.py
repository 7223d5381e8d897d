"""Limits of the replay operators that stand in more than one place, without a GPU."""
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
