"""Rotary positions where a dimension has one entry: its stride says nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"


@pytest.mark.parametrize("shape", [(1, 30, 2, 64), (2, 1, 3, 64), (2, 30, 1, 64), (1, 1, 1, 64)])
def test_in_place(shape):
    """In place through two views that differ in the stride of such a dimension alone."""
    print("CASE", shape, flush=True)
    x = torch.randn(shape, generator=torch.Generator().manual_seed(111)).bfloat16().to(DEV)
    pos, f = torch.arange(shape[1], device=DEV) + 5, replay.rotary_frequencies(64)
    want = replay.rotary(x, pos, f)
    other = x.as_strided(shape, [s if n > 1 or i == 3 else 7 for i, (n, s) in enumerate(zip(shape, x.stride()))])
    assert torch.equal(replay.rotary(x, pos, f, out=other), want)
    assert torch.equal(x, want)
