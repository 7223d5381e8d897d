"""More tokens than one launch dimension has workgroups of 256 threads for (2^24)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF = torch.bfloat16


def test_rotary():
    """A workgroup a token, in place: tokens on both sides of 2^24 as by themselves."""
    tokens, dim = 2 ** 24 + 3, 514
    print("CASE", tokens, dim, flush=True)
    x = torch.empty((tokens, 1, dim), dtype=BF, device=DEV)          # 17 GB
    at = torch.tensor([0, 1, 2 ** 23, 2 ** 24 - 1, 2 ** 24, tokens - 1], device=DEV)
    x[at] = torch.randn((6, 1, dim), generator=torch.Generator().manual_seed(91)).to(BF).to(DEV)
    few = x[at].clone()
    pos = torch.arange(tokens, device=DEV, dtype=torch.int32)
    f = replay.rotary_frequencies(2)
    replay.rotary(x, pos, f, out=x)
    assert torch.equal(x[at], replay.rotary(few, pos[at], f))


def _order(tokens):
    """One choice a token, the experts in turn, every seventh token without one."""
    ids = torch.arange(tokens, device=DEV, dtype=torch.int32)
    ids = torch.where(ids % 7 == 3, -1, ids % 4).view(-1, 1).contiguous()
    order = replay.expert_sort(ids, 4)
    kept = int(order.offsets[-1])
    assert kept == int((ids >= 0).sum())
    return order, kept, order.source[:kept].long()


def test_rows():
    """A wave a token: to the experts and back."""
    tokens, hidden = 2 ** 26 + 5, 8
    print("CASE", tokens, hidden, flush=True)
    order, kept, source = _order(tokens)
    x = torch.randn((tokens, hidden), dtype=BF, device=DEV)
    xs = replay.expert_dispatch(x, order)
    assert torch.equal(xs[:kept], x[source]) and not bool(xs[kept:].any())
    back = replay.expert_combine(xs, order)
    assert torch.equal(back, torch.where(order.slot >= 0, x, 0.0))


def test_gradient_of_rows():
    """A workgroup a token."""
    tokens, hidden = 2 ** 24 + 3, 8
    print("CASE", tokens, hidden, flush=True)
    order, kept, source = _order(tokens)
    dout, y = (torch.randn((tokens, hidden), dtype=BF, device=DEV) for _ in range(2))
    w = torch.full((tokens, 1), 0.5, device=DEV)
    dy, dw = replay.expert_combine_grad(dout, y, order, w)
    assert torch.equal(dy[:kept], dout[source] * 0.5) and not bool(dy[kept:].any())
    want = (dout[source].double() * y[:kept].double()).sum(1)
    got = dw.view(-1)
    assert float((got[source] - want).abs().max()) <= 1e-4
    assert not bool(got[order.slot.view(-1) < 0].any())
