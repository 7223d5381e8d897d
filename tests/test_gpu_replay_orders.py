"""Orders that no expert_sort made are refused before anything runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"


def test_refusals():
    ids = torch.zeros((6, 2), dtype=torch.int32, device=DEV)
    order = replay.expert_sort(ids, 4)
    x, y, w = torch.zeros((6, 64), device=DEV), torch.zeros((12, 64), device=DEV), torch.ones((6, 2), device=DEV)
    for bad in (dict(offsets=order.offsets[:0]), dict(offsets=order.offsets[:1]), dict(offsets=order.offsets[0]),
                dict(offsets=order.offsets.long()), dict(offsets=order.offsets.cpu()), dict(offsets=order.offsets[::2]),
                dict(source=order.source[:11]), dict(source=order.source.view(6, 2)), dict(source=order.source.cpu()),
                dict(slot=order.slot.view(-1)), dict(slot=order.slot[0, 0]), dict(slot=order.slot.cpu()),
                dict(slot=order.slot.float()), dict(slot=None)):
        o = order._replace(**bad)
        for call in (lambda: replay.expert_dispatch(x, o), lambda: replay.expert_combine(y, o, w),
                     lambda: replay.expert_dispatch_grad(y, o), lambda: replay.expert_combine_grad(x, y, o, w),
                     lambda: replay.expert_combine_grad(x, None, o)):
            with pytest.raises(replay.C3Error):
                call()
    assert torch.equal(replay.expert_combine(replay.expert_dispatch(x + 1, order), order), 2 * (x + 1))
