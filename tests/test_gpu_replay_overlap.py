"""Results of attention that would lie on its inputs are refused: a unit that is repeated
reads its rows again after others were written."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"


def test_refusals():
    gen = torch.Generator().manual_seed(131)
    q, k, v, g = (torch.randn((40, 2, 64), generator=gen).bfloat16().to(DEV) for _ in range(4))
    want = [t.clone() for t in (q, k, v, g)]
    for t in (q, k, v):
        with pytest.raises(replay.C3Error):
            replay.attention(q, k, v, causal=True, out=t)
    out, lse = replay.attention(q, k, v, causal=True)
    for bad in (dict(dq=q), dict(dk=k), dict(dv=v), dict(dk=v), dict(dv=k), dict(dq=g), dict(dv=g), dict(dq=out)):
        with pytest.raises(replay.C3Error):
            replay.attention_grad(g, q, k, v, out, lse, causal=True, **bad)
    d = torch.empty_like(k)
    for bad in (dict(dk=d, dv=d), dict(dq=d, dk=d), dict(dq=d, dv=d)):
        with pytest.raises(replay.C3Error):
            replay.attention_grad(g, q, k, v, out, lse, causal=True, **bad)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((q, k, v, g), want))       # nothing ran
    # inputs may be one tensor
    a, b = replay.attention(q, q, q, causal=True), replay.attention(q, q.clone(), q.clone(), causal=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
