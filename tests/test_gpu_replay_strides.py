"""Strides that attention need not look at."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF = torch.bfloat16


def _all(q, k, v, g, **how):
    out, lse = replay.attention(q, k, v, **how)
    return (out, lse) + replay.attention_grad(g, q, k, v, out, lse, **how)


def _equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def _dense(seed, B, n, m, H, Hk, dim=64):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn((B, s, h, dim), generator=gen).to(BF).to(DEV) for s, h in ((n, H), (m, Hk), (m, Hk), (n, H))]


@pytest.mark.parametrize("n,m,H,Hk", [(40, 50, 2, 1), (1, 70, 2, 1), (1, 1, 1, 1), (33, 1, 1, 1)])
def test_dimensions_of_one_entry(n, m, H, Hk):
    """The stride of a dimension with one entry says nothing, whatever it is."""
    print("CASE", n, m, H, Hk, flush=True)
    x = _dense(101, 1, n, m, H, Hk)

    def odd(t):
        return t.as_strided(t.shape, [s if size > 1 or i == 3 else 2 ** 45 + 3
                                      for i, (size, s) in enumerate(zip(t.shape, t.stride()))])
    want = _all(*x, causal=True)
    y = [odd(t) for t in x]
    assert _equal(_all(*y, causal=True), want)
    out, lse = replay.attention(*y[:3], causal=True, out=odd(torch.empty_like(x[0])))
    grads = replay.attention_grad(y[3], *y[:3], out, lse, causal=True,
                                  **{n: odd(torch.empty_like(t)) for n, t in zip(("dq", "dk", "dv"), x)})
    assert _equal((out, lse) + grads, want)
