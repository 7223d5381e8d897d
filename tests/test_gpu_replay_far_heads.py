"""Attention on heads that lie far apart."""
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


def _far(t, big, at, apart):
    """t [1, S, H, D] with heads `apart` elements from each other in `big`."""
    _, n, h, d = t.shape
    v = big.as_strided(t.shape, (0, d, apart, 1), at)
    return v.copy_(t)


def test_heads_far_apart():
    """Heads before tokens in long caches: 2^31 bytes and more from head to head, with
    keys that several query heads share and with queries that share none."""
    big = torch.empty(2 ** 31 + 2 ** 24, dtype=BF, device=DEV)             # 4.3 GB
    apart = 2 ** 30 + 2 ** 20
    q, k, v, g = _dense(102, 1, 65, 90, 8, 2)
    want = _all(q, k, v, g, causal=True)
    K, V = _far(k, big, 0, apart), _far(v, big, 90 * 64, apart)
    assert _equal(_all(q, K, V, g, causal=True), want)
    one = _dense(103, 1, 1, 5000, 8, 2)
    K, V = _far(one[1], big, 0, apart), _far(one[2], big, 5000 * 64, apart)
    assert _equal(replay.attention(one[0], K, V, causal=True), replay.attention(*one[:3], causal=True))
    q, k, v, g = _dense(104, 1, 65, 90, 2, 2)
    want = _all(q, k, v, g, causal=True)
    y = [_far(t, big, i * 2 ** 16, apart) for i, t in enumerate((q, k, v, g))]
    assert _equal(_all(*y, causal=True), want)


def test_shared_queries_far_apart():
    """Query heads that share a key head so far apart: forward, and a refusal of the
    gradient, whose tiles hold the rows of all of them."""
    big = torch.empty(2 ** 31 + 2 ** 24, dtype=BF, device=DEV)
    q, k, v, g = _dense(105, 1, 65, 90, 2, 1)
    out, lse = replay.attention(q, k, v)
    Q = _far(q, big, 0, 2 ** 30 + 2 ** 20)
    assert _equal(replay.attention(Q, k, v), (out, lse))
    with pytest.raises(replay.C3Error):
        replay.attention_grad(g, Q, k, v, out, lse)
    G = _far(g, big, 2 ** 16, 2 ** 30 + 2 ** 20)
    with pytest.raises(replay.C3Error):
        replay.attention_grad(G, q, k, v, out, lse)
