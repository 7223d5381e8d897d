"""Lists of sequences under graph capture: those that go along as an argument are
replayed, those that are staged through host memory are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
MOST = replay.MAX_CAPTURED_SEQUENCES


def _inputs(seed, lens):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn((sum(lens), h, 64), generator=gen).bfloat16().to(DEV) for h in (2, 1, 1, 2)]


def _both(x, how):
    q, k, v, g = x
    out, lse = replay.attention(q, k, v, **how)
    return (out, lse) + replay.attention_grad(g, q, k, v, out, lse, **how)


def test_most_sequences_captured():
    """Replays after more calls that stage their lists than the ring has slots."""
    lens = [(i * 7) % 23 for i in range(MOST)]
    how = dict(causal=True, q_lens=lens, k_lens=lens)
    x = _inputs(41, lens)
    _both(x, how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _both(x, how)
    others = [(i * 5) % 9 for i in range(400)]
    y = _inputs(42, others)
    for seed in (43, 44, 45):
        for t, new in zip(x, _inputs(seed, lens)):
            t.copy_(new)
        for _ in range(20):
            _both(y, dict(causal=True, q_lens=others, k_lens=others))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, _both(x, how)))


@pytest.mark.parametrize("n", [MOST + 1, 128, 129, 500])
def test_more_sequences_are_refused(n):
    print("CASE", n, flush=True)
    lens = [i % 4 for i in range(n)]
    how = dict(q_lens=lens, k_lens=lens)
    q, k, v, g = x = _inputs(46, lens)
    want = _both(x, how)
    torch.cuda.synchronize()
    other = torch.zeros(64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(replay.C3Error):
            replay.attention(q, k, v, **how)
        with pytest.raises(replay.C3Error):
            replay.attention_grad(g, q, k, v, *want[:2], **how)
        other.add_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert float(other[0]) == 1                     # the capture itself went on
    assert all(torch.equal(a, b) for a, b in zip(want, _both(x, how)))
