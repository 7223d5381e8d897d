"""Attention's gradient where a key's scores are all -inf."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF = torch.bfloat16


def _run(x, **how):
    Q, K, V, G = (t.to(DEV) for t in x)
    how = dict(how, q_lens=[x[0].shape[0]], k_lens=[x[1].shape[0]])
    out, lse = replay.attention(Q, K, V, **how)
    return replay.attention_grad(G, Q, K, V, out, lse, **how)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [96, 97, 128, 150])
@pytest.mark.parametrize("causal", [False, True])
def test_key_of_minus_infinity(dim, rows, causal):
    """A key whose scores are all -inf takes no part: its dk and dv are zeros, whatever
    the number of rows."""
    print("CASE", dim, rows, causal, flush=True)
    gen = torch.Generator().manual_seed(72)
    q, k, v, g = (torch.randn((rows, 1, dim), generator=gen).to(BF) for _ in range(4))
    q[..., 3] = q[..., 3].abs() + 1
    at = 20
    k[at, :, 3] = -math.inf
    _, dk, dv = _run((q, k, v, g), causal=causal)
    assert not bool(dk[at].any()) and not bool(dv[at].any())
    away = [j for j in range(rows) if j != at]
    assert bool(torch.isfinite(dv[away]).all()) and bool(torch.isfinite(dk[away]).all())
