"""Attention's gradient where rows see few keys, against the plain 64-bit forms
(replay_plain)."""
import math

import pytest
import torch

import replay_plain as plain

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF, HF = torch.bfloat16, torch.float16


def _run(x, **how):
    Q, K, V, G = (t.to(DEV) for t in x)
    how = dict(how, q_lens=[x[0].shape[0]], k_lens=[x[1].shape[0]])
    out, lse = replay.attention(Q, K, V, **how)
    return replay.attention_grad(G, Q, K, V, out, lse, **how)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,window", [(600, 2), (600, 3), (40, 2)])
def test_small_windows(dtype, dim, n, window):
    """dq and dk of a small window over several tiles of rows: the output's rounding does
    not enter.  The error is that of two independent roundings of equal size, of a result
    (taken from the 64-bit one) and of a product's operand, so the square root of two
    times the first in the norm, and a quarter more for the spread; delta from the
    rounded output gives twice the first and more."""
    print("CASE", dtype, dim, n, window, flush=True)
    gen = torch.Generator().manual_seed(71)
    x = [torch.randn((n, 2, dim), generator=gen).to(dtype) for _ in range(4)]
    dq, dk, _ = _run(x, causal=True, window=window)
    want = plain.attention(*x[:3], [n], [n], True, window, dim ** -0.5, x[3], dtype)
    for name, t in (("dq", dq), ("dk", dk)):
        w = want[name]
        one = (w.to(dtype).double() - w).norm() / w.norm()
        off = (plain.d(t) - w).norm() / w.norm()
        print(name, float(off), float(one), flush=True)
        assert float(off) <= 1.25 * math.sqrt(2) * float(one)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal,window,row", [(True, 0, 0), (False, 2, 599)])
def test_ends_of_long_walks(dtype, dim, causal, window, row):
    """The first query of a causal mask that sees two keys, and the last one of a window
    without it, in tiles whose other rows see more: dq as above."""
    print("CASE", dtype, dim, causal, window, flush=True)
    n = 600
    m = n + 1 if causal else n
    gen = torch.Generator().manual_seed(73)
    q, g = (torch.randn((n, 16, dim), generator=gen).to(dtype) for _ in range(2))
    k, v = (torch.randn((m, 16, dim), generator=gen).to(dtype) for _ in range(2))
    got = plain.d(_run((q, k, v, g), causal=causal, window=window)[0])[row]
    want = plain.attention(q, k, v, [n], [m], causal, window, dim ** -0.5, g, dtype)["dq"][row]
    one = (want.to(dtype).double() - want).norm() / want.norm()
    off = (got - want).norm() / want.norm()
    print(float(off), float(one), flush=True)
    assert float(off) <= 1.25 * math.sqrt(2) * float(one)
