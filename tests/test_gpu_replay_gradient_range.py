"""The range of attention's gradient in 16 bits: gradients and probabilities far from
one, against the plain 64-bit forms (replay_plain), in the norm.

Two roundings to the inputs' type make up the error: that of a result, whose size
is taken from the 64-bit result itself, and that of a product's operand, half a unit
in the last place at most; twice the latter leaves room for the output's rounding and
for 32-bit sums.
"""
import pytest
import torch

import replay_plain as plain

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
HF, BF = torch.float16, torch.bfloat16


def _close(got, want, dtype, name):
    size = want.norm()
    bound = (want.to(dtype).double() - want).norm() / size + 2 * plain.U[dtype]
    off = (plain.d(got) - want).norm() / size
    print(name, float(off), float(bound), flush=True)
    assert float(off) <= float(bound), (name, float(off), float(bound))


def _check(q, k, v, g, names=("dq", "dk", "dv"), **how):
    Q, K, V, G = (t.to(DEV) for t in (q, k, v, g))
    n, m = q.shape[0], k.shape[0]
    how = dict(how, q_lens=[n], k_lens=[m])
    out, lse = replay.attention(Q, K, V, **how)
    got = dict(zip(("dq", "dk", "dv"), replay.attention_grad(G, Q, K, V, out, lse, **how)))
    want = plain.attention(q, k, v, [n], [m], how.get("causal", False), 0, q.shape[2] ** -0.5, g, q.dtype)
    for x in names:
        _close(got[x], want[x], q.dtype, x)


def _inputs(seed, n, m, heads, kv, dim, dtype):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn((s, h, dim), generator=gen).to(dtype)
            for s, h in ((n, heads), (m, kv), (m, kv), (n, heads))]


@pytest.mark.parametrize("sigma", [1.0, 1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("dim,causal", [(64, False), (64, True), (128, True)])
@pytest.mark.parametrize("dtype", [HF, BF])
def test_small_output_gradients(dtype, dim, causal, sigma):
    """P (dP - delta) of 4,096 keys is a ten-thousandth of the output's gradient: below
    the normal fp16 numbers."""
    print("CASE", dtype, dim, causal, sigma, flush=True)
    q, k, v, g = _inputs(61, 200, 4096, 2, 1, dim, dtype)
    _check(q, k, v, (g.float() * sigma).to(dtype), causal=causal)


def test_small_probabilities():
    """65,536 keys: probabilities below the normal fp16 numbers."""
    print("CASE", flush=True)
    _check(*_inputs(62, 70, 65536, 1, 1, 64, HF))


@pytest.mark.parametrize("dim", [64, 128])
def test_large_output_gradients(dim):
    """Few keys, large values and gradients: P (dP - delta) past fp16's largest number,
    dq and dk within it."""
    print("CASE", dim, flush=True)
    q, k, v, g = _inputs(63, 300, 4, 2, 1, dim, HF)
    _check(q * 0.01, k * 0.01, v * 30, g * 1000, names=("dq", "dk"))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_of_every_size(dim, causal):
    """Output gradients that grow and shrink by 10^7 along the rows, in each order: each
    row of dq by itself, dk and dv by the rows that see the key."""
    for order in (1, -1):
        print("CASE", dim, causal, order, flush=True)
        q, k, v, g = _inputs(64, 600, 700, 2, 1, dim, HF)
        size = torch.logspace(-5, 2, 600)
        size = size if order == 1 else size.flip(0)
        g = (g.float() * size[:, None, None]).to(HF)
        how = dict(causal=causal, q_lens=[600], k_lens=[700])
        Q, K, V, G = (t.to(DEV) for t in (q, k, v, g))
        out, lse = replay.attention(Q, K, V, **how)
        dq, dk, dv = replay.attention_grad(G, Q, K, V, out, lse, **how)
        want = plain.attention(q, k, v, [600], [700], causal, 0, dim ** -0.5, g, HF)
        for i in range(0, 600, 50):
            _close(dq[i:i + 50], want["dq"][i:i + 50], HF, f"dq {i}")
        _close(dk, want["dk"], HF, "dk")
        _close(dv, want["dv"], HF, "dv")


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_not_finite_output_gradient(value):
    """One row's gradient is not finite: the other rows keep their values."""
    print("CASE", value, flush=True)
    q, k, v, g = _inputs(65, 200, 200, 1, 1, 64, HF)
    how = dict(q_lens=[200], k_lens=[200])
    Q, K, V, G = (t.to(DEV) for t in (q, k, v, g))
    out, lse = replay.attention(Q, K, V, **how)
    clean = replay.attention_grad(G, Q, K, V, out, lse, **how)[0]
    G[77, 0, 5] = value
    dq, dk, dv = replay.attention_grad(G, Q, K, V, out, lse, **how)
    away = torch.arange(200) != 77
    assert torch.equal(dq.cpu()[away], clean.cpu()[away])
    assert not bool(torch.isfinite(dq[77]).any()) and not bool(torch.isfinite(dk).any())
    assert not bool(torch.isfinite(dv[:, 0, 5]).any()) and bool(torch.isfinite(dv[:, 0, 6]).all())
