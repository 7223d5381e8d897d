"""Attention walks that are divided among workgroups, in padded batches, and the
memory and arguments of calls on another stream, against the plain 64-bit forms
(replay_plain)."""
import math

import pytest
import torch

import replay_plain as plain

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("S,M,H,Hk,D,q_lens,k_lens", [
    (4, 4099, 8, 2, 128, [4, 2, 0], [4099, 900, 700]),        # 16 rows of a key head
    (7, 2500, 4, 4, 64, [1, 7, 3], [2500, 2500, 5]),
    (200, 4096, 8, 2, 128, [200, 50, 0], [4096, 3000, 100]),  # tiles of 128 rows, cut by the padding
    (300, 3001, 2, 2, 64, [299, 1, 130], [3001, 2900, 0]),
])
def test_divided_walks_and_padding(S, M, H, Hk, D, q_lens, k_lens, causal):
    """Padding that shares a tile with queries comes back as zeros and -inf also
    where the walk over the keys is divided; what it holds does not matter."""
    print("CASE", S, M, H, Hk, D, causal, flush=True)
    B = len(q_lens)
    gen = torch.Generator().manual_seed(31)
    q, g = (torch.full((B, S, H, D), math.nan, dtype=BF) for _ in range(2))
    k, v = (torch.full((B, M, Hk, D), math.nan, dtype=BF) for _ in range(2))
    for b in range(B):
        for t, n in ((q, q_lens), (g, q_lens), (k, k_lens), (v, k_lens)):
            t[b, :n[b]] = torch.randn(t[b, :n[b]].shape, generator=gen).to(BF)
    Q, K, V, Gd = (x.to(DEV) for x in (q, k, v, g))
    how = dict(causal=causal, q_lens=q_lens, k_lens=k_lens)
    out, lse = replay.attention(Q, K, V, **how)
    dq, dk, dv = replay.attention_grad(Gd, Q, K, V, out, lse, **how)
    torch.cuda.synchronize()

    def packed(t, n):
        return torch.cat([t[b, :n[b]] for b in range(B)]).cpu()
    want = plain.attention(packed(q, q_lens), packed(k, k_lens), packed(v, k_lens), q_lens, k_lens, causal, 0,
                           D ** -0.5, packed(g, q_lens), BF)
    for n, t, lens in (("out", out, q_lens), ("lse", lse, q_lens), ("dq", dq, q_lens), ("dk", dk, k_lens),
                       ("dv", dv, k_lens)):
        plain.within(packed(t, lens), want[n], want[n + "_bound"], n)
    for b in range(B):
        for t, n in ((out, q_lens), (dq, q_lens), (dk, k_lens), (dv, k_lens)):
            assert not bool(t[b, n[b]:].any())
        assert bool((lse[b, q_lens[b]:] == -math.inf).all())


def test_memory_comes_from_the_stream_of_the_call():
    """Results and workspaces that a call on another stream makes belong to that
    stream: memory freed there is not given to the current one."""
    gen = torch.Generator().manual_seed(32)
    q = torch.randn((64, 2, 64), generator=gen).to(BF).to(DEV)
    want = replay.attention(q, q, q, causal=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out, lse = replay.attention(q, q, q, causal=True, stream=s)
    s.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    at = out.data_ptr()
    del out, lse
    here = [torch.empty_like(q) for _ in range(64)]
    assert at not in [t.data_ptr() for t in here]


def test_argument_ranges():
    """Numbers that the call's 32-bit fields cannot hold are refused, not cut off."""
    q = torch.zeros((8, 2, 64), dtype=BF, device=DEV)
    bad = pytest.raises(replay.C3Error)
    for window in (2 ** 32, 2 ** 32 + 5, 2.5, "1", None):
        with bad:
            replay.attention(q, q, q, causal=True, window=window)
    for lens in ([2 ** 32 + 8], [8.0], [-(2 ** 32) + 8], ["8"]):
        with bad:
            replay.attention(q, q, q, q_lens=lens, k_lens=[8])
        with bad:
            replay.attention(q, q, q, q_lens=[8], k_lens=lens)
    ids = torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    for n in (2 ** 32 + 4, 0, -1, replay.MAX_EXPERTS + 1, 4.0, "4"):
        with bad:
            replay.expert_sort(ids, n)


@pytest.mark.parametrize("window", [0, 5000])
@pytest.mark.parametrize("k_len,heads,dim", [(70001, 2, 64), (33000, 1, 128), (3100, 3, 72), (257, 1, 8)])
def test_many_parts(k_len, heads, dim, window):
    """One token against caches that are divided into few and into many parts, some of
    which a window leaves empty; the same bits every time."""
    print("CASE", k_len, heads, dim, window, flush=True)
    gen = torch.Generator().manual_seed(33)
    q = torch.randn((1, heads, dim), generator=gen).to(BF)
    k, v = (torch.randn((k_len, 1, dim), generator=gen).to(BF) for _ in range(2))
    k[k_len // 3] *= 4                      # one part's maximum stands out
    how = dict(causal=True, window=window, q_lens=[1], k_lens=[k_len])
    x = [t.to(DEV) for t in (q, k, v)]
    out, lse = replay.attention(*x, **how)
    want = plain.attention(q, k, v, [1], [k_len], True, window, dim ** -0.5, None, BF)
    plain.within(out, want["out"], want["out_bound"], "out")
    plain.within(lse, want["lse"], want["lse_bound"], "lse")
    again = replay.attention(*x, **how)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_workgroups_of_every_length_and_head():
    """Key heads and sequences that are no multiple of the eight dies, of very different
    lengths: every unit is done once."""
    q_lens, k_lens = [260, 1, 130, 0, 515], [260, 77, 600, 9, 515]
    gen = torch.Generator().manual_seed(34)
    H, Hk, D = 9, 3, 64
    q, g = (torch.randn((sum(q_lens), H, D), generator=gen).to(BF) for _ in range(2))
    k, v = (torch.randn((sum(k_lens), Hk, D), generator=gen).to(BF) for _ in range(2))
    how = dict(causal=True, q_lens=q_lens, k_lens=k_lens)
    Q, K, V, Gd = (t.to(DEV) for t in (q, k, v, g))
    out, lse = replay.attention(Q, K, V, **how)
    dq, dk, dv = replay.attention_grad(Gd, Q, K, V, out, lse, **how)
    want = plain.attention(q, k, v, q_lens, k_lens, True, 0, D ** -0.5, g, BF)
    for n, t in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        plain.within(t, want[n], want[n + "_bound"], n)


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window", [0, 90])
def test_hidden_values_in_large_grids(value, dim, window):
    """More workgroups than compute units: units that met a hidden value which is not
    finite are marked and repeated with care, and rows that do not see it keep their bits."""
    n, H, bad = 600, 64, 301
    gen = torch.Generator().manual_seed(35)
    x = {c: torch.randn((n, H, dim), generator=gen).to(BF).to(DEV) for c in "qkvg"}
    how = dict(causal=True, window=window)

    def run(t):
        out, lse = replay.attention(t["q"], t["k"], t["v"], **how)
        return dict(zip(("out", "lse", "dq", "dk", "dv"),
                        (out, lse) + replay.attention_grad(t["g"], t["q"], t["k"], t["v"], out, lse, **how)))
    clean = run(x)
    see = plain.seen(n, n, True, window)
    for which in "vkgq":
        print("CASE", which, value, dim, window, flush=True)
        y = dict(x)
        y[which] = x[which].clone()
        y[which][bad, 5::7, 3] = value
        got = run(y)
        torch.cuda.synchronize()
        if which in "vk":
            away_q = ~see[:, bad]
            away_k = ~(see[~away_q].any(0))
        else:
            away_q = torch.arange(n) != bad
            away_k = ~see[bad]
        touched = torch.zeros(H, dtype=torch.bool)
        touched[5::7] = True
        for name, rows in (("out", away_q), ("lse", away_q), ("dq", away_q), ("dk", away_k), ("dv", away_k)):
            a, b = got[name].cpu(), clean[name].cpu()
            assert torch.equal(a[rows], b[rows]), (which, name)
            assert torch.equal(a[:, ~touched], b[:, ~touched]), (which, name)
        if which == "v":
            assert not bool(torch.isfinite(got["out"].cpu()[~away_q][:, touched, 3]).any())
