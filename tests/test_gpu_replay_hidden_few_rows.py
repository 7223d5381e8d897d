"""Hidden values that are not finite: few rows against many keys, and both 16-bit types."""
import math

import pytest
import torch

import replay_plain as plain

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("k_len", [40, 5000])                # a whole walk and a divided one
@pytest.mark.parametrize("window", [0, 30])
def test_new_tokens(dtype, value, dim, k_len, window):
    """Four queries of 8 heads on 2: a value or a key that only the later queries see, and
    with a window one that only the earlier ones see."""
    print("CASE", dtype, value, dim, k_len, window, flush=True)
    n, H, Hk = 4, 8, 2
    gen = torch.Generator().manual_seed(81)
    x = dict(q=torch.randn((n, H, dim), generator=gen).to(dtype).to(DEV),
             k=torch.randn((k_len, Hk, dim), generator=gen).to(dtype).to(DEV),
             v=torch.randn((k_len, Hk, dim), generator=gen).to(dtype).to(DEV))
    how = dict(causal=True, window=window, q_lens=[n], k_lens=[k_len])
    clean = replay.attention(x["q"], x["k"], x["v"], **how)
    see = plain.seen(n, k_len, True, window)
    for bad in [k_len - 2] + ([k_len - n - window + 2] if window else []):
        away = ~see[:, bad]
        assert 0 < int(away.sum()) < n
        for which in "vk":
            y = dict(x)
            y[which] = x[which].clone()
            y[which][bad, 1, 3] = value
            got = replay.attention(y["q"], y["k"], y["v"], **how)
            torch.cuda.synchronize()
            for a, b in zip(got, clean):
                a, b = a.cpu(), b.cpu()
                assert torch.equal(a[away], b[away]) and torch.equal(a[:, :H // Hk], b[:, :H // Hk]), which
            if which == "v":
                # where it is seen it shows with its sign, in its column alone
                seen = got[0].cpu()[~away][:, H // Hk:]
                want = torch.full_like(seen[..., 3], value)
                assert torch.equal(seen[..., 3].isnan(), want.isnan())
                assert math.isnan(value) or torch.equal(seen[..., 3], want)
                rest = torch.arange(dim) != 3
                assert bool(torch.isfinite(seen[..., rest]).all())


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,H,window", [(100, 2, 0), (100, 2, 20), (600, 64, 0), (600, 64, 90)])
def test_half_precision(value, dim, n, H, window):
    """fp16, in grids that take care from the start and in those that repeat marked units:
    rows that do not see the value keep their bits, forward and backward."""
    bad = n // 2 + 11
    gen = torch.Generator().manual_seed(82)
    x = {c: torch.randn((n, H, dim), generator=gen).to(HF).to(DEV) for c in "qkvg"}
    how = dict(causal=True, window=window)

    def run(t):
        q, k, v, g = (t[c][None] for c in "qkvg")
        out, lse = replay.attention(q, k, v, **how)
        r = (out, lse) + replay.attention_grad(g, q, k, v, out, lse, **how)
        return dict(zip(("out", "lse", "dq", "dk", "dv"), (a[0].cpu() for a in r)))
    clean = run(x)
    see = plain.seen(n, n, True, window)
    for which in "vkgq":
        print("CASE", which, value, dim, n, window, flush=True)
        y = dict(x)
        y[which] = x[which].clone()
        y[which][bad, 1::7, 3] = value
        got = run(y)
        if which in "vk":
            away_q = ~see[:, bad]
            away_k = ~(see[~away_q].any(0))
        else:
            away_q = torch.arange(n) != bad
            away_k = ~see[bad]
        touched = torch.zeros(H, dtype=torch.bool)
        touched[1::7] = True
        for name, rows in (("out", away_q), ("lse", away_q), ("dq", away_q), ("dk", away_k), ("dv", away_k)):
            a, b = got[name], clean[name]
            assert torch.equal(a[rows], b[rows]), (which, name)
            assert torch.equal(a[:, ~touched], b[:, ~touched]), (which, name)
        if which == "v":
            assert not bool(torch.isfinite(got["out"][~away_q][:, touched, 3]).any())
