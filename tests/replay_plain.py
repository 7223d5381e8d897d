"""Plain 64-bit forms of the replay operators and bounds on what 16- or 32-bit
kernels may be off by, written from the definitions.  CPU tensors in fp64.

Each bound is an elementwise sum of first-order rounding errors: u, the unit
roundoff of the element type, once for the result and once for each operand that
is rounded to that type on the way, times the sum of magnitudes that it enters;
fp32 accumulation adds terms near 2^-24 times the number of terms, which SLACK
covers generously.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}
SLACK = 1e-4          # fp32 accumulation and exp of scores of a few hundred at most


def d(x):
    return x.detach().cpu().double()


def within(got, want, bound, what=""):
    """Equal where `want` is not finite, within `bound` elsewhere."""
    got, want = d(got), d(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    assert bool(torch.isfinite(got[fine]).all()), f"{what}: not finite"
    over = (got - want).abs()[fine] - d(bound).expand(want.shape)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (
        f"{what}: over the bound by {float(over.max()):.3g}, "
        f"error {float((got - want).abs()[fine].max()):.3g}")


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def rotary(x, positions, freqs, layout, inverse=False, amplitude=1.0):
    """(turned x, magnitude of each pair's terms); x [B, S, H, D], positions [B, S]."""
    y, mag = d(x).clone(), d(x).abs().clone()
    rot = 2 * len(freqs)
    angle = positions.cpu().double()[..., None] * d(freqs)
    cos, sin = amplitude * angle.cos()[:, :, None], amplitude * angle.sin()[:, :, None]
    sin = -sin if inverse else sin
    i = torch.arange(rot // 2)
    a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    p, q = d(x)[..., a], d(x)[..., b]
    y[..., a], y[..., b] = p * cos - q * sin, q * cos + p * sin
    mag[..., a] = mag[..., b] = abs(amplitude) * (p.abs() + q.abs())
    return y, mag


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def seen(n, m, causal, window):
    """[n, m]: whether query i sees key j."""
    at = torch.arange(n)[:, None] + (m - n)
    j = torch.arange(m)[None, :]
    s = torch.ones((n, m), dtype=torch.bool)
    if causal:
        s &= j <= at
    if window:
        s &= j > at - window
    return s


def one_head(q, k, v, see, scale):
    """P, S and lse of one head; pairs that are not seen are left out, not
    multiplied by zero."""
    s = torch.where(see, (q @ k.T) * scale, -math.inf)
    s = torch.where(see, s, -math.inf)
    top = s.amax(1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf).double()
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.where(see, (s - top).exp(), 0.0)
    total = p.sum(1, keepdim=True)
    lse = total.log() + top
    return torch.where(total == 0, 0.0, p / total), lse[:, 0]


def product(p, v, see):
    """p @ v over the seen pairs only: hidden infinities and NaN do not reach."""
    out = torch.where(see, p, 0.0) @ torch.where(torch.isfinite(v), v, 0.0)
    for j in (~torch.isfinite(v)).any(1).nonzero()[:, 0].tolist():
        bad = torch.where(torch.isfinite(v[j]), 0.0, v[j])
        out = out + torch.where(see[:, j:j + 1] & (bad != 0)[None], p[:, j:j + 1] * bad[None], 0.0)
    return out


def attention(q, k, v, q_lens, k_lens, causal, window, scale, dout=None, dtype=torch.bfloat16):
    """Packed tensors [tokens, heads, D].  Returns a dict of values and bounds:
    out, lse and, with dout, dq, dk, dv; each with a *_bound beside it."""
    H, D = q.shape[1], q.shape[2]
    G = H // k.shape[1]
    u = 1.05 * U[dtype]
    q, k, v = d(q), d(k), d(v)
    g = d(dout) if dout is not None else None
    r = {n: torch.zeros_like(t) for n, t in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    r |= {n + "_bound": torch.zeros_like(t) for n, t in r.items()}
    r["lse"] = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    q0 = k0 = 0
    for n, m in zip(q_lens, k_lens):
        see = seen(n, m, causal, window)
        for h in range(H):
            qs, ks = (slice(q0, q0 + n), h), (slice(k0, k0 + m), h // G)
            Q, K, V = q[qs], k[ks], v[ks]
            P, r["lse"][qs] = one_head(Q, K, V, see, scale)
            O = product(P, V, see)
            A = P @ V.abs().nan_to_num(0, 0, 0)
            r["out"][qs] = O
            r["out_bound"][qs] = u * (O.abs().nan_to_num(0, 0, 0) + A) + SLACK * A + TINY[dtype]
            if g is None:
                continue
            g_ = g[qs]
            r["dv"][ks] += product(P.T, g_, see.T)
            dP = torch.where(see, g_ @ V.T, 0.0)
            delta = torch.where(P > 0, P * dP, 0.0).sum(1, keepdim=True)
            dS = torch.where(see, P * (dP - delta), 0.0)
            r["dq"][qs] = scale * product(dS, K, see)
            r["dk"][ks] += scale * product(dS.T, Q, see.T)
            # first-order errors of P, delta (through the rounded output) and dS
            ga, va = g_.abs().nan_to_num(0, 0, 0), V.abs().nan_to_num(0, 0, 0)
            e_delta = (ga * (u * (O.abs().nan_to_num(0, 0, 0) + A) + SLACK * A)).sum(1, keepdim=True)
            size = P * (ga @ va.T + (ga * A).sum(1, keepdim=True))
            e = (u * dS.abs() + P * e_delta + SLACK * size + TINY[dtype]).nan_to_num(0, 0, 0)
            r["dv_bound"][ks] += (u + SLACK) * (P.T.nan_to_num(0) @ ga) + n * TINY[dtype]
            r["dq_bound"][qs] = scale * (e @ K.abs().nan_to_num(0, 0, 0))
            r["dk_bound"][ks] += scale * (e.T @ Q.abs().nan_to_num(0, 0, 0))
        q0, k0 = q0 + n, k0 + m
    for n in ("dq", "dk", "dv"):
        r[n + "_bound"] += u * r[n].abs().nan_to_num(0, 0, 0) + TINY[dtype]
    r["lse_bound"] = 2e-5 * (1 + r["lse"].abs().nan_to_num(0, 0, 0))
    return r


# ---------------------------------------------------------------------------
# tokens to their experts and back
# ---------------------------------------------------------------------------
def order(ids, experts):
    flat = ids.cpu().reshape(-1).tolist()
    lists = [[c for c, e in enumerate(flat) if e == x] for x in range(experts)]
    offsets = [0]
    for some in lists:
        offsets.append(offsets[-1] + len(some))
    source = [c for some in lists for c in some]
    slot = [-1] * len(flat)
    for p, c in enumerate(source):
        slot[c] = p
    source += [-1] * (len(flat) - len(source))
    return offsets, source, torch.tensor(slot, dtype=torch.long).view(ids.shape)


def gather(rows, slot, weights=None):
    """(sum over a token's kept choices of weight * row, the magnitudes' sum)."""
    T, top = slot.shape
    rows = d(rows)
    out, mag = torch.zeros((T, rows.shape[1]), dtype=torch.float64), None
    mag = out.clone()
    for i in range(top):
        kept = slot[:, i] >= 0
        part = rows[slot[kept, i]]
        if weights is not None:
            part = part * d(weights)[kept, i][:, None]
        out[kept] += part
        mag[kept] += part.abs()
    return out, mag
