"""Plain 64-bit forms of the embedding, the residual norm and the loss over a
vocabulary, from their definitions, and bounds on what the kernels may be off by.
CPU tensors in fp64.

U32 is half a step of fp32.  A sum of n terms in any order is off by at most n - 1
of it times the sum of the terms' magnitudes; a product, a root and a quotient by one
each of their size; the result by half a step of its type.
"""
import torch

from replay_plain import TINY, U, d

U32 = 2.0 ** -24


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def embedding(ids, table, scale):
    out = torch.zeros((len(ids), table.shape[1]), dtype=torch.float64)
    for t, i in enumerate(ids.tolist()):
        if 0 <= i < table.shape[0]:
            out[t] = scale * d(table[i])
    # the scale as fp32 and the product are rounded, then the result
    return out, out.abs() * (2 * U32 + U[table.dtype]) * 1.01 + TINY[table.dtype]


def embedding_grad(dout, ids, rows, scale, dtype, into=None):
    out = torch.zeros((rows, dout.shape[1]), dtype=torch.float64)
    mag, count = torch.zeros_like(out), torch.zeros((rows, 1), dtype=torch.float64)
    for t, i in enumerate(ids.tolist()):
        if 0 <= i < rows:
            out[i] += d(dout[t])
            mag[i] += d(dout[t]).abs()
            count[i] += 1
    out, mag = scale * out, abs(scale) * mag
    if into is not None:
        out, mag = out + d(into), mag + d(into).abs()
    return out, out.abs() * U[dtype] * 1.01 + mag * (count + 3) * U32 + TINY[dtype]


# ---------------------------------------------------------------------------
# residual norm
# ---------------------------------------------------------------------------
# Terms that one sum of a row or a mean adds up one after the other: 16 of a thread's
# own, 6 and 15 of the butterfly and the waves; and the products, root and quotient
# around it.
ROW = (16 + 6 + 15 + 8) * U32


def residual_norm(x, y, weight, post, gate, scale, eps, dn=None, dh=None):
    """{name: (value, bound)} of n, h and stats and, with dn, of all gradients."""
    X, W = d(x), d(weight)
    T, H = X.shape
    dt, rt = weight.dtype, x.dtype
    ry = torch.ones((T, 1), dtype=torch.float64)
    if y is None:
        h, mag = X, X.abs()
    else:
        Y = d(y)
        if post is not None:
            ry = (Y.square().mean(1, keepdim=True) + eps).rsqrt()
        yhat = Y * ry
        z = yhat * (d(post) if post is not None else 1.0)
        g = d(gate) if gate is not None else torch.ones((1, H), dtype=torch.float64)
        h = X + scale * g * z
        mag = X.abs() + (scale * g * z).abs()
    rh = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    # h is off by e_h; rh by half the share that the sum of squares is off by, and ROW
    e_h = (ROW + 4 * U32) * mag
    e_r = rh * ((h.abs() * e_h).mean(1, keepdim=True) * rh.square() + ROW)
    hhat = h * rh
    e_hat = e_h * rh + h.abs() * e_r + U32 * hhat.abs()
    n = hhat * W
    out = {"n": (n, U[dt] * n.abs() + W.abs() * (e_hat + 2 * U32 * hhat.abs()) + TINY[dt]),
           "h": (h, U[rt] * h.abs() + e_h + TINY[rt]),
           "stats": (torch.cat([rh, ry], 1), torch.cat([e_r, ROW * ry], 1) + U32 * torch.cat([rh, ry], 1))}
    if dn is None:
        return out
    D, dH0 = d(dn), d(dh) if dh is not None else torch.zeros_like(h)
    a = D * W
    c = (a * hhat).mean(1, keepdim=True)
    e_c = (a.abs() * (e_hat + (ROW + 2 * U32) * hhat.abs())).mean(1, keepdim=True)
    dH = dH0 + rh * (a - hhat * c)
    size = dH0.abs() + rh * (a.abs() + (hhat * c).abs())
    e_H = 6 * U32 * size + rh * (e_hat * c.abs() + hhat.abs() * e_c) + e_r * (a.abs() + (hhat * c).abs())
    out["dx"] = (dH, 1.01 * U[rt] * dH.abs() + 1.01 * e_H + TINY[rt])

    def column(value, size, e):
        return value.sum(0), 1.01 * e.sum(0) + (T + 4) * U32 * size.sum(0) + TINY[torch.float32]
    out["dweight"] = column(D * hhat, (D * hhat).abs(), D.abs() * e_hat)
    if y is None:
        return out
    dz, e_z = scale * dH, abs(scale) * (e_H + U32 * dH.abs())
    e_y = (ROW + U32) * yhat.abs() if post is not None else torch.zeros_like(yhat)
    e_zz = (e_y + U32 * yhat.abs()) * (d(post).abs() if post is not None else 1.0)
    if gate is not None:
        dg, e_g = dz * z, e_z * z.abs() + dz.abs() * (e_zz + 2 * U32 * z.abs())
        if gate.dim() == 1:
            out["dgate"] = column(dg, dg.abs(), e_g)
        else:
            out["dgate"] = (dg, 1.01 * (U[dt] * dg.abs() + e_g) + TINY[dt])
        dz, e_z = dz * g, (e_z + 2 * U32 * dz.abs()) * g.abs()
    if post is None:
        out["dy"] = (dz, 1.01 * (U[dt] * dz.abs() + e_z) + TINY[dt])
        return out
    P = d(post)
    out["dpost"] = column(dz * yhat, (dz * yhat).abs(), e_z * yhat.abs() + dz.abs() * e_y)
    a, e_a = dz * P, (e_z + U32 * dz.abs()) * P.abs()
    c = (a * yhat).mean(1, keepdim=True)
    e_c = (e_a * yhat.abs() + a.abs() * (e_y + (ROW + 2 * U32) * yhat.abs())).mean(1, keepdim=True)
    dy = ry * (a - yhat * c)
    e = ry * (e_a + yhat.abs() * e_c + e_y * c.abs()) + (ROW + 5 * U32) * ry * (a.abs() + (yhat * c).abs())
    out["dy"] = (dy, 1.01 * (U[dt] * dy.abs() + e) + TINY[dt])
    return out


# ---------------------------------------------------------------------------
# loss over a vocabulary
# ---------------------------------------------------------------------------
def vocab_loss(x, weight, targets, scale, dloss=None):
    """{name: (value, bound)} of loss and lse and, with dloss, dx and dweight.

    A logit is a sum of hidden exact products in fp32, off by (hidden + 2) U32 of the sum
    of their magnitudes at most; exp of an argument a is off by (|a| + 4) U32 of itself,
    and the sum over the vocabulary, of positive terms, by as much as its terms and 512
    U32 (2 x 128 in a lane, then tiles: far fewer than that one after the other).  d is
    rounded once to the inputs' type, and the results once."""
    T, (V, H) = x.shape[0], weight.shape
    dt = x.dtype
    kept = (targets >= 0) & (targets < V)
    X = torch.where(kept[:, None], d(x), 0.0)
    W = d(weight)
    z = scale * (X @ W.T)
    e_z = ((H + 2) * U32 * abs(scale) * (X.abs() @ W.abs().T) + 2 * U32 * z.abs()).amax(1)
    lse = torch.logsumexp(z, 1)
    at = targets.clamp(0, V - 1).long()[:, None]
    picked = z.gather(1, at)[:, 0]
    spread = (z.amax(1) - z.amin(1)).clamp(max=90.0)
    e_lse = e_z + (spread + 4 + 512) * U32 + 2 * U32 * lse.abs()
    out = {"lse": (torch.where(kept, lse, 0.0), torch.where(kept, e_lse, 0.0)),
           "loss": (torch.where(kept, lse - picked, 0.0),
                    torch.where(kept, e_lse + e_z + U32 * (lse - picked).abs(), 0.0))}
    if dloss is None:
        return out
    g = torch.where(kept, d(dloss), 0.0)[:, None] * scale
    p = (z - lse[:, None]).exp()
    D = p.clone()
    D.scatter_add_(1, at, torch.full((T, 1), -1.0, dtype=torch.float64))
    e_p = p * (e_z + e_lse + (spread + 4) * U32)[:, None] + U32 * D.abs()
    u = U[dt]
    # in fp16 the largest d is raised to 2^13 at least, so the smallest step, 2^-24, is
    # 2^-37 of it; in bf16 nothing is below its numbers
    small = 2.0 ** -37 * g.abs().max() if dt == torch.float16 else 0.0
    e_d = (u * D.abs() + e_p) * 1.01 * g.abs() + small
    D = D * g
    dx, dw = D @ W, D.T @ X
    # sums in fp32: hidden or tokens or vocabulary terms, at most (n + 8) U32 of their size
    out["dx"] = (dx, 1.01 * (u * dx.abs() + e_d @ W.abs() + (V + 8) * U32 * (D.abs() @ W.abs())) + TINY[dt])
    out["dx"] = (out["dx"][0], torch.where(kept[:, None], out["dx"][1], 0.0))
    out["dweight"] = (dw, 1.01 * (u * dw.abs() + e_d.T @ X.abs() + (T + 8) * U32 * (D.abs().T @ X.abs())) + TINY[dt])
    return out
