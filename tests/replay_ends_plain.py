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
