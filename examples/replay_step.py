"""A training step of a small language model replayed on every replica, and a vote on it.

Tokens come in through an embedding, blocks of attention and of a gated product are
joined to a residual stream with norms before and after them, and the loss goes over the
vocabulary with the embedding's own rows as output weights.  All of it, forward and
backward, runs through operators of ``paper_2608_11034_amd.replay`` and library matrix
products, so equal replicas give equal losses and gradients bit by bit, and exact C3
names the replica and the tensors where one differs.

    python examples/replay_step.py          # one bit of one replica's embedding flipped
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for path in (ROOT, os.path.join(ROOT, "examples")):
    sys.path.insert(0, path)

from paper_2608_11034_amd import replay  # noqa: E402
from replay_layer import vote  # noqa: E402


class Model:
    """Sizes and bf16 weights: ``layers`` layers of ``heads`` query heads of ``dim`` that
    share ``kv_heads`` key heads, each followed by a product of width ``inner`` and back."""

    WEIGHTS = ("wq", "wk", "wv", "wo", "w1", "w2", "norm1", "norm2", "post", "gate")

    def __init__(self, vocab=1000, hidden=256, layers=2, heads=4, kv_heads=2, dim=64, inner=512, seed=1, device="cuda"):
        self.vocab, self.hidden, self.layers = vocab, hidden, layers
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.scale = hidden ** 0.5
        gen = torch.Generator().manual_seed(seed)

        def weight(*shape, sigma=None, mean=0.0):
            sigma = shape[-2] ** -0.5 if sigma is None else sigma
            return (torch.randn(shape, generator=gen) * sigma + mean).to(torch.bfloat16).to(device)
        self.embed = weight(vocab, hidden, sigma=hidden ** -0.5)
        self.norm0 = weight(hidden, sigma=0.1, mean=1.0)
        self.layer = [dict(wq=weight(hidden, heads * dim), wk=weight(hidden, kv_heads * dim),
                           wv=weight(hidden, kv_heads * dim), wo=weight(heads * dim, hidden),
                           w1=weight(hidden, inner), w2=weight(inner, hidden),
                           norm1=weight(hidden, sigma=0.1, mean=1.0), norm2=weight(hidden, sigma=0.1, mean=1.0),
                           post=weight(hidden, sigma=0.1, mean=1.0), gate=weight(hidden, sigma=0.1, mean=0.7))
                      for _ in range(layers)]
        self.freqs = replay.rotary_frequencies(dim, device=device)

    def copy(self):
        other = object.__new__(Model)
        other.__dict__ = dict(vars(self))
        for name in ("embed", "norm0", "freqs"):
            setattr(other, name, getattr(self, name).clone())
        other.layer = [{n: t.clone() for n, t in w.items()} for w in self.layer]
        return other


def step(model, ids, targets, positions, lens):
    """Forward and backward of packed sequences of ``lens`` tokens; the loss is the mean
    over the tokens that have a target.  Returns a dict of the losses and all gradients."""
    M, T = model, ids.shape[0]
    how = dict(causal=True, q_lens=lens, k_lens=lens)
    x = replay.embedding(ids, M.embed, scale=M.scale)
    n, h, stats = replay.residual_norm(x, None, M.norm0)
    kept = []                           # what the way back needs
    for w in M.layer:
        q0, k0 = torch.mm(n, w["wq"]).view(T, M.heads, M.dim), torch.mm(n, w["wk"]).view(T, M.kv_heads, M.dim)
        v = torch.mm(n, w["wv"]).view(T, M.kv_heads, M.dim)
        q, k = replay.rotary((q0, k0), positions, M.freqs)
        o, lse = replay.attention(q, k, v, **how)
        y1 = torch.mm(o.view(T, -1), w["wo"])
        n1, h1, stats1 = replay.residual_norm(h, y1, w["norm1"], post=w["post"], gate=w["gate"])
        u = torch.mm(n1, w["w1"])
        r = u.clamp(min=0)
        y2 = torch.mm(r, w["w2"])
        n2, h2, stats2 = replay.residual_norm(h1, y2, w["norm2"], scale=0.5)
        kept.append((n, h, q, k, v, o, lse, y1, n1, h1, stats1, u, r, y2, stats2))
        n, h = n2, h2
    loss, lse_v = replay.vocab_loss(n, M.embed, targets)

    # and back
    counts = ((targets >= 0) & (targets < M.vocab)).sum()
    dloss = (1.0 / counts.float()).expand(T)
    dn, dembed = replay.vocab_loss_grad(dloss, n, M.embed, targets, lse_v)
    grads, dh = {}, None
    for i in reversed(range(M.layers)):
        w = M.layer[i]
        n, h, q, k, v, o, lse, y1, n1, h1, stats1, u, r, y2, stats2 = kept[i]
        g2 = replay.residual_norm_grad(dn, dh, h1, y2, w["norm2"], stats2, scale=0.5)
        dr = torch.mm(g2.dy, w["w2"].t())
        du = torch.where(u > 0, dr, torch.zeros_like(dr))
        g1 = replay.residual_norm_grad(torch.mm(du, w["w1"].t()), g2.dx, h, y1, w["norm1"], stats1, post=w["post"],
                                       gate=w["gate"])
        do = torch.mm(g1.dy, w["wo"].t()).view(T, M.heads, M.dim)
        dq, dk, dv = replay.attention_grad(do, q, k, v, o, lse, **how)
        dq, dk = (t.view(T, -1) for t in replay.rotary((dq, dk), positions, M.freqs, inverse=True))
        dv, dh = dv.view(T, -1), g1.dx
        dn = torch.mm(dq, w["wq"].t()) + torch.mm(dk, w["wk"].t()) + torch.mm(dv, w["wv"].t())
        grads |= {f"{i}.{name}": t for name, t in dict(
            wq=torch.mm(n.t(), dq), wk=torch.mm(n.t(), dk), wv=torch.mm(n.t(), dv),
            wo=torch.mm(o.view(T, -1).t(), g1.dy), w1=torch.mm(n1.t(), du), w2=torch.mm(r.t(), g2.dy),
            norm1=g1.dweight, norm2=g2.dweight, post=g1.dpost, gate=g1.dgate).items()}
    g0 = replay.residual_norm_grad(dn, dh, x, None, M.norm0, stats)
    # the embedding's rows are the output's weights too: one gradient for both
    replay.embedding_grad(g0.dx, ids, M.vocab, scale=M.scale, dtable=dembed, accumulate=True)
    return dict(grads, loss=loss, norm0=g0.dweight, embed=dembed)


def inputs(model, lens, seed=2, device="cuda"):
    """Tokens, the next token of each as its target (none for the last of a sequence) and
    positions."""
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, model.vocab, (sum(lens),), generator=gen)
    targets, at = torch.cat([ids[1:], ids[:1]]), 0
    for n in lens:
        at += n
        if n:
            targets[at - 1] = -100
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens])
    return ids.to(device), targets.to(device), positions.to(device), lens


def main():
    models = [Model()]
    models += [models[0].copy() for _ in range(2)]
    args = inputs(models[0], [300, 1, 211])
    print("equal replicas:", vote([step(m, *args) for m in models]))
    models[1].embed.view(torch.int16)[7, 9] ^= 1 << 6       # one bit of one replica's embedding
    where, undecided = vote([step(m, *args) for m in models])
    print("one bit flipped on replica 1:", where, "undecided:", undecided)
    assert {replica for replica, _ in where} == {1} and undecided == 0


if __name__ == "__main__":
    main()
