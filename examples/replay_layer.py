"""A transformer layer replayed on every replica, and a vote on what it gives.

Each replica runs the same layer forward and backward on the same packed
sequences: projections, rotary positions, attention, a router that sends tokens
to experts, and all their gradients, with the operators of
``paper_2608_11034_amd.replay`` between library matrix products.  Operators whose
bits depend on their inputs alone make equal replicas equal bit by bit, so exact
C3 (``c3.check``) on outputs and gradients names the replica that differs and the
chunks where it does.

    python examples/replay_layer.py          # one bit of one replica's weights flipped
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_11034_amd import c3, replay  # noqa: E402

CHUNK_BYTES = 65536


class Layer:
    """Sizes and weights of one layer: bf16, ``heads`` query heads of ``dim`` that share
    ``kv_heads`` key heads, ``experts`` experts of one product each, ``top`` a token."""

    def __init__(self, hidden=512, heads=8, kv_heads=2, dim=64, experts=8, top=2, seed=1, device="cuda"):
        self.hidden, self.heads, self.kv_heads, self.dim = hidden, heads, kv_heads, dim
        self.experts, self.top = experts, top
        gen = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen) * shape[-2] ** -0.5).to(torch.bfloat16).to(device)
        self.wq, self.wo = weight(hidden, heads * dim), weight(heads * dim, hidden)
        self.wk, self.wv = weight(hidden, kv_heads * dim), weight(hidden, kv_heads * dim)
        self.router = weight(hidden, experts)
        self.we = weight(experts, hidden, hidden)
        self.freqs = replay.rotary_frequencies(dim, device=device)

    def copy(self):
        other = object.__new__(Layer)
        other.__dict__ = {n: x.clone() if isinstance(x, torch.Tensor) else x for n, x in vars(self).items()}
        return other


def _runs(order):
    """(expert, first, end) of the sorted rows, on the host."""
    at = order.offsets.tolist()
    return [(e, a, b) for e, (a, b) in enumerate(zip(at, at[1:])) if b > a]


def step(layer, x, positions, lens, dout):
    """Forward and backward of packed tokens x [tokens, hidden] of sequences of ``lens``
    tokens each, for the output's gradient ``dout``.  Returns a dict of tensors: the
    output, the gradients of x and of every weight but the router's (the choices are
    taken as given)."""
    L, T = layer, x.shape[0]
    how = dict(causal=True, q_lens=lens, k_lens=lens)
    # attention
    q0 = torch.mm(x, L.wq).view(T, L.heads, L.dim)
    k0 = torch.mm(x, L.wk).view(T, L.kv_heads, L.dim)
    v = torch.mm(x, L.wv).view(T, L.kv_heads, L.dim)
    q, k = replay.rotary((q0, k0), positions, L.freqs)
    o, lse = replay.attention(q, k, v, **how)
    a = torch.mm(o.view(T, -1), L.wo) + x
    # experts
    top = torch.mm(a, L.router).float().topk(L.top, dim=1)
    weights = top.values.softmax(1)
    order = replay.expert_sort(top.indices.to(torch.int32), L.experts)
    xs = replay.expert_dispatch(a, order)
    ys = torch.zeros_like(xs)
    for e, i, j in _runs(order):
        torch.mm(xs[i:j], L.we[e], out=ys[i:j])
    out = replay.expert_combine(ys, order, weights) + a

    # and back
    dys, dweights = replay.expert_combine_grad(dout, ys, order, weights)
    dxs, dwe = torch.zeros_like(xs), torch.zeros_like(L.we)
    for e, i, j in _runs(order):
        torch.mm(dys[i:j], L.we[e].t(), out=dxs[i:j])
        torch.mm(xs[i:j].t(), dys[i:j], out=dwe[e])
    da = replay.expert_dispatch_grad(dxs, order) + dout
    do = torch.mm(da, L.wo.t()).view(T, L.heads, L.dim)
    dq, dk, dv = replay.attention_grad(do, q, k, v, o, lse, **how)
    dq0, dk0 = replay.rotary((dq, dk), positions, L.freqs, inverse=True)
    dq0, dk0, dv = (t.view(T, -1) for t in (dq0, dk0, dv))
    dx = da + torch.mm(dq0, L.wq.t()) + torch.mm(dk0, L.wk.t()) + torch.mm(dv, L.wv.t())
    return dict(out=out, dx=dx, dweights=dweights, dwq=torch.mm(x.t(), dq0), dwk=torch.mm(x.t(), dk0),
                dwv=torch.mm(x.t(), dv), dwo=torch.mm(o.view(T, -1).t(), da), dwe=dwe)


def vote(results, chunk_bytes=CHUNK_BYTES):
    """Exact C3 on the results of all replicas: (outliers as replica and tensor name,
    number of undecided chunks)."""
    names = list(results[0])
    replicas = [[r[n].contiguous() for n in names] for r in results]
    plan = c3.SignaturePlan(replicas, chunk_bytes)
    outs = plan.new_check_outputs()
    ws = torch.empty((plan.check_workspace_size(),), dtype=torch.uint8, device=plan.device)
    plan.run_check(outs, ws)
    torch.cuda.synchronize()
    first, chunks = [], 0
    for t in replicas[0]:               # chunks do not cross tensors
        first.append(chunks)
        chunks += -(-t.numel() * t.element_size() // chunk_bytes)
    found = c3.outliers_numpy(outs[4], outs[6])
    where = [(int(o["replica"]), names[max(i for i, f in enumerate(first) if f <= int(o["chunk"]))]) for o in found]
    return sorted(set(where)), int(outs[6][1])


def inputs(layer, lens, seed=2, device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lens)
    x, dout = (torch.randn((T, layer.hidden), generator=gen).to(torch.bfloat16).to(device) for _ in range(2))
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(device)
    return x, positions, lens, dout


def main():
    layers = [Layer() for _ in range(3)]
    args = inputs(layers[0], [700, 1, 323])
    print("equal replicas:", vote([step(layer, *args) for layer in layers]))
    layers[1].wv.view(torch.int16)[7, 9] ^= 1 << 6      # one bit of one replica's weights
    where, undecided = vote([step(layer, *args) for layer in layers])
    print("one bit flipped on replica 1:", where, "undecided:", undecided)
    assert {replica for replica, _ in where} == {1} and undecided == 0


if __name__ == "__main__":
    main()
