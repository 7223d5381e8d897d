"""The replayed layer of examples/replay_layer.py: its gradients against torch's in
64 bits, and the vote on its replicas."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

replay_layer = pytest.importorskip("replay_layer")


def _reference(L, x, positions, lens, dout, ids):
    """The layer in fp64 on the CPU, its gradients by torch; the choices are given."""
    names = ("wq", "wk", "wv", "wo", "we", "router")
    w = {n: getattr(L, n).cpu().double().requires_grad_() for n in names}
    x = x.cpu().double().requires_grad_()
    T, D, G = x.shape[0], L.dim, L.heads // L.kv_heads
    angle = positions.cpu().double()[:, None, None] * L.freqs.cpu()

    def turned(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)
    q = turned((x @ w["wq"]).view(T, L.heads, D))
    k = turned((x @ w["wk"]).view(T, L.kv_heads, D)).repeat_interleave(G, 1)
    v = (x @ w["wv"]).view(T, L.kv_heads, D).repeat_interleave(G, 1)
    parts, at = [], 0
    for n in lens:
        s = torch.matmul(q[at:at + n].transpose(0, 1), k[at:at + n].transpose(0, 1).transpose(1, 2)) * D ** -0.5
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), -torch.inf)
        parts.append(torch.matmul(s.softmax(-1), v[at:at + n].transpose(0, 1)).transpose(0, 1))
        at += n
    a = torch.cat(parts).reshape(T, -1) @ w["wo"] + x
    weights = (a.detach() @ w["router"]).gather(1, ids).softmax(1).detach().requires_grad_()
    out = a
    for i in range(L.top):
        y = torch.stack([a[t] @ w["we"][int(ids[t, i])] for t in range(T)])
        out = out + weights[:, i:i + 1] * y
    out.backward(dout.cpu().double())
    r = {"d" + n: w[n].grad for n in names if n != "router"}
    return dict(r, out=out.detach(), dx=x.grad, dweights=weights.grad)


def test_gradients():
    """A chain of bf16 products: each result is off by a few roundings of 2^-8 of its
    size; 16 of them, in the norm, leave room for the 14 roundings on the longest way."""
    L = replay_layer.Layer(hidden=64, heads=4, kv_heads=2, dim=32, experts=4, top=2)
    x, positions, lens, dout = replay_layer.inputs(L, [37, 1, 50])
    seen = {}
    sort = replay_layer.replay.expert_sort

    def keep(ids, n):
        seen["ids"] = ids
        return sort(ids, n)
    replay_layer.replay.expert_sort = keep
    try:
        got = replay_layer.step(L, x, positions, lens, dout)
    finally:
        replay_layer.replay.expert_sort = sort
    want = _reference(L, x, positions, lens, dout, seen["ids"].cpu().long())
    assert set(got) == set(want)
    for n in got:
        off = (got[n].cpu().double() - want[n]).norm() / want[n].norm()
        assert float(off) <= 16 * 2.0 ** -8, (n, float(off))


def test_vote():
    layers = [replay_layer.Layer(hidden=256, heads=4, kv_heads=2) for _ in range(3)]
    args = replay_layer.inputs(layers[0], [300, 1, 0, 211])
    results = [replay_layer.step(layer, *args) for layer in layers]
    assert replay_layer.vote(results) == ([], 0)
    layers[2].we.view(torch.int16)[3, 5, 7] ^= 1 << 6
    where, undecided = replay_layer.vote(results[:2] + [replay_layer.step(layers[2], *args)])
    assert undecided == 0 and {replica for replica, _ in where} == {2}
    assert (2, "out") in where and (2, "dwe") not in where      # dwe does not read we
