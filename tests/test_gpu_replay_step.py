"""The replayed training step of examples/replay_step.py: its losses and gradients against
torch's in 64 bits, and the vote on its replicas."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

replay_step = pytest.importorskip("replay_step")


def _reference(M, ids, targets, positions, lens):
    """The step in fp64 on the CPU, its gradients by torch."""
    w = {"embed": M.embed, "norm0": M.norm0}
    for i, layer in enumerate(M.layer):
        w |= {f"{i}.{n}": t for n, t in layer.items()}
    w = {n: t.cpu().double().requires_grad_() for n, t in w.items()}
    T, D, G = ids.shape[0], M.dim, M.heads // M.kv_heads
    ids, targets = ids.cpu(), targets.cpu()
    angle = positions.cpu().double()[:, None, None] * M.freqs.cpu()

    def turned(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    def normed(a):
        return a * (a.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    h = M.scale * w["embed"][ids]
    n = w["norm0"] * normed(h)
    for i in range(M.layers):
        p = {name: w[f"{i}.{name}"] for name in M.WEIGHTS}
        q = turned((n @ p["wq"]).view(T, M.heads, D))
        k = turned((n @ p["wk"]).view(T, M.kv_heads, D)).repeat_interleave(G, 1)
        v = (n @ p["wv"]).view(T, M.kv_heads, D).repeat_interleave(G, 1)
        parts, at = [], 0
        for m in lens:
            s = torch.matmul(q[at:at + m].transpose(0, 1), k[at:at + m].transpose(0, 1).transpose(1, 2)) * D ** -0.5
            s = s.masked_fill(torch.ones(m, m).triu(1).bool(), -torch.inf)
            parts.append(torch.matmul(s.softmax(-1), v[at:at + m].transpose(0, 1)).transpose(0, 1))
            at += m
        y = torch.cat(parts).reshape(T, -1) @ p["wo"]
        h = h + p["gate"] * (p["post"] * normed(y))
        u = (p["norm1"] * normed(h)) @ p["w1"]
        h = h + 0.5 * (u.clamp(min=0) @ p["w2"])
        n = p["norm2"] * normed(h)
    z = n @ w["embed"].t()
    kept = targets >= 0
    loss = torch.where(kept, torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    (loss.sum() / kept.sum()).backward()
    return dict({n: t.grad for n, t in w.items()}, loss=loss.detach())


def test_losses_and_gradients():
    """A chain of bf16 results: on the longest way, in the first layer's weights, some 30 of
    them are rounded by 2^-8 of their size at most; 32 in the norm."""
    M = replay_step.Model(vocab=300, hidden=64, layers=2, heads=4, kv_heads=2, dim=16, inner=96)
    args = replay_step.inputs(M, [37, 1, 50])
    got, want = replay_step.step(M, *args), _reference(M, *args)
    assert set(got) == set(want)
    for n in got:
        off = (got[n].cpu().double() - want[n]).norm() / want[n].norm()
        assert float(off) <= 32 * 2.0 ** -8, (n, float(off))


def test_vote():
    models = [replay_step.Model(vocab=500, hidden=128, heads=2, kv_heads=1)]
    models += [models[0].copy() for _ in range(2)]
    args = replay_step.inputs(models[0], [200, 1, 0, 99])
    results = [replay_step.step(m, *args) for m in models]
    assert replay_step.vote(results) == ([], 0)
    models[2].layer[1]["norm2"].view(torch.int16)[5] ^= 1 << 6
    where, undecided = replay_step.vote(results[:2] + [replay_step.step(models[2], *args)])
    assert undecided == 0 and {replica for replica, _ in where} == {2}
    assert (2, "loss") in where and (2, "0.wq") in where
