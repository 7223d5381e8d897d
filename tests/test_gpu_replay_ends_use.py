"""The embedding, the residual norm and the vocabulary loss as programs use them: on
streams, captured into graphs, inside autograd functions, in large memory; and what the
binding refuses."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF16 = torch.bfloat16


def _inputs(seed, T=300, H=136, V=700):
    g = torch.Generator().manual_seed(seed)

    def randn(*shape, sigma=1.0):
        return (torch.randn(shape, generator=g) * sigma).to(BF16).to(DEV)
    ids = torch.randint(0, V, (T,), generator=g)
    ids[torch.rand((T,), generator=g) < 0.2] = -1
    return dict(ids=ids.to(DEV), table=randn(V, H, sigma=H ** -0.5), y=randn(T, H), weight=randn(H), post=randn(H),
                gate=randn(T, H), dloss=torch.rand((T,), generator=g).to(DEV), targets=ids.roll(1).to(DEV))


def _run(v, stream=None):
    """All six, one on the results of the other."""
    T, V = v["ids"].numel(), v["table"].shape[0]
    how = dict(post=v["post"], gate=v["gate"], scale=0.5)
    x = replay.embedding(v["ids"], v["table"], scale=4.0, stream=stream)
    n, h, stats = replay.residual_norm(x, v["y"], v["weight"], stream=stream, **how)
    loss, lse = replay.vocab_loss(n, v["table"], v["targets"], stream=stream)
    dn, dw = replay.vocab_loss_grad(v["dloss"], n, v["table"], v["targets"], lse, stream=stream)
    g = replay.residual_norm_grad(dn, h, x, v["y"], v["weight"], stats, stream=stream, **how)
    apart = replay.embedding_grad(g.dx, v["ids"], V, scale=4.0, stream=stream)
    replay.embedding_grad(g.dx, v["ids"], V, scale=4.0, dtable=dw, accumulate=True, stream=stream)
    return [x, n, h, stats, loss, lse, dn, dw, apart, *g]


@pytest.mark.parametrize("T", [5, 300, 5000])
def test_captured(T):
    """Replays on new inputs, with eager calls and synchronizations between them."""
    print("CASE", T, flush=True)
    v = _inputs(1, T)
    _run(v)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _run(v)
    w = _inputs(2, T)
    with torch.cuda.graph(other):       # a second graph beside it
        got_w = _run(w)
    for seed in (3, 4, 5):
        new = _inputs(seed, T)
        for n in v:
            v[n].copy_(new[n])
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        want = _run(new)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(got_w, _run(w)))


def test_streams():
    """Calls on a stream that is not the current one, two at a time."""
    v, w = _inputs(6), _inputs(7)
    want = _run(v), _run(w)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got = [_run(u, stream=s) for u, s in zip((v, w), streams)]
        for s in streams:
            s.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


class _Loss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets):
        loss, lse = replay.vocab_loss(x, weight, targets)
        ctx.save_for_backward(x, weight, targets, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        x, weight, targets, lse = ctx.saved_tensors
        return *replay.vocab_loss_grad(dloss, x, weight, targets, lse), None


def test_in_an_autograd_function():
    """The gradient that torch hands over for a mean is one number expanded."""
    v = _inputs(8)
    x, weight = v["y"].clone().requires_grad_(), v["table"].clone().requires_grad_()
    _Loss.apply(x, weight, v["targets"]).mean().backward()
    loss, lse = replay.vocab_loss(v["y"], v["table"], v["targets"])
    dloss = torch.full_like(loss, 1.0 / loss.numel())
    dx, dw = replay.vocab_loss_grad(dloss, v["y"], v["table"], v["targets"], lse)
    assert torch.equal(x.grad, dx) and torch.equal(weight.grad, dw)


def test_large_tables():
    """Offsets past 32 bits: 600,000 rows of 4,096 are 4.9 GB."""
    V, H, T = 600_000, 4096, 70
    g = torch.Generator(device=DEV).manual_seed(9)
    table = torch.empty((V, H), dtype=BF16, device=DEV)
    for part in table.split(100_000):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV, dtype=torch.float32) * H ** -0.5)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    ids[:6] = torch.tensor([V - 1, V - 1, 0, V - 2, V // 2, 1], device=DEV)
    assert torch.equal(replay.embedding(ids, table), table[ids])
    dout = torch.randn((T, H), generator=g, device=DEV).to(BF16)
    grad = replay.embedding_grad(dout, ids, V)
    rows = ids.unique()
    for r in rows.tolist():
        want = dout[ids == r].double().sum(0)
        assert float((grad[r].double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-6
    assert int((grad.view(torch.int16) != 0).any(1).sum()) == rows.numel()
    del grad
    x = (torch.randn((T, H), generator=g, device=DEV) + 5 * table[ids].float()).to(BF16)
    for n in (5, T):
        print("CASE", n, flush=True)
        loss, lse = replay.vocab_loss(x[:n], table, ids[:n])
        dloss = torch.ones((n,), device=DEV)
        dx, dw = replay.vocab_loss_grad(dloss, x[:n], table, ids[:n], lse)
        z = torch.cat([torch.mm(x[:n].float(), part.float().t()) for part in table.split(100_000)], 1).double()
        want = torch.logsumexp(z, 1)
        assert float((lse.double() - want).abs().max()) <= 2e-5 * float(want.abs().max())
        p = (z - want[:, None]).exp()
        p[torch.arange(n, device=DEV), ids[:n]] -= 1
        # d is rounded once and the result once: half a step of bf16 each of the sum of sizes
        for r in (0, 1, V // 2, V - 2, V - 1):
            size = (p[:, r, None].abs() * x[:n].double().abs()).sum(0)
            off = (dw[r].double() - (p[:, r, None] * x[:n].double()).sum(0)).abs()
            assert bool((off <= 2.1 * 2.0 ** -8 * size + 1e-6).all()), r
        want_dx = sum(torch.mm(q.float(), part.float()) for q, part in zip(p.split(100_000, 1), table.split(100_000)))
        off = (dx.double() - want_dx.double()).norm() / want_dx.double().norm()
        assert float(off) <= 2 * 2.0 ** -8
        del z, p, dw


def test_many_tokens():
    """dx and d past 2^31 elements of offset: 70,000 tokens, d of 7,600 rows a piece."""
    T, H, V = 70_000, 64, 8000
    g = torch.Generator(device=DEV).manual_seed(10)
    weight = (torch.randn((V, H), generator=g, device=DEV) * H ** -0.5).to(BF16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    x = torch.randn((T, H), generator=g, device=DEV).to(BF16)
    loss, lse = replay.vocab_loss(x, weight, targets)
    dx, dw = replay.vocab_loss_grad(torch.full((T,), 1.0, device=DEV), x, weight, targets, lse)
    at = torch.tensor([0, 1, T // 2, T - 2, T - 1], device=DEV)
    z = torch.mm(x[at].double(), weight.double().t())
    want = torch.logsumexp(z, 1)
    assert float((lse[at].double() - want).abs().max()) <= 2e-5 * float(want.abs().max())
    p = (z - want[:, None]).exp()
    p[torch.arange(5, device=DEV), targets[at]] -= 1
    want = torch.mm(p, weight.double())
    assert float((dx[at].double() - want).norm() / want.norm()) <= 2 * 2.0 ** -8
    # every token's softmax sums to one less its target's one: over all rows dweight sums to 0
    total = dw.double().sum(0)
    size = dw.double().abs().sum(0)
    assert bool((total.abs() <= 2.0 ** -8 * size).all())


def test_most_tokens_of_a_loss():
    """2^24 workgroups of 256 threads for the rows that take part: more than one launch
    dimension holds.  Logits of 8 products: bounds as in replay_ends_plain, |z| below 64."""
    T, H, V = (1 << 26) - 1, 8, 5
    print("CASE", T, H, V, flush=True)
    g = torch.Generator(device=DEV).manual_seed(13)
    x = torch.randn((T, H), generator=g, device=DEV, dtype=BF16)
    weight = torch.randn((V, H), generator=g, device=DEV, dtype=BF16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    targets[5:9] = -1
    loss, lse = replay.vocab_loss(x, weight, targets)
    at = torch.cat((torch.arange(0, 12, device=DEV), torch.arange(T // 2, T // 2 + 12, device=DEV),
                    torch.arange(T - 12, T, device=DEV)))
    z = torch.mm(x[at].double(), weight.double().t())
    assert float(z.abs().max()) < 64
    kept = targets[at] >= 0
    want = torch.where(kept, torch.logsumexp(z, 1), 0.0)
    picked = torch.where(kept, z.gather(1, targets[at].long().clamp(min=0)[:, None])[:, 0], 0.0)
    # a logit is off by (8 + 8) 2^-24 of 8 products below 64 in all, exp's argument by as much
    bound = 4 * 16 * 64 * 2.0 ** -24
    assert float((lse[at].double() - want).abs().max()) <= bound
    assert float((loss[at].double() - (want - picked)).abs().max()) <= bound


def test_refusals():
    v = _inputs(11)
    T, H = v["y"].shape

    def refuse(call):
        with pytest.raises(replay.C3Error):
            call()
    e, r, loss = replay.embedding, replay.residual_norm, replay.vocab_loss
    refuse(lambda: e(v["ids"].float(), v["table"]))
    refuse(lambda: e(v["ids"][None], v["table"]))
    refuse(lambda: e(v["ids"].cpu(), v["table"]))
    refuse(lambda: e(v["ids"], v["table"].double()))
    refuse(lambda: e(v["ids"], v["table"].t()))
    refuse(lambda: e(v["ids"], v["table"].clone().requires_grad_()))
    refuse(lambda: e(v["ids"], v["table"], scale=float("inf")))
    refuse(lambda: e(v["ids"], v["table"], scale="two"))
    refuse(lambda: e(v["ids"], v["table"][:0]))
    refuse(lambda: e(v["ids"], v["table"], out=v["table"][:T]))
    refuse(lambda: e(v["ids"], v["table"], out=torch.empty((T, H + 1), dtype=BF16, device=DEV)))
    refuse(lambda: replay.embedding_grad(v["y"], v["ids"][1:], 700))
    refuse(lambda: replay.embedding_grad(v["y"], v["ids"], 0))
    refuse(lambda: replay.embedding_grad(v["y"], v["ids"], 2.5))
    refuse(lambda: replay.embedding_grad(v["y"], v["ids"], 700, accumulate=True))
    refuse(lambda: replay.embedding_grad(v["y"], v["ids"], 700, dtype=torch.float16))
    refuse(lambda: replay.embedding_grad(v["y"], v["ids"], 700, workspace=torch.empty(8, device=DEV)))
    refuse(lambda: r(v["y"], None, v["weight"][1:]))
    refuse(lambda: r(v["y"], v["y"][1:], v["weight"]))
    refuse(lambda: r(v["y"].half(), v["y"], v["weight"]))
    refuse(lambda: r(v["y"], None, v["weight"], post=v["post"]))
    refuse(lambda: r(v["y"], v["y"], v["weight"], gate=v["gate"][:, :1]))
    refuse(lambda: r(v["y"], v["y"], v["weight"], gate=v["gate"][:1]))
    refuse(lambda: r(v["y"], v["y"], v["weight"], eps=-1.0))
    refuse(lambda: r(v["y"], v["gate"], v["weight"], n=v["gate"]))
    refuse(lambda: r(v["y"], None, v["weight"], h=v["gate"]))
    wide = torch.zeros((2, 16400), dtype=BF16, device=DEV)
    refuse(lambda: r(wide, None, wide[0]))
    n, h, stats = r(v["y"], v["gate"], v["weight"])
    g = replay.residual_norm_grad
    refuse(lambda: g(v["y"], None, v["y"], v["gate"], v["weight"], stats[1:]))
    refuse(lambda: g(None, None, v["y"], v["gate"], v["weight"], stats))
    refuse(lambda: g(v["y"], None, v["y"], None, v["weight"], stats, dy=v["gate"]))
    refuse(lambda: g(v["y"], None, v["y"], v["gate"], v["weight"], stats, dgate=torch.empty_like(v["y"])))
    refuse(lambda: loss(v["y"].float(), v["table"].float(), v["targets"]))
    refuse(lambda: loss(v["y"], v["table"].half(), v["targets"]))
    refuse(lambda: loss(v["y"][:, :60], v["table"][:, :60], v["targets"]))      # no multiple of 8
    refuse(lambda: loss(v["y"], v["table"][:, :128], v["targets"]))
    refuse(lambda: loss(v["y"], v["table"], v["targets"][1:]))
    refuse(lambda: loss(v["y"][:, 4:132], v["table"][:, 4:132], v["targets"]))  # not on 16 bytes
    refuse(lambda: loss(v["y"], v["table"], v["targets"], loss=torch.empty((T,), device=DEV, dtype=torch.float64)))
    one, lse = loss(v["y"], v["table"], v["targets"])
    lg = replay.vocab_loss_grad
    refuse(lambda: lg(v["dloss"].double(), v["y"], v["table"], v["targets"], lse))
    refuse(lambda: lg(v["dloss"][0], v["y"], v["table"], v["targets"], lse))
    refuse(lambda: lg(v["dloss"], v["y"], v["table"], v["targets"], None))
    refuse(lambda: lg(v["dloss"], v["y"], v["table"], v["targets"], lse, dx=v["y"]))
    refuse(lambda: lg(v["dloss"], v["y"], v["table"], v["targets"], lse, dweight=v["table"]))
    refuse(lambda: lg(v["dloss"].clone().requires_grad_(), v["y"], v["table"], v["targets"], lse))


def test_what_the_loss_refuses_it_names():
    v = _inputs(12)
    y, table, targets = v["y"], v["table"], v["targets"]
    lse = torch.zeros((len(y),), device=DEV)
    for call in (lambda a, b: replay.vocab_loss(a, b, targets),
                 lambda a, b: replay.vocab_loss_grad(v["dloss"], a, b, targets, lse)):
        with pytest.raises(replay.C3Error, match="bf16 or fp16"):
            call(y.float(), table.float())
        with pytest.raises(replay.C3Error, match="multiple of 8"):
            call(y[:, :60], table[:, :60])
        with pytest.raises(replay.C3Error, match="same hidden size"):
            call(y, table[:, :128])
