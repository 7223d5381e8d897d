"""The operators at the ends of a replayed model and between its blocks, and how
their speed is measured.

A replayed training step needs, beside the layer's own operators, the way of
tokens into the model, what joins its blocks, and the loss: the embedding and its
gradient, the residual sum with the norms around a block and its gradient, and
the softmax cross entropy over a vocabulary, from the last hidden states and the
output weights, with its gradient.

A case is one pass through one of them.  With ``own`` false ``run`` computes it
in plain torch operations in 32 bits, with ``own`` true through
``paper_2608_11034_amd.replay``.  ``exact`` computes the same in 64 bits from the
definitions.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda"
MOST_LOSS = 8192 * 4096 * 131072        # tokens x hidden x rows of the largest case


def listed():
    return [
        # one new token of each of 16 sequences, a 4096-wide model: all latency
        dict(name="embedding_tokens", kind="embedding", dtype="bf16", tokens=16, rows=32000, hidden=4096,
             scale=1.0, padded=0.0),
        # an odd number of packed tokens in fp32, scaled by the root of the
        # width, some of them padding
        dict(name="embedding_packed", kind="embedding", dtype="f32", tokens=8191, rows=50001, hidden=2048,
             scale=2048 ** 0.5, padded=0.1),
        # the gradient of a micro-batch of 4 x 4096 tokens: frequent tokens
        # many times over, most rows not at all
        dict(name="embedding_grad_batch", kind="embedding_grad", dtype="bf16", tokens=16384, rows=32000,
             hidden=4096, scale=1.0, padded=0.0, sum="bf16"),
        # fp16 gradients summed into fp32 rows, an odd width, a large vocabulary
        # and padding
        dict(name="embedding_grad_wide", kind="embedding_grad", dtype="f16", tokens=4095, rows=131072,
             hidden=1000, scale=1000 ** 0.5, padded=0.2, sum="f32"),
        # the sum and the norm before a block for 8 new tokens: latency
        dict(name="norm_tokens", kind="norm", dtype="bf16", residual="bf16", tokens=8, hidden=4096,
             block=True, post=False, gate="none", scale=1.0),
        # the same for a micro-batch
        dict(name="norm_batch", kind="norm", dtype="bf16", residual="bf16", tokens=16384, hidden=4096,
             block=True, post=False, gate="none", scale=1.0),
        # forward and gradient of norms before and after a block, a gate for
        # every channel, an fp32 residual, an odd number of tokens
        dict(name="norm_grad_gated", kind="norm_grad", dtype="f16", residual="f32", tokens=8191, hidden=2048,
             block=True, post=True, gate="channels", scale=0.5),
        # forward and gradient of norm_batch: one training step's worth
        dict(name="norm_grad_batch", kind="norm_grad", dtype="bf16", residual="bf16", tokens=16384,
             hidden=4096, block=True, post=False, gate="none", scale=1.0),
        # the log-probability of one token of each of 8 sequences: the
        # weights are read once for few rows
        dict(name="loss_tokens", kind="loss", dtype="bf16", tokens=8, hidden=4096, rows=32000, ignored=0.0),
        # scoring an odd number of packed tokens over an odd vocabulary, fp16
        dict(name="loss_packed", kind="loss", dtype="f16", tokens=2047, hidden=2048, rows=50001, ignored=0.0),
        # forward and gradient of a short batch, prompts left out of the loss
        dict(name="loss_grad_short", kind="loss_grad", dtype="f16", tokens=333, hidden=1000, rows=32000,
             ignored=0.3),
        # forward and gradient of a micro-batch of 2 x 4096 tokens over a large
        # vocabulary, the largest
        dict(name="loss_grad_batch", kind="loss_grad", dtype="bf16", tokens=8192, hidden=4096, rows=131072,
             ignored=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["embedding", "embedding_grad", "norm", "norm_grad", "loss", "loss_grad", "loss_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("embedding", "embedding_grad"):
        hidden = rng.choice([512, 1000, 2048, 2048, 4096, 4097])
        case = dict(kind=kind, dtype=dtype, tokens=_log(rng, 1, min(65536, 2 ** 27 // hidden)),
                    rows=_log(rng, 1000, min(262144, 2 ** 29 // hidden)), hidden=hidden,
                    scale=rng.choice([1.0, 1.0, hidden ** 0.5]), padded=rng.choice([0.0, 0.0, 0.1, 0.5]))
        if kind == "embedding_grad":
            case["sum"] = rng.choice([dtype, dtype, "f32"])
        return case
    if kind in ("norm", "norm_grad"):
        hidden = rng.choice([512, 1000, 2048, 4096, 4096, 4100, 8192])
        case = dict(kind=kind, dtype=dtype, residual=rng.choice([dtype, dtype, "f32"]),
                    tokens=_log(rng, 1, 2 ** 26 // hidden), hidden=hidden, block=rng.random() < 0.85,
                    post=False, gate="none", scale=1.0)
        if case["block"]:
            case |= dict(post=rng.random() < 0.4, gate=rng.choice(["none", "none", "channels", "tokens"]),
                         scale=rng.choice([1.0, 1.0, 0.25]))
        return case
    hidden = rng.choice([512, 1000, 2048, 2048, 4096])
    rows = _log(rng, 1000, 131072)
    return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16"]),
                tokens=_log(rng, 1, min(16384, MOST_LOSS // 4 // hidden // rows)), hidden=hidden, rows=rows,
                ignored=rng.choice([0.0, 0.0, 0.25, 0.75]))


# ---------------------------------------------------------------------------
# prepare: what the program has in hand before the call
# ---------------------------------------------------------------------------
def _randn(gen, shape, dtype, sigma=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device=DEV).mul_(sigma).add_(mean).to(DTYPES[dtype])


def _tokens(gen, n, rows, left_out):
    """Token numbers, the low ones frequent (number i about in proportion to
    1 / (i + 1)), a share of them -100."""
    u = torch.rand((n,), generator=gen, device=DEV, dtype=torch.float64)
    ids = ((rows + 1.0) ** u - 1.0).long().clamp(0, rows - 1)
    if left_out:
        ids = torch.where(torch.rand((n,), generator=gen, device=DEV) < left_out, -100, ids)
    return ids


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    st = dict(case=case)
    kind, t, h, dt = case["kind"], case["tokens"], case["hidden"], case["dtype"]
    if kind in ("embedding", "embedding_grad"):
        st["ids"] = _tokens(gen, t, case["rows"], case["padded"])
        if kind == "embedding":
            st["table"] = _randn(gen, (case["rows"], h), dt, 0.02)
        else:
            st["dout"] = _randn(gen, (t, h), dt, 0.1)
        return st
    if kind in ("norm", "norm_grad"):
        st["x"] = _randn(gen, (t, h), case["residual"], 2.0)
        st["weight"] = _randn(gen, (h,), dt, 0.1, 1.0)
        st["y"] = _randn(gen, (t, h), dt) if case["block"] else None
        st["post"] = _randn(gen, (h,), dt, 0.1, 1.0) if case["post"] else None
        gate = dict(none=None, channels=(h,), tokens=(t, h))[case["gate"]]
        st["gate"] = None if gate is None else _randn(gen, gate, dt, 0.5)
        if kind == "norm_grad":
            st["dn"] = _randn(gen, (t, h), dt, 0.1)
            st["dh"] = _randn(gen, (t, h), case["residual"], 0.1)
        return st
    rows = case["rows"]
    st["weight"] = _randn(gen, (rows, h), dt, h ** -0.5)
    st["targets"] = _tokens(gen, t, rows, case["ignored"])
    # hidden states that point to their target by more or less: its logit is
    # up to 6 above the others', which spread by 1
    sure = 6.0 * torch.rand((t, 1), generator=gen, device=DEV)
    x = torch.randn((t, h), generator=gen, device=DEV)
    st["x"] = (x + sure * st["weight"][st["targets"].clamp(min=0)].float()).to(DTYPES[dt])
    if kind == "loss_grad":
        # the mean over tokens with weights near one; fp16 gradients are scaled
        # by a power of two, as training in fp16 does
        w = 0.5 + torch.rand((t,), generator=gen, device=DEV)
        st["dloss"] = w * ((1024.0 if dt == "f16" else 1.0) / t)
    return st


# ---------------------------------------------------------------------------
# the plain forms, in 32 bits
# ---------------------------------------------------------------------------
def _plain_embedding(st):
    table, ids, case = st["table"], st["ids"], st["case"]
    kept = (ids >= 0) & (ids < case["rows"])
    rows = table[ids.clamp(0, case["rows"] - 1)].float() * case["scale"]
    return torch.where(kept[:, None], rows, 0.0).to(table.dtype)


def _plain_embedding_grad(st):
    ids, case = st["ids"], st["case"]
    kept = (ids >= 0) & (ids < case["rows"])
    part = torch.where(kept[:, None], st["dout"].float() * case["scale"], 0.0)
    total = torch.zeros((case["rows"], case["hidden"]), device=DEV)
    total.index_add_(0, ids.clamp(0, case["rows"] - 1), part)
    return total.to(DTYPES[case["sum"]])


def _plain_norm_sum(st):
    """(h, 1 / rms of h, z, y / rms of y, 1 / rms of y) in 32 bits."""
    case = st["case"]
    h = st["x"].float()
    if st["y"] is None:
        return h, (h.square().mean(1, keepdim=True) + 1e-6).rsqrt(), None, None, None
    y = st["y"].float()
    r = (y.square().mean(1, keepdim=True) + 1e-6).rsqrt() if case["post"] else None
    yhat = y * r if case["post"] else None
    z = yhat * st["post"].float() if case["post"] else y
    h = h + case["scale"] * (z if st["gate"] is None else st["gate"].float() * z)
    return h, (h.square().mean(1, keepdim=True) + 1e-6).rsqrt(), z, yhat, r


def _plain_norm(st):
    h, r, _, _, _ = _plain_norm_sum(st)
    n = (h * r * st["weight"].float()).to(st["weight"].dtype)
    return n, h.to(st["x"].dtype)


def _plain_norm_grad(st):
    case, dt = st["case"], st["weight"].dtype
    h, r, z, yhat, ry = _plain_norm_sum(st)
    hhat, dn = h * r, st["dn"].float()
    n = (hhat * st["weight"].float()).to(dt)
    g = dn * st["weight"].float()
    dh = st["dh"].float() + r * (g - hhat * (g * hhat).mean(1, keepdim=True))
    out = dict(n=n, h=h.to(st["x"].dtype), dx=dh.to(st["x"].dtype), dweight=(dn * hhat).sum(0))
    if st["y"] is None:
        return out
    dz = case["scale"] * dh
    if st["gate"] is not None:
        dgate = dz * z
        out["dgate"] = dgate.sum(0) if case["gate"] == "channels" else dgate.to(dt)
        dz = dz * st["gate"].float()
    if case["post"]:
        out["dpost"] = (dz * yhat).sum(0)
        g = dz * st["post"].float()
        dz = ry * (g - yhat * (g * yhat).mean(1, keepdim=True))
    out["dy"] = dz.to(dt)
    return out


def _plain_logits(st):
    """(logits, lse, loss, target or 0, whether it counts) in 32 bits."""
    t, rows = st["targets"], st["case"]["rows"]
    z = torch.mm(st["x"].float(), st["weight"].float().t())
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1, keepdim=True).log() + top
    kept, at = ((t >= 0) & (t < rows))[:, None], t.clamp(0, rows - 1)[:, None]
    return z, lse, torch.where(kept, lse - z.gather(1, at), 0.0)[:, 0], at, kept


def _plain_loss(st):
    _, lse, loss, _, kept = _plain_logits(st)
    return loss, torch.where(kept, lse, 0.0)[:, 0]


def _plain_loss_grad(st):
    z, lse, loss, at, kept = _plain_logits(st)
    p = (z - lse).exp_()
    p.scatter_add_(1, at, torch.full_like(lse, -1.0))
    p *= torch.where(kept, st["dloss"][:, None], 0.0)
    dx, dw = torch.mm(p, st["weight"].float()), torch.mm(p.t(), st["x"].float())
    return loss, dx.to(st["x"].dtype), dw.to(st["x"].dtype)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return dict(embedding=_plain_embedding, embedding_grad=_plain_embedding_grad, norm=_plain_norm,
                    norm_grad=_plain_norm_grad, loss=_plain_loss, loss_grad=_plain_loss_grad)[kind](st)
    from paper_2608_11034_amd import replay
    if kind == "embedding":
        return replay.embedding(st["ids"], st["table"], scale=case["scale"])
    if kind == "embedding_grad":
        return replay.embedding_grad(st["dout"], st["ids"], case["rows"], scale=case["scale"],
                                     dtype=DTYPES[case["sum"]])
    if kind in ("norm", "norm_grad"):
        how = dict(post=st["post"], gate=st["gate"], scale=case["scale"], eps=1e-6)
        n, h, stats = replay.residual_norm(st["x"], st["y"], st["weight"], **how)
        if kind == "norm":
            return n, h
        g = replay.residual_norm_grad(st["dn"], st["dh"], st["x"], st["y"], st["weight"], stats, **how)
        out = dict(n=n, h=h, dx=g.dx, dweight=g.dweight, dgate=g.dgate, dpost=g.dpost, dy=g.dy)
        return {name: x for name, x in out.items() if x is not None}
    loss, lse = replay.vocab_loss(st["x"], st["weight"], st["targets"])
    if kind == "loss":
        return loss, lse
    return (loss,) + replay.vocab_loss_grad(st["dloss"], st["x"], st["weight"], st["targets"], lse)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    t, h, es = case["tokens"], case["hidden"], SIZE[case["dtype"]]
    if case["kind"] == "embedding":
        return dict(bytes=2 * t * h * es + 8 * t, flops=t * h)
    if case["kind"] == "embedding_grad":
        return dict(bytes=t * h * es + 8 * t + case["rows"] * h * SIZE[case["sum"]], flops=2 * t * h)
    if case["kind"] in ("norm", "norm_grad"):
        rs, grad = SIZE[case["residual"]], case["kind"] == "norm_grad"
        stream = h * t * rs * (2 if case["block"] else 1)           # x and h
        block = h * t * es * ((2 if case["block"] else 1) + (case["gate"] == "tokens"))     # y, n and gate
        if grad:
            stream += 2 * h * t * rs                                # dh and dx
            block += h * t * es * ((2 if case["block"] else 1) + (case["gate"] == "tokens"))
        return dict(bytes=stream + block, flops=(20 if grad else 6) * t * h)
    kept = max(1, round(t * (1 - case["ignored"])))
    product, x, w = 2 * kept * h * case["rows"], kept * h * es, case["rows"] * h * es
    if case["kind"] == "loss":
        return dict(bytes=x + w + 16 * t, flops=product)
    return dict(bytes=2 * x + 2 * w + 16 * t, flops=3 * product)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_embedding(st):
    case, out = st["case"], torch.zeros((st["case"]["tokens"], st["case"]["hidden"]), dtype=torch.float64,
                                        device=DEV)
    some = (st["ids"] >= 0).nonzero()[:, 0]
    out[some] = st["table"][st["ids"][some]].double() * case["scale"]
    return out


def _exact_embedding_grad(st):
    case = st["case"]
    out = torch.zeros((case["rows"], case["hidden"]), dtype=torch.float64, device=DEV)
    some = (st["ids"] >= 0).nonzero()[:, 0]
    if not some.numel():
        return out
    order = some[st["ids"][some].sort()[1]]
    ids = st["ids"][order]
    count = torch.bincount(ids, minlength=case["rows"])
    first = count.cumsum(0) - count
    nth = torch.arange(ids.numel(), device=DEV) - first[ids]       # of its row
    for i in range(int(count.max())):                               # every row once at most
        mine = order[nth == i]
        out[st["ids"][mine]] += st["dout"][mine].double()
    return out * case["scale"]


def _exact_norm(st, grad):
    """The definition differentiated by torch, in 64 bits."""
    case = st["case"]
    names = [n for n in ("x", "y", "weight", "post", "gate") if st[n] is not None]
    v = {n: st[n].double().requires_grad_(grad) for n in names}

    def normed(a):
        return a / torch.sqrt((a * a).sum(1, keepdim=True) / a.shape[1] + 1e-6)
    h = v["x"]
    if "y" in v:
        z = normed(v["y"]) * v["post"] if "post" in v else v["y"]
        h = v["x"] + (z * v["gate"] if "gate" in v else z) * case["scale"]
    n = normed(h) * v["weight"]
    if not grad:
        return n, h
    torch.autograd.backward([n, h], [st["dn"].double(), st["dh"].double()])
    return dict({"d" + a: v[a].grad for a in names}, n=n.detach(), h=h.detach())


def _exact_loss(st, grad):
    """A block of tokens at a time."""
    case = st["case"]
    t, rows = case["tokens"], case["rows"]
    w = st["weight"].double()
    loss, lse = (torch.zeros((t,), dtype=torch.float64, device=DEV) for _ in range(2))
    dx = torch.zeros((t, case["hidden"]), dtype=torch.float64, device=DEV)
    dw = torch.zeros_like(w) if grad else None
    some = ((st["targets"] >= 0) & (st["targets"] < rows)).nonzero()[:, 0]
    for at in some.split(max(1, 2 ** 28 // rows)):
        x, target = st["x"][at].double(), st["targets"][at]
        z = torch.mm(x, w.t())
        lse[at] = torch.logsumexp(z, 1)
        loss[at] = lse[at] - (x * w[target]).sum(1)
        if grad:
            d = torch.exp(z - lse[at][:, None])
            d[torch.arange(at.numel(), device=DEV), target] -= 1.0
            d *= st["dloss"][at].double()[:, None]
            dx[at] = torch.mm(d, w)
            dw += torch.mm(d.t(), x)
    return (loss, dx, dw) if grad else (loss, lse)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "embedding":
        return _exact_embedding(st)
    if kind == "embedding_grad":
        return _exact_embedding_grad(st)
    if kind in ("norm", "norm_grad"):
        return _exact_norm(st, kind == "norm_grad")
    return _exact_loss(st, kind == "loss_grad")
