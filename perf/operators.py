"""The operators of a replayed transformer layer, and how their speed is measured.

A replay runs one layer again on every replica and compares outputs and
gradients bit by bit.  Four operators of the layer are measured here, over the
sizes that such a replay meets: rotary positions on queries and keys, attention
with its row statistic, attention's gradient, and the path of tokens to their
experts and back with its gradient.

A case is one pass through one of them.  With ``own`` false ``run`` computes it
in plain torch operations in 32 bits (the angles of rotary positions, which 32
bits cannot hold at long contexts, in 64), with ``own`` true through
``paper_2608_11034_amd.replay``.  ``exact`` computes the same in 64 bits,
sequence by sequence and head by head, from the definitions.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda"
MOST_SCORES = 16 * 16384 * 16384      # padded scores of the largest case


def listed():
    return [
        # one new token of each of 8 sequences, queries and keys of a layer
        # with 32 heads that share 8 key heads: all latency
        dict(name="rotary_tokens", kind="rotary", dtype="bf16", batch=8, length=1, heads=32,
             kv_heads=8, dim=128, rot=128, layout="half", base=10000.0, factor=1.0, span=131072,
             inverse=False),
        # a micro-batch of a 4096-wide layer (32 heads of 128), the ordinary
        # call before attention
        dict(name="rotary_layer", kind="rotary", dtype="bf16", batch=4, length=4096, heads=32,
             kv_heads=32, dim=128, rot=128, layout="half", base=10000.0, factor=1.0, span=0,
             inverse=False),
        # the gradient, fp32, odd length, a quarter of each head rotated in
        # neighbouring pairs, frequencies stretched for a long context
        dict(name="rotary_long_grad", kind="rotary", dtype="f32", batch=1, length=16383, heads=32,
             kv_heads=4, dim=64, rot=16, layout="interleaved", base=500000.0, factor=8.0, span=0,
             inverse=True),
        # one new token of each of 16 sequences of very different lengths
        # against their keys and values
        dict(name="attention_tokens", kind="attention", dtype="bf16", heads=32, kv_heads=8, dim=128,
             q_lens=",".join(["1"] * 16), causal=True, window=0,
             k_lens="32768,1,17,129,4096,8191,20011,511,12345,2048,30000,777,65,16384,9999,1023"),
        # the layer of rotary_layer: 2 sequences of 4096 tokens
        dict(name="attention_layer", kind="attention", dtype="bf16", batch=2, q_len=4096, k_len=4096,
             heads=32, kv_heads=32, dim=128, causal=True, window=0),
        # packed documents of odd lengths in fp16, a 2048-wide layer with 32
        # heads of 64 that share 8, a sliding window, one document that has
        # more queries than keys (rows that see nothing)
        dict(name="attention_packed", kind="attention", dtype="f16", heads=32, kv_heads=8, dim=64,
             q_lens="1,37,1023,500,3001,130,2047,1453", k_lens="1,37,1023,333,3001,130,2047,1453",
             causal=True, window=1024),
        # forward and gradient of a small cross attention with a head size
        # that is no power of two
        dict(name="attention_grad_small", kind="attention_grad", dtype="f16", batch=2, q_len=333,
             k_len=190, heads=8, kv_heads=4, dim=80, causal=False, window=0),
        # forward and gradient of the layer of attention_layer: one training
        # step's worth
        dict(name="attention_grad_layer", kind="attention_grad", dtype="bf16", batch=2, q_len=4096,
             k_len=4096, heads=32, kv_heads=32, dim=128, causal=True, window=0),
        # a long context with few key heads, the largest
        dict(name="attention_grad_long", kind="attention_grad", dtype="bf16", batch=1, q_len=16384,
             k_len=16384, heads=16, kv_heads=2, dim=128, causal=True, window=0),
        # a few tokens to 2 of 8 experts and back: latency
        dict(name="experts_tokens", kind="experts", dtype="bf16", tokens=32, top=2, experts=8,
             hidden=4096, dropped=0.0),
        # a micro-batch of a 2048-wide layer to 8 of 64 experts and back
        dict(name="experts_layer", kind="experts", dtype="bf16", tokens=16384, top=8, experts=64,
             hidden=2048, dropped=0.0),
        # the gradient of the whole path, an odd number of tokens, 160
        # experts, one choice in ten dropped (tokens without any expert too)
        dict(name="experts_grad", kind="experts_grad", dtype="f16", tokens=8191, top=6, experts=160,
             hidden=4096, dropped=0.1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _length(rng, lo, hi):
    n = _log(rng, lo, hi)
    return n + (n == 3 * 1024)


def _heads(rng, dims):
    kv = rng.choice([1, 2, 4, 8, 8, 16])
    heads, dim = kv * rng.choice([1, 1, 2, 3, 4, 8] if kv <= 8 else [1, 2]), rng.choice(dims)
    return heads, kv, dim if heads * dim != 3 * 1024 else 64


def draw(rng):
    kind = rng.choice(["rotary", "attention", "attention", "attention_grad", "attention_grad",
                       "experts", "experts_grad"])
    if kind == "rotary":
        heads, kv, dim = _heads(rng, [64, 80, 96, 128, 128])
        batch = rng.choice([1, 1, 2, 4, 8])
        length = _length(rng, 1, max(1, 524288 // (heads + kv) // batch * 128 // dim))
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), batch=batch,
                    length=length, heads=heads, kv_heads=kv, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, dim // 4]),
                    layout=rng.choice(["half", "interleaved"]),
                    base=rng.choice([10000.0, 500000.0]), factor=rng.choice([1.0, 1.0, 4.0, 8.0]),
                    span=rng.choice([0, 0, 131072]), inverse=rng.random() < 0.4)
    if kind in ("attention", "attention_grad"):
        heads, kv, dim = _heads(rng, [64, 64, 80, 96, 128, 128, 128])
        case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16"]), heads=heads, kv_heads=kv,
                    dim=dim, causal=rng.random() < 0.75)
        case["window"] = rng.choice([0, 0, 0, 128, 1000]) if case["causal"] else 0
        form = rng.choice(["tokens", "packed", "dense", "dense"] if kind == "attention"
                          else ["packed", "dense", "dense"])
        if form == "tokens":
            n = rng.randint(1, 16)
            case["q_lens"] = ",".join(str(rng.choice([1, 1, 1, 4])) for _ in range(n))
            case["k_lens"] = ",".join(str(_length(rng, 4, 32768)) for _ in range(n))
        elif form == "packed":
            n = rng.randint(2, 8)
            most = int(min(4096, math.sqrt(MOST_SCORES / 4 / n / heads)))
            case["k_lens"] = ",".join(str(_length(rng, 1, most)) for _ in range(n))
            case["q_lens"] = (case["k_lens"] if rng.random() < 0.7 else
                              ",".join(str(_length(rng, 1, most)) for _ in range(n)))
        else:
            batch = rng.choice([1, 1, 2, 4])
            most = int(min(8192, math.sqrt(MOST_SCORES / 4 / batch / heads)))
            length = _length(rng, 16, most)
            case |= dict(batch=batch, q_len=length, k_len=length)
            if rng.random() < 0.25:
                case["k_len"] = _length(rng, 16, most)
        return case
    hidden = rng.choice([512, 1000, 2048, 2048, 4096, 4100])
    top = rng.choice([1, 2, 4, 6, 8])
    tokens = _length(rng, 16, min(65536, 268435456 // hidden // top))
    return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                tokens=tokens, top=top,
                experts=max(top, rng.choice([8, 16, 60, 64, 128, 160, 256])), hidden=hidden,
                dropped=rng.choice([0.0, 0.0, 0.1]))


# ---------------------------------------------------------------------------
# prepare: what the program has in hand before the call
# ---------------------------------------------------------------------------
def _randn(gen, shape, dtype, sigma=1.0):
    return torch.randn(shape, generator=gen, device=DEV).mul_(sigma).to(DTYPES[dtype])


def _frequencies(rot, base, factor):
    """Radians a position of each pair, in 64 bits.  A factor over 1 stretches
    the slow pairs for a context that many times the trained 4096 positions and
    leaves the fast ones, with a ramp between 1 and 32 turns in the context."""
    i = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
    f = base ** (-2.0 * i / rot)
    if factor != 1.0:
        keep = ((4096 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
    return f


def _lens(case, name):
    return [int(x) for x in case[name].split(",")]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    st = dict(case=case)
    if case["kind"] == "rotary":
        b, n = case["batch"], case["length"]
        st["q"] = _randn(gen, (b, n, case["heads"], case["dim"]), case["dtype"])
        st["k"] = _randn(gen, (b, n, case["kv_heads"], case["dim"]), case["dtype"])
        if case["span"]:
            st["pos"] = torch.randint(0, case["span"], (b, n), generator=gen, device=DEV,
                                      dtype=torch.int32)
        else:
            st["pos"] = torch.arange(n, device=DEV, dtype=torch.int32).expand(b, n).contiguous()
        st["freqs"] = _frequencies(case["rot"], case["base"], case["factor"])
        return st
    if case["kind"] in ("attention", "attention_grad"):
        d, dt = case["dim"], case["dtype"]
        if "q_lens" in case:
            st["q_lens"], st["k_lens"] = _lens(case, "q_lens"), _lens(case, "k_lens")
            q, k = (sum(st["q_lens"]),), (sum(st["k_lens"]),)
            for x in ("q_lens", "k_lens"):       # where each sequence starts, and its length
                n = torch.tensor(st[x], device=DEV)
                st["at_" + x] = (n.cumsum(0) - n, n)
        else:
            q, k = (case["batch"], case["q_len"]), (case["batch"], case["k_len"])
        st["q"] = _randn(gen, q + (case["heads"], d), dt)
        st["k"] = _randn(gen, k + (case["kv_heads"], d), dt)
        st["v"] = _randn(gen, k + (case["kv_heads"], d), dt)
        if case["kind"] == "attention_grad":
            st["dout"] = _randn(gen, q + (case["heads"], d), dt)
        return st
    t, top, e, h = case["tokens"], case["top"], case["experts"], case["hidden"]
    # a router's scores with a few experts in favour
    logits = torch.randn((t, e), generator=gen, device=DEV)
    logits += torch.randn((e,), generator=gen, device=DEV)
    w, ids = logits.topk(top, dim=1)
    st["weights"] = w.softmax(1)
    st["ids"] = ids.to(torch.int32)
    if case["dropped"]:
        gone = torch.rand((t, top), generator=gen, device=DEV) < case["dropped"]
        gone[torch.rand((t,), generator=gen, device=DEV) < case["dropped"] / 4] = True
        st["ids"] = st["ids"].masked_fill(gone, -1)
    st["x"] = _randn(gen, (t, h), case["dtype"])
    st["y"] = _randn(gen, (t * top, h), case["dtype"])       # the experts' outputs
    if case["kind"] == "experts_grad":
        st["dout"] = _randn(gen, (t, h), case["dtype"])
        st["dxs"] = _randn(gen, (t * top, h), case["dtype"])
    return st


# ---------------------------------------------------------------------------
# the plain forms, in 32 bits
# ---------------------------------------------------------------------------
def _plain_rotary(x, pos, freqs, layout, inverse):
    r = 2 * freqs.numel()
    angle = pos.double()[..., None] * freqs
    cos, sin = angle.cos().float()[:, :, None, :], angle.sin().float()[:, :, None, :]
    if inverse:
        sin = -sin
    y = x.float()
    a, b = (y[..., :r // 2], y[..., r // 2:r]) if layout == "half" else (y[..., 0:r:2], y[..., 1:r:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, v], -1) if layout == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_padded(x, at):
    """Packed tokens [sum of lengths, ...] as [sequences, longest, ...] in 32 bits."""
    start, n = at
    i = torch.arange(int(n.max()), device=DEV)
    return x.float()[(start[:, None] + i).clamp(max=max(x.shape[0] - 1, 0))]


def _plain_packed(x, at):
    """[sequences, longest, ...] back to [sum of lengths, ...]."""
    start, n = at
    return x[torch.arange(x.shape[1], device=DEV) < n[:, None]]


def _plain_shapes(st):
    """Queries [B, key heads, group * length, D] and keys and values
    [B, key heads, length, D] in 32 bits, and where a query sees a key."""
    case = st["case"]
    if "q_lens" in st:
        pq, pk = (lambda x: _plain_padded(x, st["at_q_lens"])), (lambda x: _plain_padded(x, st["at_k_lens"]))
        nq, nk = st["at_q_lens"][1], st["at_k_lens"][1]
    else:
        pq = pk = lambda x: x.float()
        nq = torch.full((case["batch"],), case["q_len"], device=DEV)
        nk = torch.full((case["batch"],), case["k_len"], device=DEV)
    hk = case["kv_heads"]

    def rows(x):
        x = pq(x)
        b, n, h, d = x.shape
        return x.view(b, n, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, h // hk * n, d)

    def keys(x):
        return pk(x).transpose(1, 2).contiguous()
    q, k, v = rows(st["q"]), keys(st["k"]), keys(st["v"])
    g = case["heads"] // hk
    i = torch.arange(q.shape[2] // g, device=DEV)[None, :, None]
    j = torch.arange(k.shape[2], device=DEV)[None, None, :]
    n, m = nq[:, None, None], nk[:, None, None]
    sees = (i < n) & (j < m)
    if case["causal"]:
        sees = sees & (j <= i + m - n)
    if case["window"]:
        sees = sees & (j > i + m - n - case["window"])
    return q, k, v, rows, sees[:, None, None]


def _plain_rows_back(x, st):
    """[B, key heads, group * length, ...] as the queries lie."""
    case = st["case"]
    hk, g = case["kv_heads"], case["heads"] // case["kv_heads"]
    b, n = x.shape[0], x.shape[2] // g
    x = x.view(b, hk, g, n, -1).permute(0, 3, 1, 2, 4).reshape(b, n, hk * g, -1)
    return _plain_packed(x, st["at_q_lens"]) if "q_lens" in st else x


def _plain_keys_back(x, st):
    x = x.transpose(1, 2)
    return _plain_packed(x, st["at_k_lens"]) if "k_lens" in st else x


def _plain_softmax(st):
    q, k, v, rows, sees = _plain_shapes(st)
    case = st["case"]
    g = case["heads"] // case["kv_heads"]
    b, hk, n, _ = q.shape
    s = (q * case["dim"] ** -0.5) @ k.transpose(2, 3)
    s = s.view(b, hk, g, n // g, -1).masked_fill(~sees, -math.inf).view(s.shape)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (s - top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    return q, k, v, rows, p, total.log() + top


def _plain_attention(st):
    _, _, v, _, p, lse = _plain_softmax(st)
    dt = DTYPES[st["case"]["dtype"]]
    return _plain_rows_back(p @ v, st).to(dt), _plain_rows_back(lse, st)[..., 0]


def _plain_attention_grad(st):
    q, k, v, rows, p, _ = _plain_softmax(st)
    dt, scale = DTYPES[st["case"]["dtype"]], st["case"]["dim"] ** -0.5
    out, dout = p @ v, rows(st["dout"])
    dv = p.transpose(2, 3) @ dout
    ds = dout @ v.transpose(2, 3)
    ds -= (dout * out).sum(-1, keepdim=True)
    ds *= p
    dq, dk = (ds @ k) * scale, (ds.transpose(2, 3) @ q) * scale
    return (_plain_rows_back(out, st).to(dt), _plain_rows_back(dq, st).to(dt),
            _plain_keys_back(dk, st).to(dt), _plain_keys_back(dv, st).to(dt))


def _plain_order(ids, experts):
    """offsets [E + 1]; for each choice its place in the sorted list, -1 where
    it has no expert; for each place its choice, -1 behind the last."""
    flat = ids.reshape(-1).long()
    kept = (flat >= 0) & (flat < experts)
    key = torch.where(kept, flat, experts)
    choice = key.sort(stable=True)[1]
    offsets = (key[:, None] == torch.arange(experts, device=DEV)).sum(0).cumsum(0)
    offsets = torch.cat([offsets.new_zeros(1), offsets])
    place = torch.empty_like(choice)
    place[choice] = torch.arange(flat.numel(), device=DEV)
    source = torch.where(torch.arange(flat.numel(), device=DEV) < offsets[-1], choice, -1)
    return (offsets.to(torch.int32), source.to(torch.int32),
            torch.where(kept, place, -1).to(torch.int32).view(ids.shape))


def _plain_gather(y, slot, weights):
    """Sum over a token's choices of weight times the row at its place."""
    rows = torch.where((slot >= 0)[..., None], y.float()[slot.clamp(min=0).long()], 0.0)
    return (rows if weights is None else rows * weights[..., None]).sum(1)


def _plain_experts(st):
    offsets, source, slot = _plain_order(st["ids"], st["case"]["experts"])
    x, top = st["x"], st["case"]["top"]
    xs = torch.where((source >= 0)[:, None], x.float()[source.clamp(min=0).long() // top], 0.0)
    return (offsets, source, slot, xs.to(x.dtype),
            _plain_gather(st["y"], slot, st["weights"]).to(x.dtype))


def _plain_experts_grad(st):
    _, source, slot = _plain_order(st["ids"], st["case"]["experts"])
    top, dt, w = st["case"]["top"], st["x"].dtype, st["weights"]
    there, choice = (source >= 0)[:, None], source.clamp(min=0).long()
    dy = torch.where(there, st["dout"].float()[choice // top] * w.reshape(-1)[choice][:, None], 0.0)
    rows = torch.where((slot >= 0)[..., None], st["y"].float()[slot.clamp(min=0).long()], 0.0)
    dw = (rows * st["dout"].float()[:, None]).sum(-1)
    return dy.to(dt), dw, _plain_gather(st["dxs"], slot, None).to(dt)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        from paper_2608_11034_amd import replay
        if kind == "rotary":
            return replay.rotary((st["q"], st["k"]), st["pos"], st["freqs"], layout=case["layout"],
                                 inverse=case["inverse"])
        if kind in ("attention", "attention_grad"):
            how = dict(causal=case["causal"], window=case["window"], q_lens=st.get("q_lens"),
                       k_lens=st.get("k_lens"))
            out, lse = replay.attention(st["q"], st["k"], st["v"], **how)
            if kind == "attention":
                return out, lse
            return (out,) + replay.attention_grad(st["dout"], st["q"], st["k"], st["v"], out, lse,
                                                  **how)
        order = replay.expert_sort(st["ids"], case["experts"])
        if kind == "experts":
            return (order.offsets, order.source, order.slot, replay.expert_dispatch(st["x"], order),
                    replay.expert_combine(st["y"], order, st["weights"]))
        dy, dw = replay.expert_combine_grad(st["dout"], st["y"], order, st["weights"])
        return dy, dw, replay.expert_dispatch_grad(st["dxs"], order)
    if kind == "rotary":
        return tuple(_plain_rotary(st[x], st["pos"], st["freqs"], case["layout"], case["inverse"])
                     for x in ("q", "k"))
    return dict(attention=_plain_attention, attention_grad=_plain_attention_grad,
                experts=_plain_experts, experts_grad=_plain_experts_grad)[kind](st)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def _pairs(case):
    """(query, key) pairs of one head that the mask leaves."""
    if "q_lens" in case:
        lens = zip(_lens(case, "q_lens"), _lens(case, "k_lens"))
    else:
        lens = [(case["q_len"], case["k_len"])] * case["batch"]
    total = 0
    for n, m in lens:
        for i in range(n):
            hi = min(m, i + m - n + 1) if case["causal"] else m
            lo = max(0, i + m - n - case["window"] + 1) if case["window"] else 0
            total += max(0, hi - lo)
    return total


def work(case):
    es = SIZE[case["dtype"]]
    if case["kind"] == "rotary":
        tokens, heads = case["batch"] * case["length"], case["heads"] + case["kv_heads"]
        return dict(bytes=2 * tokens * heads * case["dim"] * es + 4 * tokens + 4 * case["rot"],
                    flops=3 * tokens * heads * case["rot"])
    if case["kind"] in ("attention", "attention_grad"):
        if "q_lens" in case:
            nq, nk = sum(_lens(case, "q_lens")), sum(_lens(case, "k_lens"))
        else:
            nq, nk = case["batch"] * case["q_len"], case["batch"] * case["k_len"]
        q, k = nq * case["heads"] * case["dim"] * es, nk * case["kv_heads"] * case["dim"] * es
        product = 2 * _pairs(case) * case["heads"] * case["dim"]
        if case["kind"] == "attention":
            return dict(bytes=2 * q + 2 * k + 4 * nq * case["heads"], flops=2 * product)
        return dict(bytes=4 * q + 4 * k, flops=7 * product)
    t, h = case["tokens"], case["hidden"]
    n = t * case["top"]
    if case["kind"] == "experts":
        # tokens and results, the sorted rows written and read, choices and weights
        return dict(bytes=2 * t * h * es + 2 * n * h * es + 16 * n, flops=2 * n * h)
    return dict(bytes=2 * t * h * es + 3 * n * h * es + 12 * n, flops=4 * n * h)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_rotary(st):
    case = st["case"]
    half = case["rot"] // 2
    out = []
    for x in (st["q"], st["k"]):
        y = x.double().clone()
        for i in range(half):
            a, b = (i, i + half) if case["layout"] == "half" else (2 * i, 2 * i + 1)
            # the pair as a complex number, turned by the angle
            turn = torch.polar(torch.ones_like(st["pos"], dtype=torch.float64),
                               st["pos"].double() * st["freqs"][i])
            z = torch.complex(x[..., a].double(), x[..., b].double())
            z = z * (turn.conj() if case["inverse"] else turn)[..., None]
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_attention(st, grad):
    case = st["case"]
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    q, k, v = (st[x].reshape(-1, st[x].shape[-2], d) for x in "qkv")
    dout = st["dout"].reshape(q.shape) if grad else None
    out, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.full(
        q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in (q, k, v))
    if "q_lens" in st:
        lens = list(zip(st["q_lens"], st["k_lens"]))
    else:
        lens = [(case["q_len"], case["k_len"])] * case["batch"]
    q0 = k0 = 0
    for n, m in lens:
        at = torch.arange(n, device=DEV)[:, None] + m - n      # the key that a query stands at
        j = torch.arange(m, device=DEV)[None, :]
        hidden = torch.zeros((n, m), dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= j > at
        if case["window"]:
            hidden |= j <= at - case["window"]
        some = (~hidden).any(1)
        for a in range(h if n and m else 0):
            c = a // (h // hk)
            Q, K, V = (x.double() for x in (q[q0:q0 + n, a], k[k0:k0 + m, c], v[k0:k0 + m, c]))
            s = torch.mm(Q, K.t()).div_(math.sqrt(d)).masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(s, 1)
            lse[q0:q0 + n, a] = z
            p = torch.exp(s.sub_(torch.where(some, z, 0.0)[:, None]))
            out[q0:q0 + n, a] = p @ V
            if grad:
                G = dout[q0:q0 + n, a].double()
                dv[k0:k0 + m, c] += p.t() @ G
                dp = G @ V.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                dq[q0:q0 + n, a] = ds @ K
                dk[k0:k0 + m, c] += ds.t() @ Q
        q0, k0 = q0 + n, k0 + m
    if not grad:
        return out.view(st["q"].shape), lse.view(st["q"].shape[:-1])
    return out.view(st["q"].shape), dq.view(st["q"].shape), dk.view(st["k"].shape), dv.view(st["k"].shape)


def _exact_experts(st, grad):
    case = st["case"]
    top, e = case["top"], case["experts"]
    ids = st["ids"].reshape(-1).tolist()
    lists = [[] for _ in range(e)]
    for n, i in enumerate(ids):
        if 0 <= i < e:
            lists[i].append(n)
    offsets, source = [0], []
    for some in lists:
        source += some
        offsets.append(len(source))
    slot = [-1] * len(ids)
    for p, n in enumerate(source):
        slot[n] = p
    at, n = torch.tensor(source, device=DEV, dtype=torch.long), len(source)
    w = st["weights"].double().reshape(-1)
    big = torch.zeros((len(ids), case["hidden"]), dtype=torch.float64, device=DEV)
    small = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device=DEV)
    if not grad:
        xs, back = big, small
        xs[:n] = st["x"].double()[at // top]
        for t in range(top):        # the rows of every token's choice t
            mine = (at % top == t).nonzero()[:, 0]
            back[at[mine] // top] += w[at[mine]][:, None] * st["y"][mine].double()
        as_int = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (
            offsets, source + [-1] * (len(ids) - n), slot)]
        return as_int[0], as_int[1], as_int[2].view(st["ids"].shape), xs, back
    dy, dx = big, small
    g = st["dout"].double()[at // top]
    dy[:n] = w[at][:, None] * g
    dw = torch.zeros(len(ids), dtype=torch.float64, device=DEV)
    dw[at] = (g * st["y"][:n].double()).sum(1)
    for t in range(top):
        mine = (at % top == t).nonzero()[:, 0]
        dx[at[mine] // top] += st["dxs"][mine].double()
    return dy, dw.view(st["ids"].shape), dx


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(st)
    if case["kind"] in ("attention", "attention_grad"):
        return _exact_attention(st, case["kind"] == "attention_grad")
    return _exact_experts(st, case["kind"] == "experts_grad")
