"""The replay operators record no graph: what requires a gradient is refused where
torch would record one, and taken where it would not."""
import pytest
import torch

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"


def _tensors():
    gen = torch.Generator().manual_seed(121)

    def make(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen).to(dtype).to(DEV)
    t = dict(q=make(9, 2, 64), k=make(9, 1, 64), v=make(9, 1, 64), g=make(9, 2, 64), x=make(6, 64), y=make(12, 64),
             w=make(6, 2, dtype=torch.float32), freqs=replay.rotary_frequencies(64))
    t["out"], t["lse"] = replay.attention(t["q"], t["k"], t["v"])
    t["pos"] = torch.arange(9, device=DEV)
    t["order"] = replay.expert_sort(torch.zeros((6, 2), dtype=torch.int32, device=DEV), 4)
    return t


CALLS = {
    "rotary": (lambda t: replay.rotary((t["q"], t["k"]), t["pos"], t["freqs"]), ("q", "k", "freqs")),
    "attention": (lambda t: replay.attention(t["q"], t["k"], t["v"]), ("q", "k", "v")),
    "attention_grad": (lambda t: replay.attention_grad(t["g"], t["q"], t["k"], t["v"], t["out"], t["lse"]),
                       ("g", "q", "k", "v", "out", "lse")),
    "dispatch": (lambda t: replay.expert_dispatch(t["x"], t["order"]), ("x",)),
    "combine": (lambda t: replay.expert_combine(t["y"], t["order"], t["w"]), ("y", "w")),
    "combine_grad": (lambda t: replay.expert_combine_grad(t["x"], t["y"], t["order"], t["w"]), ("x", "y", "w")),
    "dispatch_grad": (lambda t: replay.expert_dispatch_grad(t["y"], t["order"]), ("y",)),
}


def _flat(r):
    return [r] if isinstance(r, torch.Tensor) else list(r)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refused_where_a_graph_is_recorded(name):
    call, which = CALLS[name]
    t = _tensors()
    want = _flat(call(t))
    for n in which:
        print("CASE", name, n, flush=True)
        y = dict(t)
        y[n] = t[n].clone().requires_grad_()
        with pytest.raises(replay.C3Error, match="gradient"):
            call(y)
        with torch.no_grad():
            got = _flat(call(y))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_inside_a_function():
    """A torch function of forward and backward, which record no graph inside."""
    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            out, lse = replay.attention(q, k, v, causal=True)
            ctx.save_for_backward(q, k, v, out, lse)
            return out

        @staticmethod
        def backward(ctx, g):
            return replay.attention_grad(g, *ctx.saved_tensors, causal=True)
    t = _tensors()
    q, k, v = (t[n].clone().requires_grad_() for n in "qkv")
    Attention.apply(q, k, v).backward(t["g"])
    out, lse = replay.attention(t["q"], t["k"], t["v"], causal=True)
    want = replay.attention_grad(t["g"], t["q"], t["k"], t["v"], out, lse, causal=True)
    assert all(torch.equal(a.grad, b) for a, b in zip((q, k, v), want))
