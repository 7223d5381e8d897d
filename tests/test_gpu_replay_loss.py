"""The loss over a vocabulary and its gradient against plain 64-bit forms: one token to
many, odd vocabularies, widths that end inside a tile, ignored tokens and what they hold."""
import pytest
import torch

import replay_ends_plain as plain
from replay_plain import within

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
BF16, F16 = torch.bfloat16, torch.float16


def _inputs(T, H, V, dtype, ignored=0.0, seed=1, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    weight = (torch.randn((V, H), generator=g) * H ** -0.5).to(dtype)
    targets = torch.randint(0, V, (T,), generator=g)
    x = torch.randn((T, H), generator=g) + 5 * torch.rand((T, 1), generator=g) * weight[targets].float()
    targets[torch.rand((T,), generator=g) < ignored] = -100
    targets[torch.rand((T,), generator=g) < ignored / 4] = V
    dloss = (0.5 + torch.rand((T,), generator=g)) * ((64.0 if dtype == F16 else 1.0) / max(T, 1))
    return x.to(dtype), weight, targets, dloss


def _both(x, weight, targets, dloss, scale=1.0, **how):
    x, weight, targets, dloss = (t.to(DEV) for t in (x, weight, targets, dloss))
    loss, lse = replay.vocab_loss(x, weight, targets, scale=scale)
    dx, dweight = replay.vocab_loss_grad(dloss, x, weight, targets, lse, scale=scale, **how)
    return dict(loss=loss, lse=lse, dx=dx, dweight=dweight)


def _compare(got, want, what=""):
    for name, (value, bound) in want.items():
        within(got[name], value, bound, f"{what} {name}")


SIZES = [(1, 8, 1), (1, 64, 300), (2, 8, 3), (5, 72, 17), (31, 128, 255), (32, 200, 256), (33, 64, 257),
         (64, 136, 513), (65, 1000, 700), (255, 64, 100), (256, 128, 64), (257, 520, 1000), (600, 264, 1031),
         (7, 2048, 2500), (16, 64, 5003), (1500, 64, 40), (2100, 136, 300), (3, 4104, 9)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,H,V", SIZES)
def test_sizes(dtype, T, H, V):
    for ignored, scale in ((0.0, 1.0), (0.4, 0.7)):
        print("CASE", dtype, T, H, V, ignored, flush=True)
        v = _inputs(T, H, V, dtype, ignored)
        _compare(_both(*v, scale=scale), plain.vocab_loss(*v[:3], scale, v[3]), f"{T} {H} {V}")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_pieces(dtype):
    """More of the vocabulary than the softmax of one piece holds."""
    T, H, V = 33000, 16, 9000
    print("CASE", dtype, T, H, V, flush=True)
    v = _inputs(T, H, V, dtype, 0.2, seed=2)
    _compare(_both(*v), plain.vocab_loss(*v[:3], 1.0, v[3]))


@pytest.mark.parametrize("T,H,V,ignored", [(333, 64, 32000, 0.4), (880, 72, 20000, 0.0), (1010, 8, 20001, 0.01)])
def test_last_round(T, H, V, ignored):
    """Tiles in whole rounds of the device and a few more, which two workgroups share."""
    print("CASE", T, H, V, flush=True)
    v = _inputs(T, H, V, BF16, ignored, seed=10)
    _compare(_both(*v), plain.vocab_loss(*v[:3], 1.0, v[3]))


def test_ignored_tokens():
    """What an ignored token holds enters nothing, and the others' bits do not go by it."""
    T, H, V = 300, 136, 500
    x, weight, targets, dloss = _inputs(T, H, V, BF16, 0.3, seed=3)
    gone = (targets < 0) | (targets >= V)
    clean = _both(x, weight, targets, dloss)
    x, dloss = x.clone(), dloss.clone()
    x[gone] = float("nan")
    dloss[gone] = float("inf")
    got = _both(x, weight, targets, dloss)
    for name, t in clean.items():
        assert torch.equal(got[name], t), name
    for name in ("loss", "lse", "dx"):
        assert bool((got[name].cpu()[gone] == 0).all()), name
    # alone, the others give the same rows
    alone = _both(x[~gone], weight, targets[~gone], dloss[~gone])
    for name in ("loss", "lse"):
        assert torch.equal(alone[name].cpu(), got[name].cpu()[~gone])


@pytest.mark.parametrize("T", [128, 129, 500, 4096, 4097, 6000])
def test_few_of_many_take_part(T):
    """The number of tokens that take part decides what is kept of them, not T: 1, 64, 65,
    128 and 129 of them."""
    H, V = 72, 300
    x, weight, targets, dloss = _inputs(T, H, V, BF16, seed=10)
    for n in (1, 64, 65, 128, 129):
        if n > T:
            continue
        print("CASE", T, n, flush=True)
        some = torch.randperm(T, generator=torch.Generator().manual_seed(n))[:n].sort()[0]
        left = torch.full_like(targets, -1)
        left[some] = targets[some]
        got = _both(x, weight, left, dloss)
        want = plain.vocab_loss(x[some], weight, targets[some], 1.0, dloss[some])
        for name in ("loss", "lse", "dx"):
            rest = torch.ones((T,), dtype=torch.bool)
            rest[some] = False
            assert bool((got[name].cpu()[rest] == 0).all()), name
            got[name] = got[name][some.to(DEV)]
        _compare(got, want, f"{T} {n}")


def test_rounding_of_few_tokens():
    """Up to 128 tokens d is kept twice over, and dx takes the target's entry in full: both
    gradients then are off by little more than rounding the result, half a step of each
    element, and not by the rounding of one large entry of d in all of a row."""
    for T, names in ((1, ("dx", "dweight")), (7, ("dx", "dweight")), (128, ("dx", "dweight")), (700, ("dx",))):
        v = _inputs(T, 256, 3000, BF16, seed=11)
        got, want = _both(*v), plain.vocab_loss(*v[:3], 1.0, v[3])
        for name in names:
            value = want[name][0]
            rounded = (value.to(BF16).double() - value).norm()
            off = (got[name].cpu().double() - value).norm()
            assert float(off) <= 1.1 * float(rounded), (T, name, float(off / rounded))


def test_all_ignored_and_none():
    x, weight, targets, dloss = _inputs(40, 64, 300, BF16, seed=4)
    got = _both(torch.full_like(x, float("nan")), weight, torch.full_like(targets, -1), dloss)
    for t in got.values():
        assert bool((t == 0).all())
    got = _both(x[:0], weight, targets[:0], dloss[:0])
    assert got["dx"].shape == (0, 64) and bool((got["dweight"] == 0).all())


def test_strides_and_types_of_targets():
    T, H, V = 70, 136, 400
    v = _inputs(T, H, V, BF16, 0.2, seed=5)
    want = _both(*v)
    kept = []

    def moved(t):
        big = torch.full((t.shape[0], H + 24), 77.0, dtype=t.dtype, device=DEV)
        y = big[:, 8:8 + H]
        y.copy_(t)
        kept.append((y, big))
        return y
    x, weight = moved(v[0]), moved(v[1])
    dx, dweight = moved(torch.zeros((T, H), dtype=BF16)), moved(torch.zeros((V, H), dtype=BF16))
    targets, dloss = v[2].to(torch.int32).to(DEV), v[3].to(DEV)
    loss, lse = replay.vocab_loss(x, weight, targets)
    replay.vocab_loss_grad(dloss, x, weight, targets, lse, dx=dx, dweight=dweight)
    for name, t in dict(loss=loss, lse=lse, dx=dx, dweight=dweight).items():
        assert torch.equal(t, want[name]), name
    # one number for all tokens, not laid out
    one = torch.full((1,), 0.25, device=DEV)
    a = replay.vocab_loss_grad(one.expand(T), x, weight, targets, lse)
    b = replay.vocab_loss_grad(one.expand(T).contiguous(), x, weight, targets, lse)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    for y, big in kept:
        y.fill_(77.0)
        assert bool((big == 77.0).all())


def test_stride_of_a_single_row():
    """Nothing goes by it."""
    x, weight, targets, dloss = (t.to(DEV) for t in _inputs(1, 72, 1, BF16, seed=12))
    want = _both(x, weight, targets, dloss)
    for n in (0, 8, 4096):
        odd = [t.as_strided(t.shape, (n, 1)) for t in (x, weight)]
        got = _both(odd[0], odd[1], targets, dloss)
        assert all(torch.equal(got[name], t) for name, t in want.items()), n


def test_more_rows_than_a_piece():
    """5,000,000 rows for two tokens: d of 2^22 rows at most."""
    V, H = 5_000_000, 8
    g = torch.Generator(device=DEV).manual_seed(13)
    weight = torch.randn((V, H), generator=g, device=DEV).to(BF16)
    x = torch.randn((2, H), generator=g, device=DEV).to(BF16)
    targets = torch.tensor([V - 1, 2 ** 22 + 5], device=DEV)
    dloss = torch.ones((2,), device=DEV)
    got = _both(x, weight, targets, dloss)
    z = torch.mm(x.double(), weight.double().t())
    lse = torch.logsumexp(z, 1)
    assert float((got["lse"].double() - lse).abs().max()) <= 2e-5
    p = (z - lse[:, None]).exp()
    p[torch.arange(2, device=DEV), targets] -= 1
    for name, want in (("dx", torch.mm(p, weight.double())), ("dweight", torch.mm(p.t(), x.double()))):
        assert float((got[name].double() - want).norm() / want.norm()) <= 2.0 ** -8, name


@pytest.mark.parametrize("factor", [2.0 ** -20, 2.0 ** 12])
def test_gradients_of_any_size_in_fp16(factor):
    """dx and dweight scale with dloss: a power of two on it is one on them, as long as
    fp16 holds the results (normal numbers: compared where they are)."""
    x, weight, targets, dloss = _inputs(200, 64, 3000, F16, seed=6)
    one = _both(x, weight, targets, dloss)
    other = _both(x, weight, targets, dloss * factor)
    for name in ("dx", "dweight"):
        a, b = one[name].double() * factor, other[name].double()
        fine = (a.abs() > 2.0 ** -14) & (a.abs() < 60000) & (one[name].double().abs() > 2.0 ** -14)
        assert factor < 1 or bool(fine.any())
        assert torch.equal(a[fine], b[fine]), name


def test_dloss_up_to_the_largest_of_fp32_in_fp16():
    """Columns where the weights are zero have zeros in dx, and nothing is NaN."""
    x, weight, targets, _ = _inputs(100, 64, 500, F16, seed=9)
    weight[:, ::2] = 0
    got = _both(x, weight, targets, torch.full((100,), 2.0 ** 127))
    assert int((got["dx"][:, ::2] != 0).sum()) == 0
    assert not bool(got["dx"].isnan().any()) and not bool(got["dweight"].isnan().any())


def test_sure_and_far_logits():
    """Logits of a few hundred: one row takes all of the sum, or the target has none."""
    T, H, V = 64, 64, 1000
    g = torch.Generator().manual_seed(7)
    weight = torch.randn((V, H), generator=g).to(BF16)
    targets = torch.randint(0, V, (T,), generator=g)
    x = (6 * weight[targets].float()).to(BF16)
    targets[::2] = (targets[::2] + 1) % V
    dloss = torch.ones((T,))
    _compare(_both(x, weight, targets, dloss), plain.vocab_loss(x, weight, targets, 1.0, dloss))


def test_against_differences():
    """Differences of the mean loss along the gradient; bf16 steps that the inputs hold
    exactly (multiples of 2^-4 added to multiples of 2^-4)."""
    T, H, V = 48, 64, 120
    g = torch.Generator().manual_seed(8)
    x = torch.randint(-16, 17, (T, H), generator=g).double() / 16
    weight = torch.randint(-16, 17, (V, H), generator=g).double() / 16
    targets = torch.randint(0, V, (T,), generator=g)
    dloss = torch.ones((T,))
    got = _both(x.to(BF16), weight.to(BF16), targets, dloss)

    def f(a, b):
        loss, _ = replay.vocab_loss(a.to(BF16).to(DEV), b.to(BF16).to(DEV), targets.to(DEV))
        return float(loss.double().sum())
    for name, (da, db) in dict(dx=(1, 0), dweight=(0, 1)).items():
        grad = got[name].cpu().double()
        step = torch.zeros_like(grad)
        # one entry a row, so that the step is short: the largest of each
        at = grad.abs().argmax(1, keepdim=True)
        step.scatter_(1, at, grad.gather(1, at).sign() / 16)
        quotient = (f(x + da * (step if da else 0), weight + db * (step if db else 0)) -
                    f(x - da * (step if da else 0), weight - db * (step if db else 0))) / 2
        want = float((grad * step).sum())
        assert abs(quotient - want) <= 0.02 * abs(want), (name, quotient, want)


def test_same_bits_every_time():
    v = _inputs(700, 264, 1500, BF16, 0.2, seed=9)
    first = _both(*v)
    for _ in range(3):
        again = _both(*v)
        assert all(torch.equal(again[n], t) for n, t in first.items())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,V", [(129, 3000), (700, 3000), (4096, 3000), (5000, 3000), (3000, 200)])
def test_rounding_of_targets_entries(dtype, T, V):
    """Beyond 128 tokens both gradients take the target's entry of d in full.  The others'
    rounding is off by half a step of each at most, one apart from the other, so the squares of
    what it leaves in a gradient add up; so do they with those of rounding the result.  The
    norm of 33,000 elements or more strays from that by a percent or two: 1.05."""
    print("CASE", dtype, T, V, flush=True)
    x, weight, targets, dloss = v = _inputs(T, 256, V, dtype, seed=14)
    got, want = _both(*v), plain.vocab_loss(*v[:3], 1.0, v[3])
    g, W, X = dloss.double()[:, None], weight.double(), x.double()
    p = (X @ W.T - want["lse"][0][:, None]).exp()
    off_d = torch.finfo(dtype).eps / 2 * p * g + (2.0 ** -38 * g.max() if dtype == F16 else 0.0)
    off_d.scatter_(1, targets[:, None], 0.0)
    left = dict(dx=(off_d.square() @ W.square().sum(1)).sum().sqrt(),
                dweight=(off_d.square().T @ X.square().sum(1)).sum().sqrt())
    for name, rest in left.items():
        value = want[name][0]
        rounded = (value.to(dtype).double() - value).norm()
        off = (got[name].cpu().double() - value).norm()
        print(name, float(off / rounded), float(rest / rounded), flush=True)
        assert float(off) <= 1.05 * float((rounded.square() + rest.square()).sqrt()), (name, float(off / rounded))


@pytest.mark.parametrize("T,V", [(200, 40), (1500, 129), (4096, 700), (4097, 700), (9000, 513)])
def test_targets_in_one_place(T, V):
    """All targets one row, the first or the last; or each other one of a few."""
    for n, share in enumerate((torch.zeros(T), torch.full((T,), V - 1.0), torch.arange(T) % 3 * (V // 2 - 1))):
        print("CASE", T, V, n, flush=True)
        x, weight, targets, dloss = _inputs(T, 72, V, BF16, 0.1, seed=15)
        targets = torch.where((targets >= 0) & (targets < V), share.long(), targets)
        _compare(_both(x, weight, targets, dloss), plain.vocab_loss(x, weight, targets, 1.0, dloss), f"{T} {V} {n}")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T", [7, 100, 129, 300, 5000])
def test_dloss_that_is_not_finite(dtype, T):
    """An infinite dloss makes its token's share of dweight infinite, and the other tokens' rows
    of dx are what they are without it, also in fp16 where dloss is past what it holds."""
    x, weight, targets, dloss = _inputs(T, 72, 300, dtype, seed=16)
    weight = weight * 2.0 ** -6             # dx within fp16
    dloss = dloss * (100.0 / dloss.max())
    dloss[3] = float("inf")
    print("CASE", dtype, T, flush=True)
    got = _both(x, weight, targets, dloss)
    rest = torch.arange(T) != 3
    want, bound = plain.vocab_loss(x[rest], weight, targets[rest], 1.0, dloss[rest])["dx"]
    within(got["dx"].cpu()[rest], want, bound, "dx")
    sign = torch.ones((300, 1))
    sign[targets[3]] = -1.0
    share = sign * x[3].float() * float("inf")
    assert torch.equal(got["dweight"].cpu().float()[:, x[3] != 0], share[:, x[3] != 0])
    dloss[3] = float("nan")
    got = _both(x, weight, targets, dloss)
    within(got["dx"].cpu()[rest], want, bound, "dx")
    assert bool(got["dx"][3].isnan().all()) and bool(got["dweight"].isnan().all())


@pytest.mark.parametrize("factor", [2.0 ** -20, 2.0 ** -14])
def test_small_gradients_in_fp16(factor):
    """As test_gradients_of_any_size_in_fp16, from gradients so large that fp16 holds a part of
    the small ones in full."""
    x, weight, targets, dloss = _inputs(200, 64, 3000, F16, seed=6)
    one = _both(x, weight, targets, dloss * 2.0 ** 14)
    other = _both(x, weight, targets, dloss * (2.0 ** 14 * factor))
    for name in ("dx", "dweight"):
        a, b = one[name].double() * factor, other[name].double()
        fine = (a.abs() > 2.0 ** -14) & (one[name].double().abs() < 60000)
        assert int(fine.sum()) > 100, (name, int(fine.sum()))
        assert torch.equal(a[fine], b[fine]), name


def _against_plain_on_the_device(x, weight, targets, dloss, some, row_parts):
    """dx of the tokens `some` and dweight's parts in 64 bits: d is rounded once and the results
    once, half a step of each, so an error in the norm is below 2 half steps."""
    got = _both(x, weight, targets, dloss)
    W, dw = weight.double(), torch.zeros(weight.shape, dtype=torch.float64, device=DEV)
    for at in torch.arange(len(x), device=DEV).split(max(1, 2 ** 28 // len(weight))):
        p = torch.mm(x[at].double(), W.t())
        p = (p - torch.logsumexp(p, 1, keepdim=True)).exp()
        p[torch.arange(len(at), device=DEV), targets[at].long()] -= 1.0
        p *= dloss[at].double()[:, None]
        dw += torch.mm(p.t(), x[at].double())
        mine = some[(some >= at[0]) & (some <= at[-1])]
        want = torch.mm(p[mine - at[0]], W)
        off = (got["dx"][mine].double() - want).norm(dim=1) / want.norm(dim=1)
        assert bool((off <= 2 * 2.0 ** -8).all()), (mine, off)
    for part in row_parts:
        off = (got["dweight"][part].double() - dw[part]).norm() / dw[part].norm()
        assert float(off) <= 2 * 2.0 ** -8, (part, float(off))


def test_second_rows_of_d_in_pieces():
    """100 tokens, each with two rows of d, over 3,000,000 rows: three pieces."""
    T, H, V = 100, 8, 3_000_000
    print("CASE", T, H, V, flush=True)
    g = torch.Generator(device=DEV).manual_seed(17)
    weight = torch.randn((V, H), generator=g, device=DEV).to(BF16)
    x = torch.randn((T, H), generator=g, device=DEV).to(BF16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    targets[:2] = torch.tensor([V - 1, 0], device=DEV)
    _against_plain_on_the_device(x, weight, targets, torch.ones((T,), device=DEV), torch.arange(T, device=DEV),
                                 [targets, slice(0, 1 << 20), slice(1 << 20, 2 << 20), slice(2 << 20, V)])


def test_d_past_32_bits():
    """2^20 + 77 tokens: pieces of 2,048 rows, d of more than 2^31 elements in each."""
    T, H, V = (1 << 20) + 77, 8, 5000
    print("CASE", T, H, V, flush=True)
    g = torch.Generator(device=DEV).manual_seed(18)
    weight = torch.randn((V, H), generator=g, device=DEV).to(BF16)
    x = torch.randn((T, H), generator=g, device=DEV).to(BF16)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    dloss = 0.5 + torch.rand((T,), generator=g, device=DEV)
    order = targets.argsort()
    some = torch.cat((torch.tensor([0, 1, T // 2, T - 2, T - 1], device=DEV), order[:3], order[-3:])).unique()
    _against_plain_on_the_device(x, weight, targets, dloss, some,
                                 [slice(0, 2048), slice(2048, 4096), slice(4096, V), slice(V - 100, V)])


@pytest.mark.parametrize("T", [129, 4096, 5000])
def test_targets_of_none_and_of_four_bytes(T):
    """Tokens placed by their targets: none takes part, or targets are int32 and dloss is one
    number for all."""
    print("CASE", T, flush=True)
    x, weight, targets, _ = (t.to(DEV) for t in _inputs(T, 72, 300, BF16, 0.1, seed=19))
    one = torch.full((1,), 0.25, device=DEV)
    _, lse = replay.vocab_loss(x, weight, targets)
    for t in replay.vocab_loss_grad(one.expand(T), x, weight, torch.full_like(targets, 300), lse):
        assert bool((t == 0).all())
    want = replay.vocab_loss_grad(one.expand(T).contiguous(), x, weight, targets, lse)
    got = replay.vocab_loss_grad(one.expand(T), x, weight, targets.to(torch.int32), lse)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
