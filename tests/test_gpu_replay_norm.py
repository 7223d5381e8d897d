"""The residual norm and its gradient against plain 64-bit forms: every form, type
and a range of widths, odd ones and strides among them."""
import pytest
import torch

import replay_ends_plain as plain
from replay_plain import within

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)]     # residual, block
FORMS = [(False, False, None), (True, False, None), (True, False, "channels"), (True, False, "tokens"),
         (True, True, None), (True, True, "channels"), (True, True, "tokens")]


def _inputs(T, H, residual, block, form, seed=1):
    g = torch.Generator().manual_seed(seed)

    def randn(*shape, sigma=1.0, mean=0.0, dtype=block):
        return (torch.randn(shape, generator=g) * sigma + mean).to(dtype)
    there, post, gate = form
    return dict(x=randn(T, H, sigma=2.0, dtype=residual), y=randn(T, H) if there else None,
                weight=randn(H, sigma=0.1, mean=1.0), post=randn(H, sigma=0.1, mean=1.0) if post else None,
                gate={None: None, "channels": randn(H, sigma=0.5), "tokens": randn(T, H, sigma=0.5)}[gate],
                dn=randn(T, H), dh=randn(T, H, dtype=residual))


def _dev(v):
    return {n: t.to(DEV) if t is not None else None for n, t in v.items()}


def _both(v, scale, eps, dh=True, **out):
    how = dict(post=v["post"], gate=v["gate"], scale=scale, eps=eps)
    n, h, stats = replay.residual_norm(v["x"], v["y"], v["weight"], **how)
    g = replay.residual_norm_grad(v["dn"], v["dh"] if dh else None, v["x"], v["y"], v["weight"], stats, **how)
    return dict(g._asdict(), n=n, h=h, stats=stats)


def _compare(got, want, what=""):
    for name, (value, bound) in want.items():
        within(got[name], value, bound, f"{what} {name}")
    for name in ("dy", "dpost", "dgate"):
        assert (got[name] is None) == (name not in want), name


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("residual,block", TYPES)
def test_forms(residual, block, form):
    for T, H in ((1, 8), (3, 200), (70, 513), (37, 2048)):
        print("CASE", residual, block, form, T, H, flush=True)
        v = _inputs(T, H, residual, block, form)
        want = plain.residual_norm(v["x"], v["y"], v["weight"], v["post"], v["gate"], 0.5, 1e-5, v["dn"], v["dh"])
        _compare(_both(_dev(v), 0.5, 1e-5), want, f"{T} {H}")


@pytest.mark.parametrize("H", [1, 2, 7, 64, 65, 511, 512, 520, 1000, 1024, 1025, 4096, 4100, 8192, 8200, 16384, 16383])
@pytest.mark.parametrize("residual,block", [(BF16, BF16), (F32, F16), (F32, F32)])
def test_widths(residual, block, H):
    for form in (FORMS[1], FORMS[5]):
        print("CASE", residual, block, H, form, flush=True)
        v = _inputs(5, H, residual, block, form, seed=2)
        want = plain.residual_norm(v["x"], v["y"], v["weight"], v["post"], v["gate"], 1.0, 1e-6, v["dn"], v["dh"])
        _compare(_both(_dev(v), 1.0, 1e-6), want, f"{H}")


@pytest.mark.parametrize("T,H", [(1500, 256), (2049, 64), (700, 4096), (1025, 8200)])
def test_many_tokens(T, H):
    """More rows than the gradient's workgroups walk at once."""
    print("CASE", T, H, flush=True)
    v = _inputs(T, H, BF16, BF16, FORMS[5], seed=3)
    want = plain.residual_norm(v["x"], v["y"], v["weight"], v["post"], v["gate"], 0.25, 1e-6, v["dn"], v["dh"])
    _compare(_both(_dev(v), 0.25, 1e-6), want)


def test_no_other_reader():
    """dh missing is dh of zeros."""
    v = _inputs(9, 136, BF16, BF16, FORMS[1], seed=4)
    want = plain.residual_norm(v["x"], v["y"], v["weight"], None, None, 1.0, 1e-6, v["dn"], None)
    _compare(_both(_dev(v), 1.0, 1e-6, dh=False), want)


@pytest.mark.parametrize("residual,block", TYPES)
@pytest.mark.parametrize("H", [64, 1000, 4099])
def test_strides_and_alignment(residual, block, H):
    """Rows further apart and starting anywhere: the same bits, nothing beside the rows."""
    print("CASE", residual, block, H, flush=True)
    form, T = (True, True, "tokens"), 11
    v = _dev(_inputs(T, H, residual, block, form, seed=5))
    want = _both(v, 0.5, 1e-6)
    kept = []

    def moved(t, value=77.0):
        if t.dim() == 1:
            big = torch.full((t.shape[0] + 1,), value, dtype=t.dtype, device=DEV)
            y = big[1:]
        else:
            big = torch.full((t.shape[0] * (H + 5) + 3,), value, dtype=t.dtype, device=DEV)
            y = big[3:].view(t.shape[0], H + 5)[:, :H]
        y.copy_(t)
        kept.append((y, big))
        return y
    w = {n: moved(t) for n, t in v.items()}
    how = dict(post=w["post"], gate=w["gate"], scale=0.5, eps=1e-6)
    out = {n: moved(torch.zeros_like(v["x" if n in ("h", "dx") else "y"])) for n in ("h", "n", "dx", "dy", "dgate")}
    n, h, stats = replay.residual_norm(w["x"], w["y"], w["weight"], h=out["h"], n=out["n"], **how)
    g = replay.residual_norm_grad(w["dn"], w["dh"], w["x"], w["y"], w["weight"], stats, dx=out["dx"], dy=out["dy"],
                                  dgate=out["dgate"], **how)
    got = dict(g._asdict(), n=n, h=h, stats=stats)
    for name, t in want.items():
        assert torch.equal(got[name], t), name
    for y, big in kept:
        y.fill_(77.0)
        assert bool((big == 77.0).all())


def test_in_place():
    v = _dev(_inputs(300, 520, BF16, BF16, FORMS[5], seed=6))
    want = _both(v, 1.0, 1e-6)
    x, dh, dn = v["x"].clone(), v["dh"].clone(), v["dn"].clone()
    how = dict(post=v["post"], gate=v["gate"])
    n, h, stats = replay.residual_norm(x, v["y"], v["weight"], h=x, **how)
    assert h is x and torch.equal(n, want["n"]) and torch.equal(h, want["h"])
    g = replay.residual_norm_grad(dn, dh, v["x"], v["y"], v["weight"], stats, dx=dh, dy=dn, **how)
    assert g.dx is dh and g.dy is dn
    for name in ("dx", "dy", "dweight", "dpost", "dgate"):
        assert torch.equal(getattr(g, name), want[name]), name


def test_nothing():
    v = _dev(_inputs(0, 40, F32, F32, FORMS[5], seed=7))
    got = _both(v, 1.0, 1e-6)
    assert got["n"].shape == (0, 40) and got["dx"].shape == (0, 40)
    for name in ("dweight", "dpost", "dgate"):
        assert bool((got[name] == 0).all())


def test_rows_of_zeros_and_infinities():
    """A row of zeros is normed by eps alone; an infinity stays in its row."""
    v = _dev(_inputs(4, 72, BF16, BF16, FORMS[0], seed=8))
    clean = _both(v, 1.0, 1e-6)
    v["x"] = v["x"].clone()
    v["x"][1] = 0.0
    v["x"][2, 5] = float("inf")
    got = _both(v, 1.0, 1e-6)
    assert bool((got["n"][1] == 0).all()) and bool(torch.isfinite(got["dx"][1]).all())
    assert bool(torch.isnan(got["n"][2, 5]))
    for name in ("n", "dx", "stats"):
        for row in (0, 3):
            assert torch.equal(got[name][row], clean[name][row])


@pytest.mark.parametrize("form", FORMS)
def test_against_differences(form):
    """Central differences of a weighted sum of n and h, along a direction of each input:
    the kernels in fp32, sums in fp64.  With steps of 2^-6 of the direction the cubic term
    leaves about 1e-4 of the quotient, and rounding 2^-24 of the sum over the step: 2e-5."""
    v = _dev(_inputs(6, 136, F32, F32, form, seed=9))
    got = _both(v, 0.5, 1e-3)

    def f(u):
        n, h, _ = replay.residual_norm(u["x"], u["y"], u["weight"], post=u["post"], gate=u["gate"], scale=0.5, eps=1e-3)
        return float((n.double() * v["dn"].double()).sum() + (h.double() * v["dh"].double()).sum())
    for name in ("x", "y", "weight", "post", "gate"):
        if v[name] is None:
            continue
        g = got["d" + name].double()
        # along the gradient, so that the quotient is not small
        step = (g / g.abs().max() * 2.0 ** -6).float()
        quotient = (f(dict(v, **{name: v[name] + step})) - f(dict(v, **{name: v[name] - step}))) / 2
        want = float((g * step.double()).sum())
        assert abs(quotient - want) <= 2e-3 * abs(want), (name, quotient, want)


def test_same_bits_every_time():
    v = _dev(_inputs(1300, 1032, BF16, BF16, FORMS[5], seed=10))
    first = _both(v, 1.0, 1e-6)
    for _ in range(3):
        again = _both(v, 1.0, 1e-6)
        assert all(torch.equal(again[n], t) for n, t in first.items())
