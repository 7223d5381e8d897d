"""The embedding and its gradient against plain 64-bit forms: widths, alignments,
frequent rows that many waves share, rows without a token, ids outside the table."""
import pytest
import torch

import replay_ends_plain as plain
from replay_plain import within

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def _randn(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _ids(seed, n, rows, hot=0.0, out=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, rows, (n,), generator=g)
    ids[torch.rand((n,), generator=g) < hot] = rows - 1
    ids[torch.rand((n,), generator=g) < out] = -100
    ids[torch.rand((n,), generator=g) < out / 4] = rows
    return ids


def _strided(x, extra, shift=0):
    """x with rows `extra` elements further apart, the first one `shift` elements in."""
    big = torch.full((x.shape[0] * (x.shape[1] + extra) + shift,), 77.0, dtype=x.dtype, device=DEV)
    y = big[shift:].view(x.shape[0], -1)[:, :x.shape[1]]
    y.copy_(x)
    return y, big


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,rows,hidden", [(1, 1, 8), (1, 7, 1), (5, 3, 64), (16, 100, 1000), (300, 50, 513),
                                           (3000, 1000, 2048)])
def test_lookup(dtype, n, rows, hidden):
    print("CASE", dtype, n, rows, hidden, flush=True)
    table = _randn(1, rows, hidden, dtype=dtype)
    for wide, scale, out in ((torch.int64, 1.0, 0.0), (torch.int32, 0.3, 0.3)):
        ids = _ids(2, n, rows, out=out).to(wide)
        want, bound = plain.embedding(ids, table, scale)
        got = replay.embedding(ids.to(DEV), table.to(DEV), scale=scale)
        within(got, want, bound, "lookup")
        # other strides and alignment: the same bits, and nothing beside the rows
        t, _ = _strided(table, 3, 1)
        o, big = _strided(torch.zeros((n, hidden), dtype=dtype), 5, 3)
        replay.embedding(ids.to(DEV), t, scale=scale, out=o)
        assert torch.equal(o, got)
        o.fill_(77.0)
        assert bool((big == 77.0).all())


def test_lookup_of_nothing():
    table = _randn(1, 5, 16, dtype=torch.bfloat16).to(DEV)
    assert replay.embedding(torch.zeros((0,), dtype=torch.int64, device=DEV), table).shape == (0, 16)
    assert replay.embedding(torch.zeros((3,), dtype=torch.int64, device=DEV), table[:, :0]).shape == (3, 0)


GRADS = [  # tokens, rows, width, share of the most frequent row, share without a row
    (1, 1, 8, 0, 0), (1, 9, 24, 0, 0), (2, 1, 16, 0, 0), (15, 4, 40, 0, 0), (16, 4, 40, 0, 0), (17, 4, 40, 0.5, 0),
    (33, 1, 520, 0, 0), (200, 1000, 1000, 0.3, 0.2), (1025, 37, 65, 0.2, 0.1), (4097, 5000, 96, 0.5, 0.0),
    (1000, 3, 33, 0, 1.0), (16384, 300, 24, 0.1, 0.1), (16385, 300, 24, 0.1, 0.1), (40000, 70000, 16, 0.3, 0.0),
    (20000, 2, 8, 0, 0.5)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,rows,hidden,hot,out", GRADS)
def test_gradient(dtype, n, rows, hidden, hot, out):
    print("CASE", dtype, n, rows, hidden, hot, out, flush=True)
    ids, dout = _ids(3, n, rows, hot, out), _randn(4, n, hidden, dtype=dtype)
    for to in {dtype, torch.float32}:
        want, bound = plain.embedding_grad(dout, ids, rows, 0.7, to)
        got = replay.embedding_grad(dout.to(DEV), ids.to(DEV), rows, scale=0.7, dtype=to)
        assert got.dtype == to
        within(got, want, bound, "gradient")
        # other strides and alignment, 4-byte ids: the same bits
        g, _ = _strided(dout, 3, 1)
        o, big = _strided(torch.zeros((rows, hidden), dtype=to), 5, 3)
        replay.embedding_grad(g, ids.to(torch.int32).to(DEV), rows, scale=0.7, dtable=o)
        assert torch.equal(o, got)
        o.fill_(77.0)
        assert bool((big == 77.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,rows,hidden,hot,out", [(1, 3, 8, 0, 0), (100, 7, 40, 0.4, 0.3), (5000, 9000, 520, 0.3, 0.1),
                                                   (17000, 50, 24, 0.3, 0.1), (50, 7, 9, 0.3, 0.1),
                                                   (600, 300, 513, 0.3, 0.1), (4100, 900, 257, 0.3, 0.1),
                                                   (5000, 100, 1021, 0.3, 0.1)])
def test_accumulated(dtype, n, rows, hidden, hot, out):
    print("CASE", dtype, n, rows, hidden, flush=True)
    ids, dout, old = _ids(5, n, rows, hot, out), _randn(6, n, hidden, dtype=dtype), _randn(7, rows, hidden, dtype=dtype)
    want, bound = plain.embedding_grad(dout, ids, rows, 1.0, dtype, into=old)
    into = old.to(DEV)
    assert replay.embedding_grad(dout.to(DEV), ids.to(DEV), rows, dtable=into, accumulate=True) is into
    within(into, want, bound, "accumulated")
    idle = torch.ones((rows,), dtype=torch.bool)
    idle[ids[(ids >= 0) & (ids < rows)]] = False
    assert torch.equal(into.cpu()[idle], old[idle])         # bit by bit
    # with no tokens nothing happens
    before = into.clone()
    replay.embedding_grad(dout.to(DEV)[:0], ids.to(DEV)[:0], rows, dtable=into, accumulate=True)
    assert torch.equal(into, before)


def test_gradient_of_nothing():
    old = torch.full((5, 16), 3.0, device=DEV)
    dout, ids = torch.zeros((0, 16), device=DEV), torch.zeros((0,), dtype=torch.int32, device=DEV)
    replay.embedding_grad(dout, ids, 5, dtable=old)
    assert bool((old == 0).all())


def test_infinities_stay_in_their_row():
    ids = torch.tensor([2, 0, 2, -1, 1], device=DEV)
    dout = torch.ones((5, 24), dtype=torch.bfloat16, device=DEV)
    dout[3] = float("nan")          # of no row
    dout[1] = float("inf")
    got = replay.embedding_grad(dout, ids, 4).float().cpu()
    assert bool((got[0] == float("inf")).all()) and bool((got[1] == 1).all()) and bool((got[2] == 2).all())
    assert bool((got[3] == 0).all())


def test_against_differences():
    """A linear function: its difference quotient is its gradient, up to rounding."""
    table, g = _randn(8, 6, 16), _randn(9, 20, 16)
    ids = _ids(10, 20, 6)
    grad = replay.embedding_grad(g.to(DEV), ids.to(DEV), 6, scale=2.0).cpu().double()

    def f(t):
        return float((replay.embedding(ids.to(DEV), t.to(DEV), scale=2.0).cpu().double() * g.double()).sum())
    step = torch.randn((6, 16), generator=torch.Generator().manual_seed(11))
    got, want = f(table + step) - f(table - step), 2 * float((grad * step.double()).sum())
    assert abs(got - want) <= 1e-4 * float((grad * step.double()).abs().sum())


def test_same_bits_every_time():
    ids, dout = _ids(12, 30000, 500, 0.2).to(DEV), _randn(13, 30000, 264, dtype=torch.bfloat16).to(DEV)
    first = replay.embedding_grad(dout, ids, 500)
    for _ in range(3):
        assert torch.equal(replay.embedding_grad(dout, ids, 500), first)


@pytest.mark.parametrize("dtype,to", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32),
                                      (torch.float32, torch.float32)])
@pytest.mark.parametrize("n,rows,hidden", [(5000, 32000, 4097), (5000, 32000, 4096), (4097, 10000, 4099),
                                           (300, 40000, 4097), (20000, 100000, 1021)])
def test_zeros_beside_the_sums(dtype, to, n, rows, hidden):
    """Tables of more zeros than the sort's launches take (72 MiB in 16 bits, or 144 MiB for up to
    4,096 tokens): the sums' launch leaves out the rows that the sort has marked.  Rows with a
    token and rows without, over the whole table, which holds something else before."""
    print("CASE", dtype, to, n, rows, hidden, flush=True)
    ids, dout = _ids(14, n, rows, 0.05, 0.1).to(DEV), _randn(15, n, hidden, dtype=dtype).to(DEV)
    ids[:2] = torch.tensor([1, 0], device=DEV)
    kept = (ids >= 0) & (ids < rows)
    at, part = ids[kept], dout[kept].double()
    want = torch.zeros((rows, hidden), dtype=torch.float64, device=DEV).index_add_(0, at, part)
    mag = torch.zeros((rows, hidden), dtype=torch.float64, device=DEV).index_add_(0, at, part.abs_())
    count = torch.bincount(at, minlength=rows)
    assert int((count > 0).sum()) > 100 and int((count == 0).sum()) > 100
    got = torch.full((rows, hidden), 77.0, dtype=to, device=DEV)
    replay.embedding_grad(dout, ids, rows, dtable=got)
    assert bool((got[count == 0] == 0).all())
    # bounds as of the plain 64-bit form: the sum's order, then the rounding to the result's type
    half = torch.finfo(to).eps / 2
    bound = want.abs() * half * 1.01 + mag.mul_((count[:, None] + 3) * 2.0 ** -24) + plain.TINY[to]
    assert bool(((got.double() - want).abs_() <= bound).all())


def test_marks_of_rows_wider_than_the_zeros_beside_the_sort():
    """Rows of more than 24 MiB are all left to the sums' launch, also row 0, whose only token
    stands second in its wave behind another row's."""
    n, hidden = 4097, 6_291_464
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("dout takes 52 GB")
    dout = torch.empty((n, hidden), dtype=torch.bfloat16, device=DEV)
    dout[:2] = torch.tensor([[1.0], [2.0]], device=DEV)
    ids = torch.full((n,), -100, dtype=torch.int64, device=DEV)
    ids[:2] = torch.tensor([1, 0], device=DEV)
    got = torch.full((3, hidden), 77.0, device=DEV)
    replay.embedding_grad(dout, ids, 3, dtable=got)
    for row, value in enumerate((2.0, 1.0, 0.0)):
        assert bool((got[row] == value).all()), row
    del dout
    torch.cuda.empty_cache()
