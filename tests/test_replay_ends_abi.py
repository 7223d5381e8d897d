"""The embedding, residual norm and vocabulary loss of include/c3_replay.h without a
GPU: structure sizes, packed arguments and the refusals that return before any GPU work."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "c3_replay.h")

replay = pytest.importorskip("paper_2608_11034_amd.replay")
INVAL, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4
P = ctypes.c_void_p
F32, BF16, F16 = replay.F32, replay.BF16, replay.F16
NAN, INF = float("nan"), float("inf")


def test_struct_sizes_match_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "c3_replay.h"\nint main(void) { printf("%zu %zu %zu %zu\\n", '
                   "sizeof(c3_embedding_t), sizeof(c3_residual_norm_t), sizeof(c3_rows_t), "
                   "sizeof(c3_vocab_loss_t)); return 0; }\n")
    exe = tmp_path / "sizes"
    assert os.system(f"gcc -std=c11 -Wall -Wextra -pedantic -I {ROOT}/include {src} -o {exe}") == 0
    want = [int(x) for x in os.popen(str(exe)).read().split()]
    assert want == [ctypes.sizeof(t) for t in (replay.Embedding, replay.ResidualNorm, replay.RowsOf, replay.VocabLoss)]
    assert f"#define C3_MAX_NORM_HIDDEN {replay.MAX_NORM_HIDDEN}\n" in open(HEADER).read()


@pytest.mark.parametrize("form,struct", [(replay._EMBEDDING, replay.Embedding),
                                         (replay._RESIDUAL_NORM, replay.ResidualNorm),
                                         (replay._ROWS, replay.RowsOf), (replay._VOCAB_LOSS, replay.VocabLoss)])
def test_packed_arguments(form, struct):
    values = list(range(1, len(struct._fields_) + 1))
    raw = form.pack(*values)
    assert len(raw) == ctypes.sizeof(struct)
    s = struct.from_buffer_copy(raw)
    assert [getattr(s, n) for n, _ in struct._fields_] == values


def _struct(cls, values):
    s = cls()
    for n, v in values.items():
        setattr(s, n, v)
    return s


def _embedding(ids=64, table=256, out=512, null=False, **k):
    a = _struct(replay.Embedding, {**dict(dtype=BF16, id_bytes=8, tokens=4, rows=10, hidden=16, row_stride=16,
                                          table_stride=16, scale=1.0), **k})
    return replay._lib().c3_embedding(None if null else ctypes.byref(a), P(ids), P(table), P(out), P(0))


def _embedding_grad(dout=256, ids=64, dtable=512, table_dtype=BF16, accumulate=0, ws=256, ws_bytes=1 << 30, null=False,
                    size=False, **k):
    a = _struct(replay.Embedding, {**dict(dtype=BF16, id_bytes=8, tokens=4, rows=10, hidden=16, row_stride=16,
                                          table_stride=16, scale=1.0), **k})
    p = None if null else ctypes.byref(a)
    if size:
        return replay._lib().c3_embedding_grad_workspace_size(p)
    return replay._lib().c3_embedding_grad(p, P(dout), P(ids), P(dtable), table_dtype, accumulate, P(ws), ws_bytes, P(0))


@pytest.mark.parametrize("call", [_embedding, _embedding_grad])
def test_embedding_refusals(call):
    assert call(null=True) == INVAL
    for k in (dict(tokens=-1), dict(tokens=1 << 31), dict(rows=0), dict(rows=1 << 31), dict(hidden=-1),
              dict(hidden=1 << 31), dict(id_bytes=2), dict(scale=NAN), dict(scale=INF), dict(row_stride=15),
              dict(table_stride=15), dict(row_stride=-16), dict(ids=0)):
        assert call(**k) == INVAL, k
    assert call(dtype=7) == UNSUPPORTED
    assert call(ids=68) == ALIGN and call(id_bytes=4, ids=66) == ALIGN
    assert call(hidden=0) == 0                                      # nothing to do
    assert call(tokens=(1 << 31) - 1, hidden=1 << 20, row_stride=1 << 20, table_stride=1 << 20,
                **({"ws_bytes": 1 << 62} if call is _embedding_grad else {})) == UNSUPPORTED


def test_embedding_pointers():
    assert _embedding(table=0) == INVAL and _embedding(out=0) == INVAL and _embedding(out=256) == INVAL
    assert _embedding(table=257) == ALIGN and _embedding(out=513) == ALIGN and _embedding(tokens=0, ids=0) == 0
    assert _embedding_grad(dout=0) == INVAL and _embedding_grad(dtable=0) == INVAL
    assert _embedding_grad(dtable=256) == INVAL                     # the output's gradient itself
    assert _embedding_grad(dout=257) == ALIGN and _embedding_grad(dtable=513) == ALIGN
    assert _embedding_grad(dtable=514, table_dtype=F32) == ALIGN
    assert _embedding_grad(table_dtype=F16) == UNSUPPORTED
    assert _embedding_grad(ws=0) == WORKSPACE and _embedding_grad(ws=64) == WORKSPACE
    assert _embedding_grad(ws_bytes=8) == WORKSPACE
    assert _embedding_grad(tokens=0, accumulate=1) == 0
    assert _embedding_grad(size=True) >= 256 and _embedding_grad(size=True, rows=0) == 0
    assert _embedding_grad(size=True, null=True) == 0
    assert _embedding_grad(size=True, tokens=100000) > _embedding_grad(size=True, tokens=1000)


ROWS = dict(x=256, y=512, gate=0, h=1024, n=2048, dn=4096, dh=8192, dx=16384, dy=32768, dgate=0)


def _norm(grad, size=False, null=False, weight=64, post=0, stats=64, sums=64, ws=256, ws_bytes=1 << 30, stride=16, **k):
    names = {n: k.pop(n) for n in list(k) if n in ROWS}
    a = _struct(replay.ResidualNorm, {**dict(dtype=BF16, residual=BF16, tokens=4, hidden=16, scale=1.0, eps=1e-6,
                                             gate=0), **{("gate" if n == "kind" else n): v for n, v in k.items()}})
    p = None if null else ctypes.byref(a)
    L = replay._lib()
    if size:
        return L.c3_residual_norm_grad_workspace_size(p)
    keep = {}
    for n, v in {**ROWS, **names}.items():
        at, st = v if isinstance(v, tuple) else (v, stride)
        keep[n] = _struct(replay.RowsOf, dict(ptr=at, stride=st))
    r = {n: ctypes.byref(v) for n, v in keep.items()}
    if grad:
        return L.c3_residual_norm_grad(p, r["dn"], r["dh"], r["x"], r["y"], r["gate"], P(weight), P(post), P(stats),
                                       r["dx"], r["dy"], r["dgate"], P(sums), P(ws), ws_bytes, P(0))
    return L.c3_residual_norm(p, r["x"], r["y"], r["gate"], P(weight), P(post), r["h"], r["n"], P(stats), P(0))


@pytest.mark.parametrize("grad", [False, True])
def test_norm_refusals(grad):
    def rc(**k):
        return _norm(grad, **k)
    assert rc(null=True) == INVAL
    for k in (dict(tokens=-1), dict(tokens=1 << 31), dict(hidden=0), dict(kind=-1), dict(kind=3), dict(scale=NAN),
              dict(scale=INF), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(weight=0), dict(stats=0), dict(x=0),
              dict(stride=15), dict(kind=1), dict(kind=2),                       # a gate that is not there
              dict(y=0, post=64), dict(y=0, kind=1, gate=64)):
        assert rc(**k) == INVAL, k
    assert rc(dtype=9) == UNSUPPORTED and rc(dtype=F32) == UNSUPPORTED and rc(residual=F16) == UNSUPPORTED
    assert rc(hidden=16385, stride=20000) == UNSUPPORTED
    assert rc(x=257) == ALIGN and rc(residual=F32, x=258) == ALIGN and rc(weight=65) == ALIGN and rc(stats=68) == ALIGN
    assert rc(post=65) == ALIGN and rc(kind=1, gate=65) == ALIGN
    outs = ("dx", "dy") if grad else ("h", "n")
    ins = ("x", "y") + (("dn", "dh") if grad else ())
    for o in outs:
        assert rc(**{o: 0}) == INVAL, o
        for i in ins:
            if (o, i) in (("h", "x"), ("dx", "dh"), ("dy", "dn")):
                assert rc(**{o: (ROWS[i], 24)}) == INVAL, (o, i)    # in place with another stride
            else:
                assert rc(**{o: ROWS[i]}) == INVAL, (o, i)
    assert rc(**{outs[1]: ROWS[outs[0]]}) == INVAL
    if grad:
        assert rc(dn=0) == INVAL and rc(sums=0) == INVAL and rc(sums=66) == ALIGN
        assert rc(kind=2, gate=128, dgate=0) == INVAL
        assert rc(ws=0) == WORKSPACE and rc(ws=64) == WORKSPACE and rc(ws_bytes=8) == WORKSPACE
        assert _norm(True, size=True) >= 256 and _norm(True, size=True, hidden=0) == 0
    else:
        assert rc(tokens=0) == 0


def _loss(grad, size=False, null=False, x=256, weight=512, targets=64, loss=64, lse=128, dloss=64, dloss_stride=1,
          dx=1024, dx_stride=16, dweight=2048, dweight_stride=16, ws=256, ws_bytes=1 << 40, **k):
    a = _struct(replay.VocabLoss, {**dict(dtype=BF16, target_bytes=8, tokens=4, hidden=16, rows=10, x_stride=16,
                                          weight_stride=16, scale=1.0), **k})
    p = None if null else ctypes.byref(a)
    L = replay._lib()
    if size:
        return (L.c3_vocab_loss_grad_workspace_size if grad else L.c3_vocab_loss_workspace_size)(p)
    if grad:
        return L.c3_vocab_loss_grad(p, P(dloss), dloss_stride, P(x), P(weight), P(targets), P(lse), P(dx), dx_stride,
                                    P(dweight), dweight_stride, P(ws), ws_bytes, P(0))
    return L.c3_vocab_loss(p, P(x), P(weight), P(targets), P(loss), P(lse), P(ws), ws_bytes, P(0))


@pytest.mark.parametrize("grad", [False, True])
def test_loss_refusals(grad):
    def rc(**k):
        return _loss(grad, **k)
    assert rc(null=True) == INVAL
    for k in (dict(tokens=-1), dict(tokens=1 << 31), dict(rows=0), dict(rows=1 << 31), dict(hidden=0),
              dict(target_bytes=2), dict(scale=NAN), dict(scale=INF), dict(x_stride=8), dict(weight_stride=8),
              dict(x_stride=-16), dict(x=0), dict(weight=0), dict(targets=0), dict(lse=0)):
        assert rc(**k) == INVAL, k
    for k in (dict(dtype=F32), dict(hidden=12), dict(hidden=1 << 20), dict(rows=(1 << 31) - 1),
              dict(tokens=1 << 24, rows=1 << 24), dict(x_stride=1 << 22), dict(weight_stride=1 << 22)):
        assert rc(**k) == UNSUPPORTED, k
    for k in (dict(x=264), dict(weight=264), dict(x_stride=20), dict(weight_stride=20), dict(targets=68), dict(lse=66)):
        assert rc(**k) == ALIGN, k
    assert rc(ws=0) == WORKSPACE and rc(ws=64) == WORKSPACE and rc(ws_bytes=8) == WORKSPACE
    assert _loss(grad, size=True) >= 256 and _loss(grad, size=True, rows=0) == 0 and _loss(grad, size=True, null=True) == 0
    if grad:
        for k in (dict(dloss=0), dict(dloss_stride=-1), dict(dx=0), dict(dweight=0), dict(dx=256), dict(dx=512),
                  dict(dx=2048), dict(dweight=256), dict(dweight=512), dict(dx_stride=8), dict(dweight_stride=8)):
            assert rc(**k) == INVAL, k
        for k in (dict(dx=1032), dict(dweight=2056), dict(dx_stride=20), dict(dweight_stride=20), dict(dloss=66)):
            assert rc(**k) == ALIGN, k
    else:
        assert rc(loss=0) == INVAL and rc(loss=128) == INVAL and rc(loss=66) == ALIGN
        assert rc(tokens=0) == 0


def test_loss_workspace_holds_a_piece():
    """The softmax of 512 MiB at a time, not of the whole vocabulary."""
    some = _loss(True, size=True, tokens=8192, hidden=4096, rows=1 << 20, x_stride=4096, weight_stride=4096)
    assert (512 << 20) < some < (900 << 20)


def test_loss_workspace_of_few_and_many_tokens():
    """512 MiB of d with the second rows that up to 128 tokens have, and beyond 131,072 tokens
    2,048 rows of the vocabulary: 4 KiB a token."""
    def size(tokens, rows):
        return _loss(True, size=True, tokens=tokens, hidden=16, rows=rows)
    for tokens in (64, 127, 128):
        assert size(tokens, 3_000_000) <= (512 << 20) + (1 << 20), tokens
    for tokens in (129, 1000, 131_072):
        assert size(tokens, 1_000_000) <= (512 << 20) + 2048 * tokens + (64 << 20), tokens
    for tokens in (200_000, 1 << 20):
        assert 4096 * tokens < size(tokens, 8000) <= (4096 + 2048) * tokens + (64 << 20), tokens


def test_cpu_tensors_and_graphs_are_refused():
    x = torch.zeros((4, 16), dtype=torch.bfloat16)
    ids, w = torch.zeros((4,), dtype=torch.int64), torch.ones((16,), dtype=torch.bfloat16)
    for call in (lambda: replay.embedding(ids, x), lambda: replay.embedding_grad(x, ids, 3),
                 lambda: replay.residual_norm(x, None, w),
                 lambda: replay.residual_norm_grad(x, None, x, None, w, torch.zeros((4, 2))),
                 lambda: replay.vocab_loss(x, x, ids),
                 lambda: replay.vocab_loss_grad(torch.zeros(4), x, x, ids, torch.zeros(4))):
        with pytest.raises(replay.C3Error):
            call()
