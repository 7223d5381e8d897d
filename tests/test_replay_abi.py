"""The replay operators' C ABI (include/c3_replay.h) without a GPU: symbols,
structure sizes and the refusals that return before any GPU work."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "c3_replay.h")

replay = pytest.importorskip("paper_2608_11034_amd.replay")
INVAL, ALIGN, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4
NULL = ctypes.c_void_p(0)
P = ctypes.c_void_p


def _declared():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"^\s*[A-Za-z_][\w\s\*]*?\b(c3_\w+)\s*\(", src, flags=re.M)))


def test_library_exports_every_declared_symbol():
    names = _declared()
    assert "c3_rotary" in names and "c3_attention_grad" in names and "c3_expert_sort" in names
    for n in names:
        assert hasattr(replay._lib(), n), n


def test_struct_sizes_match_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "c3_replay.h"\nint main(void) { printf("%zu %zu %zu %zu\\n", '
                   "sizeof(c3_heads_t), sizeof(c3_attention_t), sizeof(c3_attn_tensor_t), "
                   "sizeof(c3_expert_rows_t)); return 0; }\n")
    exe = tmp_path / "sizes"
    assert os.system(f"gcc -std=c11 -Wall -Wextra -pedantic -I {ROOT}/include {src} -o {exe}") == 0
    want = [int(x) for x in os.popen(str(exe)).read().split()]
    assert want == [ctypes.sizeof(t) for t in (replay.Heads, replay.Attention, replay.AttnTensor,
                                               replay.ExpertRows)]
    assert f"#define C3_MAX_EXPERTS {replay.MAX_EXPERTS}\n" in open(HEADER).read()
    assert f"#define C3_MAX_EXPERT_TOP {replay.MAX_TOP}\n" in open(HEADER).read()


def _rotary(heads=2, dtype=1, batch=1, length=4, dim=64, pos=P(64), pos_bytes=4, freqs=P(64), rot=64,
            layout=0, inverse=0, amplitude=1.0, n=1, in_=256, out=512, stride=(0, 128, 64), out_stride=None,
            table=True):
    t = (replay.Heads * 2)()
    for h in t:
        h.in_, h.out, h.heads = in_, out, heads
        h.in_stride[:] = stride
        h.out_stride[:] = stride if out_stride is None else out_stride
    return replay._lib().c3_rotary(t if table else None, n, dtype, batch, length, dim, pos, pos_bytes,
                                   (ctypes.c_int64 * 2)(0, 1), freqs, rot, layout, inverse, amplitude, NULL)


def test_rotary_refusals():
    assert _rotary(table=False) == INVAL
    assert _rotary(n=0) == INVAL and _rotary(n=3) == INVAL
    assert _rotary(dtype=3) == UNSUPPORTED and _rotary(dtype=9) == UNSUPPORTED
    assert _rotary(dim=0) == INVAL and _rotary(dim=5000) == INVAL
    assert _rotary(rot=0) == INVAL and _rotary(rot=3) == INVAL and _rotary(rot=66) == INVAL
    assert _rotary(pos=NULL) == INVAL and _rotary(freqs=NULL) == INVAL
    assert _rotary(pos_bytes=2) == INVAL and _rotary(pos=P(66)) == ALIGN and _rotary(freqs=P(68)) == ALIGN
    assert _rotary(layout=2) == INVAL and _rotary(amplitude=float("inf")) == INVAL
    assert _rotary(batch=-1) == INVAL and _rotary(heads=-1) == INVAL
    assert _rotary(batch=2 ** 20, length=2 ** 20) == INVAL
    assert _rotary(in_=0) == INVAL and _rotary(in_=257) == ALIGN
    assert _rotary(in_=512, out_stride=(0, 64, 64)) == INVAL      # in place with other strides
    assert _rotary(batch=0) == 0 and _rotary(heads=0) == 0        # nothing to do


def _attention(lens=None, size_only=False, grad=False, ws=P(256), ws_bytes=1 << 30, lse=P(256), ptr=256,
               stride=(8192, 128, 64), **k):
    a = replay.Attention()
    for n, v in dict(dtype=1, heads=4, kv_heads=2, dim=64, causal=1, window=0, scale=0.125, batch=2,
                     q_tokens=32, k_tokens=32, packed=0) .items():
        setattr(a, n, k.get(n, v))
    keep = []
    if lens is not None:
        for n, x in zip(("q_lens", "k_lens"), lens):
            if x is not None:
                keep.append((ctypes.c_int32 * max(1, len(x)))(*x))
                setattr(a, n, ctypes.cast(keep[-1], ctypes.c_void_p))
    L = replay._lib()
    if size_only:
        f = L.c3_attention_grad_workspace_size if grad else L.c3_attention_workspace_size
        return f(ctypes.byref(a))
    t = replay.AttnTensor()
    t.ptr = ptr
    t.stride[:] = stride
    r = ctypes.byref(t)
    if grad:
        return L.c3_attention_grad(ctypes.byref(a), r, r, r, r, r, lse, r, r, r, ws, ws_bytes, NULL)
    return L.c3_attention(ctypes.byref(a), r, r, r, r, lse, ws, ws_bytes, NULL)


@pytest.mark.parametrize("grad", [False, True])
def test_attention_refusals(grad):
    def rc(**k):
        return _attention(grad=grad, **k)
    assert rc(heads=0) == INVAL and rc(kv_heads=0) == INVAL and rc(heads=3) == INVAL
    assert rc(dtype=0) == UNSUPPORTED and rc(dim=60) == UNSUPPORTED and rc(dim=136) == UNSUPPORTED
    assert rc(dim=0) == INVAL and rc(batch=-1) == INVAL and rc(window=-1) == INVAL
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert rc(scale=s) == INVAL
    assert rc(q_tokens=-1) == INVAL and rc(q_tokens=1 << 40) == UNSUPPORTED and rc(k_tokens=1 << 40) == UNSUPPORTED
    assert rc(packed=1) == INVAL                                   # without lengths
    assert rc(lens=([3, 4], None)) == INVAL
    assert rc(lens=([3, -1], [3, 4])) == INVAL and rc(lens=([3, 33], [3, 4])) == INVAL
    assert rc(packed=1, lens=([16, 15], [16, 16])) == INVAL        # sums must meet the tokens
    assert rc(packed=1, lens=([16, 17], [16, 16])) == INVAL
    assert rc(packed=1, lens=([2 ** 31 - 1, 2 ** 31 - 1], [16, 16])) == INVAL
    assert rc(packed=1, batch=0) == INVAL
    assert rc(ptr=0) == INVAL and rc(ptr=264) == ALIGN
    assert rc(stride=(8192, 128, 60)) == ALIGN and rc(stride=(8192, -128, 64)) == INVAL
    assert rc(stride=(8192, 1 << 30, 64)) == UNSUPPORTED
    assert rc(lse=NULL) == INVAL and rc(lse=P(258)) == ALIGN
    assert rc(ws=NULL) == WORKSPACE and rc(ws=P(128)) == WORKSPACE and rc(ws_bytes=8) == WORKSPACE
    assert rc(batch=0) == 0                                        # nothing to do


def test_attention_workspace_sizes():
    for grad in (False, True):
        assert _attention(size_only=True, grad=grad) >= 256
        assert _attention(size_only=True, grad=grad, heads=3) == 0
        many = [1] * 500
        some = _attention(size_only=True, grad=grad, packed=1, batch=100, q_tokens=100, k_tokens=100,
                          lens=(many[:100], many[:100]))
        more = _attention(size_only=True, grad=grad, packed=1, batch=500, q_tokens=500, k_tokens=500,
                          lens=(many, many))
        assert more > some


def _rows(call, tokens=4, top=2, dtype=1, hidden=64, ts=64, ss=64, slot=64, kept=64, args=(P(64), P(64))):
    r = replay.ExpertRows()
    r.dtype, r.top, r.tokens, r.hidden, r.token_stride, r.sorted_stride = dtype, top, tokens, hidden, ts, ss
    r.slot, r.kept = slot, kept
    return getattr(replay._lib(), call)(ctypes.byref(r), *args, NULL)


def test_expert_refusals():
    L = replay._lib()

    def sort(ids=P(64), n=100, e=8, offsets=P(64), source=P(64), slot=P(64), ws=P(256), ws_bytes=1 << 20):
        return L.c3_expert_sort(ids, n, e, offsets, source, slot, ws, ws_bytes, NULL)
    assert L.c3_expert_sort_workspace_size(100, 8) >= 256
    assert L.c3_expert_sort_workspace_size(-1, 8) == 0 and L.c3_expert_sort_workspace_size(1 << 31, 8) == 0
    assert L.c3_expert_sort_workspace_size(100, 0) == 0
    assert L.c3_expert_sort_workspace_size(100, replay.MAX_EXPERTS + 1) == 0
    assert sort(e=0) == INVAL and sort(n=-1) == INVAL and sort(n=1 << 31) == INVAL
    for n in ("ids", "offsets", "source", "slot"):
        assert sort(**{n: NULL}) == INVAL and sort(**{n: P(66)}) == ALIGN
    assert sort(ws=NULL) == WORKSPACE and sort(ws=P(64)) == WORKSPACE and sort(ws_bytes=8) == WORKSPACE
    calls = {"c3_expert_dispatch": (P(64), P(64)), "c3_expert_combine": (P(64), NULL, P(64)),
             "c3_expert_combine_grad": (P(64), P(64), P(64), P(64), P(64))}
    for call, args in calls.items():
        def rc(**k):
            return _rows(call, **{"args": args, **k})
        assert rc(dtype=3) == UNSUPPORTED and rc(top=0) == INVAL and rc(top=65) == INVAL
        assert rc(tokens=-1) == INVAL and rc(tokens=1 << 31) == INVAL and rc(hidden=-1) == INVAL
        assert rc(tokens=1 << 30, top=4) == INVAL
        assert rc(ts=63) == INVAL and rc(ss=0) == INVAL
        assert rc(slot=0) == INVAL and rc(kept=0) == INVAL and rc(slot=66) == ALIGN
        assert rc(tokens=0) == 0
        for i in range(len(args)):
            if args[i] is not NULL and not (call == "c3_expert_combine_grad" and i in (2, 4)):
                assert rc(args=args[:i] + (NULL,) + args[i + 1:]) == INVAL, (call, i)
            if args[i] is not NULL:
                assert rc(args=args[:i] + (P(65),) + args[i + 1:]) == ALIGN, (call, i)


def test_null_structures():
    L = replay._lib()
    assert L.c3_attention_workspace_size(None) == 0 and L.c3_attention_grad_workspace_size(None) == 0
    assert L.c3_expert_dispatch(None, P(64), P(64), NULL) == INVAL


def test_cpu_tensors_are_refused():
    import torch
    x = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16)
    f = torch.ones(32, dtype=torch.float64)
    with pytest.raises(replay.C3Error):
        replay.rotary(x, torch.arange(4), f)
    with pytest.raises(replay.C3Error):
        replay.attention(x, x, x)
    with pytest.raises(replay.C3Error):
        replay.attention_grad(x, x, x, x, x, x)
    with pytest.raises(replay.C3Error):
        replay.expert_sort(torch.zeros((4, 2), dtype=torch.int32), 4)
