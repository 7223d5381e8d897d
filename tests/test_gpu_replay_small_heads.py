"""Attention of small heads on walks that are divided into few and many parts, against
the plain 64-bit forms (replay_plain)."""
import pytest
import torch

import replay_plain as plain

pytestmark = pytest.mark.gpu

replay = pytest.importorskip("paper_2608_11034_amd.replay")
DEV = "cuda"


@pytest.mark.parametrize("parts", [2, 5, 9, 13, 16, 17])
@pytest.mark.parametrize("dim", [8, 16, 24, 40])
@pytest.mark.parametrize("q_len,keys", [(1, 256), (130, 512)])      # the keys of a part
def test_every_part_is_joined(q_len, keys, dim, parts):
    """The parts of a walk reach the output whatever the head's size, of one row and of
    tiles of 128."""
    print("CASE", q_len, dim, parts, flush=True)
    k_len = keys * (parts - 1) + 100
    gen = torch.Generator().manual_seed(51)
    q, g = (torch.randn((q_len, 1, dim), generator=gen).to(torch.bfloat16) for _ in range(2))
    k, v = (torch.randn((k_len, 1, dim), generator=gen).to(torch.bfloat16) for _ in range(2))
    v += 1                              # a part left out shows in every element
    Q, K, V, G = (t.to(DEV) for t in (q, k, v, g))
    how = dict(q_lens=[q_len], k_lens=[k_len])
    out, lse = replay.attention(Q, K, V, **how)
    grads = replay.attention_grad(G, Q, K, V, out, lse, **how)
    want = plain.attention(q, k, v, [q_len], [k_len], False, 0, dim ** -0.5, g, torch.bfloat16)
    for n, t in zip(("out", "lse", "dq", "dk", "dv"), (out, lse) + grads):
        plain.within(t, want[n], want[n + "_bound"], n)
