"""Attention of more sequences than have their slots divided: a workgroup takes a row tile whole.  To the bounds
of cache_ref, with several key heads and row tiles, short and empty sequences among them."""
import numpy as np
import pytest

from test_gpu_attend import _check, _compare, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,N,Hq,Hk,D,dtype,tree", [
    (257, 7, 27, 3, 64, "bfloat16", True),       # 63 rows of a head: one tile of 64
    (257, 13, 15, 3, 64, "float16", False),      # 65: one of 128
    (263, 20, 21, 3, 128, "bfloat16", True),     # 140: two of 128
    (300, 20, 14, 2, 128, "float16", True),
    (258, 43, 9, 3, 64, "float16", True),        # 129: two of 128, the second of one row
    (257, 11, 18, 3, 256, "bfloat16", True),     # 66: two of 64
    (259, 24, 16, 2, 200, "float16", False),     # 192: three of 64
    (261, 3, 2, 2, 24, "bfloat16", True),
    (1000, 1, 4, 1, 128, "bfloat16", False)])
def test_row_tiles_taken_whole(B, N, Hq, Hk, D, dtype, tree):
    _check(B, N, Hq, Hk, D, 16, 40, dtype, tree=tree, seed=B + N)


def test_many_empty_sequences():
    # all of a sequence's tiles are padding, or all but the first one
    d = _inputs(260, 20, 28, 2, 64, 16, 30, "bfloat16", 1, True)
    d["k"], d["v"] = d["k"].nan_to_num(0.3), d["v"].nan_to_num(0.3)
    M = d["pages"].shape[1]
    d["pages"] = np.arange(260 * M).reshape(260, M)
    d["lengths"] = np.arange(260) % 4
    _compare(d, _run(d))
    d["lengths"][:] = 0
    out, lse = _run(d)
    assert not out.any() and (lse == -float("inf")).all()


def test_the_same_bits_with_kept_buffers_and_in_a_graph():
    import torch
    from paper_2002_00876_amd import binding
    from test_gpu_attend import _ints
    d = _inputs(270, 20, 14, 2, 128, 16, 60, "bfloat16", 2, True)
    want = _run(d)
    assert binding.tree_workspace_bytes(270, 20, 14, 2, 128) == 0
    out = (torch.full_like(want[0], 7), torch.full_like(want[1], 7))
    t = {x: d[x].cuda() if x in "qkv" else _ints(d[x]) for x in d}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.tree_attention(t["q"], t["k"], t["v"], t["pages"], t["starts"], t["parents"], t["lengths"],
                               out=out)
    for _ in range(3):
        out[0].fill_(5), out[1].fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
