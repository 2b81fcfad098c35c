"""Attention of drafted tokens over a paged cache against float64, to the bounds of cache_ref."""
import numpy as np
import pytest

import cache_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

NONE = -1


def _inputs(B, N, Hq, Hk, D, S, past, dtype, seed, tree, spare=2, wide=1):
    """Host arrays of a cache in use: pages anywhere, everything that is not seen is NaN."""
    import torch
    rng = np.random.default_rng(seed)
    starts = rng.integers(0, past, endpoint=True, size=B)
    starts[0] = past
    lengths = rng.integers(0, N, endpoint=True, size=B)
    lengths[-1] = N
    M = -(-(past + N) // S) + wide
    P = B * M + spare
    pages = rng.permutation(P)[:B * M].reshape(B, M)
    t = getattr(torch, dtype)

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(t)

    k, v = normal(P, S, Hk, D), normal(P, S, Hk, D) + 0.5
    seen = torch.zeros(P, S, dtype=torch.bool)
    for b in range(B):
        j = np.arange(starts[b] + lengths[b])
        seen[pages[b, j // S], j % S] = True
        pages[b, -(-(int(starts[b]) + int(lengths[b])) // S):] = rng.choice([-1, P + 7, 2 ** 31 - 1])
    k[~seen], v[~seen] = float("nan"), float("nan")
    parents = None
    if tree:
        parents = np.maximum(np.arange(N)[None] - rng.integers(1, 9, size=(B, N)), -1)
    return dict(q=normal(B, N, Hq, D) * 1.5, k=k, v=v, pages=pages, starts=starts, lengths=lengths,
                parents=parents)


def _ints(x):
    import torch
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _run(d, scale=None, **kw):
    import torch
    from paper_2002_00876_amd import binding
    out = binding.tree_attention(d["q"].cuda(), d["k"].cuda(), d["v"].cuda(), _ints(d["pages"]),
                                 _ints(d["starts"]), _ints(d["parents"]), _ints(d["lengths"]),
                                 scale=scale, **kw)
    torch.cuda.synchronize()
    return out


def _compare(d, got, scale=None):
    dtype = str(d["q"].dtype).replace("torch.", "")
    B, N, _, D = d["q"].shape
    lengths = [N] * B if d["lengths"] is None else d["lengths"]
    nan = np.nan_to_num
    out, lse, off, loff = R.attend(d["q"].double().numpy(), nan(d["k"].double().numpy()),
                                   nan(d["v"].double().numpy()), d["pages"], d["starts"], lengths,
                                   d["parents"], D ** -0.5 if scale is None else scale, dtype)
    o, l = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
    none = lse == -np.inf
    assert np.all(l[none] == -np.inf) and np.all(o[none] == 0)
    with np.errstate(invalid="ignore"):
        far, lfar = np.abs(o - out) - off, np.where(none, 0, np.abs(l - lse) - loff)
    assert not np.isnan(o).any() and far.max() <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))
    assert not np.isnan(l).any() and lfar.max() <= 0, lfar.max()


def _check(B, N, Hq, Hk, D, S, past, dtype="bfloat16", tree=True, scale=None, seed=0, **kw):
    say(f"attend B={B} N={N} Hq={Hq} Hk={Hk} D={D} S={S} past={past} {dtype} tree={tree}")
    d = _inputs(B, N, Hq, Hk, D, S, past, dtype, seed, tree, **kw)
    _compare(d, _run(d, scale), scale)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("D", [8, 24, 64, 80, 96, 128, 136, 256])
@pytest.mark.parametrize("N,Hq,Hk", [(1, 4, 4), (5, 8, 2), (3, 21, 3), (16, 4, 1), (33, 8, 2)])
def test_heads(dtype, D, N, Hq, Hk):
    _check(3, N, Hq, Hk, D, 16, 300, dtype, seed=D + N)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("past", [0, 1, 31, 32, 63, 64, 65, 127, 128, 129, 1000])
@pytest.mark.parametrize("N", [1, 2, 16, 31, 32, 33, 64, 65])
def test_lengths(past, N, tree):
    _check(2, N, 2, 1, 64, 16, past, tree=tree, seed=past + N)


@pytest.mark.parametrize("S", [1, 3, 16, 48, 64, 100, 256, 4096])
@pytest.mark.parametrize("N,G", [(4, 2), (40, 2)])
def test_pages(S, N, G):
    _check(2, N, 2 * G, 2, 64, S, 777, seed=S)


@pytest.mark.parametrize("N,Hq,Hk,D", [(255, 2, 1, 64), (256, 1, 1, 128), (256, 8, 1, 64), (129, 7, 1, 256)])
@pytest.mark.parametrize("tree", [False, True])
def test_most_drafts(N, Hq, Hk, D, tree):
    _check(2, N, Hq, Hk, D, 64, 500, tree=tree, seed=N)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,Hq,Hk,D", [(1, 2, 1, 64), (7, 4, 1, 128), (24, 4, 1, 128), (40, 4, 1, 64)])
def test_long_contexts(dtype, N, Hq, Hk, D):
    _check(2, N, Hq, Hk, D, 48, 30000, dtype, seed=N)


def test_sharp_and_flat():
    # scores whose softmax is one slot's, and scores that are all alike
    for scale in (1e-6, 3.0, 30.0):
        for N in (2, 20, 50):
            _check(2, N, 2, 1, 128, 16, 400, "float16", scale=scale, seed=N)


def test_many_small_numerators():
    # one slot far above 40000 others that together weigh as much as it does
    import torch
    for N, G in ((1, 2), (20, 2), (40, 2)):
        for dtype in ("float16", "bfloat16"):
            d = _inputs(1, N, G, 1, 64, 64, 40000, dtype, 1, False)
            d["q"].zero_()
            d["q"][..., 0] = 8.0
            d["k"][~d["k"].isnan()] = 0.0
            d["k"][int(d["pages"][0, 0]), 3, 0, 0] = 10.6       # exp(-10.6) = 1 / 40000
            _compare(d, _run(d))


@pytest.mark.parametrize("B", [1, 5, 63, 64, 65, 129, 255, 256, 257, 700])
@pytest.mark.parametrize("N,tree", [(1, False), (6, True)])
def test_batches(B, N, tree):
    _check(B, N, 2, 1, 64, 16, 150, tree=tree, seed=B)


def test_one_long_sequence_among_short_ones():
    d = _inputs(40, 3, 4, 2, 64, 16, 6000, "bfloat16", 5, True)
    d["starts"] = np.where(np.arange(40) == 7, 6000, np.minimum(d["starts"], 20))
    rng = np.random.default_rng(0)
    M, P = d["pages"].shape[1], d["k"].shape[0]
    d["pages"] = rng.permutation(P)[:40 * M].reshape(40, M)
    d["k"], d["v"] = d["k"].nan_to_num(0.3), d["v"].nan_to_num(0.3)
    _compare(d, _run(d))


@pytest.mark.parametrize("D", [64, 128, 200])
@pytest.mark.parametrize("N,G", [(3, 2), (40, 2), (60, 5)])
def test_stretches_of_several_sequences(D, N, G):
    # more units than workgroups: stretches that end within one sequence and begin within another
    _check(90, N, G, 1, D, 16, 900, seed=D + N, wide=0)


@pytest.mark.parametrize("Hk", [3, 7, 12, 40])
def test_heads_that_do_not_divide_the_workgroups(Hk):
    for N in (2, 70):
        _check(5, N, Hk, Hk, 64, 16, 700, seed=Hk)


def test_more_heads_than_workgroups():
    _check(2, 2, 600, 600, 8, 16, 300, seed=1)


def test_empty_rows():
    # no drafts at all, nothing before the drafts, slots past the table
    d = _inputs(3, 4, 4, 2, 64, 16, 40, "bfloat16", 2, True)
    d["lengths"] = np.array([0, 0, 0])
    o, l = _run(d)
    assert (o == 0).all() and (l == -float("inf")).all()
    d = _inputs(3, 4, 4, 2, 64, 16, 0, "bfloat16", 2, True, wide=0)
    _compare(d, _run(d))
    d = _inputs(2, 20, 4, 2, 64, 16, 30, "bfloat16", 2, False, wide=0)
    d["k"], d["v"] = d["k"].nan_to_num(0.3), d["v"].nan_to_num(0.3)
    d["pages"] = np.arange(8).reshape(2, 4)[:, :3]
    d["starts"], d["lengths"] = np.array([40, 48]), np.array([20, 20])    # 48 slots in all
    _compare(d, _run(d))
    d["starts"], d["lengths"] = np.array([-5, 4000]), np.array([-2, 99])  # clamped
    _compare(d, _run(d))


def test_pages_that_are_not_there_are_zeros():
    for N in (3, 40):
        d = _inputs(2, N, 4, 2, 64, 16, 200, "bfloat16", 2, True)
        d["pages"][0, 2], d["pages"][1, 1] = -1, d["k"].shape[0]
        _compare(d, _run(d))


def test_parents_out_of_range_continue_the_text():
    for N in (6, 70):
        d = _inputs(2, N, 2, 1, 64, 16, 50, "bfloat16", 3, True)
        d["parents"][:, 1], d["parents"][:, 2], d["parents"][:, 3] = 1, 5, -2 ** 31
        d["parents"][:, 4] = 2 ** 31 - 1
        _compare(d, _run(d))


def test_strides():
    # a cache with heads before tokens, queries that are a view of a wider product, no lengths
    import torch
    from paper_2002_00876_amd import binding
    for N in (3, 40):
        d = _inputs(2, N, 4, 2, 64, 16, 200, "float16", 4, True)
        d["lengths"] = None
        d["k"], d["v"] = d["k"].nan_to_num(0.1), d["v"].nan_to_num(0.1)
        P, M = d["k"].shape[0], d["pages"].shape[1]
        d["pages"] = np.random.default_rng(1).permutation(P)[:2 * M].reshape(2, M)
        k = d["k"].transpose(1, 2).contiguous().cuda().transpose(1, 2)
        v = d["v"].transpose(1, 2).contiguous().cuda().transpose(1, 2)
        wide = torch.full((2, N, 9, 64), float("nan"), dtype=torch.float16, device="cuda")
        wide[:, :, 2:6] = d["q"].cuda()
        got = binding.tree_attention(wide[:, :, 2:6], k, v, _ints(d["pages"]), _ints(d["starts"]),
                                     _ints(d["parents"]))
        _compare(d, got)
        odd = torch.zeros((2, N, 4, 65), dtype=torch.float16, device="cuda")   # heads not aligned
        odd[..., 1:] = d["q"].cuda()
        again = binding.tree_attention(odd[..., 1:], k, v, _ints(d["pages"]), _ints(d["starts"]),
                                       _ints(d["parents"]))
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_the_same_bits_again_and_in_kept_buffers():
    import torch
    from paper_2002_00876_amd import binding
    for N, Hq in ((2, 4), (30, 8)):
        d = _inputs(9, N, Hq, 2, 128, 16, 3000, "bfloat16", 6, True)
        a = _run(d)
        ws = torch.full((binding.tree_workspace_bytes(9, N, Hq, 2, 128),), 255, dtype=torch.uint8,
                        device="cuda")
        out = (torch.full_like(a[0], 7), torch.full_like(a[1], 7))
        b = _run(d, ws=ws, out=out)
        assert b[0] is out[0] and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_captured():
    """One graph of two calls that share a workspace, replayed as the lengths and the cache change."""
    import torch
    from paper_2002_00876_amd import binding
    d = _inputs(4, 5, 8, 2, 64, 16, 900, "bfloat16", 8, True)
    d["k"], d["v"] = d["k"].nan_to_num(0.3), d["v"].nan_to_num(0.3)
    P, M = d["k"].shape[0], d["pages"].shape[1]
    d["pages"] = np.random.default_rng(1).permutation(P)[:4 * M].reshape(4, M)
    t = {x: d[x].cuda() if x in "qkv" else _ints(d[x]) for x in d}
    ws = torch.empty(binding.tree_workspace_bytes(4, 5, 8, 2, 64), dtype=torch.uint8, device="cuda")

    def call(q):
        return binding.tree_attention(q, t["k"], t["v"], t["pages"], t["starts"], t["parents"],
                                      t["lengths"], ws=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(t["q"])
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = call(t["q"])
        two = call(one[0])
    for step in range(4):
        t["starts"].copy_(_ints(np.clip(d["starts"] - 100 * step, 0, None)))
        t["lengths"].copy_(_ints((d["lengths"] + step) % 6))
        t["k"].mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        want = call(t["q"])
        again = call(want[0])
        torch.cuda.synchronize()
        assert torch.equal(one[0], want[0]) and torch.equal(one[1], want[1]), step
        assert torch.equal(two[0], again[0]) and torch.equal(two[1], again[1]), step


def test_a_cache_past_32_bits():
    # pages more than 2^32 bytes, and 2^31 elements, from the cache's start
    import torch
    from paper_2002_00876_amd import binding
    P, S, Hk, D = 1100, 1024, 16, 128
    k = torch.zeros((P, S, Hk, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    at = [1099, 1050]
    for p in at:
        k[p] = torch.randn((S, Hk, D), generator=g, device="cuda")
        v[p] = torch.randn((S, Hk, D), generator=g, device="cuda")
    for N in (2, 48):
        q = torch.randn((1, N, 16, D), generator=g, device="cuda").to(torch.bfloat16)
        far = binding.tree_attention(q, k, v, _ints([at]), _ints([1500]))
        near = binding.tree_attention(q, k[at].clone(), v[at].clone(), _ints([[0, 1]]), _ints([1500]))
        torch.cuda.synchronize()
        assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
        assert far[0].float().abs().max() > 0.01


def test_another_stream():
    import torch
    d = _inputs(3, 5, 8, 2, 64, 16, 900, "bfloat16", 9, True)
    want = _run(d)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _run(d)
    side.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_checked(monkeypatch):
    from paper_2002_00876_amd import binding
    monkeypatch.setenv("TS_CHECK", "1")
    d = _inputs(2, 5, 4, 2, 64, 16, 90, "bfloat16", 9, True)
    _run(d)
    for name, at, value, code in (("starts", 1, -1, -4), ("starts", 0, 10 ** 6, -4),
                                  ("lengths", 1, 6, -4), ("pages", (0, 0), -1, -6),
                                  ("parents", (1, 2), 2, -6), ("parents", (1, 2), -2, -6)):
        bad = {**d, name: d[name].copy()}
        bad[name][at] = value
        with pytest.raises(binding.TsError) as e:
            _run(bad)
        assert e.value.code == code, name


def test_shared_pages():
    # two sequences whose text begins alike read the same pages; their drafts lie in pages of their own
    d = _inputs(2, 20, 4, 2, 64, 16, 200, "bfloat16", 11, True)
    d["k"], d["v"] = d["k"].nan_to_num(0.2), d["v"].nan_to_num(0.2)
    P, M = d["k"].shape[0], d["pages"].shape[1]
    d["pages"] = np.random.default_rng(2).permutation(P)[:2 * M].reshape(2, M)
    d["pages"][1, :9] = d["pages"][0, :9]
    d["starts"], d["lengths"] = np.array([150, 144]), np.array([20, 17])
    _compare(d, _run(d))


def test_two_streams_at_once():
    import torch
    from paper_2002_00876_amd import binding
    cases = [_inputs(12, N, 8, 2, 128, 16, 3000, "bfloat16", N, True) for N in (4, 40)]
    want = [_run(d) for d in cases]
    args = [(d["q"].cuda(), d["k"].cuda(), d["v"].cuda(), _ints(d["pages"]), _ints(d["starts"]),
             _ints(d["parents"]), _ints(d["lengths"])) for d in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = []
        for s, a in zip(streams, args):
            with torch.cuda.stream(s):
                got.append(binding.tree_attention(*a))
        torch.cuda.synchronize()
        for g, x in zip(got, want):
            assert torch.equal(g[0], x[0]) and torch.equal(g[1], x[1])
