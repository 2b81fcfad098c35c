"""Attention whose scores are as large as they may be, against float64."""
import numpy as np
import pytest

import cache_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _large(sizes, dtype, N, G, scale, past=200, S=16, D=64, seed=0):
    """(q, k, v) of one key head a sequence, which lies in pages of its own: even drafts' scores are
    +-2^size times up to 4 and have two values, the larger one at some slots, the smaller one at the others;
    odd drafts' are ordinary.  Every other sequence has positive ones."""
    import torch
    rng = np.random.default_rng(seed)
    t = getattr(torch, dtype)
    B, M = len(sizes), -(-(past + N) // S)
    q = torch.from_numpy(rng.standard_normal((B, N, G, D))).to(t)
    k = torch.from_numpy(rng.standard_normal((B * M, S, 1, D))).to(t)
    v = torch.from_numpy(rng.standard_normal((B * M, S, 1, D)) + 0.5).to(t)
    q[:, 1::2, :, 1:] *= 0.2
    q[:, 1::2, :, 0] = 0
    q[:, ::2] = 0
    step = 2.0 ** (-7 if dtype == "bfloat16" else -10)
    for b, size in enumerate(sizes):
        e = size - int(np.log2(scale))
        sign = 1 if b % 2 else -1
        for i in range(0, N, 2):
            a = 1 + step * rng.integers(0, int(1 / step), size=G)
            q[b, i, :, 0] = torch.from_numpy(a * sign * 2.0 ** (e // 2)).to(t)
        top = 1 + step * rng.integers(1, int(1 / step) - 1)
        level = top + step * sign * np.where(rng.random((M, S)) < 0.1, 0, -1)
        k[b * M:(b + 1) * M, :, 0, 0] = torch.from_numpy(level).to(t) * 2.0 ** (e - e // 2)
    return q, k, v, np.arange(B * M).reshape(B, M), np.full(B, past)


def _check(sizes, dtype, N, G, scale, parents=None, seed=0):
    import torch
    from paper_2002_00876_amd import binding
    say(f"attend limits {dtype} N={N} G={G} scale={scale} 2^{sizes[0]}..{sizes[-1]}")
    q, k, v, pages, starts = _large(sizes, dtype, N, G, scale, seed=seed)
    assert torch.isfinite(q).all() and torch.isfinite(k).all()
    got, got_lse = binding.tree_attention(q.cuda(), k.cuda(), v.cuda(), _ints(pages), _ints(starts),
                                          None if parents is None else _ints(parents), scale=scale)
    got, got_lse = got.double().cpu().numpy(), got_lse.double().cpu().numpy()
    B = len(sizes)
    out, lse, off, loff = R.attend(q.double().numpy(), k.double().numpy(), v.double().numpy(), pages, starts,
                                   [N] * B, parents, scale, dtype)
    # a large score is one exact product: equal ones have equal numerators, and the smaller ones, at
    # least 2^-11 of their size below, none.  What is left is the rounding of numerators and of sums
    u, L = R.HALF_STEP[dtype], int(starts[0]) + N
    most = float(v.double().abs().max())
    off[:, ::2] = u * np.abs(out[:, ::2]) + (u + 2.0 ** -21 + 2 * L * 2.0 ** -24) * most + 2.0 ** -24
    loff[:, ::2] = 2.0 ** -22 * np.abs(lse[:, ::2])
    far, lfar = np.abs(got - out) - off, np.abs(got_lse - lse) - loff
    assert not np.isnan(got).any() and far.max() <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))
    assert not np.isnan(got_lse).any() and lfar.max() <= 0, (lfar.max(), np.unravel_index(lfar.argmax(), lfar.shape))


SHAPES = [(2, 1), (3, 8), (40, 2), (65, 2)]


@pytest.mark.parametrize("N,G", SHAPES)
@pytest.mark.parametrize("scale", [0.125, 2.0 ** 10])
def test_large_scores(N, G, scale):
    _check([19, 20, 21, 22, 23, 24, 25, 26, 27, 28, 29, 30, 31, 32, 34, 40, 60, 60, 80, 80], "bfloat16", N, G, scale)


@pytest.mark.parametrize("N,G", SHAPES)
@pytest.mark.parametrize("scale,sizes", [(0.125, [19, 20, 21, 22, 23, 24, 25, 26, 26]),
                                         (2.0 ** 12, [21, 22, 23, 24, 25, 26, 27, 28, 29, 30, 31, 32, 34, 35, 40, 40])])
def test_large_scores_of_float16(N, G, scale, sizes):
    _check(sizes, "float16", N, G, scale, seed=1)


def test_large_scores_of_trees():
    N = 24
    rng = np.random.default_rng(3)
    sizes = [19, 24, 25, 26, 27, 28, 30, 31, 50, 51]
    parents = np.maximum(np.arange(N)[None] - rng.integers(1, 9, size=(len(sizes), N)), -1)
    _check(sizes, "bfloat16", N, 2, 1.0, parents, seed=2)
    _check(sizes[:6], "float16", N, 2, 1.0, parents[:6], seed=2)


@pytest.mark.parametrize("dtype", ["bfloat16"])
@pytest.mark.parametrize("N,G", SHAPES)
@pytest.mark.parametrize("scale", [5e5, 1e6])
def test_scores_at_the_lower_end(dtype, N, G, scale):
    # every score of every row is -9.2e29 before the scale: the mean of the values that are seen, and a
    # log-sum-exp whose rounding is that of its size
    import torch
    from paper_2002_00876_amd import binding
    say(f"attend lower end N={N} G={G} scale={scale}")
    D, S, past = 64, 16, 150
    M = -(-(past + N) // S)
    rng = np.random.default_rng(N)
    q = torch.zeros((1, N, G, D), dtype=torch.bfloat16)
    k = torch.zeros((M, S, 1, D), dtype=torch.bfloat16)
    v = torch.from_numpy(rng.standard_normal((M, S, 1, D))).to(torch.bfloat16)
    q[..., 0], k[..., 0] = -2.0 ** 50, 2.0 ** 49 * 1.453125
    score = float(q[0, 0, 0, 0].double() * k[0, 0, 0, 0].double())
    assert -1e30 < score < -9e29
    out, lse = binding.tree_attention(q.cuda(), k.cuda(), v.cuda(), _ints([np.arange(M)]), _ints([past]), scale=scale)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    flat = v.double().numpy().reshape(-1, D)
    u = R.HALF_STEP["bfloat16"]
    for i in range(N):
        seen = flat[:past + i + 1]
        want, mean = seen.mean(0), np.abs(seen).mean(0)
        off = u * np.abs(want) + (u + 2.0 ** -21 + 2 * len(seen) * 2.0 ** -24) * mean + 2.0 ** -24
        assert np.all(np.abs(out[0, i] - want) <= off), i
    assert np.all(np.abs(lse - score * float(np.float32(scale))) <= 2.0 ** -22 * abs(score) * scale)


@pytest.mark.parametrize("N,G", SHAPES)
def test_values_of_any_size(N, G):
    # values times a power of two: outputs are the same bits times it, up to the stated size
    import torch
    from test_gpu_attend import _inputs, _run
    d = _inputs(2, N, G, 1, 64, 16, 300, "bfloat16", N, True)
    d["q"] = d["q"] * 4
    want, lse = _run(d)
    for e in (-60, 60, 86):
        large = dict(d, v=d["v"] * 2.0 ** e)
        got, other = _run(large)
        assert float(large["v"].nan_to_num(0).abs().max()) <= 1e27
        assert torch.equal(got.double(), want.double() * 2.0 ** e) and torch.equal(lse, other), e
