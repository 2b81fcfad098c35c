"""The K largest logits of a row and its log-sum-exp against a sort in float64: values and
indices exactly (they are decided by comparisons alone), the log-sum-exp to the bound of
token_ref."""
import numpy as np
import pytest

import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]


def _run(x, K, lens=None, T=1.0, **kw):
    import torch
    from paper_2002_00876_amd import binding
    tl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = binding.top_logits(x, K, tl, temperature=T, **kw)
    torch.cuda.synchronize()
    return out


def _check(x, K, lens=None, T=1.0, tag=""):
    """x: device tensor [B, N, V]."""
    import torch
    say(f"top {tag}: {tuple(x.shape)} {x.dtype} K={K} T={T}")
    v, i, l = _run(x, K, lens, T)
    assert v.dtype == x.dtype and i.dtype == torch.int32 and l.dtype == torch.float32
    h = x.double().cpu().numpy()
    v, i, l = v.double().cpu().numpy(), i.cpu().numpy(), l.double().cpu().numpy()
    B, N, _ = h.shape
    for b in range(B):
        L = N if lens is None else min(max(lens[b], 0), N)
        assert np.all(v[b, L:] == -np.inf) and np.all(i[b, L:] == -1) and np.all(l[b, L:] == -np.inf)
        for n in range(L):
            rv, ri, rl = R.top(h[b, n], K, T)
            assert np.array_equal(i[b, n], ri), f"indices of row {b}, {n}"
            assert np.array_equal(v[b, n], rv), f"values of row {b}, {n}"
            if rl == -np.inf:
                assert l[b, n] == -np.inf
            else:
                most = R.EPS * (R.UNITS + abs(rl) + R.span(h[b, n], T))
                assert abs(l[b, n] - rl) <= most, (b, n)


def _normal(shape, dtype, seed=0, sigma=3.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * sigma).to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (20, 5), (63, 63), (65, 1), (128, 128), (129, 7),
                                 (256, 256), (511, 100), (513, 256), (1000, 32), (4099, 256),
                                 (8192, 17), (8193, 256), (50001, 100), (131073, 256)])
def test_sizes(dtype, V, K):
    _check(_normal((2, 3, V), dtype, V + K), K, [3, 2], tag="sizes")


@pytest.mark.parametrize("V,K", [(300, 50), (5000, 64), (40000, 128), (524288, 256)])
def test_few_different_values(V, K):
    # many equal logits: the lowest indices are taken, past what any list holds too
    x = _normal((1, 4, V), "float32", V)
    x[0, 0] = x[0, 0].round()
    x[0, 1] = 1.5
    x[0, 2] = (x[0, 2] > 8).float()
    x[0, 3] = -0.0
    x[0, 3, ::2] = 0.0
    _check(x, K, tag="ties")


@pytest.mark.parametrize("V,K", [(20, 5), (700, 80), (9000, 256), (131072, 128)])
def test_masked_tokens(V, K):
    import torch
    x = _normal((1, 6, V), "bfloat16", V)
    x[0, 0] = -float("inf")                                  # nothing can follow
    x[0, 1, 1:] = -float("inf")
    x[0, 2, :-3] = -float("inf")                             # fewer than K can
    x[0, 3, V // 2:] = -float("inf")
    x[0, 4] = torch.finfo(torch.bfloat16).min
    x[0, 5, 3:] = torch.finfo(torch.bfloat16).min
    _check(x, K, tag="masked")


@pytest.mark.parametrize("V,K", [(3000, 256), (60000, 200)])
def test_large_logits_together(V, K):
    # the largest lie side by side (few threads' maxima see them), ascending and descending rows
    import torch
    x = _normal((1, 3, V), "float32", V, 0.1)
    x[0, 0, 100:100 + 2 * K] += 50
    x[0, 1] = torch.arange(V, device="cuda")
    x[0, 2] = -torch.arange(V, device="cuda")
    _check(x, K, tag="together")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [1025, 1500, 2047, 3001, 6151, 8200, 9000, 12345, 20008, 32000, 36860])
def test_rows_that_end_within_a_wave(V, dtype):
    # the K largest spread over the row's last few thousand logits, in rows whose last vectors are
    # those of a part of a wave, and enough rows that none is divided
    x = _normal((1, 2100, V), dtype, V)
    x[0, :, max(0, V - 3000):] += 6
    few = x[:, ::300].contiguous()
    _check(few, 40, tag="ends")
    for a, b in zip(_run(x, 40)[:2], _run(few, 40)[:2]):
        assert bool((a[:, ::300] == b).all())


@pytest.mark.parametrize("T", [0.1, 0.7, 3.0])
def test_temperature(T):
    _check(_normal((1, 3, 9001), "float16", 5), 20, T=T, tag="temperature")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(20, 4), (600, 9), (9001, 40)])
def test_strides_and_masked_places(dtype, V, K):
    # a padded vocabulary, sequences apart, and NaN wherever nothing may be read
    import torch
    big = torch.full((3, 5, V + 7), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    x = big[:, 1:4, 3:3 + V]
    clean = _normal((3, 3, V), dtype, 1)
    x.copy_(clean)
    lens = [3, 0, 1]
    x[1] = float("nan")
    x[2, 1:] = float("nan")
    got = _run(x, K, lens)
    want = _run(clean, K, lens)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    _check(clean, K, lens, tag="strides")
    # rows of one tensor for every sequence, and logits that are not contiguous along V
    one = clean[:1, :1].expand(2, 3, V)
    assert all(torch.equal(a[0, 0], a[1, 2]) for a in _run(one, K))
    turned = clean.transpose(1, 2).contiguous().transpose(1, 2)
    assert all(torch.equal(a, b) for a, b in zip(_run(turned, K), _run(clean, K)))


def test_rows_past_32_bit_offsets():
    import torch
    V, K = 1000, 10
    rows = _normal((1, 2, V), "bfloat16", 3)
    big = torch.empty(2 ** 32 + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((1, 2, V), (0, 2 ** 32 + 5, 1))
    x.copy_(rows)
    for a, b in zip(_run(x, K), _run(rows, K)):
        assert torch.equal(a, b)


def test_out_and_repeats():
    import torch
    x = _normal((3, 40, 32000), "bfloat16", 9)
    first = _run(x, 32)
    out = tuple(torch.empty_like(t) for t in first)
    again = _run(x, 32, out=out)
    for a, b, c in zip(first, again, out):
        assert torch.equal(a, b) and b.data_ptr() == c.data_ptr()
