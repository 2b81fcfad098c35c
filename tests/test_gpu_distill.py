"""Distillation from a teacher's top logits against float64, row by row, and its gradient against
the formula's and against differences of the loss."""
import math

import numpy as np
import pytest

import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]


def _case(B, N, V, K, dtype, seed=0, empty=0.0, rest=True, T=1.0, tail=0.2):
    """Student logits, a teacher's values, distinct indices and log-sum-exp, row weights."""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 2.5, (B, N, V))
    at = np.stack([rng.permutation(V)[:K] for _ in range(B * N)]).reshape(B, N, K)
    t = -np.sort(-(rng.normal(0, 2.0, (B, N, K)) + 4), axis=2)
    np.put_along_axis(x, at, 0.8 * t + rng.normal(0, 1, t.shape), 2)
    slots = rng.random((B, N, K)) < empty
    at = np.where(slots, -1, at)
    dt = getattr(torch, dtype)
    x, t = torch.tensor(x).to(dt).cuda(), torch.tensor(t).to(dt).cuda()
    l = None
    if rest:
        kept = np.where(at >= 0, t.double().cpu().numpy() / T, -np.inf)
        with np.errstate(divide="ignore"):
            l = np.array([R.lse(r) for r in kept.reshape(-1, K)]).reshape(B, N)
        l = np.where(np.isfinite(l), l, 0.0) - math.log(1 - tail)
        l = torch.tensor(l, dtype=torch.float32).cuda()
    return (x, t, torch.tensor(at, dtype=torch.int32).cuda(), l,
            torch.tensor(rng.random((B, N)) + 0.5, dtype=torch.float32).cuda())


def _check(x, t, at, l=None, w=None, lens=None, T=1.0, tag=""):
    import torch
    from paper_2002_00876_amd import binding
    say(f"distill {tag}: {tuple(x.shape)} {x.dtype} K={t.shape[2]} rest={l is not None} T={T}")
    tl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    alone = binding.distill(x, t, at, l, tl, temperature=T)
    loss, grad = binding.distill_grad(x, t, at, l, tl, w, temperature=T)
    torch.cuda.synchronize()
    assert torch.equal(alone, loss), "the loss differs between the two calls"
    assert grad.dtype == x.dtype and grad.shape == x.shape
    half, least = R.ROUND[str(x.dtype).split(".")[1]]
    hx, ht, hat = (y.double().cpu().numpy() if y.is_floating_point() else y.cpu().numpy()
                   for y in (x, t, at))
    hl = None if l is None else l.double().cpu().numpy()
    hw = np.ones(x.shape[:2]) if w is None else w.double().cpu().numpy()
    loss, grad = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    for b in range(x.shape[0]):
        L = x.shape[1] if lens is None else min(max(lens[b], 0), x.shape[1])
        assert np.all(loss[b, L:] == 0) and np.all(grad[b, L:] == 0), "padding is not exactly 0"
        for n in range(L):
            row = hx[b, n]
            rl, ls, rg, scale = R.distill(row, ht[b, n], hat[b, n], T,
                                          None if hl is None else hl[b, n])
            tf = ht[b, n][(hat[b, n] >= 0) & np.isfinite(ht[b, n])]
            span = R.span(row, T) + np.abs(tf).max(initial=0) / T
            if hl is not None and np.isfinite(hl[b, n]):
                span += abs(hl[b, n])
            eps = R.EPS * (R.UNITS + span)
            if math.isinf(rl):
                assert loss[b, n] == rl, (b, n)
            else:
                assert abs(loss[b, n] - rl) <= eps * ls, (b, n, loss[b, n], rl)
            off = np.abs(grad[b, n] - hw[b, n] * rg)
            most = hw[b, n] * scale * eps + hw[b, n] * np.abs(rg) * half * (1 + eps) + least
            assert np.all(off <= most), (b, n, int((off - most).argmax()), float((off - most).max()))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(1, 1), (2, 1), (20, 4), (20, 20), (63, 9), (65, 64), (256, 256),
                                 (1000, 100), (1025, 3), (4097, 256), (8193, 64), (50001, 100)])
def test_sizes(V, K, dtype, rest):
    c = _case(2, 3, V, K, dtype, V + K, empty=0.2, rest=rest and K < V)
    _check(*c, lens=[3, 2], tag="sizes")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V", [262144, 262145, 524288])
def test_largest_vocabularies(V, rest):
    import torch
    from paper_2002_00876_amd import binding
    c = _case(1, 2, V, 256, "bfloat16", V, rest=rest)
    _check(*c, tag="largest")
    # as many rows as are not divided for their number
    x, t, at, l, _ = (None if y is None else y[:, :1].expand(1, 1100, *y.shape[2:]) for y in c)
    loss = binding.distill(x, t, at, l)
    few = binding.distill(*(None if y is None else y[:, :1] for y in c[:4]))
    assert torch.equal(loss, loss[:, :1].expand_as(loss))
    assert (loss[0, 0] - few[0, 0]).abs() <= R.EPS * (R.UNITS + 64) * (1 + few[0, 0].abs())


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [0.5, 2.0, 4.0])
def test_temperature(T, rest):
    for dtype in TYPES:
        _check(*_case(2, 2, 3001, 40, dtype, 7, rest=rest, T=T), T=T, tag="temperature")


@pytest.mark.parametrize("V", [30, 2000, 9000])
def test_teacher_rows_that_say_nothing(V):
    import torch
    for rest in (False, True):
        x, t, at, l, w = _case(1, 5, V, 8, "float32", 3, rest=rest)
        at[0, 0] = -1                                  # no slots
        at[0, 1] = V                                   # none inside the vocabulary
        at[0, 2, 1:] = -1
        t[0, 3] = -float("inf")                        # a masked teacher's row
        if rest:
            l[0, 3] = -float("inf")
        t[0, 4, 2:] = -float("inf")
        _check(x, t, at, l, w, tag="empty teacher")
        # what an empty slot holds is not used
        from paper_2002_00876_amd import binding
        t2 = torch.where(at.ge(0) & at.lt(V), t, float("nan"))
        for a, b in zip(binding.distill_grad(x, t, at, l, weights=w),
                        binding.distill_grad(x, t2, at, l, weights=w)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [30, 2000, 9000])
def test_student_rows_with_masked_tokens(V, dtype):
    import torch
    for rest in (False, True):
        x, t, at, l, w = _case(1, 6, V, 8, dtype, 4, rest=rest)
        x[0, 0] = -float("inf")
        x[0, 1, at[0, 1, 0].long()] = -float("inf")    # the student cannot say what the teacher does
        keep = x[0, 2, at[0, 2].long()].clone()
        x[0, 2] = -float("inf")                        # nor anything else
        x[0, 2, at[0, 2].long()] = keep
        x[0, 3] = torch.finfo(x.dtype).min
        x[0, 4, ::2] = torch.finfo(x.dtype).min
        x[0, 5, at[0, 5].long()] += 60                 # nearly all of it on the slots
        _check(x, t, at, l, w, tag="masked student")


def test_rest_that_is_nearly_nothing():
    # the teacher's slots hold all but 1e-5 of it, the student's all but e^-40
    import torch
    x, t, at, l, w = _case(1, 3, 5000, 30, "float32", 8, rest=True, tail=1e-5)
    x.clamp_(max=1.0)
    x.scatter_(2, at.long(), 45 + torch.rand(at.shape, device="cuda"))
    _check(x, t, at, l, w, tag="small rest")
    x2, t2, at2, l2, w2 = _case(1, 3, 5000, 30, "float32", 9, rest=True, tail=0.0)
    l2 -= 2e-7
    _check(x2, t2, at2, l2, w2, tag="no rest")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,K", [(21, 4), (900, 9), (9001, 40)])
def test_strides_and_masked_places(V, K, dtype):
    import torch
    from paper_2002_00876_amd import binding
    x, t, at, l, w = _case(3, 3, V, K, dtype, 2)
    lens = torch.tensor([3, 0, 1], dtype=torch.int32, device="cuda")
    big = torch.full((3, 5, V + 7), float("nan"), dtype=x.dtype, device="cuda")
    y = big[:, 1:4, 3:3 + V]
    y.copy_(x)
    y[1] = float("nan")
    y[2, 1:] = float("nan")
    l2, w2 = l.clone(), w.clone()
    for z in (l2, w2):
        z[1], z[2, 1:] = float("nan"), float("nan")
    for a, b in zip(binding.distill_grad(x, t, at, l, lens, w),
                    binding.distill_grad(y, t, at, l2, lens, w2)):
        assert torch.equal(a, b)
    # one row for all: its gradient is every row's
    one = x[:1, :1].expand(3, 3, V)
    g = binding.distill_grad(one, t[:1, :1].expand(3, 3, K), at[:1, :1].expand(3, 3, K),
                             l[:1, :1].expand(3, 3))[1]
    assert torch.equal(g[0, 0], g[2, 1])


def test_teacher_of_another_type_and_from_top_logits():
    # the calls as they follow each other: the teacher's rows, their top logits, the student
    import torch
    from paper_2002_00876_amd import binding
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    teacher = torch.randn((2, 4, 7001), generator=g, device="cuda").mul_(3).bfloat16()
    student = teacher.float() + torch.randn((2, 4, 7001), generator=g, device="cuda")
    lens = [4, 3]
    v, i, l = binding.top_logits(teacher, 50, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                 temperature=2.0)
    _check(student, v, i, l, None, lens, T=2.0, tag="from top_logits")
    _check(student.half(), v, i, None, None, lens, T=2.0, tag="from top_logits")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V,K", [(20, 5), (700, 30), (9001, 100)])
def test_gradient_against_differences(V, K, rest):
    # along a direction of entries within [-1, 1]: the third derivative of the loss along it is
    # at most 2 (differences of third cumulants of variables within [-1, 1]), so differences over
    # 2h are off by at most h^2 / 3, and by the loss's own error over h
    import torch
    from paper_2002_00876_amd import binding
    x, t, at, l, w = _case(1, 4, V, K, "float32", 11, rest=rest)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    d = torch.rand(x.shape, generator=g, device="cuda") * 2 - 1
    d.scatter_(2, at.long().clamp(min=0), 1.0)
    h = 2.0 ** -6
    up, down = (binding.distill(x + s * h * d, t, at, l).double() for s in (1, -1))
    grad = binding.distill_grad(x, t, at, l)[1].double()
    span = float(x.max() - x.min()) + float(t.abs().max()) + (float(l.abs().max()) if rest else 0)
    tol = h * h / 3 + R.EPS * (R.UNITS + span) * (1 + float(up.abs().max())) / h
    off = ((up - down) / (2 * h) - (grad * d.double()).sum(2)).abs().max().item()
    assert off <= tol, (off, tol)
    assert (grad * d.double()).sum(2).abs().max().item() > 20 * tol


def test_gradient_written_past_32_bit_offsets():
    import torch
    from paper_2002_00876_amd import binding
    V, rows = 131072, 16400                             # 2^31 + 2^21 elements
    x, t, at, l, w = _case(1, 2, V, 16, "bfloat16", 5)
    at2, t2, l2, w2 = (torch.cat([y[:, :1].expand(1, rows - 1, *y.shape[2:]), y[:, 1:]], 1)
                       for y in (at, t, l, w))
    # two rows in memory: the first for all but the last one
    first, second = (binding.distill_grad(x[:, k:k + 1], t[:, k:k + 1], at[:, k:k + 1],
                                          l[:, k:k + 1], weights=w[:, k:k + 1]) for k in (0, 1))
    loss, grad = binding.distill_grad(x[:, :1].expand(1, rows, V), t2, at2, l2, weights=w2)
    torch.cuda.synchronize()
    assert torch.equal(grad[0, 0], first[1][0, 0]) and torch.equal(grad[0, rows - 2], first[1][0, 0])
    assert torch.equal(loss[0, : rows - 1], first[0][0].expand(rows - 1))
    del grad
    big = torch.empty(2 ** 32 + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    y = big.as_strided((1, 2, V), (0, 2 ** 32 + 5, 1))
    y.copy_(x)
    got = binding.distill_grad(y, t, at, l, weights=w)
    assert torch.equal(got[1][0, 1], second[1][0, 0]) and torch.equal(got[0][0, 1], second[0][0, 0])


def test_out_repeats_and_no_loss():
    import torch
    from paper_2002_00876_amd import binding
    x, t, at, l, w = _case(2, 30, 32000, 64, "bfloat16", 6)
    first = binding.distill_grad(x, t, at, l, weights=w)
    out = tuple(torch.empty_like(y) for y in first)
    again = binding.distill_grad(x, t, at, l, weights=w, out=out)
    for a, b, c in zip(first, again, out):
        assert torch.equal(a, b) and b.data_ptr() == c.data_ptr()
    none, grad = binding.distill_grad(x, t, at, l, weights=w, want_loss=False)
    assert none is None and torch.equal(grad, first[1])
