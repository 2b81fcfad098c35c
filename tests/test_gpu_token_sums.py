"""The sums of a row's softmax (log-sum-exps of top logits; distillation's loss and gradient) over
temperatures, dispatch branches and masks that leave threads without a token to sum, against
float64, to the bounds of token_ref."""
import math

import numpy as np
import pytest

import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

# log2(e) / T times a power of ten is rounded up for some of these and down for the others
TEMPERATURES = [0.3, 0.6, 0.9, 1.1, 1.3]


def _logits(N, V, dtype, seed):
    import torch
    rng = np.random.default_rng(seed)
    return torch.tensor(rng.normal(0, 2.5, (1, N, V))).to(getattr(torch, dtype)).cuda()


def _teacher(x, K, T, seed):
    """Values, tokens and a log-sum-exp that leaves a fifth, of each of x's rows; the student's
    logits of these tokens are drawn near them."""
    import torch
    rng = np.random.default_rng(seed)
    _, N, V = x.shape
    at = np.stack([rng.permutation(V)[:K] for _ in range(N)])[None]
    t = torch.tensor(-np.sort(-(rng.normal(0, 2.0, (1, N, K)) + 4), axis=2), dtype=torch.float32)
    at = torch.tensor(at).cuda()
    x.scatter_(2, at, (0.8 * t + torch.tensor(rng.normal(0, 1, t.shape)).float()).to(x.dtype).cuda())
    l = (torch.logsumexp(t.double() / T, 2) - math.log(0.8)).float()
    return t.cuda(), at.int(), l.cuda()


def _check_lse(x, K, T, B=1):
    from paper_2002_00876_amd import binding
    say(f"lse: {B} x {tuple(x.shape[1:])} {x.dtype} K={K} T={T}")
    v, i, l = binding.top_logits(x.expand(B, *x.shape[1:]), K, temperature=T)
    assert bool((l == l[:1]).all()) and bool((i == i[:1]).all())
    h = x.double().cpu().numpy()[0]
    for n, row in enumerate(h):
        rv, ri, rl = R.top(row, K, T)
        assert np.array_equal(i[0, n].cpu().numpy(), ri)
        got = l[0, n].item()
        if rl == -math.inf:
            assert got == rl, (n, got)
        else:
            assert abs(got - rl) <= R.EPS * (R.UNITS + abs(rl) + R.span(row, T)), (n, got, rl)


def _check_distill(x, teacher, T, rest, B=1):
    import torch
    from paper_2002_00876_amd import binding
    say(f"distill: {B} x {tuple(x.shape[1:])} {x.dtype} T={T} rest={rest}")
    t, at, l = teacher
    wide = [y.expand(B, *y.shape[1:]) for y in (x, t, at)] + [l.expand(B, -1) if rest else None]
    alone = binding.distill(*wide, temperature=T)
    loss, grad = binding.distill_grad(*wide, temperature=T)
    assert torch.equal(alone, loss)
    assert bool((loss == loss[:1]).all()) and bool((grad == grad[:1]).all())
    half, least = R.ROUND[str(x.dtype).split(".")[1]]
    hx, ht, hat, hl = (y.double().cpu().numpy()[0] for y in (x, t, at, l))
    loss, grad = loss[0].double().cpu().numpy(), grad[0].double().cpu().numpy()
    for n, row in enumerate(hx):
        rl, ls, rg, scale = R.distill(row, ht[n], hat[n].astype(np.int64), T, hl[n] if rest else None)
        span = R.span(row, T) + np.abs(ht[n]).max() / T + (abs(hl[n]) if rest else 0)
        eps = R.EPS * (R.UNITS + span)
        if math.isinf(rl):
            assert loss[n] == rl, (n, loss[n])
        else:
            assert abs(loss[n] - rl) <= eps * ls, (n, loss[n], rl)
        off = np.abs(grad[n] - rg)
        most = scale * eps + np.abs(rg) * half * (1 + eps) + least
        assert np.all(off <= most), (n, int((off - most).argmax()), float((off - most).max()))


# (a sequence's rows, sequences): few rows, which are divided where they are long, and many
SHAPES = [(V, 1) for V in (20, 256, 1025, 9001, 70000)] + [(V, 720) for V in (1500, 9001, 30011)]


def _holes(x, keep):
    """-inf over the first half of one row and all but the start of another, kept tokens aside."""
    import torch
    V = x.shape[2]
    hole = torch.zeros(x.shape, dtype=torch.bool, device=x.device)
    hole[0, 1, : V // 2] = True
    hole[0, 2, V // 7 + 1:] = True
    if keep is not None:
        hole.scatter_(2, keep.long(), False)
    return x.masked_fill_(hole, -math.inf)


@pytest.mark.parametrize("T", TEMPERATURES)
@pytest.mark.parametrize("V,B", SHAPES)
def test_log_sum_exp_at_any_temperature(V, B, T):
    for dtype in ("float32", "bfloat16"):
        _check_lse(_holes(_logits(3, V, dtype, V), None), 3, T, B)


@pytest.mark.parametrize("T", TEMPERATURES)
@pytest.mark.parametrize("V,B", [(1, 1)] + SHAPES)
def test_distillation_at_any_temperature(V, B, T):
    K = min(5, V)
    for dtype in ("float32", "float16"):
        x = _logits(3, V, dtype, V)
        teacher = _teacher(x, K, T, V)
        _holes(x, teacher[1])
        for rest in (False, True) if K < V else (False,):
            _check_distill(x, teacher, T, rest, B)


# ---- logits so large that their exponents pass 2^31 ----

def _masked(x, mask, keep):
    """Rows of x [1, 6, V] with a finite mask: everywhere, over the first half, over all but the last
    few, at every other token, its opposite at one token and everywhere.  keep [1, 6, K]: tokens that
    stay in the rows that are not of one value."""
    import torch
    V = x.shape[2]
    hole = torch.zeros(x.shape, dtype=torch.bool, device=x.device)
    hole[0, 1, : V // 2] = True
    hole[0, 2, : V - 3] = True
    hole[0, 3, ::2] = True
    if keep is not None:
        hole[0, 1:4].scatter_(1, keep[0, 1:4].long(), False)
    x.masked_fill_(hole, mask)
    x[0, 0] = mask
    x[0, 4, V // 3] = -mask
    x[0, 5] = -mask
    return x


@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e12, -1e20, -1e30])
@pytest.mark.parametrize("V,B", SHAPES)
def test_log_sum_exp_of_finite_masks(V, B, mask):
    for dtype, T in (("float32", 1.0), ("bfloat16", 1.0), ("float32", 0.6)):
        _check_lse(_masked(_logits(6, V, dtype, V), mask, None), 3, T, B)


@pytest.mark.parametrize("V,B", SHAPES)
def test_log_sum_exp_at_the_least_temperature(V, B):
    # logits of some thousands have exponents of 10^9 here
    _check_lse(_logits(4, V, "float32", V) * 2 + 3000, 3, 1e-6, B)
    _check_lse(_logits(4, V, "float16", V) * 2 - 3000, 3, 1e-6, B)


@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e12, -1e20, -1e30])
@pytest.mark.parametrize("V,B", SHAPES)
def test_distillation_of_finite_masks(V, B, mask):
    for dtype, T in (("float32", 1.0), ("bfloat16", 1.0), ("float32", 0.6)):
        x = _logits(6, V, dtype, V)
        teacher = _teacher(x, 5, T, V)
        x = _masked(x, mask, teacher[1])
        for rest in (False, True):
            # (in float64 a sum over masks of 10^20 would lose its logarithm beside unmasked slots:
            # every row here has other tokens outside the slots, or one value throughout)
            _check_distill(x, teacher, T, rest, B)


@pytest.mark.parametrize("V,B", SHAPES)
def test_distillation_of_far_logits_at_a_low_temperature(V, B):
    x = _logits(3, V, "float32", V)
    teacher = _teacher(x, 5, 1e-3, V)
    _check_distill(x + 4e6, teacher, 1e-3, False, B)
