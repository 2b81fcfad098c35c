"""Distillation with the teacher's log-sum-exp where its slots leave nothing, or next to nothing:
every token in a slot, both models masked alike, and rows that say nothing; against float64.

What the slots leave, 1 - sum p, is known to the rounding of p_k = exp(t_k / T - lse), which grows
with |lse|: below 2^-22 (8 + |lse|) it counts as 0, and it is 0 where no token is outside."""
import math

import numpy as np
import pytest

import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

INF = math.inf


def _reference(row, t, at, T, l):
    """(loss, d loss / d row) of one row in float64; loss +inf where q is 0 and p is not."""
    V = row.size
    keep = (at >= 0) & (at < V)
    p = np.zeros(V)
    if l > -INF:
        p[at[keep]] = np.exp(t[keep] / T - l)
    if l == -INF or not np.isfinite(row).any():
        return (INF if (p > 0).any() else 0.0), np.zeros(V)
    outside = np.ones(V, bool)
    outside[at[keep]] = False
    z = (row - row[np.isfinite(row)].max()) / T
    z -= R.lse(z)
    q = np.exp(z)
    p_r = 1.0 - p.sum()
    if not outside.any() or p_r < 2.0 ** -22 * (8 + abs(l)):
        p_r = 0.0
    low = -INF
    if np.isfinite(z[outside]).any():
        m = z[outside].max()
        low = m + R.lse(z[outside] - m)
    on = p > 0
    loss = float((p[on] * (np.log(p[on]) - z[on])).sum())
    if p_r > 0:
        loss += p_r * (math.log(p_r) - low)
    g = (q - p) / T
    if low > -INF:
        g[outside] = np.exp((row[outside] - row[outside].max()) / T)
        g[outside] *= (math.exp(low) - p_r) / (g[outside].sum() * T)
    return loss, g


def _check(x, t, at, l, T, tag, repeat=1):
    import torch
    from paper_2002_00876_amd import binding
    say(f"rest {tag}: {repeat} x {tuple(x.shape)} {x.dtype} K={t.shape[2]} T={T}")
    wide = [y.repeat(repeat, *[1] * (y.dim() - 1)) for y in (x, t, at, l)]
    alone = binding.distill(*wide, temperature=T)
    loss, grad = binding.distill_grad(*wide, temperature=T)
    assert torch.equal(alone, loss)
    B = x.shape[0]
    for b in range(0, repeat * B, B):
        assert torch.equal(loss[b:b + B], loss[:B]) and torch.equal(grad[b:b + B], grad[:B])
    half, least = R.ROUND[str(x.dtype).split(".")[1]]
    loss, grad = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    hx, ht, hat, hl = (y.cpu() if y.dtype == torch.int32 else y.double().cpu() for y in (x, t, at, l))
    hx, ht, hat, hl = (y.numpy() for y in (hx, ht, hat, hl))
    for b in range(B):
        for n in range(x.shape[1]):
            rl, rg = _reference(hx[b, n], ht[b, n], hat[b, n], T, hl[b, n])
            used = ht[b, n][(hat[b, n] >= 0) & (ht[b, n] > -1e9)]
            span = R.span(hx[b, n], T) + np.abs(used).max(initial=0) / T
            span += abs(hl[b, n]) if hl[b, n] > -INF else 0
            eps = R.EPS * (R.UNITS + span)
            if math.isinf(rl):
                assert loss[b, n] == rl, (b, n, loss[b, n])
            else:
                assert abs(loss[b, n] - rl) <= eps * (1 + abs(rl)), (b, n, loss[b, n], rl)
            # p and q are each at most 1, each off by eps of itself, the rest by eps
            off = np.abs(grad[b, n] - rg)
            most = 3 * eps / T + np.abs(rg) * half * (1 + eps) + least
            assert np.all(off <= most), (b, n, int((off - most).argmax()), float((off - most).max()))


def _rows(B, N, V, dtype, seed, lse, T):
    """A teacher's rows whose log-sum-exps are about lse, a student's near them."""
    import torch
    rng = np.random.default_rng(seed)
    t = rng.normal(0, 3, (B, N, V))
    t += T * lse - t.max(2, keepdims=True)
    x = t + rng.normal(0, 1, t.shape)
    return (torch.tensor(y).to(getattr(torch, dtype)).cuda() for y in (t, x))


@pytest.mark.parametrize("lse", [0, 10, 40, 200, -200])
@pytest.mark.parametrize("T", [0.1, 0.7, 1.0])
@pytest.mark.parametrize("V", [1, 2, 20, 256])
def test_every_token_in_a_slot(V, T, lse):
    from paper_2002_00876_amd import binding
    for dtype in ("float32", "bfloat16", "float16"):
        teacher, student = _rows(3, 40, V, dtype, V, lse, T)
        v, i, l = binding.top_logits(teacher, V, temperature=T)
        _check(student, v, i, l, T, f"all, lse {lse}")


@pytest.mark.parametrize("lse", [0, 10, 40, 200, -200])
@pytest.mark.parametrize("T", [0.1, 0.7])
@pytest.mark.parametrize("V,repeat", [(60, 1), (1000, 1), (9001, 1), (1500, 120), (30011, 60)])
def test_both_masked_alike(V, repeat, T, lse):
    # the teacher's slots hold all that is possible; the rest is masked on both sides, by -inf or the
    # type's lowest value
    import torch
    from paper_2002_00876_amd import binding
    for dtype in ("float32", "bfloat16"):
        for mask in (-INF, torch.finfo(getattr(torch, dtype)).min):
            teacher, student = _rows(1, 20, V, dtype, V, lse, T)
            on = torch.zeros(V, dtype=torch.bool, device="cuda")
            on[torch.randperm(V, generator=torch.Generator().manual_seed(V))[:40].cuda()] = True
            teacher.masked_fill_(~on, mask)
            student.masked_fill_(~on, mask)
            v, i, l = binding.top_logits(teacher, 50, temperature=T)
            _check(student, v, i, l, T, f"masked, lse {lse}", repeat)


@pytest.mark.parametrize("lse", [0, 40, 200])
@pytest.mark.parametrize("V", [60, 1000, 9001])
def test_a_rest_that_is_there(V, lse):
    # it stays a class: impossible for a student that masks it, far off for one that all but does
    import torch
    T, K = 1.0, 30
    teacher, student = _rows(1, 4, V, "float32", V, lse, T)
    v, i = teacher.topk(K, 2)
    for left in (1e-3, 0.2):
        l = (torch.logsumexp(v.double() / T, 2) - math.log(1 - left)).float()
        low = student - 45
        low.scatter_(2, i, student.gather(2, i))
        low[0, 0] = -INF
        low[0, 0].scatter_(0, i[0, 0], student[0, 0].gather(0, i[0, 0]))
        _check(low, v, i.int(), l, T, f"rest {left}, lse {lse}")


@pytest.mark.parametrize("V,repeat", [(1, 1), (30, 1), (2000, 1), (9000, 1), (2000, 600), (30011, 300)])
def test_neither_side_says_anything(V, repeat):
    # a teacher's row without a finite logit has no probability to compare with: loss and gradient
    # are 0, whatever the student's row is
    import torch
    teacher, student = _rows(1, 4, V, "float32", V, 0, 1.0)
    K = min(V, 5)
    v, i = teacher.topk(K, 2)
    l = torch.logsumexp(v, 2) + 0.1
    v[0, :3] = -INF
    l[0, :3] = -INF
    student[0, 0] = -INF
    student[0, 1] = torch.finfo(torch.float32).min
    _check(student, v, i.int(), l, 1.0, "nothing", repeat)
    from paper_2002_00876_amd import binding
    loss, grad = binding.distill_grad(student, v, i.int(), l)
    assert not loss[0, :3].any() and not grad[0, :3].any()
