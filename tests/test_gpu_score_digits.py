"""What scores of given tokens and their gradient keep where numbers nearly cancel, against float64."""
import numpy as np
import pytest

import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _row(row, T):
    """(d = (x - max) / T, log sum exp d, X = -sum p d, p) of a row: log p = d - log s, the entropy is log s + X."""
    d = (row - row.max()) / T
    e = np.exp(d)
    p = e / e.sum()
    return d, np.log(e.sum()), -(p * d).sum(), p


@pytest.mark.parametrize("sigma,T", [(0.002, 1.0), (3.0, 1e4), (0.5, 10.0)])
@pytest.mark.parametrize("V,N", [(20, 2), (700, 2), (4001, 2), (9000, 2), (131072, 1)])
def test_entropy_gradient_of_rows_that_are_nearly_uniform(V, N, sigma, T):
    # -u p (log p + H) / T = -u p (d + X) / T: log s, which is large here, is no part of it.  X is the
    # quotient of two sums, each off by eps; p is off by eps, d by 2^-23 of its size (a difference of
    # logits and its product), and the result by half a step and that of the sum d + X
    import torch
    from paper_2002_00876_amd import binding
    say(f"entropy gradient V={V} sigma={sigma} T={T}")
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    x = torch.randn((2, N, V), generator=g, device="cuda") * sigma
    z = np.full((2, N), V // 3)
    u = np.array([[1.0] * N, [-2.5] * N], np.float32)
    none = torch.zeros((2, N), device="cuda")
    grad = binding.score_grad(x, _ints(z), None, none, torch.tensor(u, device="cuda"), temperature=T)[2]
    rows, grad = x.double().cpu().numpy(), grad.double().cpu().numpy()
    for b in range(2):
        for n in range(N):
            d, _, X, p = _row(rows[b, n], T)
            eps = R.EPS * (R.UNITS + R.span(rows[b, n], T))
            scale = abs(u[b, n]) / T
            want = -u[b, n] / T * p * (d + X)
            off = scale * p * ((eps + 2.0 ** -22) * np.abs(d + X) + 2 * eps * X + 2.0 ** -23 * np.abs(d)) + \
                2.0 ** -24 * np.abs(want) + R.ROUND["float32"][1]
            far = np.abs(grad[b, n] - want) - off
            assert far.max() <= 0, (b, n, int(far.argmax()), far.max())
            # the values' own error is common to them: their sum, 0, shows it
            assert abs(grad[b, n].sum()) <= off.sum(), (b, n)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V,gap", [(2, 30.0), (20, 20.0), (64, 24.0), (700, 25.0), (1024, 40.0), (4001, 30.0),
                                   (9001, 30.0), (50001, 34.0), (131072, 40.0)])
def test_rows_with_a_token_that_is_nearly_certain(V, gap, dtype):
    # rest = sum of the others' numerators, off by eps relative; log p of the sure token is -log1p(rest), the
    # entropy log1p(rest) - sum p d: both are as small as rest, and off by their own size only, whichever token
    # is given and whether alternatives are asked for
    import torch
    from paper_2002_00876_amd import binding
    for T in (1.0, 0.5):
        places = sorted({0, 1, V // 3, V // 2, max(V - 2, 0), V - 1})
        say(f"sure tokens V={V} gap={gap} {dtype} T={T}")
        x = torch.zeros((1, len(places), V), dtype=getattr(torch, dtype), device="cuda")
        for n, at in enumerate(places):
            x[0, n, at] = gap
            x[0, n, (at + 1) % V] = -2.0
        rows = x.double().cpu().numpy()[0]
        for step in (0, 1, 2):     # the sure token itself, its neighbour, one of the others
            z = np.array([[(at + step) % V for at in places]])
            calls = [binding.score(x, _ints(z), K, temperature=T) for K in (0, 1, min(V, 3))]
            grads = binding.score_grad(x, _ints(z), temperature=T)
            for logp, H in [c[:2] for c in calls] + [grads[:2]]:
                logp, H = logp.double().cpu().numpy()[0], H.double().cpu().numpy()[0]
                for n, at in enumerate(places):
                    d = (rows[n] - rows[n, at]) / T
                    rest = np.exp(np.delete(d, at)).sum()
                    p = np.exp(d) / (1 + rest)
                    eps = R.EPS * (R.UNITS + R.span(rows[n], T))
                    want = d[z[0, n]] - np.log1p(rest)
                    assert abs(logp[n] - want) <= (eps if z[0, n] == at else 2.0 ** -22) * abs(want), (n, step)
                    want = np.log1p(rest) - (p * d).sum()
                    assert abs(H[n] - want) <= 2 * eps * want, (n, step, H[n], want)
            for _, _, alt, alt_logp in calls[1:]:
                assert alt[0, :, 0].tolist() == places
                for n, at in enumerate(places):
                    rest = np.exp(np.delete((rows[n] - rows[n, at]) / T, at)).sum()
                    eps = R.EPS * (R.UNITS + R.span(rows[n], T))
                    assert abs(float(alt_logp[0, n, 0]) + np.log1p(rest)) <= eps * np.log1p(rest), n


def test_many_rows_with_a_token_that_is_nearly_certain():
    # rows that are not divided among workgroups: the kernels of many rows
    import torch
    from paper_2002_00876_amd import binding
    for V in (1000, 9000, 30000):
        N, gap = 1100, 30.0
        x = torch.zeros((1, N, V), dtype=torch.bfloat16, device="cuda")
        at = (torch.arange(N, device="cuda") * 7919) % V
        x[0, torch.arange(N), at] = gap
        rest = (V - 1) * np.exp(-gap)
        eps = R.EPS * (R.UNITS + gap)
        H = np.log1p(rest) + gap * rest / (1 + rest)
        for K, z in ((0, at), (2, at), (0, (at + 5) % V), (2, (at + 5) % V)):
            logp, ent, _, _ = binding.score(x, z.int()[None], K)
            want = -np.log1p(rest) - (0 if z is at else gap)
            assert float((logp.double() - want).abs().max()) <= (eps if z is at else 2.0 ** -22) * abs(want), (V, K)
            assert float((ent.double() - H).abs().max()) <= 2 * eps * H, (V, K)


def test_rows_with_several_largest_logits():
    # one of them is left out of the sums, wherever the others lie
    import torch
    from paper_2002_00876_amd import binding
    rng = np.random.default_rng(0)
    for V in (20, 700, 5000, 40000):
        x = torch.full((1, 12, V), -40.0, device="cuda")
        for n in range(12):
            at = rng.choice(min(V, 9 if n % 2 else V), size=2 + n % 3, replace=False)
            x[0, n, torch.tensor(at)] = 1.5
        x[0, 10], x[0, 11] = 0.25, torch.finfo(torch.float32).min
        for K in (0, 4):
            z = torch.argmax(x, dim=2).int()
            logp, ent, _, _ = binding.score(x, z, K)
            for n in range(12):
                count = 2 + n % 3 if n < 10 else V
                assert abs(float(logp[0, n]) + np.log(count)) <= R.EPS * R.UNITS, (V, K, n)
                assert abs(float(ent[0, n]) - np.log(count)) <= 3 * R.EPS * R.UNITS, (V, K, n)
