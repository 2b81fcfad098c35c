"""Scores of given tokens and their gradient in calls of so many rows that none is divided among workgroups: the
kernels of 64, 256 and 512 threads, whose rows are held in LDS in part and read again backwards.  Rows of a
call's own output are compared with float64, to the bounds of test_gpu_score."""
import numpy as np
import pytest

import test_gpu_score as S
import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu


def _compare(x, z, T, w, u, picked, scores, grads, K, tag):
    """Rows `picked` of [1, N, V] logits: logp, entropy, alternatives, and the gradient against float64."""
    logp, ent, alt, alt_lp = [None if t is None else t[0, picked].double().cpu().numpy() for t in scores]
    glogp, gent, grad = [t[0, picked].double().cpu().numpy() for t in grads]
    rows, dtype = x[0, picked].double().cpu().numpy(), str(x.dtype).replace("torch.", "")
    z, w, u = [None if t is None else t[0, picked].cpu().numpy().astype(np.float64) for t in (z, w, u)]
    half, least = R.ROUND[dtype]
    V = rows.shape[1]
    for i in range(len(picked)):
        at, zi = (tag, picked[i]), int(z[i])
        lp_z, H, lp = S._row(rows[i], zi, T)
        # the lowest bfloat16 over T lies beyond the 32-bit floats: -inf there
        lowest = float(np.finfo(np.float32).min)
        lp = np.where(lp < lowest, -np.inf, lp)
        lp_z = -np.inf if lp_z is not None and lp_z < lowest else lp_z
        eps = R.EPS * (R.UNITS + R.span(rows[i], T))
        for got in (logp[i], glogp[i]):
            if lp_z is None:
                assert got == 0, at
            elif lp_z == -np.inf:
                assert got == -np.inf, at
            else:
                assert abs(got - lp_z) <= eps + 2.0 ** -22 * abs(lp_z), at
        for got in (ent[i], gent[i]):
            assert got >= 0 and abs(got - H) <= eps * (2 + H), at
        if K:
            order = np.lexsort((np.arange(V), -rows[i]))[:K]
            assert np.array_equal(alt[i], order), at
            on = lp[order] > -np.inf
            assert np.all(alt_lp[i][~on] == -np.inf), at
            assert np.all(np.abs(alt_lp[i][on] - lp[order][on]) <= eps + 2.0 ** -22 * np.abs(lp[order][on])), at
        p = np.exp(lp)
        wi = (1.0 if w is None else w[i]) if lp_z is not None else 0.0
        ui = 0.0 if u is None else u[i]
        own = np.zeros(V)
        if np.isfinite(rows[i]).any():
            if lp_z is not None:
                own[zi] = wi
            on = p > 0
            # log p + H is off by eps of both its parts, as t / s is, and by 2^-23 of (x - max) / T
            part, size = np.zeros(V), np.zeros(V)
            part[on] = p[on] * (lp[on] + H)
            size[on] = p[on] * (np.abs(lp[on] + H) + 2 * H + np.abs(lp[on]))
            want = (own - wi * p - ui * part) / T
        else:
            want, size = own, own
        # a numerator below 2^-126, the least normal float, may be 0: that is off by it times what it is multiplied by
        times = (abs(wi) + abs(ui) * (np.where(lp > -200, np.abs(lp), 0.0) + H + 2)) / T
        off = half * np.abs(want) + least + 2.0 ** -126 * times + 2 * eps * (abs(wi) * p + abs(ui) * size) / T
        if lp_z is not None:
            # (w / T) (s - e) / s: 1 / T, its product with w, 1 / s and two more products are rounded
            off[zi] += 2 * eps * abs(wi) * p[zi] / T + 2.0 ** -22 * abs(want[zi])
        far = np.abs(grad[i] - want) - off
        assert not np.isnan(grad[i]).any() and far.max() <= 0, (at, int(far.argmax()), far.max())


@pytest.mark.parametrize("pitch", [0, 7, 8])
@pytest.mark.parametrize("V,N,dtype", [(200, 3000, "bfloat16"), (8191, 2100, "bfloat16"), (4097, 2049, "float32"),
                                       (9001, 1100, "bfloat16"), (24570, 1030, "float16"), (24577, 1025, "bfloat16"),
                                       (50001, 1024, "bfloat16"), (50000, 1024, "float32"), (131072, 1024, "bfloat16")])
def test_rows_of_a_large_call(V, N, dtype, pitch):
    # (the pitch is odd where it is V itself or V + 7, and aligned where it is made a multiple of 8)
    import torch
    from paper_2002_00876_amd import binding
    say(f"many rows V={V} N={N} {dtype} pitch={pitch}")
    g = torch.Generator(device="cuda")
    g.manual_seed(V + pitch)
    stride = {0: V, 7: V + 7, 8: (V + 15) // 8 * 8}[pitch]
    t = getattr(torch, dtype)
    wide = torch.full((1, N, stride), float("nan"), dtype=t, device="cuda")
    wide[0, :, :V] = torch.randn((N, V), generator=g, device="cuda") * 3
    x = wide[:, :, :V]
    n = N - 3                                                  # the last rows are padding
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    z = torch.randint(0, V, (1, N), generator=g, device="cuda", dtype=torch.int32)
    w, u = torch.randn((2, 1, N), generator=g, device="cuda")
    x[0, 5] = -float("inf")                                    # nothing can follow
    x[0, 6, : V - 2] = -float("inf")                           # two tokens can
    x[0, 7, ::2] = torch.finfo(t).min                          # masked by the lowest value
    x[0, 8] = 2.5                                              # all alike
    x[0, 9, V // 2] = 60.0                                     # one that is nearly certain
    z[0, 6], z[0, 9], z[0, 10], z[0, 11], z[0, 12] = 0, V // 2, V - 1, -1, V
    if dtype == "float32":
        x[0, 13] *= 1e9                                        # sums are taken again another way
    picked = [0, 1, 5, 6, 7, 8, 9, 10, 11, 12, 13, n // 2, n - 2, n - 1]
    T = float(np.float32(0.7))
    for K, uu in ((0, u), (5, None)):
        scores = binding.score(x, z, K, lens, temperature=T)
        grads = binding.score_grad(x, z, lens, w, uu, temperature=T)
        torch.cuda.synchronize()
        _compare(x, z, T, w, uu, picked, scores, grads, K, (V, K))
        assert all((a[0, n:] == 0).all() for a in (scores[0], scores[1], *grads))
        assert (scores[2][0, n:] == -1).all() and (scores[3][0, n:] == -float("inf")).all()
        # every row's gradient adds up to 0 but for its rounding, given tokens within the vocabulary or not
        # (sum p |log p| = H <= log V; half a step of each value, but at least that of the smallest floats)
        half, least = R.ROUND[dtype]
        total = grads[2].double().sum(2)[0, :n]
        size = grads[2].double().abs().sum(2)[0, :n]
        masked = torch.zeros(n, dtype=torch.bool, device="cuda")
        masked[[5, 6, 7, 13]] = True                           # (a masked given token has no p to balance it)
        parts = w[0, :n].abs() + (0 if uu is None else 5 * np.log(V) * uu[0, :n].abs())
        slack = half * size + V * least + 2 * R.EPS * (R.UNITS + 110) * parts / T
        assert bool((total.abs()[~masked] <= slack[~masked]).all())


@pytest.mark.parametrize("V,rows", [(300, 4000), (9001, 1300), (50001, 1030)])
def test_many_sequences_and_two_strides(V, rows):
    # the same rows as sequences of different lengths, from a batch of a strided view: the same bits
    import torch
    from paper_2002_00876_amd import binding
    B = 10
    N = rows // B
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    x = (torch.randn((B, N, V), generator=g, device="cuda") * 3).to(torch.bfloat16)
    z = torch.randint(0, V, (B, N), generator=g, device="cuda", dtype=torch.int32)
    w, u = torch.randn((2, B, N), generator=g, device="cuda")
    lens = torch.arange(N - B + 1, N + 1, device="cuda", dtype=torch.int32)
    a = binding.score_grad(x, z, lens, w, u)
    flat = binding.score_grad(x.view(1, B * N, V), z.view(1, -1), None, w.view(1, -1), u.view(1, -1))
    s, t = binding.score(x, z, 0, lens), binding.score(x.view(1, B * N, V), z.view(1, -1), 0)
    torch.cuda.synchronize()
    for b in range(B):
        n = int(lens[b])
        for got, want in ((a[0], flat[0]), (a[1], flat[1]), (a[2], flat[2]), (s[0], t[0]), (s[1], t[1])):
            assert torch.equal(got[b, :n], want[0, b * N:b * N + n]) and not got[b, n:].any()
