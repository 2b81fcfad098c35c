"""Attention of few rows: numerators keep more digits than the cache's type has.

A bfloat16 numerator is cut (off by less than 2^-7 of itself) and its rest rounded (by 2^-8 of that): 2^-15.  A
float16 one: 2^-10 and 2^-11, 2^-21, and where it is below 2^-28 of its row's largest 2^-39 of that.  The other
terms are those of cache_ref.attend, whose result is rounded to the type once."""
import numpy as np
import pytest

import cache_ref as R
from test_gpu_attend import _inputs, _run
from gpu_util import say

pytestmark = pytest.mark.gpu

NUMERATOR = {"bfloat16": 2.0 ** -15, "float16": 2.0 ** -21}


def _bounds(d, dtype):
    """(out, bound) in float64 of a call without a scale."""
    q, k, v = (np.nan_to_num(d[x].double().numpy()) for x in "qkv")
    B, N, Hq, D = q.shape
    S, Hk = k.shape[1:3]
    scale, most = D ** -0.5, d["pages"].shape[1] * S
    out, off = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        n, start = int(d["lengths"][b]), int(d["starts"][b])
        end = min(start + n, most)
        kk, vv = R.slots(k, d["pages"], S, b, end), R.slots(v, d["pages"], S, b, end)
        for i in range(n):
            to = R.sees(i, start, n, None if d["parents"] is None else d["parents"][b])
            for h in range(Hq):
                g = h // (Hq // Hk)
                s = scale * (kk[to, g] @ q[b, i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                e = D * 2.0 ** -24 * scale * (np.abs(kk[to, g]) @ np.abs(q[b, i, h])).max() + 2.0 ** -22 + \
                    2.0 ** -23 * np.abs(s).max() * 1.5 + len(to) * 2.0 ** -24
                out[b, i, h] = p @ vv[to, g]
                off[b, i, h] = R.HALF_STEP[dtype] * np.abs(out[b, i, h]) + \
                    (NUMERATOR[dtype] + 2 * e) * (p @ np.abs(vv[to, g])) + 2.0 ** -24
                if dtype == "float16":
                    off[b, i, h] += len(to) * 2.0 ** -39 * np.abs(vv[to, g]).max(0)
    return out, off


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("N,Hq,Hk,D,past", [(1, 4, 4, 64, 40), (5, 8, 2, 128, 300), (16, 4, 1, 64, 1000), (7, 9, 1, 80, 130),
                                            (70, 1, 1, 256, 200), (3, 6, 2, 136, 2000)])
def test_outputs_near_0(dtype, N, Hq, Hk, D, past):
    # values whose mean is 0: the result's own rounding is small beside that of its parts
    say(f"attend digits N={N} Hq={Hq} Hk={Hk} D={D} past={past} {dtype}")
    d = _inputs(3, N, Hq, Hk, D, 16, past, dtype, N + D, True)
    d["v"] = d["v"] - 0.5
    got = _run(d)[0].double().cpu().numpy()
    out, off = _bounds(d, dtype)
    far = np.abs(got - out) - off
    assert not np.isnan(got).any() and far.max() <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("B,N,Hq,past", [(200, 8, 16, 3), (20, 33, 5, 0), (300, 8, 4, 3)])
def test_log_sum_exp_near_0(B, N, Hq, past, dtype):
    # few slots, whose scores are one exact product each.  An exponent to base 2 is rounded once (a float16's by
    # 2^-21, for 2^14 is made of its row's largest), the factor to base 2 by 2^-24 of the score; the hardware
    # exponential and logarithm are off by 2^-23 (of a sum of up to 2^3), sums by 2^-24 a slot, and the result,
    # of m + log2 and its product with ln 2, by 2^-23 of itself and of m
    D = 8
    say(f"attend lse B={B} N={N} Hq={Hq} past={past} {dtype}")
    d = _inputs(B, N, Hq, 1, D, 16, past, dtype, N, True)
    d["q"][..., 1:], d["k"][..., 1:] = 0, d["k"][..., 1:] * 0     # (NaN stays where nothing is seen)
    d["q"] *= 0.25
    got = _run(d)[1].double().cpu().numpy()
    q, k = (np.nan_to_num(d[x].double().numpy()) for x in "qk")
    scale = float(np.float32(D ** -0.5))
    for b in range(B):
        n, start = int(d["lengths"][b]), int(d["starts"][b])
        kk = R.slots(k, d["pages"], 16, b, start + n)[:, 0]
        assert np.all(got[b, n:] == -np.inf)
        for i in range(n):
            to = R.sees(i, start, n, d["parents"][b])
            for h in range(Hq):
                s = scale * (kk[to] @ q[b, i, h])
                want, size = np.log(np.exp(s).sum()), np.abs(s).max()
                off = np.log(2) * (2.0 ** -21 if dtype == "float16" else 2.0 ** -23) + 2.0 ** -24 * size + 2.0 ** -23 + \
                    max(1, np.log2(len(to))) * 2.0 ** -23 + len(to) * 2.0 ** -24 + 2.0 ** -23 * (abs(want) + size)
                assert abs(got[b, i, h] - want) <= off, (b, i, h, got[b, i, h] - want, off)
