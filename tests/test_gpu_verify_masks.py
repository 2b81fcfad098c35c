"""Verification of drafts whose logits are masked, by -inf or by the type's lowest value, on either
side, or whose probabilities are below the 32-bit floats; against float64."""
import pytest

import token_ref as R
from test_gpu_verify import _case, _check

pytestmark = pytest.mark.gpu

INF = float("inf")


def _sums(d, dT):
    import torch
    return torch.logsumexp(d.double() / dT, 2).float()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T", [1.0, 0.7, 2.0])
@pytest.mark.parametrize("V", [50, 20000])
def test_masked_drafts(V, T, dtype):
    import torch
    x, d, z, u, noise = _case(5, 2, V, dtype, 20 + V, T=T, dT=T)
    lowest = torch.finfo(x.dtype).min
    at = z[:, 0].long()
    for b, (p, q) in enumerate([(None, lowest), (None, -INF), (lowest, lowest), (-INF, lowest),
                                (-INF, -INF)]):
        # q = 0: accepted where p > 0, whatever the uniform, and refused where p = 0
        if p is not None:
            x[b, 0, at[b]] = p
        d[b, 0, at[b]] = q
    u[:, 0] = 1 - 2.0 ** -24
    _check(x, d, z, u, noise, T=T, dT=T, tag="masked drafts")
    _check(x, d, z, u, noise, dl=_sums(d, T), T=T, dT=T, tag="masked drafts, their sums")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T", [1.0, 0.7, 2.0])
@pytest.mark.parametrize("V", [50, 20000])
def test_drafts_masked_on_both_sides_in_different_ways(V, T, dtype):
    # p of the type's lowest value is 0 in 64 bits too: it refuses a draft of q = 0
    import torch
    x, d, z, u, noise = _case(2, 2, V, dtype, 50 + V, T=T, dT=T)
    at = z[:, 0].long()
    x[0, 0, at[0]] = torch.finfo(x.dtype).min
    d[0, 0, at[0]] = -INF
    x[1, 0, at[1]] = x[1, 0].max() - 600 * T             # e^-600 is not, and does not
    d[1, 0, at[1]] = -INF
    _check(x, d, z, u, noise, T=T, dT=T, tag="masked twice")
    _check(x, d, z, u, noise, dl=_sums(d, T), T=T, dT=T, tag="masked twice, their sums")


@pytest.mark.parametrize("V", [50, 20000])
def test_drafts_far_below_the_maximum(V):
    # p and q of e^-200 and e^-300: neither is a 32-bit float, which is larger is decided all the same
    x, d, z, u, noise = _case(4, 2, V, "float32", 40 + V)
    at = z[:, 0].long()
    for b, (p, q) in enumerate([(200, 300), (300, 200), (95, 200), (200, 95)]):
        x[b, 0, at[b]] = x[b, 0].max() - p
        d[b, 0, at[b]] = d[b, 0].max() - q
    _check(x, d, z, u, noise, tag="far drafts")
    _check(x, d, z, u, noise, dl=_sums(d, 1.0), tag="far drafts, their sums")


@pytest.mark.parametrize("V", [50, 20000])
def test_drafts_from_nowhere_with_their_sums(V):
    # a draft's row without a finite logit has a log-sum-exp of -inf and q = 0: what remains of a
    # refused draft is the target's row
    x, d, z, u, noise = _case(5, 2, V, "float32", 30 + V)
    d[:, 0] = -INF
    x[1, 0, z[1, 0].long()] = -INF
    x[2, 0] = -INF
    z[3, 0] = -1
    _check(x, d, z, u, noise, tag="nowhere")
    _check(x, d, z, u, noise, dl=_sums(d, 1.0), tag="nowhere, its sums")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [1, 50, 20000])
def test_drafts_whose_sums_underflow(V, dtype):
    # a draft's row of the type's lowest value has a log-sum-exp below the floats at T < 1: given as
    # -inf it says q = 0
    import torch
    x, d, z, u, noise = _case(3, 2, V, dtype, 60 + V, T=0.5, dT=0.5)
    d[:, 0] = torch.finfo(d.dtype).min
    x[1, 0, z[1, 0].long()] = -INF
    sums = _sums(d, 0.5)
    assert bool((sums[:, 0] == -INF).all())
    _check(x, d, z, u, noise, dl=sums, T=0.5, dT=0.5, tag="sums of -inf")


@pytest.mark.parametrize("V", [50, 20000])
def test_sums_of_nothing_beside_large_logits(V):
    # q = 0 is what a log-sum-exp of -inf says, whatever the draft's logits: a refused draft leaves p
    import torch
    x, d, z, u, noise = _case(4, 2, V, "float32", 70 + V)
    d[:, 0, ::2] += 300
    sums = _sums(d, 1.0)
    sums[:, 0] = -INF
    x[:, 0] = torch.where(x[:, 0] == x[:, 0].amax(1, keepdim=True), 2.0, x[:, 0].clamp(max=2.0))
    z[:2, 0] = -1
    _check(x, d, z, u, noise, dl=sums, tag="sums of nothing")
