"""Verification of drafted tokens against float64, sequence by sequence.  What is decided are
whole tokens: an outcome may differ only where a decision's margin (the relative distance from
going the other way) is below what 32-bit sums may be off by, and the seeds here leave no such
case."""
import math

import numpy as np
import pytest

import token_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
MARGIN = 64 * R.EPS


def _case(B, G, V, dtype, seed=0, sigma=0.7, ddtype=None, T=1.0, dT=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((B, G + 1, V), generator=g, device="cuda") * 2
    x[..., : min(V, 5)] += 6
    d = x[:, :G] + sigma * torch.randn((B, G, V), generator=g, device="cuda")
    x, d = x.to(getattr(torch, dtype)), d.to(getattr(torch, ddtype or dtype))
    e = torch.empty((B, G, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    z = (d.float() / dT - e.log()).argmax(2).to(torch.int32) if G else torch.empty(
        (B, 0), dtype=torch.int32, device="cuda")
    u = torch.rand((B, G), generator=g, device="cuda")
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    return x, d, z, u, noise


def _check(x, d, z, u, noise, lens=None, dl=None, T=1.0, dT=1.0, tag=""):
    import torch
    from paper_2002_00876_amd import binding
    say(f"verify {tag}: {tuple(x.shape)} {x.dtype} {d.dtype}")
    tl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, acc, logp = binding.verify(x, d, z, u, noise, tl, dl, T, dT)
    torch.cuda.synchronize()
    B, G = x.shape[0], x.shape[1] - 1
    assert out.shape == (B, G + 1) and out.dtype == torch.int32
    out, acc, logp = out.cpu().numpy(), acc.cpu().numpy(), logp.double().cpu().numpy()
    hx, hd, hu, hn = (y.double().cpu().numpy() for y in (x, d, u, noise))
    hz, hl = z.cpu().numpy(), None if dl is None else dl.double().cpu().numpy()
    some = 0
    for b in range(B):
        n = G if lens is None else min(max(lens[b], 0), G)
        ro, ra, rl, margin = R.verify(hx[b], hd[b], hz[b], hu[b], hn[b], n, T, dT,
                                      None if hl is None else hl[b])
        assert margin > MARGIN, f"the seed leaves a margin of {margin:.1e} in sequence {b}"
        assert acc[b] == ra and out[b, : ra + 1].tolist() == ro, (b, out[b], ro)
        assert np.all(out[b, ra + 1:] == -1) and np.all(logp[b, ra + 1:] == 0)
        for t, r in enumerate(rl):
            if math.isinf(r):
                assert logp[b, t] == r
            else:
                most = R.EPS * (R.UNITS + R.span(hx[b, t], T) + abs(r))
                assert abs(logp[b, t] - r) <= most, (b, t)
        some += ra
    return some / max(1, B * G)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,V", [(0, 20), (1, 1), (1, 2), (3, 20), (4, 256), (2, 257), (5, 1000),
                                 (3, 16385), (8, 50001), (2, 140001)])
def test_sizes(G, V, dtype):
    _check(*_case(5, G, V, dtype, 100 * G + V), tag="sizes")


def test_some_are_accepted_and_some_are_not():
    share = _check(*_case(64, 6, 300, "float32", 1), tag="share")
    assert 0.2 < share < 0.95


@pytest.mark.parametrize("V", [33, 3000, 40000])
def test_lengths_and_types(V):
    for dtype in TYPES:
        for ddtype in TYPES:
            _check(*_case(6, 4, V, dtype, V, ddtype=ddtype), lens=[4, 0, 1, 2, 3, 4],
                   tag=f"lengths {ddtype}")


@pytest.mark.parametrize("T,dT", [(0.5, 1.0), (2.0, 2.0), (0.7, 1.3)])
def test_temperatures(T, dT):
    _check(*_case(8, 3, 2000, "bfloat16", 3, T=T, dT=dT), T=T, dT=dT, tag="temperatures")


@pytest.mark.parametrize("V", [50, 20000])
def test_known_sums_of_the_drafts(V):
    # normalised drafts: no sum over their rows; others with their own log-sum-exp
    import torch
    x, d, z, u, noise = _case(12, 4, V, "float32", 4)
    want = torch.logsumexp(d.double(), 2)
    _check(x, d, z, u, noise, dl=want.float(), tag="draft_lse")
    _check(x, (d.double() - want[..., None]).float(), z, u, noise,
           dl=torch.zeros((12, 4), device="cuda"), tag="normalised")


@pytest.mark.parametrize("V", [50, 20000])
def test_masked_tokens_and_empty_rows(V):
    import torch
    inf = float("inf")
    x, d, z, u, noise = _case(7, 2, V, "float32", 6)
    x[0, 0] = -inf                                     # nothing can follow: token 0
    x[1, 0, z[1, 0].long()] = -inf                     # the draft cannot
    d[2, 0] = -inf                                     # a draft from nowhere
    x[3, :, 1:] = -inf                                 # only one can
    x[4, :, ::2] = torch.finfo(torch.float32).min
    z[5, 0], z[6, 1] = -1, V                           # no tokens: refused
    _check(x, d, z, u, noise, tag="masked")


def test_equal_rows_accept_everything_and_opposite_rows_nothing():
    import torch
    x, d, z, u, noise = _case(6, 5, 900, "float32", 8, sigma=0.0)
    from paper_2002_00876_amd import binding
    out, acc, _ = binding.verify(x, d, z, u, noise)
    assert torch.equal(acc, torch.full_like(acc, 5)) and torch.equal(out[:, :5], z)
    x.scatter_(2, torch.cat([z, z[:, :1]], 1).long()[..., None], -float("inf"))
    out, acc, _ = binding.verify(x, d, z, u, noise)
    assert torch.equal(acc, torch.zeros_like(acc)) and bool((out[:, 0] != z[:, 0]).all())


def test_residual_of_equal_rows_falls_back_to_the_target():
    # p = q refused by a uniform of 1: what is left is nothing, the draw is the target's
    import torch
    from paper_2002_00876_amd import binding
    for V in (40, 30000):
        x, d, z, u, noise = _case(4, 1, V, "float32", 9, sigma=0.0)
        out, acc, _ = binding.verify(x, d, z, torch.ones_like(u), noise)
        p = torch.softmax(x[:, 0].double(), 1)
        assert torch.equal(acc, torch.zeros_like(acc))
        assert torch.equal(out[:, 0].long(), (p / noise.double()).argmax(1))


def test_emitted_tokens_follow_the_target():
    # 20000 sequences of the same rows: the first emitted token's frequencies are the target's
    # within 5 standard deviations
    import torch
    from paper_2002_00876_amd import binding
    B, V = 20000, 12
    x, d, _, _, _ = _case(1, 1, V, "float32", 10, sigma=1.5)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    q = torch.softmax(d[0, 0].double(), 0)
    z = torch.multinomial(q, B, True, generator=g).to(torch.int32)[:, None]
    u = torch.rand((B, 1), generator=g, device="cuda")
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    out, acc, _ = binding.verify(x.expand(B, 2, V), d.expand(B, 1, V), z, u, noise)
    p = torch.softmax(x[0, 0].double(), 0)
    got = torch.bincount(out[:, 0].long(), minlength=V).double() / B
    assert bool(((got - p).abs() <= 5 * (p * (1 - p) / B).sqrt()).all())
    want = torch.minimum(p, q).sum()
    assert abs(acc.double().mean() - want) <= 5 * (want * (1 - want) / B).sqrt()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [31, 16391])
def test_strides_and_masked_places(V, dtype):
    import torch
    from paper_2002_00876_amd import binding
    x, d, z, u, noise = _case(3, 3, V, dtype, 12)
    lens = torch.tensor([3, 0, 1], dtype=torch.int32, device="cuda")
    bx = torch.full((3, 6, V + 9), float("nan"), dtype=x.dtype, device="cuda")
    bd = torch.full((4, 3, V + 3), float("nan"), dtype=x.dtype, device="cuda")
    x2, d2 = bx[:, 1:5, 5:5 + V], bd[1:, :, 1:1 + V]
    x2.copy_(x)
    d2.copy_(d)
    for b, n in enumerate([3, 0, 1]):
        x2[b, n + 1:] = float("nan")
        d2[b, n:] = float("nan")
    for a, b in zip(binding.verify(x, d, z, u, noise, lens),
                    binding.verify(x2, d2, z, u, noise, lens)):
        assert torch.equal(a, b)


def test_rows_past_32_bit_offsets():
    import torch
    from paper_2002_00876_amd import binding
    V = 3000
    x, d, z, u, noise = _case(2, 1, V, "bfloat16", 13)
    big = torch.empty(2 ** 32 + 2 ** 21, dtype=torch.bfloat16, device="cuda")
    x2 = big.as_strided((2, 2, V), (2 ** 32 + 3, V, 1))
    d2 = big[2 * V:].as_strided((2, 1, V), (2 ** 32 + 3, V, 1))
    x2.copy_(x)
    d2.copy_(d)
    for a, b in zip(binding.verify(x, d, z, u, noise), binding.verify(x2, d2, z, u, noise)):
        assert torch.equal(a, b)


def test_out_workspace_and_repeats():
    import torch
    from paper_2002_00876_amd import binding
    x, d, z, u, noise = _case(20, 4, 50001, "bfloat16", 14)
    first = binding.verify(x, d, z, u, noise)
    out = tuple(torch.empty_like(t) for t in first)
    ws = torch.full((max(1, binding.token_workspace_bytes(binding.TOKEN_VERIFY, 20, 4, 50001)),), 0xA5,
                    dtype=torch.uint8, device="cuda")
    for _ in range(3):
        again = binding.verify(x, d, z, u, noise, out=out, ws=ws)
        for a, b, c in zip(first, again, out):
            assert torch.equal(a, b) and b.data_ptr() == c.data_ptr()
