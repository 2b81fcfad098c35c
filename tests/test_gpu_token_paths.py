"""Branches of the calls on rows of token logits that only large calls take: verification with its
positions divided among launches, more drafts than a wave has lanes, more long rows than the top
logits' workspace holds at once, a wave a row in distillation of medium vocabularies."""
import math

import numpy as np
import pytest

import token_ref as R
from gpu_util import say
from test_gpu_distill import _case as distill_case, _check as check_distill
from test_gpu_top_logits import _check as check_top, _normal
from test_gpu_verify import MARGIN, _case as verify_case, _check as check_verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sums", [False, True])
@pytest.mark.parametrize("G,sigma", [(8, 0.7), (20, 0.05), (100, 0.01), (240, 0.005)])
def test_positions_divided_among_launches(G, sigma, sums):
    # more than 16e6 elements a position; four sequences, repeated, some with fewer drafts
    import torch
    from paper_2002_00876_amd import binding
    V = 131072 if G <= 100 else 65537
    copies = math.ceil(16.01e6 / (4 * V))
    say(f"verify in launches: {4 * copies} x {G} x {V}, sums {sums}")
    few = verify_case(4, G, V, "bfloat16", G, sigma=sigma)
    x, d, z, u, noise = (y.repeat(copies, *[1] * (y.dim() - 1)) for y in few)
    lens = [G] * 4 + [0, 1, 2, 5] + [min(G, n) for n in (11, 47, 64, 95)]
    tl = torch.tensor(lens + [G] * (4 * copies - 12), dtype=torch.int32, device="cuda")
    few_dl = torch.logsumexp(few[1].double(), 2).float() if sums else None
    dl = few_dl.repeat(copies, 1) if sums else None
    out, acc, logp = binding.verify(x, d, z, u, noise, tl, dl)
    for b in range(12, 4 * copies, 4):
        for y in (out, acc, logp):
            assert torch.equal(y[b:b + 4], y[:4])
    out, acc, logp = out[:12].cpu().numpy(), acc[:12].cpu().numpy(), logp[:12].double().cpu().numpy()
    hx, hd, hu, hn = (few[k].float().cpu().numpy() for k in (0, 1, 3, 4))
    hz, hl = few[2].cpu().numpy(), few_dl.double().cpu().numpy() if sums else None
    stops = set()
    for b in range(12):
        k = b % 4
        ro, ra, rl, margin = R.verify(hx[k].astype(np.float64), hd[k].astype(np.float64), hz[k],
                                      hu[k].astype(np.float64), hn[k].astype(np.float64), lens[b],
                                      1.0, 1.0, hl[k] if sums else None)
        assert margin > MARGIN, f"the seed leaves a margin of {margin:.1e} in sequence {b}"
        assert acc[b] == ra and out[b, : ra + 1].tolist() == ro, (b, acc[b], ra)
        assert np.all(out[b, ra + 1:] == -1) and np.all(logp[b, ra + 1:] == 0)
        for t, r in enumerate(rl):
            most = R.EPS * (R.UNITS + R.span(hx[k, t].astype(np.float64), 1.0) + abs(r))
            assert abs(logp[b, t] - r) <= most, (b, t)
        stops.add(ra)
    say(f"accepted: {sorted(stops)}")
    assert len(stops) >= 4


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [24, 50, 3000])
def test_more_drafts_than_lanes(V, dtype):
    import torch
    G = 150
    x, d, z, u, noise = verify_case(6, G, V, dtype, V, sigma=0.002)
    lens = [150, 63, 64, 65, 128, 129]
    share = check_verify(x, d, z, u, noise, lens=lens, tag="many drafts")
    assert share > 0.3
    check_verify(x, d, z, u, noise, lens=lens, dl=torch.logsumexp(d.double(), 2).float(),
                 tag="many drafts, their sums")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_more_long_rows_than_the_workspace_holds(dtype):
    check_top(_normal((3, 1500, 1100), dtype, 17), 40, [1500, 700, 1500], tag="slabs")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("V", [1025, 8191])
def test_a_wave_a_row_of_medium_vocabularies(V, rest):
    for dtype in ("float32", "bfloat16"):
        c = distill_case(3, 700, V, 70, dtype, V, empty=0.2, rest=rest)
        check_distill(*c, lens=[700, 650, 0], tag="a wave a row")
