"""Appending to a paged cache with the rotation of positions against float64."""
import numpy as np
import pytest

import cache_ref as R
from gpu_util import say

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _inputs(B, N, Hq, Hk, D, S, past, dtype, R_, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    starts = rng.integers(0, past, endpoint=True, size=B)
    lengths = rng.integers(0, N, endpoint=True, size=B)
    lengths[-1] = N
    M = -(-(past + N) // S)
    P = B * M + 2
    pages = rng.permutation(P)[:B * M].reshape(B, M)

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(getattr(torch, dtype))

    freqs = (10000.0 ** (-np.arange(0, R_, 2) / max(R_, 1))).astype(np.float32)
    return dict(q=normal(B, N, Hq, D) if Hq else None, k=normal(B, N, Hk, D), v=normal(B, N, Hk, D),
                kc=normal(P, S, Hk, D), vc=normal(P, S, Hk, D), pages=pages, starts=starts,
                lengths=lengths, freqs=freqs, positions=None)


def _run(d, neighbours=False, kc=None, vc=None, out=None, q=None):
    import torch
    from paper_2002_00876_amd import binding
    kc = d["kc"].cuda() if kc is None else kc
    vc = d["vc"].cuda() if vc is None else vc
    q = d["q"].cuda() if q is None and d["q"] is not None else q
    freqs = torch.from_numpy(d["freqs"]).cuda() if len(d["freqs"]) else None
    got = binding.cache_append(d["k"].cuda(), d["v"].cuda(), kc, vc, _ints(d["pages"]),
                               _ints(d["starts"]), _ints(d["lengths"]), q=q, freqs=freqs,
                               positions=_ints(d["positions"]), neighbours=neighbours, out=out)
    torch.cuda.synchronize()
    return got, kc, vc


def _compare(d, got, neighbours=False):
    dtype = str(d["k"].dtype).replace("torch.", "")
    B, N = d["k"].shape[:2]
    S, most = d["kc"].shape[1], d["pages"].shape[1] * d["kc"].shape[1]
    q, kc, vc = got
    k_want, v_want = d["kc"].double().numpy().copy(), d["vc"].double().numpy().copy()
    off = np.zeros(k_want.shape)
    starts = np.clip(d["starts"], 0, most)
    at = starts[:, None] + np.arange(N)[None]
    positions = at if d["positions"] is None else d["positions"]
    k, koff = R.rotate(d["k"].double().numpy(), positions, d["freqs"], neighbours, dtype)
    v = d["v"].double().numpy()
    lengths = [N] * B if d["lengths"] is None else np.clip(d["lengths"], 0, N)
    for b in range(B):
        for n in range(lengths[b]):
            j = at[b, n]
            if j < most and 0 <= d["pages"][b, j // S] < len(k_want):
                page = d["pages"][b, j // S], j % S
                k_want[page], off[page], v_want[page] = k[b, n], koff[b, n], v[b, n]
    assert np.array_equal(vc.double().cpu().numpy(), v_want)
    assert (np.abs(kc.double().cpu().numpy() - k_want) <= off).all()
    if d["q"] is None:
        assert q is None
        return
    q_want, qoff = R.rotate(d["q"].double().numpy(), positions, d["freqs"], neighbours, dtype)
    q = q.double().cpu().numpy()
    for b in range(B):
        assert (np.abs(q[b, :lengths[b]] - q_want[b, :lengths[b]]) <= qoff[b, :lengths[b]]).all()
        assert (q[b, lengths[b]:] == 0).all()


def _check(*sizes, neighbours=False, seed=0):
    say(f"append {sizes} neighbours={neighbours}")
    d = _inputs(*sizes, seed=seed)
    _compare(d, _run(d, neighbours), neighbours)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("D,R_", [(8, 0), (16, 16), (64, 64), (80, 80), (80, 32), (128, 128), (128, 16),
                                  (136, 128), (256, 256), (256, 0)])
def test_heads(dtype, neighbours, D, R_):
    _check(3, 5, 6, 2, D, 16, 200, dtype, R_, neighbours=neighbours, seed=D + R_)


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 300])
@pytest.mark.parametrize("S", [1, 3, 16, 48, 256])
def test_pages(N, S):
    _check(2, N, 4, 1, 64, S, 100, "bfloat16", 64, seed=N + S)


@pytest.mark.parametrize("Hq,Hk", [(0, 1), (0, 8), (1, 1), (71, 71), (128, 1), (28, 4)])
def test_numbers_of_heads(Hq, Hk):
    _check(2, 3, Hq, Hk, 128, 16, 40, "float16", 128, seed=Hq)


def test_far_positions():
    # angles of up to 2 10^9 turns' worth of radians, and negative ones
    d = _inputs(2, 4, 2, 1, 64, 16, 40, "float16", 64)
    d["positions"] = np.array([[10 ** 6, 2 ** 31 - 1, 123456789, 0], [-1, -10 ** 6, 7, 1 << 24]])
    for neighbours in (False, True):
        _compare(d, _run(d, neighbours), neighbours)


def test_nothing_to_write():
    d = _inputs(3, 4, 2, 2, 64, 16, 40, "bfloat16", 64)
    d["lengths"] = np.array([0, -3, 0])
    _compare(d, _run(d))
    d["lengths"], d["starts"] = np.array([4, 4, 99]), np.array([62, 4000, -5])   # past the table; clamped
    d["pages"] = d["pages"][:, :3]
    _compare(d, _run(d))
    d["starts"] = np.array([0, 16, 30])
    d["pages"][0, 0], d["pages"][1, 1] = -1, d["kc"].shape[0]                    # pages not there
    _compare(d, _run(d))


def test_strides_and_places():
    # views of one product's rows, a cache with heads before tokens, queries rotated in place
    import torch
    from paper_2002_00876_amd import binding
    for neighbours in (False, True):
        d = _inputs(2, 9, 4, 2, 64, 16, 60, "bfloat16", 32)
        qkv = torch.cat([d["q"], d["k"], d["v"]], 2).cuda()
        q, k, v = qkv.split([4, 2, 2], 2)
        kc = d["kc"].transpose(1, 2).contiguous().cuda().transpose(1, 2)
        vc = d["vc"].transpose(1, 2).contiguous().cuda().transpose(1, 2)
        freqs = torch.from_numpy(d["freqs"]).cuda()
        got = binding.cache_append(k, v, kc, vc, _ints(d["pages"]), _ints(d["starts"]),
                                   _ints(d["lengths"]), q=q, freqs=freqs, neighbours=neighbours)
        _compare(d, (got, kc, vc), neighbours)
        assert torch.equal(qkv, torch.cat([d["q"], d["k"], d["v"]], 2).cuda())
        own = d["q"].cuda()
        again, kc2, vc2 = _run(d, neighbours, q=own, out=own)
        assert again is own and torch.equal(own, got) and torch.equal(kc2, kc) and torch.equal(vc2, vc)
        odd = torch.zeros((2, 9, 2, 65), dtype=torch.bfloat16, device="cuda")   # heads not aligned
        odd[..., 1:] = d["k"].cuda()
        kc3, vc3 = d["kc"].cuda(), d["vc"].cuda()
        binding.cache_append(odd[..., 1:], v, kc3, vc3, _ints(d["pages"]), _ints(d["starts"]),
                             _ints(d["lengths"]), freqs=freqs, neighbours=neighbours)
        assert torch.equal(kc3, kc) and torch.equal(vc3, vc)


def test_captured():
    import torch
    from paper_2002_00876_amd import binding
    d = _inputs(2, 3, 4, 2, 64, 16, 200, "bfloat16", 64)
    t = {x: _ints(d[x]) if x in ("pages", "starts", "lengths") else d[x].cuda() for x in
         ("q", "k", "v", "kc", "vc", "pages", "starts", "lengths")}
    freqs = torch.from_numpy(d["freqs"]).cuda()

    def call(kc, vc):
        return binding.cache_append(t["k"], t["v"], kc, vc, t["pages"], t["starts"], t["lengths"],
                                    q=t["q"], freqs=freqs)

    call(t["kc"].clone(), t["vc"].clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q = call(t["kc"], t["vc"])
    kc, vc = d["kc"].cuda(), d["vc"].cuda()
    for step in range(4):
        t["starts"].copy_(_ints(np.minimum(d["starts"] + step * 3, 197)))
        t["k"].mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        want = call(kc, vc)
        torch.cuda.synchronize()
        assert torch.equal(q, want) and torch.equal(t["kc"], kc) and torch.equal(t["vc"], vc)


def test_checked(monkeypatch):
    from paper_2002_00876_amd import binding
    monkeypatch.setenv("TS_CHECK", "1")
    d = _inputs(2, 5, 4, 2, 64, 16, 90, "bfloat16", 64)
    d["lengths"] = np.array([5, 5])
    _run(d)
    page = int(d["starts"][0]) // 16
    for name, at, value, code in (("starts", 1, -1, -4), ("starts", 0, 10 ** 6, -4),
                                  ("lengths", 1, 6, -4), ("pages", (0, page), -1, -6)):
        bad = {**d, name: d[name].copy()}
        bad[name][at] = value
        with pytest.raises(binding.TsError) as e:
            _run(bad)
        assert e.value.code == code, name
