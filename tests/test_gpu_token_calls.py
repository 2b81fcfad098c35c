"""The calls on rows of token logits as a program makes them: on a stream that is not the default
one, inside a captured graph that is replayed, with refusals before anything is launched, and all
together in the chain drafter of examples/."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ERR_WORKSPACE, ERR_LENGTHS, ERR_LABELS = -3, -4, -6
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _tensors(V=9001, dtype="bfloat16", seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, G = 3, 4
    x = (torch.randn((B, G + 1, V), generator=g, device="cuda") * 3).to(getattr(torch, dtype))
    d = (x[:, :G].float() + torch.randn((B, G, V), generator=g, device="cuda")).to(x.dtype)
    u = torch.rand((B, G), generator=g, device="cuda")
    e = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    lens = torch.tensor([4, 2, 0], dtype=torch.int32, device="cuda")
    return x, d, d.argmax(2).to(torch.int32), u, e, lens


def _all(binding, x, d, z, u, e, lens):
    top = binding.top_logits(x, 20, lens)
    loss = binding.distill(x, top[0], top[1], top[2], lens, temperature=2.0)
    grad = binding.distill_grad(d, top[0][:, :-1].contiguous(), top[1][:, :-1].contiguous(),
                                top[2][:, :-1].contiguous(), lens)
    return (*top, loss, *grad, *binding.verify(x, d, z, u, e, lens))


@pytest.mark.parametrize("V", [40, 9001, 70000])
def test_on_another_stream(V):
    import torch
    from paper_2002_00876_amd import binding
    t = _tensors(V)
    want = _all(binding, *t)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy = torch.zeros(1 << 26, device="cuda")
        y = [busy.sum() + v if v.is_floating_point() else v for v in t]   # made on this stream
        y = [a.to(b.dtype) for a, b in zip(y, t)]
        got = _all(binding, *y)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("V", [40, 9001, 70000])
def test_in_a_graph(V):
    import torch
    from paper_2002_00876_amd import binding
    t = _tensors(V)
    _all(binding, *t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _all(binding, *t)
    for seed in (1, 2, 3):
        new = _tensors(V, seed=seed)
        want = _all(binding, *new)
        for a, b in zip(t, new):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), f"replay of seed {seed}"


def test_checked_inputs(monkeypatch):
    import torch
    from paper_2002_00876_amd import binding
    x, d, z, u, e, lens = _tensors(50)
    v, i, l = binding.top_logits(x, 6)
    plain = _all(binding, x, d, z, u, e, lens)
    monkeypatch.setenv("TS_CHECK", "1")
    for a, b in zip(_all(binding, x, d, z, u, e, lens), plain):
        assert torch.equal(a, b)

    def refused(code, call):
        with pytest.raises(binding.TsError) as ei:
            call()
        assert ei.value.code == code

    for bad in (-1, 6):
        n = lens.clone()
        n[1] = bad
        refused(ERR_LENGTHS, lambda: binding.top_logits(x, 6, n))
        refused(ERR_LENGTHS, lambda: binding.distill(x, v, i, lengths=n))
        refused(ERR_LENGTHS, lambda: binding.distill_grad(x, v, i, lengths=n))
        refused(ERR_LENGTHS, lambda: binding.verify(x, d, z, u, e, n))
    for at, bad in (((0, 1, 2), 50), ((0, 1, 2), -2), ((2, 0, 1), int(i[2, 0, 0]))):
        j = i.clone()
        j[at] = bad
        refused(ERR_LABELS, lambda: binding.distill(x, v, j))
        binding.distill(x, v, j, lengths=torch.zeros_like(lens))       # padding is not looked at
    y = z.clone()
    y[0, 1] = 50
    refused(ERR_LABELS, lambda: binding.verify(x, d, y, u, e))


def test_binding_refuses():
    import torch
    from paper_2002_00876_amd import binding
    x, d, z, u, e, lens = _tensors(9000)
    v, i, l = binding.top_logits(x, 6)
    bad = [lambda: binding.top_logits(x[0], 6), lambda: binding.top_logits(x.double(), 6),
           lambda: binding.top_logits(x, 6, lens.long()), lambda: binding.top_logits(x, 6, lens[:2]),
           lambda: binding.top_logits(x, 6, out=(v, i)),
           lambda: binding.top_logits(x, 6, out=(v.float(), i, l)),
           lambda: binding.top_logits(x, 6, out=(v.transpose(0, 1).contiguous().transpose(0, 1), i, l)),
           lambda: binding.distill(x, v, i.long()), lambda: binding.distill(x, v[:, :2], i),
           lambda: binding.distill(x, v, i, l.double()), lambda: binding.distill(x, v, i.cpu()),
           lambda: binding.distill_grad(x, v, i, weights=u),
           lambda: binding.distill_grad(x, v, i, out=(l, d)),
           lambda: binding.verify(x, d[:, :2], z, u, e), lambda: binding.verify(x, d, z, u, e[:2]),
           lambda: binding.verify(x, d, z.long(), u, e), lambda: binding.verify(x, d, z, u.double(), e),
           lambda: binding.verify(x, d, z, u, e, draft_lse=l)]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was not refused")
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.TsError) as ei:
        binding.verify(x, d, z, u, e, ws=small)
    assert ei.value.code == ERR_WORKSPACE
    with pytest.raises(binding.TsError):
        binding.top_logits(x, 257)
    with pytest.raises(binding.TsError):
        binding.distill(x, v, i, temperature=0.0)


def test_chain_drafter_example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import chain_drafter
    finally:
        sys.path.pop(0)
    losses, before, after = chain_drafter.main(steps=60, quiet=True)
    # the chain learns, and what it has learnt makes more of its drafts stand
    assert losses[-1] < 0.7 * losses[0]
    assert after > before + 0.5
