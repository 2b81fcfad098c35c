"""Workspaces that a caller gives to the calls on rows of token logits: refused where the kernels
could not write them, used where they are large enough, whatever they hold and whatever their type."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


def _calls():
    import torch
    from paper_2002_00876_amd import binding as b
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    B, G, V, K = 2, 3, 20001, 6
    x = torch.randn((B, G + 1, V), generator=g, device="cuda")
    v, i, l = b.top_logits(x, K)
    z, u = i[:, :G, 0].contiguous(), torch.rand((B, G), generator=g, device="cuda")
    e = torch.rand((B, V), generator=g, device="cuda") + 0.1
    return {b.TOKEN_TOP: (lambda **kw: b.top_logits(x, K, **kw), (B, G + 1, V, K)),
            b.TOKEN_DISTILL: (lambda **kw: (b.distill(x, v, i, l, **kw),), (B, G + 1, V, K)),
            b.TOKEN_DISTILL_GRAD: (lambda **kw: b.distill_grad(x, v, i, l, **kw), (B, G + 1, V, K)),
            b.TOKEN_VERIFY: (lambda **kw: b.verify(x, x[:, :G], z, u, e, **kw), (B, G, V, 1))}


@pytest.mark.parametrize("op", range(4))
def test_workspaces_that_kernels_cannot_write(op):
    import torch
    from paper_2002_00876_amd import binding
    call, size = _calls()[op]
    need = binding.token_workspace_bytes(op, *size)
    say(f"workspace of operation {op}: {need} bytes")
    assert need > 0
    one = torch.empty(256, dtype=torch.uint8, device="cuda")
    for bad in (torch.empty(need, dtype=torch.uint8), one[:1].expand(need),
                torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(ws=bad)


@pytest.mark.parametrize("op", range(4))
def test_workspaces_of_any_type_and_contents(op):
    import torch
    from paper_2002_00876_amd import binding
    call, size = _calls()[op]
    need = binding.token_workspace_bytes(op, *size)
    want = call()
    for dtype in (torch.uint8, torch.float32, torch.int64):
        ws = torch.full(((need + 7) // 8 * 8,), 0xFF, dtype=torch.uint8, device="cuda").view(dtype)
        for a, b in zip(call(ws=ws), want):
            assert torch.equal(a, b)
