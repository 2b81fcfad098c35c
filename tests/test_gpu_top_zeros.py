"""The K largest logits keep the sign of a zero."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V,K", [(1, 1), (20, 20), (200, 64), (900, 40), (9001, 256), (131073, 30)])
def test_kept_zeros_are_the_logits_themselves(V, K, dtype):
    import torch
    from paper_2002_00876_amd import binding
    say(f"zeros: V={V} K={K} {dtype}")
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    x = -torch.rand((1, 3, V), generator=g, device="cuda").to(getattr(torch, dtype))
    x[0, 0, ::3] = -0.0
    x[0, 1] = -0.0
    x[0, 1, ::2] = 0.0
    x[0, 2, V // 2] = -0.0
    v, i, _ = binding.top_logits(x, K)
    want = x.gather(2, i.long())
    assert torch.equal(v, want) and torch.equal(v.signbit(), want.signbit())
