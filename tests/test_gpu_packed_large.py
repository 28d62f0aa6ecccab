"""Sizes at which a launch would pass 2^32 threads, of which the hardware takes the low 32 bits alone."""
import pytest
import torch

from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def test_norms_with_rotation_of_2_26_tokens():
    """(8.6 GB, in place) every token's result is that of a smaller call"""
    ctx = binding.Context()
    some, n = 1 << 20, (1 << 26) + 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(some, 64, device="cuda", generator=gen).to(BF)
    pos, want = torch.arange(some, device="cuda", dtype=I32), torch.empty_like(x)
    ctx.glue_qk_norm_rope(None, x, pos, None, want, 64)
    k = torch.empty(n, 64, device="cuda", dtype=BF)
    parts = [(i, min(i + some, n)) for i in range(0, n, some)]
    for a, b in parts:
        k[a:b] = x[:b - a]
    ctx.glue_qk_norm_rope(None, k, pos.repeat(65)[:n].contiguous(), None, k, 64)
    assert all(torch.equal(k[a:b], want[:b - a]) for a, b in parts)
