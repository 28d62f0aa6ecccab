"""Caches whose keys and values share memory are refused by the calls that write them, and those that lie in each other's gaps are not."""
import pytest
import torch

from paper_2601_17261_amd import binding
from test_gpu_cache import ints, new_tokens

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def view(base, at, strides, shape):
    return base.as_strided(shape, strides + (1,), at)


@pytest.mark.parametrize("swap", [False, True])
def test_pages_that_reach_into_each_others_rows(swap):
    """rows 128 values apart, pages of two rows 192: the second row of a page's values is the first of the next page's keys"""
    base = torch.randn(4096, device="cuda").to(BF)
    ctx, cu, rows, kept = binding.Context(), ints([0, 3]), ints([2, -1, -1]), ints([1])
    q, k, v = new_tokens(1, 3, 1, 1, 64)
    table, k_len = ints([[0, 1, 2, 3]]), ints([8])
    for page_stride, refused in ((192, True), (256, False), (320, False)):
        a, b = (view(base, at, (page_stride, 128, 64), (4, 2, 1, 64)) for at in ((64, 0) if swap else (0, 64)))
        before = base.clone()
        cache = binding.make_cache(a, b, table, k_len)
        if refused:
            for call in (lambda: ctx.glue_cache_append(cache, None, None, k, v, None, cu), lambda: ctx.glue_cache_keep(cache, cu, rows, kept)):
                with pytest.raises(binding.AgzoError) as e:
                    call()
                assert e.value.code == binding.EINVAL
            assert torch.equal(base, before)
            out = torch.empty_like(q)
            ctx.glue_attention_paged(cache, q, out, cu)                # which only reads them
            continue
        ctx.glue_cache_append(cache, None, None, k, v, None, cu)
        for place, row in ((5, 0), (6, 1), (7, 2)):
            at = (place // 2, place % 2, 0)
            assert torch.equal(a[at], k[row]) and torch.equal(b[at], v[row])
            before.as_strided((64,), (1,), a[at].storage_offset()).copy_(k[row])
            before.as_strided((64,), (1,), b[at].storage_offset()).copy_(v[row])
        assert torch.equal(base, before)
    ctx.check()
