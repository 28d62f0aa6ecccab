"""Attention over pages at the longest sequences that the call takes: nearly 2^31 places, which a table gives few pages again and again."""
import math

import pytest
import torch

from paper_2601_17261_amd import binding
from test_gpu_cache import ints

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("page,heads,new", [(2 ** 16, 1, [1]), (2 ** 16, 7, [3]), (2 ** 16, 24, [6, 1]), (99999, 5, [4])])
def test_the_mean_of_many_values(page, heads, new):
    """queries of zeros weigh all places alike: sums of small whole numbers and their count, which are exact up to 2^24 and rounded to 2^-24 each time that parts of more are joined"""
    dim, pages = 64, (2 ** 31 - 1 - 1024) // page
    gen = torch.Generator().manual_seed(heads)
    v = torch.randint(-3, 4, (3, 1, 1, dim), generator=gen).to(BF).cuda().expand(3, page, 1, dim).contiguous()
    k = torch.randn(3, page, 1, dim, device="cuda").to(BF)
    which = torch.randint(0, 3, (len(new), pages), generator=gen, dtype=torch.int32)
    have = [pages * page, pages * page - 12345][:len(new)]
    cu = [0, *torch.tensor(new).cumsum(0).tolist()]
    q = torch.zeros(cu[-1], heads * dim, device="cuda", dtype=BF)
    out, lse = torch.full_like(q, 7.0), torch.empty(cu[-1], heads, device="cuda")
    ctx = binding.Context()
    ctx.glue_attention_paged(binding.make_cache(k, v, which.cuda(), ints(have)), q, out, ints(cu), lse=lse)
    ctx.check()
    value = v[:, 0, 0].double()
    for s, m in enumerate(new):
        for i in range(m):
            seen = have[s] - m + i + 1
            full, rest = seen // page, seen % page
            count = torch.bincount(which[s, :full].long(), minlength=3).double() * page
            if rest:
                count[which[s, full]] += rest
            o = count.cuda() @ value / seen
            # the result's rounding; some 2^10 parts joined, of sums of up to three a place
            assert ((out[cu[s] + i].double().view(heads, dim) - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** 11 * 2.0 ** -24 * 3).all()
            assert (lse[cu[s] + i].double() - math.log(seen)).abs().max() <= 2.0 ** 11 * 2.0 ** -24
