"""Attention over pages with many rows a sequence where sequences have room for thousands of keys (row tiles of 256): lengths, trees, masks, values that are not finite, replays."""
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_cache import Pages, ints, offsets
from test_gpu_paged_attention import check, queries, trees, words

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def room(page):
    return 4096 // page


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 48, 64, 256])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2), (7, 1)])
def test_pieces_of_prompts(dim, page, heads, kv):
    new, have = [0, 1, 330, 264, 233, 7, 257, 256, 600], [5, 1, 330, 364, 900, 1007, 257, 256 + 64, 663]
    check(Pages(page, have, page, kv, dim, more=room(page)), queries(12, sum(new), heads, dim), new, have, dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("keys", [1, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 321, 449])
def test_few_tiles_of_keys(dim, keys):
    """as many as are on their way at a time, one less, one more"""
    check(Pages(keys, [keys], 16, 1, dim, more=room(16)), queries(keys, keys, 140, dim) if keys < 3 else queries(keys, keys, 130 // keys + 4, dim), [keys], [keys], dim)


@pytest.mark.parametrize("layout", ["heads", "pages", "rows", "pairs"])
def test_layouts(layout):
    new, have = [150, 3, 200], [270, 3, 500]
    for dim in (64, 128):
        check(Pages(1, have, 32, 2, dim, layout, more=room(32)), queries(1, sum(new), 6, dim), new, have, dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv", [(8, 1), (14, 2)])
def test_trees(dim, heads, kv):
    new, have = [1, 2, 31, 32, 33, 64, 65, 100], [1, 40, 31, 90, 33 + 31, 64 + 64, 500, 1000]
    check(Pages(2, have, 16, kv, dim, more=room(16)), queries(3, sum(new), heads, dim), new, have, dim, bits=trees(5, new))


@pytest.mark.parametrize("kind", ["tree", "chunk"])
@pytest.mark.parametrize("dim,heads,kv", [(128, 16, 2), (64, 12, 4), (128, 7, 1)])
def test_in_shares(kind, dim, heads, kv):
    have = [9000, 3, 2500, 700, 64]
    new = [60, 3, 37, 64, 1] if kind == "tree" else [300, 2, 330, 500, 64]
    check(Pages(5, have, 16, kv, dim, more=20), queries(4, sum(new), heads, dim), new, have, dim, bits=trees(4, new) if kind == "tree" else None)


def test_many_sequences():
    rng = random.Random(5)
    for n in (64, 65, 150):
        have = [rng.choice([1, 65, 140, 900]) for _ in range(n)]
        new = [min(h, rng.choice([0, 1, 90, 160])) for h in have]
        assert sum(new) * 4 > 128 * n
        check(Pages(n, have, 16, 1, 64, more=room(16)), queries(n, sum(new), 4, 64), new, have, 64)


def test_rows_that_see_nothing():
    new, have = [300, 3, 340, 2], [2, 0, 10, 1000]
    c = Pages(1, [2, 1, 10, 20], 16, 2, 64, more=room(16))
    c.k_len = ints([2, -9, 10, 1000])
    q = queries(1, sum(new), 4, 64)
    out, lse = check(c, q, new, have, 64)
    assert (out[:298] == 0).all() and torch.isinf(lse[:298]).all() and (out[300:303] == 0).all()
    rng = random.Random(3)
    bits = [rng.choice([0, 1, 1 << 299, 0b10, (1 << 300) - 1, 1 << 40]) for _ in range(sum(new))]
    check(c, q, new, have, 64, bits=[b & (1 << 320) - 1 for b in bits])
    check(c, q, new, have, 64, bits=[0] * sum(new), tree=torch.empty(sum(new), 0, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_is_not_seen_takes_no_part(bad, dim):
    new, have, heads, kv = [6, 40, 1, 270], [50, 40, 33, 2500], 8, 2
    c = Pages(3, have, 16, kv, dim, more=room(16))
    q, bits = queries(3, sum(new), heads, dim, 0.3), trees(7, new)
    used = torch.zeros(c.k.shape[:2], dtype=torch.bool, device="cuda")
    for s, h in enumerate(have):
        for p in range(h):
            used[ref.slot(c.table, 16, c.k.shape[0], s, p)] = True
    c.k[~used], c.v[~used] = bad, bad
    check(c, q, new, have, dim)
    check(c, q, new, have, dim, bits=bits)
    for s, i in ((0, 3), (1, 20), (3, 269), (3, 10), (3, 150)):
        c.v[ref.slot(c.table, 16, c.k.shape[0], s, have[s] - new[s] + i)][0, 5] = bad
    check(c, q, new, have, dim)
    check(c, q, new, have, dim, bits=bits)
    c = Pages(4, have, 16, kv, dim, more=room(16))
    bits = [b & ~(1 << 2) for b in bits]
    for s in (0, 1, 3):
        at = ref.slot(c.table, 16, c.k.shape[0], s, have[s] - new[s] + 2)
        c.k[at], c.v[at] = bad, bad
    check(c, q, new, have, dim, bits=bits)


def test_scores_far_from_zero():
    new, have = [150, 5, 390], [900, 60, 3000]
    for gain, scale in ((30.0, None), (1.0, 4.0), (1.0, 1e-4), (0.0, None)):
        check(Pages(6, have, 16, 2, 128), queries(6, sum(new), 4, 128, gain), new, have, 128, scale=scale)


def test_ids_that_are_no_pages_are_the_nearest_and_rows_of_no_sequence():
    new, have = [140, 160], [240, 3060]
    c = Pages(7, have, 16, 2, 64)
    c.table[0][1], c.table[1][2], c.table[1][100] = 2 ** 31 - 1, -(2 ** 31), -1
    check(c, queries(7, 309, 4, 64), new, have, 64, tail=9)


def test_repeats_and_replays():
    """with the same bits, eager and captured, beside other calls of the context"""
    side = torch.cuda.Stream()
    ctx, plain = binding.Context(side), binding.Context()
    new, have = [300, 1, 200], [6000, 500, 2000]
    c, q, cu = Pages(9, have, 16, 2, 128), queries(9, 501, 8, 128), ints(offsets(new))
    single, cu1 = queries(10, 3, 8, 128), ints([0, 1, 2, 3])
    cache = c.cache()
    out, out1, want, want1 = torch.empty_like(q), torch.empty_like(single), torch.empty_like(q), torch.empty_like(single)
    torch.cuda.synchronize()
    ctx.glue_attention_paged(cache, q, out, cu)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.glue_attention_paged(cache, q, out, cu)
        ctx.glue_attention_paged(cache, single, out1, cu1)
    for lens in (have, [5000, 400, 1999], [1, 2, 3], [6001, 77, 2048], have):
        c.k_len.copy_(ints(lens))
        out.fill_(3), out1.fill_(3)
        torch.cuda.synchronize()
        for _ in range(3):
            g.replay()
        plain.glue_attention_paged(cache, q, want, cu)
        plain.glue_attention_paged(cache, single, want1, cu1)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out1, want1)
