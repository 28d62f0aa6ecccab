"""Attention over pages: whose probabilities keep two bf16 parts (a sequence of one new token, or of up to 16 rows), by itself and beside others.  The bound is that of two parts, which one
part alone does not keep: where a row's few large probabilities meet values of both signs, the rounding of each is a part of a small result."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_cache import Pages, ints, offsets
from test_gpu_paged_attention import queries, trees, words

BF = torch.bfloat16
HALF = 2.0 ** -8                # half a step of bf16, relative to the value


def bound(q, k, v, scale, vis, o, p):
    """What a row's results may be off by.  q [rows][dim], k, v [keys][dim], vis [rows][keys], o and p (probabilities) of the formula, all fp64:
      the result rounded to bf16:                 2^-8 |o|
      the probabilities' two parts:               2^-16 sum p |v|
      scores, sums of dim products in fp32:       dim 2^-24 sum |q k| scale, twice over (the product's order, the normalisation's sum of the same probabilities)
      their scaling, exponentials, rescaling, the sums over keys in fp32: 2^-24 of the largest score, and 2^-24 a key and sixteen more, twice over too"""
    size = (q.abs() @ k.abs().T).mul(scale).masked_fill(~vis, 0.0).amax(1)
    off = 2 * 2.0 ** -24 * (q.shape[1] * size + 4 * size + k.shape[0] + 16)
    return HALF * o.abs() + (HALF ** 2 + off)[:, None] * (p @ v.abs())


def formula(q, k, v, scale, vis):
    z = (q @ k.T * scale).masked_fill(~vis, -math.inf)
    p = torch.softmax(z, 1)
    return p, p @ v


@pytest.mark.parametrize("keys", [2, 5, 40, 700, 3000])
def test_the_bound_is_kept_by_two_parts_and_not_by_one(keys):
    """the formula with roundings planted in it"""
    gen = torch.Generator().manual_seed(keys)
    dim, rows = 64, 12
    q, k, v = ((g * torch.randn(n, dim, generator=gen)).to(BF).double() for g, n in ((4.0, rows), (1.0, keys), (1.0, keys)))
    vis = torch.ones(rows, keys, dtype=torch.bool)
    p, o = formula(q, k, v, dim ** -0.5, vis)
    off = bound(q, k, v, dim ** -0.5, vis, o, p)
    rounded = lambda x: x.float().to(BF).double()
    w = (q @ k.T * dim ** -0.5)
    w = (w - w.amax(1, keepdim=True)).exp()
    first = rounded(w)
    for parts, kept in ((first, False), (first + rounded(w - first), True)):
        got = rounded(parts @ v / w.sum(1, keepdim=True))
        assert bool(((got - o).abs() <= off).all()) == kept


def check(new, have, heads, kv, dim, page, bits=None, more=0, seed=0):
    """sequences that keep two parts by the tight bound; the call's other rows by the wide one"""
    n, G = sum(new), heads // kv
    c, q, cu = Pages(seed, have, page, kv, dim, more=more), queries(seed, n, heads, dim, 4.0), offsets(new)
    out, tree = torch.empty_like(q), None if bits is None else words(bits)
    binding.Context().glue_attention_paged(c.cache(), q, out, ints(cu), tree=tree)
    all_two = n * G <= 16 * len(new)
    found = 0
    for s, m in enumerate(new):
        if m == 0 or not (m == 1 or m * G <= 16 or all_two):
            continue
        rows = slice(cu[s], cu[s + 1])
        k, v = (ref.gather(t, c.table, page, s, have[s]).double() for t in (c.k, c.v))
        vis = ref.seen(m, have[s], None if bits is None else bits[rows], "cuda")
        x, got = q[rows].double().view(m, heads, dim), out[rows].double().view(m, heads, dim)
        for h in range(heads):
            g = h // G
            p, o = formula(x[:, h], k[:, g], v[:, g], dim ** -0.5, vis)
            off = bound(x[:, h], k[:, g], v[:, g], dim ** -0.5, vis, o, p)
            err = (got[:, h] - o).abs()
            assert (err <= off).all(), (s, h, float((err / off).max()))
        found += 1
    want = ref.attention(q, c.k, c.v, c.table, page, have, cu, dim, bits=bits)
    assert ((out.double() - want["out"]).abs() <= want["out_off"]).all()
    return found


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [5, 16])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 2), (17, 1), (32, 1), (96, 2), (150, 1)])
def test_single_tokens(dim, page, heads, kv):
    """with any number of heads on a key head"""
    have = [1, 2, 3, 17, 33, 65, 130, 700, 2500]
    assert check([1] * len(have), have, heads, kv, dim, page) == len(have)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page,more,piece", [(16, 0, 300), (16, 200, 300), (16, 200, 1500), (5, 400, 300), (64, 0, 60), (16, 0, 2200)])
@pytest.mark.parametrize("heads,kv", [(8, 2), (40, 2)])
def test_single_tokens_beside_pieces_of_prompts(dim, page, more, piece, heads, kv):
    """row tiles of 128 and 256, of one workgroup and of several"""
    new, have = [1, 1, piece, 1, 0, 1], [4, 900, piece + 200, 1, 50, 3100 if more else 70]
    assert check(new, have, heads, kv, dim, page, more=more) == 4


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page,more", [(16, 0), (16, 300), (7, 300)])
def test_few_tokens_beside_many(dim, page, more):
    """up to 16 rows: trees and ends of prompts"""
    new, have = [4, 2, 200, 3, 5], [4, 700, 900, 45, 3000 if more else 300]
    assert check(new, have, 8, 2, dim, page, more=more) == 3
    assert check(new, have, 8, 2, dim, page, bits=trees(3, new), more=more) == 3


@pytest.mark.gpu
def test_many_sequences_beside_a_piece():
    for more in (0, 200):
        new, have = [1] * 70 + [900] + [1] * 20, [7 * i + 1 for i in range(70)] + [1000] + [40 * i + 1 for i in range(20)]
        assert check(new, have, 8, 2, 64, 16, more=more) == 90


@pytest.mark.gpu
def test_all_of_a_call_with_few_rows_in_the_mean():
    new, have = [1] * 40 + [30], [100 * i + 1 for i in range(40)] + [500]
    assert check(new, have, 4, 1, 128, 16) == 41


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("more", [0, 200])
def test_with_values_that_are_not_finite_beside(dim, more):
    """a workgroup that goes over its tiles with care keeps two parts too"""
    new, have, heads, kv, page = [1, 300, 1], [900, 500, 40], 8, 2, 16
    c, q, cu = Pages(5, have, page, kv, dim, more=more), queries(5, sum(new), heads, dim, 4.0), offsets(new)
    for s, place, bad in ((0, 3, math.inf), (0, 600, math.nan), (2, 11, -math.inf)):
        at = ref.slot(c.table, page, c.k.shape[0], s, place)
        c.v[at][0, 5] = bad
    out = torch.empty_like(q)
    binding.Context().glue_attention_paged(c.cache(), q, out, ints(cu))
    for s in (0, 2):
        k, v = (ref.gather(t, c.table, page, s, have[s]).double() for t in (c.k, c.v))
        vis = torch.ones(1, have[s], dtype=torch.bool, device="cuda")
        x, got = q[cu[s]].double().view(heads, dim), out[cu[s]].double().view(heads, dim)
        fine = torch.ones(dim, dtype=torch.bool, device="cuda")
        fine[5] = False
        for h in range(heads):
            g = h * kv // heads
            cols = fine if g == 0 else torch.ones_like(fine)
            p, o = formula(x[h:h + 1], k[:, g], v[:, g][:, cols], dim ** -0.5, vis)
            off = bound(x[h:h + 1], k[:, g], v[:, g][:, cols], dim ** -0.5, vis, o, p)
            assert ((got[h, cols] - o[0]).abs() <= off[0]).all()
            assert torch.isfinite(got[h, 5]) == (g != 0)
