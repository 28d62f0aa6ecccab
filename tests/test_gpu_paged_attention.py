"""Attention of new tokens over a cache in pages (agzo_glue_attention_paged) against the formula in 64 bits: single tokens, trees of drafted ones, pieces of prompts."""
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_cache import Pages, ints, offsets

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def trees(seed, new):
    """bits of each row: itself and its ancestors"""
    rng, bits, depth = random.Random(seed), [], []
    for m in new:
        own = []
        for i in range(m):
            p = rng.randrange(-1, i) if i else -1
            own.append((own[p] if p >= 0 else 0) | 1 << i)
        bits += own
    return bits


def words(bits, n=None):
    n = n or max([b.bit_length() for b in bits] + [1]) // 32 + 1
    signed = lambda x: x - (1 << 32) if x >> 31 else x
    return ints([[signed(b >> (32 * w) & 0xFFFFFFFF) for w in range(n)] for b in bits]).reshape(len(bits), n)


def check(c, q, new, have, dim, bits=None, scale=None, tail=0, exact_rows=None, ctx=None, tree=None):
    ctx, cu = ctx or binding.Context(), offsets(new)
    n, heads = q.shape[0], q.shape[1] // dim
    out, lse = torch.full_like(q, 7.0), torch.full((n, heads), 7.0, device="cuda")
    if bits is not None and tree is None:
        tree = words(bits + [0] * (n - len(bits)))
    ctx.glue_attention_paged(c.cache(), q, out, ints(cu), scale=scale, tree=tree, lse=lse)
    want = ref.attention(q, c.k, c.v, c.table, c.page, have, cu, dim, scale, bits)
    rows = slice(0, cu[-1])
    got, w, off = out[rows].double(), want["out"][rows], want["out_off"][rows]
    fin = torch.isfinite(w)
    # (a value that is not finite: the same one)
    assert torch.equal(torch.isnan(got), torch.isnan(w))
    assert ((got == w) | torch.isnan(w) | ((got - w).abs() <= off))[fin | torch.isinf(w)].all(), float((got - w)[fin].abs().max())
    l, lw = lse[rows].double(), want["lse"][rows]
    assert torch.equal(torch.isinf(l), torch.isinf(lw))
    ok = torch.isfinite(lw)
    assert ((l - lw).abs() <= 2e-5 * (1 + lw.abs()))[ok].all()
    assert (out[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()
    return out, lse


def queries(seed, n, heads, dim, gain=1.3):
    gen = torch.Generator(device="cuda").manual_seed(seed + 77)
    return (gain * torch.randn(n, heads * dim, device="cuda", generator=gen)).to(BF)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [1, 7, 16, 48, 64, 256])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 2), (7, 1), (33, 1)])
def test_single_tokens(dim, page, heads, kv):
    have = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]
    new = [1] * len(have)
    check(Pages(page, have, page, kv, dim), queries(dim, len(have), heads, dim), new, have, dim)


@pytest.mark.parametrize("layout", ["heads", "pages", "rows", "pairs"])
@pytest.mark.parametrize("page", [5, 32])
def test_layouts(layout, page):
    new, have = [1, 3, 20, 1], [70, 3, 200, 129]
    for dim in (64, 128):
        check(Pages(page, have, page, 2, dim, layout), queries(1, sum(new), 6, dim), new, have, dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [3, 16, 64])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2), (5, 1)])
def test_pieces_of_prompts(dim, page, heads, kv):
    new, have = [0, 1, 130, 64, 33, 7, 200], [5, 1, 130, 64 + 100, 700, 1007, 331]
    check(Pages(page, have, page, kv, dim), queries(2, sum(new), heads, dim), new, have, dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [9, 16, 64])
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 2), (7, 1)])
def test_trees(dim, page, heads, kv):
    new, have = [1, 2, 31, 32, 33, 64, 65, 100], [1, 40, 31, 90, 33 + 31, 64 + 64, 500, 1000]
    check(Pages(page, have, page, kv, dim), queries(3, sum(new), heads, dim), new, have, dim, bits=trees(page, new))


@pytest.mark.parametrize("kind", ["single", "tree", "chunk"])
@pytest.mark.parametrize("dim,heads,kv", [(128, 8, 2), (64, 4, 4), (128, 7, 1)])
def test_long_caches_in_shares(kind, dim, heads, kv):
    """lengths as uneven as they get: the keys are dealt out, a sequence's in many shares beside others in one"""
    have = [9000, 3, 2500, 700, 64]
    new = [1] * 5 if kind == "single" else [40, 3, 17, 64, 1] if kind == "tree" else [300, 2, 130, 500, 64]
    check(Pages(5, have, 16, kv, dim, more=20), queries(4, sum(new), heads, dim), new, have, dim, bits=trees(4, new) if kind == "tree" else None)


def test_many_sequences():
    rng = random.Random(5)
    for n in (64, 65, 200):
        have = [rng.choice([1, 5, 40, 900]) for _ in range(n)]
        new = [min(h, rng.choice([0, 1, 1, 2])) for h in have]
        check(Pages(n, have, 16, 2, 64, more=100), queries(n, sum(new), 4, 64), new, have, 64)
    have = [3000] + [2] * 130 + [2000]
    check(Pages(9, have, 32, 1, 128, more=50), queries(9, len(have), 4, 128), [1] * len(have), have, 128)


def test_rows_that_see_nothing():
    # fewer places than new tokens, none at all, lengths outside the room
    new, have = [5, 3, 40, 2], [2, 0, 10, 1000]
    c = Pages(1, [2, 1, 10, 20], 16, 2, 64)
    c.k_len = ints([2, -9, 10, 1000])
    q = queries(1, sum(new), 4, 64)
    out, lse = check(c, q, new, have, 64)
    assert (out[:3] == 0).all() and torch.isinf(lse[:3]).all() and (out[5:8] == 0).all()
    # trees: rows without a bit, with bits behind the new tokens, of places that are not there
    bits = [0, 1 << 3, 1 << 4, 0b10, 0b11000, 0, 1, 7, *[1 << 39 if i % 2 else 0xF << i for i in range(40)], 0, 3]
    check(c, q, new, have, 64, bits=bits)
    # no words: the new tokens see none of each other
    check(c, q, new, have, 64, bits=[0] * sum(new), tree=torch.empty(sum(new), 0, dtype=torch.int32, device="cuda"))
    # fewer words than tokens, and bits past them
    full = [(1 << 64) - 1] * sum(new)
    check(c, q, new, have, 64, bits=[(1 << 32) - 1] * sum(new), tree=words(full, 2)[:, :1])
    check(c, q, new, have, 64, bits=full, tree=words(full, 2))


def test_rows_of_no_sequence():
    new, have = [3, 1], [30, 4000]
    check(Pages(2, have, 16, 2, 128), queries(2, 9, 4, 128), new, have, 128, tail=5)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 5)])
def test_what_is_not_seen_takes_no_part(bad, dim, page):
    """keys and values that no row sees, that some see, and what pages hold behind the last place"""
    new, have, heads, kv = [6, 40, 1, 70], [50, 40, 33, 1500], 4, 2
    c = Pages(3, have, page, kv, dim)
    q, bits = queries(3, sum(new), heads, dim, 0.3), trees(7, new)
    used = torch.zeros(c.k.shape[:2], dtype=torch.bool, device="cuda")
    for s, h in enumerate(have):
        for p in range(h):
            used[ref.slot(c.table, page, c.k.shape[0], s, p)] = True
    c.k[~used], c.v[~used] = bad, bad
    check(c, q, new, have, dim)
    check(c, q, new, have, dim, bits=bits)
    # values of new tokens that some rows see and others do not
    for s, i in ((0, 3), (1, 20), (3, 69), (3, 10)):
        c.v[ref.slot(c.table, page, c.k.shape[0], s, have[s] - new[s] + i)][0, 5] = bad
    check(c, q, new, have, dim)
    check(c, q, new, have, dim, bits=bits)
    # ... and keys that only some rows see
    c = Pages(4, have, page, kv, dim)
    bits = [b & ~(1 << 2) for b in bits]
    for s in (0, 1, 3):
        at = ref.slot(c.table, page, c.k.shape[0], s, have[s] - new[s] + 2)
        c.k[at], c.v[at] = bad, bad
    check(c, q, new, have, dim, bits=bits)


def test_scores_far_from_zero():
    new, have = [1, 5, 90], [900, 60, 300]
    for gain, scale in ((30.0, None), (1.0, 4.0), (1.0, 1e-4), (0.0, None)):
        check(Pages(6, have, 16, 2, 128), queries(6, sum(new), 4, 128, gain), new, have, 128, scale=scale)


def test_ids_that_are_no_pages_are_the_nearest():
    new, have = [1, 4], [40, 60]
    c = Pages(7, have, 16, 2, 64)
    c.table[0][1], c.table[1][2] = 2 ** 31 - 1, -(2 ** 31)
    check(c, queries(7, 5, 4, 64), new, have, 64)


def test_shared_pages():
    new, have = [1, 1, 2], [100, 100, 97]
    c = Pages(8, have, 16, 2, 64)
    c.table[1][:6] = c.table[2][:6] = c.table[0][:6]
    check(c, queries(8, 4, 4, 64), new, have, 64)


def test_offsets_beyond_32_bits():
    """a cache of more than 2^32 values a tensor, of which only its ends are used"""
    pages, page, kv, dim = 70000, 64, 8, 128
    assert pages * page * kv * dim > 2 ** 32
    c = Pages(1, [3], 64, 1, 64)
    c.k, c.v = (torch.zeros(pages, page, kv, dim, device="cuda", dtype=BF) for _ in range(2))
    c.page, c.pages, c.table = page, 3, [[pages - 1, 0, pages - 2], [65536, 4, 1]]
    for t in c.table:
        for i in t:
            c.k[i], c.v[i] = torch.randn(page, kv, dim, device="cuda").to(BF), torch.randn(page, kv, dim, device="cuda").to(BF)
    new, have = [1, 30], [190, 150]
    c.k_len = ints(have)
    check(c, queries(1, 31, 8, 128), new, have, 128)
    from test_gpu_cache import check_append
    check_append(c, binding.make_rope(128), new, have, 8, kv, dim, 3)


def test_repeats_bit_for_bit_alone_and_beside_others():
    ctx = binding.Context()
    new, have = [1, 30, 1, 200], [3000, 500, 64, 2000]
    c, q, cu = Pages(9, have, 16, 2, 128), queries(9, 232, 8, 128), ints(offsets(new))
    outs = []
    for _ in range(4):
        out = torch.empty_like(q)
        ctx.glue_attention_paged(c.cache(), q, out, cu)
        outs.append(out)
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_wide_rows_and_a_trees_stride():
    new, have = [10, 3], [200, 3]
    c, bits = Pages(10, have, 16, 2, 64), trees(10, new)
    wide = torch.randn(13, 4 * 64 + 64, device="cuda").to(BF)
    q, out = wide[:, 64:], torch.zeros(13, 4 * 64 + 8, device="cuda", dtype=BF)
    tree = torch.full((13, 5), -1, dtype=torch.int32, device="cuda")
    tree[:, :2] = words(bits, 2)
    ctx, want = binding.Context(), torch.empty(13, 256, device="cuda", dtype=BF)
    ctx.glue_attention_paged(c.cache(), q, out[:, :256], ints(offsets(new)), tree=tree[:, :2])
    ctx.glue_attention_paged(c.cache(), q.contiguous(), want, ints(offsets(new)), tree=words(bits, 2))
    assert torch.equal(out[:, :256], want) and (out[:, 256:] == 0).all()


def test_captured_and_replayed_beside_the_programs_own_work():
    """two graphs of one context, replayed as lengths and pages change, and eager calls of another context between them"""
    side = torch.cuda.Stream()
    ctx, plain = binding.Context(side), binding.Context()
    cases = []
    for seed, new, have, tree in ((1, [1, 1, 1], [10, 600, 2000], False), (2, [33, 5], [700, 1300], True)):
        c, q = Pages(seed, [2500] * len(have), 16, 2, 128), queries(seed, sum(new), 8, 128)
        c.k_len = ints(have)
        cases.append((c, c.cache(), q, torch.empty_like(q), ints(offsets(new)), words(trees(seed, new)) if tree else None))
    torch.cuda.synchronize()
    for c, cache, q, out, cu, tree in cases:
        ctx.glue_attention_paged(cache, q, out, cu, tree=tree)            # (the workspace grows here)
    torch.cuda.synchronize()
    graphs = []
    for c, cache, q, out, cu, tree in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            ctx.glue_attention_paged(cache, q, out, cu, tree=tree)
            c.k_len += 111
        graphs.append(g)
    for i in range(4):
        for (c, cache, q, out, cu, tree), g in zip(cases, graphs):
            q.copy_(torch.randn_like(q))
            c.k[0] = float(i)
            want = torch.empty_like(out)
            plain.glue_attention_paged(cache, q, want, cu, tree=tree)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_a_capture_that_would_grow_the_workspace_is_refused():
    side = torch.cuda.Stream()
    ctx, c = binding.Context(side), Pages(3, [5000], 16, 8, 128)
    q = queries(3, 1, 8, 128)
    out, cache, cu = torch.empty_like(q), c.cache(), ints([0, 1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        with pytest.raises(binding.AgzoError) as e:
            ctx.glue_attention_paged(cache, q, out, cu)
    assert e.value.code == binding.ENOMEM


def test_refusals():
    ctx, c = binding.Context(), Pages(4, [20, 33], 8, 2, 64)
    q, cu, E = queries(4, 7, 4, 64), ints([0, 4, 7]), binding.AgzoError
    out, tree = torch.empty_like(q), ints([[1]] * 7)
    run = lambda **o: ctx.glue_attention_paged(**{**dict(cache=c.cache(), q=q, out=out, cu_q=cu), **o})
    run()
    run(tree=tree)
    for o, error in ((dict(scale=0.0), E), (dict(scale=math.inf), E), (dict(scale=math.nan), E), (dict(out=q), E), (dict(out=c.v.view(-1, 256)[:7]), E), (dict(q=q[:, :192], out=out[:, :192]), E),
                     (dict(q=q[:, :200].contiguous(), out=out[:, :200].contiguous()), ValueError), (dict(q=q.half()), TypeError), (dict(out=out[:6]), ValueError), (dict(cu_q=ints([0, 7])), ValueError),
                     (dict(tree=tree[:6]), ValueError), (dict(tree=tree.long()), TypeError), (dict(lse=torch.empty(7, 3, device="cuda")), ValueError), (dict(q=q.cpu()), ValueError),
                     (dict(lse=out.view(torch.float32).flatten()[:28].view(7, 4)), E)):
        with pytest.raises(error):
            run(**o)
    with pytest.raises(E):
        run(cache=binding.make_cache(*(torch.zeros(4, 8, 2, 96, device="cuda").to(BF) for _ in range(2)), ints(c.table), c.k_len), q=torch.zeros(7, 384, device="cuda").to(BF),
            out=torch.zeros(7, 384, device="cuda").to(BF))


def test_nothing_to_do():
    ctx, c = binding.Context(), Pages(5, [4, 9], 4, 1, 64)
    e = torch.empty(0, 64, device="cuda", dtype=BF)
    ctx.glue_attention_paged(c.cache(), e, torch.empty_like(e), ints([0, 0, 0]))
    none = binding.make_cache(c.k[:0], c.v[:0], torch.empty(2, 0, dtype=torch.int32, device="cuda"), ints([3, 0]))
    q, out = queries(5, 2, 1, 64), torch.full((2, 64), 7.0, device="cuda").to(BF)
    ctx.glue_attention_paged(none, q, out, ints([0, 1, 2]))                 # no pages: nothing is seen
    assert (out == 0).all()
    ctx.check()
