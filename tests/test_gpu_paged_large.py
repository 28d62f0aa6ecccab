"""The calls on a cache in pages, rotation and verification at the ends of their ranges: rows more than 2^32 values apart, launches cut in several, the most sequences and tokens."""
import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_cache import Pages, ints, offsets
from test_gpu_paged_attention import words

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def wide(rows, ld, cols, dtype):
    """rows of `cols` values that lie ld apart"""
    return torch.empty(rows, ld, device="cuda", dtype=dtype)[:, :cols]


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_rotation_of_more_tokens_than_a_launch_takes(dtype):
    n, rope = 2 ** 23 + 5, binding.make_rope(16)
    q, pos = torch.randn(n, 16, device="cuda").to(dtype), torch.randint(0, 2 ** 31 - 1, (n,), device="cuda").int()
    out, back = torch.empty_like(q), torch.empty_like(q)
    ctx = binding.Context()
    ctx.glue_rope(rope, q, None, pos, out, None, 16)
    ctx.glue_rope_backward(rope, q, None, pos, back, None, 16)
    for rows in (slice(0, 1000), slice(2 ** 23 - 500, n)):
        for got, turned in ((out, False), (back, True)):
            want, off = ref.rotate(q[rows], pos[rows], rope, 16, turned)
            assert ((got[rows].double() - want).abs() <= off + ref.HALF[dtype] * want.abs()).all()


def test_rotation_of_rows_far_apart():
    n, dim, rope = 4200, 64, binding.make_rope(64, interleaved=True)
    q, out = (wide(n, 2 ** 20, 2 * dim, BF) for _ in range(2))
    q.normal_()
    pos = torch.randint(0, 5000, (n,), device="cuda").int()
    binding.Context().glue_rope(rope, q, None, pos, out, None, dim)
    want, off = ref.rotate(q, pos, rope, dim)
    assert ((out.double() - want).abs() <= off + ref.HALF[BF] * want.abs()).all()


def test_the_most_new_tokens():
    n, page, dim = 2 ** 24, 4096, 64
    lens = [n - 12345, 12345]
    q, k, v = (torch.randn(n, dim, device="cuda").to(BF) for _ in range(3))
    pages = [(m + page - 1) // page for m in lens]
    order = torch.randperm(sum(pages), generator=torch.Generator().manual_seed(0)).tolist()
    table = [order[:pages[0]], order[pages[0]:] + [-1] * (pages[0] - pages[1])]
    kc, vc = (torch.empty(sum(pages), page, 1, dim, device="cuda", dtype=BF) for _ in range(2))
    cache, rope, out = binding.make_cache(kc, vc, ints(table), ints(lens)), binding.make_rope(dim), torch.empty_like(q)
    ctx = binding.Context()
    ctx.glue_cache_append(cache, rope, q, k, v, out, ints(offsets(lens)))
    for s, at in ((0, 0), (0, lens[0] - 5000), (1, 0), (1, lens[1] - 5000)):
        row = (0, lens[0])[s] + at
        places, rows = torch.arange(at, at + 5000, device="cuda"), slice(row, row + 5000)
        where = (ints(table[s]).long()[places // page], places % page)
        for got, x in ((out[rows], q), (kc[where][:, 0], k)):
            want, off = ref.rotate(x[rows], places.int(), rope, dim)
            assert ((got.double() - want).abs() <= off + ref.HALF[BF] * want.abs()).all()
        assert torch.equal(vc[where][:, 0], v[rows])
    with pytest.raises(binding.AgzoError):
        ctx.glue_cache_append(cache, rope, q.expand(2, n, dim).reshape(2 * n, dim)[:n + 1], *(x.new_empty(n + 1, dim) for x in (k, v, q)), ints(offsets(lens)))


def test_attention_of_rows_far_apart():
    new, have, heads, dim = [1000, 40, 1], [1020, 700, 3000], 2, 64
    n, ld = sum(new), 2 ** 22 - 8
    assert n * ld > 2 ** 32
    c = Pages(3, have, 16, 1, dim)
    q, out = (wide(n, ld, heads * dim, BF) for _ in range(2))
    q.normal_()
    cu = offsets(new)
    binding.Context().glue_attention_paged(c.cache(), q, out, ints(cu))
    want = ref.attention(q.contiguous(), c.k, c.v, c.table, c.page, have, cu, dim)
    assert ((out.double() - want["out"]).abs() <= want["out_off"]).all()


@pytest.mark.parametrize("tree", [False, True])
def test_the_most_sequences(tree):
    """a token or a tree of two each, some with nothing in front of it; then the second ones together"""
    n_seq, dim, page = 65536, 64, 2
    have = [2 + s % 4 for s in range(n_seq)]
    m = 2 if tree else 1
    table = torch.randperm(3 * n_seq, generator=torch.Generator().manual_seed(1)).view(n_seq, 3).int()
    k, v = (torch.randn(3 * n_seq, page, 1, dim, device="cuda").to(BF) for _ in range(2))
    cache = binding.make_cache(k, v, table.cuda(), ints(have))
    q = torch.randn(m * n_seq, dim, device="cuda").to(BF)
    out, cu = torch.empty_like(q), ints([m * s for s in range(n_seq + 1)])
    ctx = binding.Context()
    ctx.glue_attention_paged(cache, q, out, cu, tree=words([1, 2] * n_seq) if tree else None)
    some = list(range(0, n_seq, 997)) + [n_seq - 1]
    t, h = table.tolist(), [have[s] for s in some]
    rows = torch.tensor([m * s + i for s in some for i in range(m)], device="cuda")
    want = ref.attention(q[rows], k, v, [t[s] for s in some], page, h, offsets([m] * len(some)), dim, bits=[1, 2] * len(some) if tree else None)
    assert ((out[rows].double() - want["out"]).abs() <= want["out_off"]).all()
    if not tree:
        return
    before, tokens = (k.clone(), v.clone()), ints([0] * (2 * n_seq))
    with pytest.raises(binding.AgzoError):                    # verification has a sequence less
        ctx.verify_drafts(torch.ones(2 * n_seq, 1, device="cuda"), None, tokens, torch.zeros(2 * n_seq, device="cuda"), cu, tokens + 0, tokens + 0, ints([0] * n_seq))
    ctx.glue_cache_keep(cache, cu, tokens + 1, ints([1] * n_seq))
    assert torch.equal(k, before[0]) and torch.equal(v, before[1])      # row 1 is at place 1 already


def test_probabilities_far_apart():
    vocab, ld = 5000, 2 ** 28 + 1
    cu = [0, 4, 12]
    gen = torch.Generator(device="cuda").manual_seed(4)
    p, q = (wide(12, ld, vocab, torch.float32) for _ in range(2))
    assert 12 * ld > 2 ** 31
    for x in (p, q):
        x.copy_(torch.softmax(0.5 * torch.randn(12, vocab, device="cuda", generator=gen), -1))
    q[1:] = 0.8 * p[:-1] + 0.2 * q[1:]
    ctx = binding.Context()
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        tokens = torch.multinomial(q.cpu(), 1, generator=g)[:, 0].tolist()
        u = torch.rand(12, generator=g)
        out = [torch.full((i,), 77, dtype=torch.int32, device="cuda") for i in (12, 12, 2)]
        ctx.verify_drafts(p, q, ints(tokens), u.cuda(), ints(cu), *out)
        want = ref.verify(p.double().cpu(), q.double().cpu(), tokens, u.tolist(), cu)
        assert [o.tolist() for o in out] == [want[0], want[1], list(want[2])]
