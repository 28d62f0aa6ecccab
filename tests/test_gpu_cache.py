"""New tokens on their way into a cache in pages (agzo_glue_cache_append) and a tree's accepted tokens together in it (agzo_glue_cache_keep), place by place."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(lens):
    return [int(x) for x in np.cumsum([0] + list(lens))]


class Pages:
    """A cache of garbage: pages in no order, [n_pages][page][kv][dim] seen through strides"""

    def __init__(self, seed, have, page, kv, dim, layout="tokens", spare=3, more=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.page = page
        need = [(h + page - 1) // page for h in have]
        total, self.pages = sum(need) + spare, max(need + [0]) + more
        order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table, at = [], 0
        for n in need:
            self.table.append(order[at:at + n] + [-7] * (self.pages - n))
            at += n
        shape = (total, page, kv, dim)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(BF)
        if layout == "tokens":
            self.k, self.v = rnd(*shape), rnd(*shape)
        elif layout == "heads":
            self.k, self.v = (rnd(total, kv, page, dim).transpose(1, 2) for _ in range(2))
        elif layout == "pages":                     # both in one tensor, page by page
            both = rnd(total, 2, page, kv, dim)
            self.k, self.v = both[:, 0], both[:, 1]
        elif layout == "rows":                      # token by token, with room between
            both = rnd(total, page, kv * 2 * dim + 16)
            self.k, self.v = (both[:, :, i * kv * dim:(i + 1) * kv * dim].unflatten(2, (kv, dim)) for i in range(2))
        elif layout == "pairs":                     # head by head
            both = rnd(total, page, kv, 2, dim)
            self.k, self.v = both[..., 0, :], both[..., 1, :]
        self.k_len = ints(have)

    def cache(self):
        return binding.make_cache(self.k, self.v, ints(self.table), self.k_len)


def new_tokens(seed, n, heads, kv, dim):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000)
    return [torch.randn(n, h * dim, device="cuda", generator=gen).to(BF) for h in (heads, kv, kv)]


def check_append(c, rope, new, have, heads, kv, dim, seed, positions=None, gains=(None, None), eps=None, tail=0):
    ctx, cu = binding.Context(), offsets(new)
    n = cu[-1] + tail
    q, k, v = new_tokens(seed, n, heads, kv, dim)
    out = torch.full_like(q, 7.0)
    kc, vc = c.k.clone(), c.v.clone()
    ctx.glue_cache_append(c.cache(), rope, q, k, v, out, ints(cu), positions=None if positions is None else ints(positions + [0] * tail), q_gain=gains[0], k_gain=gains[1], eps=eps)
    where = list(ref.places(cu, have, c.pages * c.page))
    pos = ints([p for _, _, p in where]) if positions is None else ints(positions)
    qn, kn = (x[:cu[-1]].double() if eps is None else ref.norm(x[:cu[-1]], g, dim, eps) for x, g in ((q, gains[0]), (k, gains[1])))
    (qw, q_off), (kw, k_off) = ((x, torch.zeros_like(x)) if rope is None else ref.rotate(x, pos, rope, dim) for x in (qn, kn))
    # (of a norm in fp32: 2^-21)
    fine = lambda got, want, off: ((got.double() - want).abs() <= off + (2.0 ** -8 + (0 if eps is None else 2.0 ** -21)) * want.abs() + (0 if eps is None else off)).all()
    assert fine(out[:cu[-1]], qw, q_off)
    assert (out[cu[-1]:] == 7.0).all()
    stored = {}
    for i, (s, _, place) in enumerate(where):
        at = ref.slot(c.table, c.page, kc.shape[0], s, place)
        if at is not None:
            stored[at] = i
    if stored:
        at, rows = ints([a[0] for a in stored]).long(), ints(list(stored.values())).long()
        slots = ints([a[1] for a in stored]).long()
        assert fine(c.k[at, slots].flatten(1), kw[rows], k_off[rows])
        assert torch.equal(c.v[at, slots].flatten(1), v[rows])
        kc[at, slots], vc[at, slots] = c.k[at, slots], c.v[at, slots]
    assert torch.equal(c.k, kc) and torch.equal(c.v, vc)      # all else as it was
    return stored


@pytest.mark.parametrize("layout", ["tokens", "heads", "pages", "rows", "pairs"])
@pytest.mark.parametrize("page,dim,heads,kv", [(16, 128, 8, 2), (1, 64, 3, 1), (12, 64, 4, 4), (64, 128, 7, 1)])
def test_append(layout, page, dim, heads, kv):
    new, have = [1, 0, 40, 3, 17], [1, 5, 40, 30, 100]
    gains = [1 + 0.1 * torch.randn(dim, device="cuda") for _ in range(2)]
    for i, (rope, g, eps) in enumerate(((binding.make_rope(dim, 1e4), gains, 1e-6), (None, (None, None), None), (binding.make_rope(32, 1e4, interleaved=True), (gains[0], None), 1e-5))):
        c = Pages(i + page, have, page, kv, dim, layout)
        stored = check_append(c, rope, new, have, heads, kv, dim, i, gains=g, eps=eps)
        assert len(stored) == sum(new)


def test_append_many_sequences_and_tokens():
    rng = np.random.default_rng(3)
    for new in ([1] * 300, rng.integers(0, 40, 130).tolist(), [4500]):
        have = [int(m + rng.integers(0, 50)) for m in new]
        check_append(Pages(len(new), have, 16, 2, 64), binding.make_rope(64), new, have, 4, 2, 64, len(new), gains=(None, None), eps=1e-6)


def test_append_with_given_positions_and_rows_of_no_sequence():
    new, have = [5, 3], [9, 3]
    c = Pages(1, have, 4, 2, 128)
    check_append(c, binding.make_rope(128), new, have, 4, 2, 128, 7, positions=[100000, 0, 1, 1, 2 ** 31 - 1, -5, 3, 3], tail=4)


def test_append_where_places_or_pages_are_missing():
    # fewer places than new tokens; lengths outside the room; ids that are no page's; a sequence without a place
    new, have = [5, 4, 3, 2], [2, 1000, -4, 8]
    c = Pages(2, [5, 8, 3, 8], 4, 1, 64)
    c.k_len = ints(have)
    c.table[1][1] = c.k.shape[0]
    c.table[3][1] = -1
    stored = check_append(c, binding.make_rope(64), new, have, 2, 1, 64, 3)
    assert len(stored) == 2


def test_append_in_place_without_queries_and_twice():
    ctx, have = binding.Context(), [20, 33]
    c = Pages(4, have, 8, 2, 64)
    q, k, v = new_tokens(4, 7, 4, 2, 64)
    cu, rope, want = ints([0, 4, 7]), binding.make_rope(64), torch.empty(7, 256, device="cuda", dtype=BF)
    ctx.glue_cache_append(c.cache(), rope, q, k, v, want, cu)
    first = c.k.clone(), c.v.clone()
    ctx.glue_cache_append(c.cache(), rope, None, k, v, None, cu)                 # again, the same
    assert torch.equal(c.k, first[0]) and torch.equal(c.v, first[1])
    ctx.glue_cache_append(c.cache(), rope, q, k, v, q, cu)
    assert torch.equal(q, want)


def test_append_wide_inputs():
    """q, k and v side by side in one tensor, the turned queries over their own"""
    ctx, c = binding.Context(), Pages(5, [30], 16, 2, 64)
    wide = torch.randn(30, 8 * 64 + 8, device="cuda").to(BF)
    q, k, v = wide[:, :256], wide[:, 256:384], wide[:, 384:512]
    parts = [t.contiguous() for t in (q, k, v)]
    rope, cu, out = binding.make_rope(64), ints([0, 30]), torch.empty(30, 256, device="cuda", dtype=BF)
    ctx.glue_cache_append(c.cache(), rope, *parts, out, cu)
    kc, vc = c.k.clone(), c.v.clone()
    c.k.zero_(), c.v.zero_()
    ctx.glue_cache_append(c.cache(), rope, q, k, v, q, cu)
    at = torch.tensor(c.table[0], device="cuda")
    assert torch.equal(q, out)
    assert torch.equal(c.k[at].flatten(0, 1)[:30], kc[at].flatten(0, 1)[:30]) and torch.equal(c.v[at].flatten(0, 1)[:30], vc[at].flatten(0, 1)[:30])


@pytest.mark.parametrize("layout", ["tokens", "heads", "pairs"])
@pytest.mark.parametrize("page", [1, 12, 16])
def test_keep(layout, page):
    new = [48, 1, 9, 0, 130, 6]
    have = [60, 1, 20, 3, 131, 5]                                            # the last: its first place is missing
    paths = [[1, 2, 9, 40], [], [8], [], list(range(1, 60)) + list(range(64, 128, 2)), [2, 4, 5]]
    for kv, dim in ((2, 128), (8, 128), (1, 64)):
        c = Pages(page, have, page, kv, dim, layout)
        kc, vc = c.k.clone(), c.v.clone()
        cu = offsets(new)
        rows, kept = ints([r for p, m in zip(paths, new) for r in p + [-1] * (m - len(p))]), ints([len(p) for p in paths])
        binding.Context().glue_cache_keep(c.cache(), ints(cu), rows, kept)
        for s, path in enumerate(paths):
            for j, r in enumerate(path):
                of, to = (ref.slot(c.table, page, c.k.shape[0], s, have[s] - new[s] + i) for i in (r, j + 1))
                if of is not None and to is not None:
                    assert torch.equal(c.k[to], kc[of]) and torch.equal(c.v[to], vc[of])
                    kc[to], vc[to] = c.k[to], c.v[to]                        # (places in front of what is read later)
        assert torch.equal(c.k, kc) and torch.equal(c.v, vc)


def test_keep_leaves_what_is_none_of_its_rows():
    """entries in front of their place, behind the new tokens, more entries than rows"""
    c = Pages(9, [30, 30], 16, 2, 64)
    kc = c.k.clone()
    binding.Context().glue_cache_keep(c.cache(), ints([0, 5, 10]), ints([1, 1, 0, 5, -3, 2 ** 31 - 1, -2 ** 31, 4, 4, 4]), ints([2 ** 31 - 1, -5]))
    assert torch.equal(c.k, kc)
    binding.Context().glue_cache_keep(c.cache(), ints([0, 5, 10]), ints([4, 4, 4, 4, 4] * 2), ints([4, 0]))
    t, base = c.table[0], 25
    last = kc[t[29 // 16], 29 % 16]
    for p in (26, 27, 28, 29):                                               # the same row several times
        assert torch.equal(c.k[t[p // 16], p % 16], last)


def test_captured_and_replayed_as_lengths_grow():
    side = torch.cuda.Stream()
    ctx, plain = binding.Context(side), binding.Context()
    have = [5, 17]
    c, d = Pages(6, [40, 40], 16, 2, 64), Pages(6, [40, 40], 16, 2, 64)
    c.k_len, d.k_len = ints(have), ints(have)
    q, k, v = new_tokens(6, 2, 4, 2, 64)
    out, want, cu, rope = torch.empty_like(q), torch.empty_like(q), ints([0, 1, 2]), binding.make_rope(64)
    cc, dc = c.cache(), d.cache()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.glue_cache_append(cc, rope, q, k, v, out, cu)
        c.k_len += 1
    for _ in range(4):
        k.copy_(torch.randn_like(k))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        plain.glue_cache_append(dc, rope, q, k, v, want, cu)
        d.k_len += 1
        assert torch.equal(c.k, d.k) and torch.equal(c.v, d.v) and torch.equal(out, want) and torch.equal(c.k_len, d.k_len)


def test_refusals():
    ctx, c = binding.Context(), Pages(7, [20, 33], 8, 2, 64)
    q, k, v = new_tokens(7, 7, 4, 2, 64)
    out, cu, rope = torch.empty_like(q), ints([0, 4, 7]), binding.make_rope(64)
    E = binding.AgzoError
    run = lambda **o: ctx.glue_cache_append(**{**dict(cache=c.cache(), rope=rope, q=q, k=k, v=v, q_out=out, cu_q=cu), **o})
    run()
    gain = torch.ones(64, device="cuda")
    for o, error in ((dict(rope=binding.make_rope(128)), E), (dict(q_gain=gain), E), (dict(eps=-1.0), E), (dict(eps=float("nan")), E), (dict(q_out=None), ValueError), (dict(v=v[:6]), ValueError),
                     (dict(k=k[:, :64].contiguous(), v=v[:, :64].contiguous()), ValueError), (dict(cu_q=ints([0, 7])), ValueError), (dict(cu_q=cu.long()), TypeError), (dict(q=q.float()), TypeError),
                     (dict(positions=ints([0])), ValueError), (dict(q_gain=gain[:32], eps=1e-6), ValueError), (dict(cu_q=cu.cpu()), ValueError),
                     (dict(k=c.k.view(-1, 128)[:7]), E), (dict(q_out=c.v.view(-1, 256)[:7]), E), (dict(q_out=q[:, ], q=out[:, ]), None)):
        if error is None:
            run(**o)
        else:
            with pytest.raises(error):
                run(**o)
    # k and v of one memory; rows that overlap each other
    with pytest.raises(E):
        run(cache=binding.make_cache(c.k, c.k, ints(c.table), c.k_len))
    with pytest.raises(E):
        run(cache=binding.make_cache(c.k[:-1], c.k[1:], ints(c.table), c.k_len))
    with pytest.raises(E):
        run(cache=binding.make_cache(c.k[:, :1].expand(-1, 8, -1, -1), c.v, ints(c.table), c.k_len))
    t = ints(c.table)
    for args, error in (((c.k.float(), c.v, t, c.k_len), TypeError), ((c.k, c.v[:, :4], t, c.k_len), ValueError), ((c.k, c.v, t.long(), c.k_len), TypeError), ((c.k, c.v, t, c.k_len[:1]), ValueError),
                        ((c.k, c.v, t.t(), c.k_len), ValueError), ((c.k, c.v, t.cpu(), c.k_len), ValueError), ((c.k[0], c.v[0], t, c.k_len), ValueError),
                        ((c.k.transpose(2, 3), c.v.transpose(2, 3), t, c.k_len), ValueError)):
        with pytest.raises(error):
            binding.make_cache(*args)
    rows, kept = ints([-1] * 7), ints([0, 0])
    ctx.glue_cache_keep(c.cache(), cu, rows, kept)
    for args, error in (((ints([0, 7]), rows, kept), ValueError), ((cu, rows.long(), kept), TypeError), ((cu, rows, kept[:1]), ValueError), ((cu, c.k.view(torch.int32).flatten()[:7], kept), E)):
        with pytest.raises(error):
            ctx.glue_cache_keep(c.cache(), *args)


def test_nothing_to_do():
    ctx, c = binding.Context(), Pages(8, [4], 4, 1, 64)
    e, cu = torch.empty(0, 64, device="cuda", dtype=BF), ints([0, 0])
    ctx.glue_cache_append(c.cache(), None, e, e, e, torch.empty_like(e), cu)
    ctx.glue_cache_keep(c.cache(), cu, ints([]), ints([0]))
    none = binding.make_cache(c.k[:0], c.v[:0], torch.empty(0, 0, dtype=torch.int32, device="cuda"), ints([]))
    ctx.glue_cache_append(none, None, e, e, e, torch.empty_like(e), ints([0]))
    ctx.check()
