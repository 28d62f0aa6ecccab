"""The calls on a cache in pages one after the other, as a program serves with them: prompts in pieces, drafted trees and chains, verification, accepted tokens kept."""
import random

import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_cache import ints, offsets
from test_gpu_paged_attention import words

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
EPS, THETA = 1e-6, 1.0e4


class Server:
    """One layer: embeddings -> q, k, v -> norms, rotation, cache -> attention -> output product and residual -> head"""

    def __init__(self, seed, n_seq, page, max_pages, d=128, heads=4, kv=2, dim=64, vocab=300, rope=None):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
        self.heads, self.kv, self.dim, self.vocab, self.page = heads, kv, dim, vocab, page
        self.emb, self.wqkv = rnd(vocab, d), rnd(d, (heads + 2 * kv) * dim) / d ** 0.5
        self.wo, self.head = rnd(heads * dim, d) / (heads * dim) ** 0.5, 0.6 * rnd(d, vocab)
        self.gains = [1 + 0.1 * rnd(dim) for _ in range(2)]
        pages = n_seq * max_pages + 2
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:n_seq * max_pages]
        self.table = order.view(n_seq, max_pages).int().cuda()
        self.k, self.v = (torch.full((pages, page, kv, dim), float("nan"), device="cuda", dtype=BF) for _ in range(2))
        self.k_len = ints([0] * n_seq)
        self.cache = binding.make_cache(self.k, self.v, self.table, self.k_len)
        self.rope = rope or binding.make_rope(dim, THETA)

    def forward(self, ctx, tokens, cu, positions=None, tree=None):
        """probabilities behind each new token; q as attention takes it and its result"""
        h = self.emb[tokens]
        q, k, v = (h @ self.wqkv).to(BF).split([self.heads * self.dim, self.kv * self.dim, self.kv * self.dim], 1)
        qr, att = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(q.shape, device="cuda", dtype=BF)
        ctx.glue_cache_append(self.cache, self.rope, q, k, v, qr, cu, positions=positions, q_gain=self.gains[0], k_gain=self.gains[1], eps=EPS)
        ctx.glue_attention_paged(self.cache, qr, att, cu, tree=tree)
        return torch.softmax((h + att.float() @ self.wo) @ self.head, -1), qr, att

    def rows(self, s, n):
        t = self.table.tolist()
        return ref.gather(self.k, t, self.page, s, n), ref.gather(self.v, t, self.page, s, n)


def check_attention(srv, q, att, cu, have, bits=None):
    want = ref.attention(q, srv.k, srv.v, srv.table.tolist(), srv.page, have, cu, srv.dim, bits=bits)
    assert ((att.double() - want["out"]).abs() <= want["out_off"]).all()


def tree_of(rng, n):
    parents = [-1] + [rng.randrange(max(0, i - 6), i) for i in range(1, n)]
    bits, depth = [], []
    for i, p in enumerate(parents):
        bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return parents, bits, depth


@pytest.mark.parametrize("page,rope", [(16, None), (5, binding.make_rope(32, THETA, interleaved=True, scaling=binding.ROPE_LINEAR, factor=2.0))])
def test_serving_with_drafts(page, rope):
    rng, gen = random.Random(page), torch.Generator().manual_seed(page)
    n_seq = 3
    srv, ctx = Server(page, n_seq, page, 400 // page + 1, rope=rope), binding.Context()
    texts = [[rng.randrange(srv.vocab) for _ in range(n)] for n in (1, 70, 200)]
    have = [0] * n_seq
    # prompts, in two pieces, but for the last token, which goes with the first drafts
    for at, to in ((0, 0.5), (0.5, 1.0)):
        pieces = [t[:-1][int(at * (len(t) - 1)):int(to * (len(t) - 1))] for t in texts]
        have = [h + len(p) for h, p in zip(have, pieces)]
        srv.k_len.copy_(ints(have))
        cu = offsets([len(p) for p in pieces])
        _, q, att = srv.forward(ctx, ints(sum(pieces, [])).long(), ints(cu))
        check_attention(srv, q, att, cu, have)
    kept_rows = [srv.rows(s, have[s]) for s in range(n_seq)]
    taken = 0
    for step in range(8):
        chain = step % 2
        trees = [tree_of(rng, rng.randint(2, 40)) for _ in range(n_seq)]
        if chain:
            trees = [([i - 1 for i in range(n)], [(2 << i) - 1 for i in range(n)], list(range(n))) for n in (4, 1, 9)]
        new = [len(t[0]) for t in trees]
        cu = offsets(new)
        n = cu[-1]
        have = [h + m for h, m in zip(have, new)]
        srv.k_len.copy_(ints(have))
        # drafts: what the model without its attention finds likely behind the token that they follow
        tokens, q_probs = [], torch.zeros(n, srv.vocab)
        for s, (parents, _, _) in enumerate(trees):
            for i, p in enumerate(parents):
                if p < 0:
                    tokens.append(texts[s][-1])
                    continue
                guess = torch.softmax(srv.emb[tokens[cu[s] + p]] @ srv.head, -1).cpu()
                q_probs[cu[s] + i] = guess
                tokens.append(int(torch.multinomial(guess, 1, generator=gen)) if chain else int(guess.topk(4).indices[rng.randrange(4)]))
        bits = sum((t[1] for t in trees), [])
        positions = ints([h - m + x for h, m, t in zip(have, new, trees) for x in t[2]])
        p, q, att = srv.forward(ctx, ints(tokens).long(), ints(cu), positions=None if chain else positions, tree=None if chain else words(bits))
        check_attention(srv, q, att, cu, have, None if chain else bits)
        u = torch.rand(n, generator=gen)
        out = [torch.full((m,), 77, dtype=torch.int32, device="cuda") for m in (n, n, n_seq)]
        parents = sum((t[0] for t in trees), [])
        ctx.verify_drafts(p, q_probs.cuda() if chain else None, ints(tokens), u.cuda(), ints(cu), *out, parents=None if chain else ints(parents))
        want = ref.verify(p.double().cpu(), q_probs.double() if chain else None, tokens, u.tolist(), cu, None if chain else parents)
        assert [o.tolist() for o in out] == [want[0], want[1], want[2]]
        drafted = [srv.rows(s, have[s]) for s in range(n_seq)]
        ctx.glue_cache_keep(srv.cache, ints(cu), out[1], out[2])
        for s in range(n_seq):
            path = [0] + want[1][cu[s]:cu[s] + want[2][s]]
            base = have[s] - new[s]
            kept_rows[s] = tuple(torch.cat((old, of[torch.tensor(path, device="cuda") + base])) for old, of in zip(kept_rows[s], drafted[s]))
            have[s] = base + len(path)
            texts[s] += [tokens[cu[s] + r] for r in path[1:]] + [want[0][cu[s] + len(path) - 1]]
            taken += len(path) - 1
            assert len(texts[s]) == have[s] + 1
        srv.k_len.copy_(ints(have))
        for s in range(n_seq):
            for got, w in zip(srv.rows(s, have[s]), kept_rows[s]):
                assert torch.equal(got, w)
    assert taken > 0
    # the cache that it has come to is that of the texts
    other = Server(page, n_seq, page, 400 // page + 1, rope=rope)
    other.k_len.copy_(ints(have))
    cu = offsets(have)
    other.forward(ctx, ints(sum((t[:-1] for t in texts), [])).long(), ints(cu))
    for s in range(n_seq):
        for a, b in zip(srv.rows(s, have[s]), other.rows(s, have[s])):
            # (products of other sizes: q, k and v may be rounded to the neighbour, and a norm and a rotation are made of them)
            assert ((a.double() - b.double()).abs() <= 4 * 2.0 ** -8 * (1 + b.double().abs())).all()


def test_a_captured_step_beside_an_eager_one():
    """append, attention, verification and keeping in one graph, two of them, replayed with other tokens and random numbers each time"""
    side = torch.cuda.Stream()
    captured, plain = binding.Context(side), binding.Context()
    graphs = []
    for seed, nodes in ((1, 7), (2, 40)):
        rng = random.Random(seed)
        parents, bits, depth = tree_of(rng, nodes)
        a, b = (Server(seed, 2, 16, 40) for _ in range(2))
        cu, n = ints([0, nodes, 2 * nodes]), 2 * nodes
        data = dict(tokens=torch.randint(0, a.vocab, (n,), device="cuda"), u=torch.rand(n, device="cuda"), parents=ints(parents * 2), tree=words(bits * 2), depth=ints(depth * 2))
        seq = torch.arange(n, device="cuda") // nodes

        def step(srv, ctx, out, cu=cu, nodes=nodes, data=data, seq=seq):
            srv.k_len += nodes
            p, _, _ = srv.forward(ctx, data["tokens"], cu, positions=srv.k_len[seq] - nodes + data["depth"], tree=data["tree"])
            ctx.verify_drafts(p, None, data["tokens"].int(), data["u"], cu, *out, parents=data["parents"])
            ctx.glue_cache_keep(srv.cache, cu, out[1], out[2])
            srv.k_len += out[2] + 1 - nodes
            return p
        for srv, ctx in ((a, captured), (b, plain)):
            srv.k.zero_(), srv.v.zero_()
            srv.k_len.copy_(ints([3, 30]))
        out, want = ([torch.empty(m, dtype=torch.int32, device="cuda") for m in (n, n, 2)] for _ in range(2))
        torch.cuda.synchronize()
        twin = Server(seed, 2, 16, 40)
        with torch.cuda.stream(side):
            step(twin, captured, out)                    # (the workspace grows here)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p = step(a, captured, out)
        graphs.append((g, a, b, step, out, want, data, p))
    for i in range(5):
        for g, a, b, step, out, want, data, p in graphs:
            data["tokens"].copy_(torch.randint(0, a.vocab, data["tokens"].shape, device="cuda"))
            data["u"].copy_(torch.rand_like(data["u"]) * 0.05)
            torch.cuda.synchronize()
            pw = step(b, plain, want)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(p, pw) and all(torch.equal(x, y) for x, y in zip(out, want))
            assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.k_len, b.k_len)


def test_two_contexts_at_once():
    """each with its own workspace, on streams of their own"""
    cases = []
    for seed in (1, 2):
        stream = torch.cuda.Stream()
        srv = Server(seed, 1, 16, 200, d=64, vocab=50)
        with torch.cuda.stream(stream):
            cases.append((stream, binding.Context(stream), srv))
    torch.cuda.synchronize()
    for _, _, srv in cases:
        srv.k.normal_(), srv.v.normal_()
        srv.k_len.fill_(3000)
    q = torch.randn(40, 256, device="cuda").to(BF)
    cu, outs = ints([0, 40]), []
    torch.cuda.synchronize()
    alone = []
    for stream, ctx, srv in cases:
        o = torch.empty_like(q)
        ctx.glue_attention_paged(srv.cache, q, o, cu)
        torch.cuda.synchronize()
        alone.append(o)
    for _ in range(20):
        for stream, ctx, srv in cases:
            o = torch.empty_like(q)
            ctx.glue_attention_paged(srv.cache, q, o, cu)
            outs.append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, alone[i % 2]) for i, o in enumerate(outs))
