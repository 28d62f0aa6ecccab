"""Drafted tokens against the target's probabilities with given random numbers (agzo_verify_drafts): the same tokens as the definition's, walked row by row in 64 bits."""
import math
import random

import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_cache import ints, offsets

pytestmark = pytest.mark.gpu


def rows_of(seed, n, vocab, dtype, spread=2.0):
    gen = torch.Generator().manual_seed(seed)
    return torch.softmax(spread * torch.randn(n, vocab, generator=gen), -1).to(dtype)


def run(p, q, tokens, u, cu, parents=None, ctx=None):
    ctx, n = ctx or binding.Context(), p.shape[0]
    dev = lambda t: None if t is None else t.cuda()
    out = [torch.full((m,), 77, dtype=torch.int32, device="cuda") for m in (n, n, len(cu) - 1)]
    ctx.verify_drafts(dev(p), dev(q), ints(tokens), torch.tensor(u, device="cuda"), ints(cu), *out, parents=None if parents is None else ints(parents))
    return [t.tolist() for t in out]


def check(p, q, tokens, u, cu, parents=None):
    u = torch.tensor(u, dtype=torch.float32).tolist()
    got = run(p, q, tokens, u, cu, parents)
    want = ref.verify(p.double(), None if q is None else q.double(), tokens, u, cu, parents)
    for g, w in zip(got[:2], want[:2]):
        assert [77 if x is None else x for x in w] == g
    assert got[2] == list(want[2])
    return got


def uniforms(seed, n):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed + 5)).tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 2047, 2048, 2049, 10007, 50000])
def test_chains(vocab, dtype):
    accepted = 0
    for seed, lens in ((1, [1, 2, 5, 9]), (2, [9] * 7), (3, [1]), (4, [70, 3])):
        n, cu = sum(lens), offsets(lens)
        p, noise = rows_of(seed, n, vocab, torch.float64), rows_of(seed + 50, n, vocab, torch.float64)
        # (row i's token is drawn from the draft's row, which is like the target's behind the row before)
        q = (0.7 * p.roll(1, 0) + 0.3 * noise)
        tokens = torch.multinomial(q, 1, generator=torch.Generator().manual_seed(seed))[:, 0].tolist()
        for with_q in (True, False):
            got = check(p.to(dtype), q.to(dtype) if with_q else None, tokens, uniforms(seed, n), cu)
            accepted += sum(got[2])
    assert accepted > 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [5, 100, 4099, 30011])
def test_trees(vocab, dtype):
    rng = random.Random(vocab)
    accepted = []
    for lens in ([1, 2, 10, 48], [64, 65], [200], [3] * 20):
        n, cu = sum(lens), offsets(lens)
        p = rows_of(n, n, vocab, dtype, 3.0)
        parents, tokens = [], []
        for s, m in enumerate(lens):
            for i in range(m):
                up = rng.randrange(max(0, i - 30), i) if i else -1
                parents.append(up)
                best = p[cu[s] + max(up, 0)].float().topk(min(vocab, 4)).indices.tolist()
                tokens.append(rng.choice(best))                          # (siblings with the same token among them)
        for seed in range(3):
            accepted += check(p, None, tokens, uniforms(seed, n), cu, parents)[2]
    assert max(accepted) > 0


def test_likely_first_children():
    """a node's first child has most of its probability"""
    rng, lens, vocab = random.Random(2), [64, 150, 30], 1000
    n, cu = sum(lens), offsets(lens)
    p, parents, tokens = 0.02 * rows_of(1, n, vocab, torch.float32), [], []
    for s, m in enumerate(lens):
        for i in range(m):
            parents.append(rng.randrange(max(0, i - 3), i) if i else -1)
            tokens.append(rng.randrange(vocab))
            if i and p[cu[s] + parents[-1]].max() < 0.9:
                p[cu[s] + parents[-1], tokens[-1]] += 0.98
    assert max(check(p, None, tokens, uniforms(4, n), cu, parents)[2]) > 1


def test_long_walks():
    """paths of more than 64 rows, unlikely leaves beside them"""
    rows, vocab = 300, 500
    p = 1e-5 * rows_of(1, rows, vocab, torch.float32)
    parents, tokens, trunk = [-1], [0], 0
    for i in range(1, rows):
        parents.append(trunk)
        tokens.append(i)
        if i % 7 != 3:
            p[trunk, i] = 0.9999
            trunk = i
    for q, of in ((None, parents), (p.roll(1, 0), None)):
        got = check(p, q, tokens, uniforms(4, rows), [0, rows], of)
        assert got[2][0] > 100 or of is None


def test_siblings_alike_far_apart():
    """a node's children in other groups of 64 rows, one token among them twice: the second has nothing left"""
    rows = 200
    p = torch.full((rows, 4), 0.25)
    parents = [-1] + [0 if i in (3, 70, 150) else 1 for i in range(1, rows)]
    tokens = [0] + [{3: 2, 70: 2, 150: 3}.get(i, 0) for i in range(1, rows)]
    for u3, u70, u150, want in ((0.5, 0.0, 0.0, [3]), (0.1, 0.9, 0.9, [2]), (0.5, 0.0, 0.9, [])):
        u = [0.6] * rows
        u[3], u[70], u[150] = u3, u70, u150
        got = check(p, None, tokens, u, [0, rows], parents)
        assert got[0][:len(want)] == want


def test_borders():
    """u q(x) = p(x) is not below it; a border that a sum meets goes to the next token; the first token with any weight, and the last one"""
    p = torch.tensor([[0.25, 0.25, 0.25, 0.25], [0.0, 0.5, 0.5, 0.0]])
    q = torch.tensor([[1.0, 0, 0, 0], [0.5, 0.25, 0.25, 0]])
    assert check(p, q, [0, 0], [0.0, 0.5], [0, 2])[2] == [0]
    assert check(p, q, [0, 0], [0.0, math.nextafter(0.5, 0) - 1e-7], [0, 2])[2] == [1]
    for u, token in ((0.0, 1), (0.499, 1), (0.5, 2), (0.999, 2), (1.0, 2), (7.0, 2), (-1.0, 1)):
        assert check(p, None, [0, 0], [u, 0.0], [0, 2])[0] == [0, token]
    # all of it refused: w = p - q has the last token only
    assert check(p, torch.tensor([[1.0, 0, 0, 0], [0.4, 0.3, 0.3, 0.0]]), [0, 1], [0.3, 0.99], [0, 2])[0][0] == 3


def test_probabilities_that_are_none():
    nan, inf = math.nan, math.inf
    p = torch.tensor([[nan, -1.0, 0.5, 0.25], [0.0, 0.0, nan, -inf], [0.0, inf, 0.0, inf]])
    assert check(p[:2], None, [0, 2], [0.5, 0.0], [0, 2])[0] == [2, -1]          # accepted, and nothing to draw from
    assert check(p[:2], None, [0, 0], [0.1, 0.0], [0, 2])[0] == [2, -1]          # NaN: refused; from the rest
    assert check(p[1:2], None, [0], [0.1], [0, 1])[0] == [-1]
    assert check(p[2:], None, [0], [0.1], [0, 1])[0] == [3]                  # (no border in infinitely much: the last)
    for bad in (-1, 4, 2 ** 31 - 1, -(2 ** 31)):
        assert check(p[:2], None, [bad, bad], [0.1, 0.0], [0, 2])[2] == [0]
        assert check(p[:2], p[:2], [bad, bad], [0.1, 0.0], [0, 2])[2] == [0]
    # refused tokens leave nothing: the target's own probabilities
    one = torch.tensor([[0.0, 0.5, 0.0], [1.0, 0, 0]])
    assert check(one, None, [0, 1], [0.3, 0.9], [0, 2])[0] == [1, -1]
    assert check(one, one, [0, 1], [0.3, 1.0], [0, 2])[2] == [1]             # (drawn where the draft has nothing: accepted)
    # random numbers that are none are refusals, and draw the last
    assert check(one, None, [0, 1], [nan, nan], [0, 2])[2] == [0]


def test_parents_that_are_none_are_not_looked_at():
    p = torch.full((5, 3), 1 / 3)
    for parents in ([7, -1, 5, 2 ** 31 - 1, 0], [0, 1, 2, 3, 4], [-9, -9, 0, 3, 2]):
        check(p, None, [0, 1, 2, 0, 1], [0.5, 0.1, 0.1, 0.1, 0.1], [0, 5], parents)


def test_rows_of_no_sequence_and_sequences_of_none():
    p = rows_of(1, 12, 300, torch.float32)
    got = check(p, None, list(range(12)), uniforms(1, 12), [2, 2, 5, 5, 9])
    assert got[0][:2] == [77] * 2 and got[1][9:] == [77] * 3 and got[2][0] == 0 and got[2][2] == 0


def test_strides_and_misaligned_rows():
    """rows of a wider tensor that no 16 bytes divide"""
    for dtype in (torch.float32, torch.bfloat16):
        wide = rows_of(2, 9, 5003, dtype).cuda()
        p, q = wide[:, 3:4500], wide.roll(1, 0)[:, 1:4498]
        tokens, u, cu = list(range(9)), uniforms(2, 9), [0, 4, 9]
        ctx, outs = binding.Context(), []
        for a, b in ((p, q), (p.contiguous(), q.contiguous())):
            out = [torch.empty(m, dtype=torch.int32, device="cuda") for m in (9, 9, 2)]
            ctx.verify_drafts(a, b, ints(tokens), torch.tensor(u, device="cuda"), ints(cu), *out)
            outs.append([t.tolist() for t in out])
        assert outs[0] == outs[1]
        want = ref.verify(p.double().cpu(), q.double().cpu(), tokens, torch.tensor(u).tolist(), cu)
        assert outs[0] == [want[0], want[1], want[2]]


def test_a_token_has_the_targets_distribution():
    """one draft and what follows it, over 40000 pairs of random numbers: the first token's frequencies are the target's"""
    n = 40000
    p, q = torch.tensor([0.1, 0.2, 0.3, 0.05, 0.35]), torch.tensor([0.3, 0.1, 0.2, 0.3, 0.1])
    gen = torch.Generator().manual_seed(3)
    tokens = torch.zeros(n, 2, dtype=torch.long)
    tokens[:, 1] = torch.multinomial(q, n, replacement=True, generator=gen)
    u = torch.rand(2 * n, generator=gen).tolist()
    counts = torch.zeros(5)
    ctx = binding.Context()
    P, Q = p.repeat(2 * n, 1), q.repeat(2 * n, 1)
    out, _, _ = run(P, Q, tokens.flatten().tolist(), u, list(range(0, 2 * n + 1, 2)), ctx=ctx)
    counts = torch.bincount(torch.tensor(out[::2]), minlength=5) / n
    # five standard deviations of a frequency, sqrt(p (1 - p) / n)
    assert ((counts - p).abs() < 5 * (p * (1 - p) / n).sqrt()).all()


def test_captured_and_replayed():
    side = torch.cuda.Stream()
    ctx, plain = binding.Context(side), binding.Context()
    n, cu = 18, ints([0, 9, 18])
    p, q = (torch.softmax(torch.randn(n, 5000, device="cuda"), -1) for _ in range(2))
    tokens, u = torch.randint(0, 5000, (n,), device="cuda").int(), torch.rand(n, device="cuda")
    out, want = ([torch.empty(m, dtype=torch.int32, device="cuda") for m in (n, n, 2)] for _ in range(2))
    torch.cuda.synchronize()
    ctx.verify_drafts(p, q, tokens, u, cu, *out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.verify_drafts(p, q, tokens, u, cu, *out)
    for i in range(4):
        u.copy_(torch.rand(n, device="cuda") ** (4 if i % 2 else 1))
        tokens.copy_(torch.randint(0, 5000, (n,), device="cuda").int())
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        plain.verify_drafts(p, q, tokens, u, cu, *want)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    ctx, E = binding.Context(), binding.AgzoError
    p = rows_of(1, 6, 50, torch.float32).cuda()
    t, u, cu = ints(range(6)), torch.rand(6, device="cuda"), ints([0, 3, 6])
    o = [torch.empty(m, dtype=torch.int32, device="cuda") for m in (6, 6, 2)]
    ok = dict(p=p, q=None, tokens=t, uniforms=u, cu=cu, out_tokens=o[0], out_rows=o[1], n_accepted=o[2])
    ctx.verify_drafts(**ok)
    for change, error in ((dict(q=p, parents=t), E), (dict(out_rows=o[0]), E), (dict(out_tokens=t), E), (dict(q=p.bfloat16()), TypeError), (dict(p=p.double()), TypeError), (dict(q=p[:, :49]), ValueError),
                          (dict(tokens=t.long()), TypeError), (dict(tokens=t[:5]), ValueError), (dict(uniforms=u.double()), TypeError), (dict(n_accepted=o[0]), ValueError), (dict(cu=cu.cpu()), ValueError),
                          (dict(parents=t[:5]), ValueError), (dict(p=p.t()), ValueError), (dict(p=p.cpu()), ValueError)):
        with pytest.raises(error):
            ctx.verify_drafts(**{**ok, **change})
    with pytest.raises(E):
        ctx.verify_drafts(**{**ok, "p": torch.empty(6, 0, device="cuda")})
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    ctx.verify_drafts(p[:0], None, e, u[:0], ints([0, 0]), e, e.clone(), o[2][:1])
    ctx.check()
