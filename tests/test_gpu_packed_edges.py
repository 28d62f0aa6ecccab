"""Packed attention at the ends of its ranges: the smallest scales, keys in many shares, and what is kept in more than one bf16 part, each against 64 bits."""
import random

import pytest
import torch

import packed_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_packed_attention import MARK, check, make, run

pytestmark = pytest.mark.gpu


def within(got, want, off, name):
    bad = ~((got.double() - want).abs() <= off)
    assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist())


def test_the_smallest_scale():
    """2^-100: every key counts the same, and gradients of q and k are as small; below it lse / scale would pass fp32"""
    ctx, scale = binding.Context(), 2.0 ** -100
    q, k, v, d, cq, ck = make(41, [40, 100], [40, 100], 4, 2, 64)
    got, want = run(ctx, q, k, v, d, cq, ck, 64, scale=scale), ref.attention(q, k, v, cq.tolist(), ck.tolist(), 64, scale=scale, dout=d)
    within(got["out"], want["out"], want["out_off"], "out")
    within(got["dv"], want["dv"], want["dv_off"], "dv")
    for name in ("dq", "dk"):
        within(got[name].double() / scale, want[name] / scale, want[name + "_off"] / scale + 1e-30, name)
    out, lse, dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, got["lse"], q, k, v))
    for small in (2.0 ** -101, 1e-38, 1e-45):
        with pytest.raises(binding.AgzoError):
            ctx.glue_attention_packed(q, k, v, out, cq, ck, 64, scale=small)
        with pytest.raises(binding.AgzoError):
            ctx.glue_attention_packed_backward(q, k, v, got["out"], got["lse"], d, dq, dk, dv, cq, ck, 64, scale=small)
    assert all((t == 7.0).all() for t in (out, dq, dk, dv))


def uneven(seed, n, total, longest=None):
    """n lengths, some of them 0 and 1, that add up to about `total`"""
    rng = random.Random(seed)
    lens = [rng.choice((0, 1, 63, 64, 65)) if rng.random() < 0.4 else int(rng.lognormvariate(0.0, 1.0) * total / n) for _ in range(n)]
    if longest:
        lens[rng.randrange(n)] = longest
    return lens


@pytest.mark.parametrize("qlens,klens,heads,kv,dim", [
    # shares of eight tiles, more of them than the lanes that join a row (16 and 32)
    ([1], [40000], 4, 1, 64), ([1, 1], [40000, 70], 2, 2, 128), ([3, 2, 1], [30000, 0, 900], 7, 1, 64),
    # larger shares
    ([1], [150001], 2, 1, 64), ([1, 1, 1, 1], [3, 140000, 0, 65], 4, 2, 128), ([150], [70000], 2, 1, 64),
    # more sequences than a wave looks at once
    ([1] * 70, uneven(1, 70, 90000), 4, 2, 64), ([1] * 131, uneven(2, 131, 180000, 30000), 2, 1, 128), ([2, 0, 1] * 30, uneven(3, 90, 120000), 2, 2, 64)])
def test_keys_in_shares(qlens, klens, heads, kv, dim):
    ctx = binding.Context()
    q, k, v, _, cq, ck = make(sum(klens) + dim, qlens, klens, heads, kv, dim, behind=2)
    check(run(ctx, q, k, v, None, cq, ck, dim), ref.attention(q, k, v, cq.tolist(), ck.tolist(), dim), cq, ck)


@pytest.mark.parametrize("n,room,dim", [(5, 20000, 64), (80, 1500, 128)])
def test_keys_in_shares_of_rooms_that_are_not_full(n, room, dim):
    """Bit for bit what the same keys give in rooms of which nothing else is left"""
    ctx, rng = binding.Context(), random.Random(n)
    have = [rng.choice((0, 1, room, rng.randint(2, room))) for _ in range(n)]
    q, k, v, _, cq, ck = make(n, [1] * n, [room] * n, 4, 2, dim)
    length = torch.tensor(have, device="cuda", dtype=torch.int32)
    got = run(ctx, q, k, v, None, cq, ck, dim, k_len=length)
    for s, h in enumerate(have):
        k[s * room + h:(s + 1) * room] = float("nan")
        v[s * room + h:(s + 1) * room] = float("nan")
    again = run(ctx, q, k, v, None, cq, ck, dim, k_len=length)
    assert all(torch.equal(got[i], again[i]) for i in got)
    there = torch.cat([torch.arange(s * room, s * room + h, device="cuda") for s, h in enumerate(have)])
    cu = [sum(have[:i]) for i in range(n + 1)]
    want = ref.attention(q, k[there], v[there], cq.tolist(), cu, dim)
    check(got, want, cq, ck)


U = 2.0 ** -24


def fp32_bounds(q, k, v, cu_q, cu_k, dim, d=None):
    """{out (, dq)} and bounds of their errors where probabilities and dS have 16 bits or more: a result's rounding to bf16; of scores, of do v and of the
    sums over keys a rounding to fp32 for each step of 16 values and as many more; exp2, lse and the parts that row terms are kept in"""
    q, k, v = (t.double().view(t.shape[0], -1, dim) for t in (q, k, v))
    heads, kv, scale, low = q.shape[1], k.shape[1], dim ** -0.5, 2.0 ** -16
    out, out_off, dq, dq_off = (torch.zeros_like(q) for _ in range(4))
    d = None if d is None else d.double().view_as(q)
    for b in range(len(cu_q) - 1):
        qs, ks = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        vis = ref.seen(nq, nk, True, q.device)
        steps = (nk // 16 + 16) * U
        for h in range(heads):
            K, V, Q = k[ks, h * kv // heads], v[ks, h * kv // heads], q[qs, h]
            s = torch.where(vis, Q @ K.T * scale, -torch.inf)
            lse = s.logsumexp(1, keepdim=True)
            p = (s - lse).exp()
            e = 2 * (dim // 16) * U * scale * (Q.abs() @ K.abs().T) + 4 * U * (torch.where(vis, s, 0.0).abs() + lse.abs()) + 8 * U
            e = e + (p * e).sum(1, keepdim=True)
            out[qs, h] = p @ V
            out_off[qs, h] = ref.HALF * out[qs, h].abs() + (1 + ref.HALF) * ((p * (e + low + steps)) @ V.abs())
            if d is None:
                continue
            D = d[qs, h]
            dp, ep = D @ V.T, 2 * (dim // 16) * U * (D.abs() @ V.abs().T)
            delta = (p * dp).sum(1, keepdim=True)
            size = dp.abs() + 1.01 * delta.abs()
            delta_off = (p * (e * size + ep)).sum(1, keepdim=True) + steps * (p * size).sum(1, keepdim=True)
            lonely = vis.sum(1, keepdim=True) == 1
            ds = torch.where(lonely, 0.0, p * (dp - delta))
            ds_off = torch.where(lonely, 0.0, ds.abs() * (e + low + steps) + p * (ep + delta_off + 4 * U * size))
            dq[qs, h] = scale * ds @ K
            dq_off[qs, h] = ref.HALF * dq[qs, h].abs() + (1 + ref.HALF) * scale * (ds_off @ K.abs())
    return {"out": (out.flatten(1), out_off.flatten(1)), "dq": (dq.flatten(1), dq_off.flatten(1))}


@pytest.mark.parametrize("klens,heads,kv,dim", [([1, 2, 64, 65, 300], 4, 2, 64), ([900, 5], 8, 1, 128), ([20000], 2, 1, 64)])
def test_probabilities_of_single_rows_have_two_parts(klens, heads, kv, dim):
    q, k, v, _, cq, ck = make(sum(klens), [1] * len(klens), klens, heads, kv, dim)
    got = run(binding.Context(), q, k, v, None, cq, ck, dim)
    want, off = fp32_bounds(q, k, v, cq.tolist(), ck.tolist(), dim)["out"]
    within(got["out"], want, off, "out")


@pytest.mark.parametrize("lens,heads,kv,dim", [([5] * 40, 4, 2, 64), ([64, 1, 33, 2, 50], 6, 2, 128)])
def test_the_queries_gradient_of_one_tile_of_keys_has_two_parts_and_its_own_delta(lens, heads, kv, dim):
    q, k, v, d, cq, ck = make(sum(lens) + 1, lens, lens, heads, kv, dim)
    got = run(binding.Context(), q, k, v, d, cq, ck, dim)
    want, off = fp32_bounds(q, k, v, cq.tolist(), ck.tolist(), dim, d)["dq"]
    within(got["dq"], want, off, "dq")


@pytest.mark.parametrize("qlens,klens", [([], []), ([0], [0]), ([0, 0], [70, 3]), ([3, 200], [0, 0]), ([0, 5, 0], [0, 0, 9])])
@pytest.mark.parametrize("dim", [64, 128])
def test_no_queries_or_no_keys(qlens, klens, dim):
    """Of rows that see nothing 0 and -inf, and of keys that nothing sees gradients of 0; where there are no sequences nothing is written"""
    ctx = binding.Context()
    for behind in (0, 4):
        q, k, v, d, cq, ck = make(7, qlens, klens, 4, 2, dim, behind=behind)
        for name, t in run(ctx, q, k, v, d, cq, ck, dim).items():
            n = sum(klens if name in ("dk", "dv") else qlens)
            assert (t[:n] == (-float("inf") if name == "lse" else 0.0)).all() and (t[n:] == MARK).all(), name
