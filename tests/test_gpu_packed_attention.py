"""Attention over packed sequences of different lengths, forward and backward, against a 64-bit form row by row, with element-wise bounds."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
MARK = -77.0        # what rows of no sequence hold, before and after


def offsets(lens, first=0):
    return torch.tensor(np.cumsum([first] + list(lens)), device="cuda", dtype=torch.int32)


def make(seed, qlens, klens, heads, kv, dim, pad=0, behind=0, spread=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n, w, c: (torch.randn(n, w + pad, device="cuda", generator=gen) * c).bfloat16()[:, :w]
    nq, nk = sum(qlens) + behind, sum(klens) + behind
    return rnd(nq, heads * dim, spread), rnd(nk, kv * dim, spread), rnd(nk, kv * dim, 1.0), rnd(nq, heads * dim, 1.0), offsets(qlens), offsets(klens)


def run(ctx, q, k, v, d, cq, ck, dim, **kw):
    heads = q.shape[1] // dim
    r = {"out": torch.full_like(q, MARK), "lse": torch.full((q.shape[0], heads), MARK, device="cuda")}
    ctx.glue_attention_packed(q, k, v, r["out"], cq, ck, dim, lse=r["lse"], **kw)
    if d is not None:
        r["dq"], r["dk"], r["dv"] = torch.full_like(q, MARK), torch.full_like(k, MARK), torch.full_like(v, MARK)
        ctx.glue_attention_packed_backward(q, k, v, r["out"], r["lse"], d, r["dq"], r["dk"], r["dv"], cq, ck, dim, **kw)
    return r


def check(got, want, cq, ck):
    cq, ck = cq.tolist(), ck.tolist()
    for name, t in got.items():
        cu, total = (ck, t.shape[0]) if name in ("dk", "dv") else (cq, t.shape[0])
        there = ref.rows_in(cu, total, t.device)
        assert (t[~there] == MARK).all(), name
        g, w = t[there].double(), want[name][there]
        if name == "lse":
            fin = torch.isfinite(w)
            assert torch.equal(g[~fin], w[~fin])
            assert ((g[fin] - w[fin]).abs() <= 2e-5 * (1 + w[fin].abs())).all(), float((g[fin] - w[fin]).abs().max())
            continue
        off = want[name + "_off"][there]
        bad = ~((g - w).abs() <= off + 1e-30)
        assert not bad.any(), (name, int(bad.sum()), bad.numel(), bad.nonzero()[:4].tolist(), g[bad][:4].tolist(), w[bad][:4].tolist(), off[bad][:4].tolist())


SHAPES = [
    # one token; odd short ones; empty sequences among others
    ([1], 1, 1, 64), ([1, 1, 1], 4, 2, 128), ([5, 77, 0, 33, 1], 6, 2, 128), ([0, 0, 3], 2, 2, 64),
    # around tiles of 64 keys and 128 rows, groups of one to seven heads
    ([63, 64, 65], 1, 1, 128), ([127, 128, 129], 2, 1, 64), ([31, 32, 33, 257], 3, 3, 128), ([300, 18], 7, 1, 64), ([200, 511], 8, 2, 128),
    # long
    ([1500, 40], 4, 2, 128), ([2049], 2, 1, 64),
]


@pytest.mark.parametrize("lens,heads,kv,dim", SHAPES)
def test_prompts(lens, heads, kv, dim):
    ctx = binding.Context()
    q, k, v, d, cq, ck = make(len(lens) + heads, lens, lens, heads, kv, dim, pad=8 * (heads % 3), behind=heads % 2 * 5)
    want = ref.attention(q, k, v, cq.tolist(), ck.tolist(), dim, dout=d)
    check(run(ctx, q, k, v, d, cq, ck, dim), want, cq, ck)


@pytest.mark.parametrize("qlens,klens,heads,kv,dim", [
    ([1, 1, 1, 1], [1, 300, 64, 1027], 8, 2, 128), ([1], [5000], 4, 1, 64), ([1] * 9, [700] * 9, 14, 2, 64),
    ([3, 17, 130], [80, 17, 1000], 4, 4, 128), ([2, 4], [9000, 20], 6, 2, 128),
    # rows that see nothing: fewer keys than queries, no keys at all
    ([5, 70, 3, 1], [2, 66, 0, 0], 2, 1, 64), ([200], [100], 4, 2, 128), ([4, 4], [0, 0], 2, 2, 64)])
def test_other_lengths_of_queries(qlens, klens, heads, kv, dim):
    ctx = binding.Context()
    q, k, v, d, cq, ck = make(sum(klens) + heads, qlens, klens, heads, kv, dim, behind=3)
    want = ref.attention(q, k, v, cq.tolist(), ck.tolist(), dim, dout=d)
    check(run(ctx, q, k, v, d, cq, ck, dim), want, cq, ck)


@pytest.mark.parametrize("qlens,klens,heads,kv,dim,scale", [([40, 1], [40, 1], 2, 1, 128, 0.3), ([65, 7], [130, 0], 4, 2, 64, 0.02), ([1, 3], [2000, 1], 4, 1, 128, None)])
def test_without_mask_and_other_scales(qlens, klens, heads, kv, dim, scale):
    ctx = binding.Context()
    q, k, v, d, cq, ck = make(9, qlens, klens, heads, kv, dim)
    want = ref.attention(q, k, v, cq.tolist(), ck.tolist(), dim, scale, False, d)
    check(run(ctx, q, k, v, d, cq, ck, dim, scale=scale, causal=False), want, cq, ck)


def test_large_scores():
    """Scores of some hundreds: nearly one-hot probabilities, and maxima that move late."""
    ctx = binding.Context()
    q, k, v, d, cq, ck = make(3, [200, 90], [200, 90], 2, 1, 128, spread=6.0)
    k[:, :] = k * torch.linspace(0.1, 1.5, k.shape[0], device="cuda")[:, None].bfloat16()
    want = ref.attention(q, k, v, cq.tolist(), ck.tolist(), 128, dout=d)
    got = run(ctx, q, k, v, None, cq, ck, 128)
    # fp32 scores of up to some 500 are off by 500 * 2^-22, and so are probabilities
    want["out_off"] += 2e-4 * (want["out_off"] / ref.HALF)
    check(got, want, cq, ck)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [64, 128])
def test_masked_values_have_no_part(value, dim):
    """Keys and values that are not finite show in the rows that see them, and in no other."""
    ctx = binding.Context()
    lens = [100, 70]
    q, k, v, d, cq, ck = make(11, lens, lens, 4, 2, dim, behind=40)
    at = 75
    clean = run(ctx, q, k, v, None, cq, ck, dim)["out"]
    v2 = v.clone()
    v2[at, 3] = value
    v2[170:] = value
    got = run(ctx, q, k, v2, None, cq, ck, dim)["out"]
    touched = torch.zeros_like(clean, dtype=torch.bool)
    for h in (0, 1):                              # the heads of key head 0
        touched[at:100, h * dim + 3] = True
    assert torch.equal(got[~touched], clean[~touched])
    t = got[touched].float()
    assert (t.isnan() if value != value else t == value).all()
    k2 = k.clone()
    k2[at, 5] = float("nan")
    k2[170:] = float("nan")
    got = run(ctx, q, k2, v, None, cq, ck, dim)["out"]
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[at:100, :2 * dim] = True
    assert torch.equal(got[~touched], clean[~touched]) and got[touched].isnan().all()


@pytest.mark.parametrize("dim", [64, 128])
def test_masked_values_have_no_part_in_gradients(dim):
    ctx = binding.Context()
    lens = [100, 70]
    q, k, v, d, cq, ck = make(12, lens, lens, 4, 2, dim, behind=40)
    r = run(ctx, q, k, v, d, cq, ck, dim)
    clean = {n: t.clone() for n, t in r.items()}
    nan = float("nan")

    def back(q, k, v, d, out=clean["out"], lse=clean["lse"]):
        g = {"dq": torch.full_like(q, MARK), "dk": torch.full_like(k, MARK), "dv": torch.full_like(v, MARK)}
        ctx.glue_attention_packed_backward(q, k, v, out, lse, d, g["dq"], g["dk"], g["dv"], cq, ck, dim)
        return g

    at = 41
    # a row's gradient that is not finite: its own dq, and the keys that it sees
    d2 = d.clone()
    d2[at] = nan
    d2[170:] = nan
    g = back(q, k, v, d2)
    keep = torch.ones(210, dtype=torch.bool, device="cuda")
    keep[at] = False
    assert torch.equal(g["dq"][keep], clean["dq"][keep]) and g["dq"][at].isnan().all()
    for n in ("dk", "dv"):
        assert torch.equal(g[n][at + 1:], clean[n][at + 1:]) and g[n][:at + 1].isnan().all(), n
    # a key and value: the rows in front of it keep their gradients
    k2, v2 = k.clone(), v.clone()
    k2[at] = nan
    v2[at] = nan
    g = back(q, k2, v2, d)
    assert torch.equal(g["dq"][:at], clean["dq"][:at]) and torch.equal(g["dq"][100:], clean["dq"][100:]) and g["dq"][at:100].isnan().all()
    assert torch.equal(g["dk"][100:], clean["dk"][100:]) and torch.equal(g["dv"][100:], clean["dv"][100:])
    # a query: the keys behind it keep theirs
    q2 = q.clone()
    q2[at] = nan
    g = back(q2, k, v, d)
    assert torch.equal(g["dk"][at + 1:], clean["dk"][at + 1:]) and torch.equal(g["dv"][at + 1:], clean["dv"][at + 1:])


def test_offsets_outside_the_tensors_are_taken_as_inside():
    ctx = binding.Context()
    q, k, v, d, cq, ck = make(13, [30, 34], [30, 34], 2, 1, 64)
    want = run(ctx, q, k, v, d, cq, ck, 64)
    far = cq.clone()
    far[0], far[2] = -5, 1 << 30
    got = run(ctx, q, k, v, d, far, far, 64)
    assert all(torch.equal(got[n], want[n]) for n in want)
    # sequences between other rows: those keep what they hold
    part = torch.tensor([10, 30, 50], device="cuda", dtype=torch.int32)
    got = run(ctx, q, k, v, d, part, part, 64)
    for t in got.values():
        assert (t[:10] == MARK).all() and (t[50:] == MARK).all() and not (t[10:50] == MARK).any()


def test_gradients_against_differences():
    """The gradient of a weighted sum of the outputs along a direction, against two more forward passes of the 64-bit form."""
    ctx = binding.Context()
    lens, dim = [50, 21], 64
    q, k, v, d, cq, ck = make(14, lens, lens, 4, 2, dim)
    got = run(ctx, q, k, v, d, cq, ck, dim)
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = 1e-4
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        way = torch.randn(t.shape, device="cuda", generator=gen).double()
        f = []
        for sign in (1, -1):
            args = {"dq": q.double(), "dk": k.double(), "dv": v.double()}
            args[name] = t.double() + sign * h * way
            f.append((ref.attention(args["dq"], args["dk"], args["dv"], cq.tolist(), ck.tolist(), dim)["out"] * d.double()).sum())
        slope, mine = (f[0] - f[1]) / (2 * h), (got[name].double() * way).sum()
        # independent roundings of 2^-8 in every element add up like their root
        assert (slope - mine).abs() <= 4 * 2 ** -8 * (got[name].double() * way).norm() + 1e-6 * slope.abs(), name


def test_same_results_again_and_on_another_stream():
    lens = [400, 3, 129]
    q, k, v, d, cq, ck = make(15, lens, lens, 8, 2, 128)
    ctx = binding.Context()
    a = run(ctx, q, k, v, d, cq, ck, 128)
    b = run(ctx, q, k, v, d, cq, ck, 128)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    other = binding.Context(stream=st)
    with torch.cuda.stream(st):
        c = run(other, q, k, v, d, cq, ck, 128)
    st.synchronize()
    for n in a:
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], c[n]), n


def test_captured_calls_replay():
    """Forward and backward in a graph, replayed with new inputs, with eager calls on the same context between."""
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = binding.Context(stream=st)
        qlens, klens = [1, 1, 1], [900, 40, 3000]
        q, k, v, d, cq, ck = make(16, qlens, klens, 8, 2, 128)
        r = run(ctx, q, k, v, d, cq, ck, 128)           # the workspace has its size
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            ctx.glue_attention_packed(q, k, v, r["out"], cq, ck, 128, lse=r["lse"])
            ctx.glue_attention_packed_backward(q, k, v, r["out"], r["lse"], d, r["dq"], r["dk"], r["dv"], cq, ck, 128)
        for seed in range(3):
            q2, k2, v2, d2, _, ck2 = make(20 + seed, qlens, [1000, 2000 - seed, 940 + seed], 8, 2, 128)
            for a, b in ((q, q2), (k, k2), (v, v2), (d, d2), (ck, ck2)):
                a.copy_(b)
            graph.replay()
            st.synchronize()
            got = {n: t.clone() for n, t in r.items()}
            # a larger call, which makes the context's workspace grow: the graph keeps the one that it was captured with
            big = make(30 + seed, [700] * (2 + seed), [700] * (2 + seed), 8, 2, 128)
            run(ctx, *big, 128)
            want = run(ctx, q, k, v, d, cq, ck, 128)
            st.synchronize()
            assert all(torch.equal(got[n], want[n]) for n in want)


def test_capture_that_would_grow_the_workspace_is_refused():
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = binding.Context(stream=st)
        q, k, v, d, cq, ck = make(17, [1], [5000], 4, 1, 64)
        out = torch.full_like(q, MARK)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            with pytest.raises(binding.AgzoError) as e:
                ctx.glue_attention_packed(q, k, v, out, cq, ck, 64)
        assert e.value.code == binding.ENOMEM
        graph.replay()
        st.synchronize()
        assert (out == MARK).all()


def test_offsets_past_32_bits():
    """Keys whose rows lie more than 2^32 bytes behind the first."""
    ctx = binding.Context()
    ld, n = 1 << 21, 1100
    store = torch.empty(n * ld, device="cuda", dtype=torch.bfloat16)          # 4.6 GB
    wide = store.view(n, ld)
    q, k, v, d, cq, ck = make(18, [1, 2], [100, 1000], 4, 1, 64)
    k2, v2 = wide[:, 64:128], wide[:, 128:192]
    k2.copy_(k)
    v2.copy_(v)
    a, b = run(ctx, q, k, v, d, cq, ck, 64), run(ctx, q, k2, v2, None, cq, ck, 64)
    assert torch.equal(a["out"], b["out"])
    dk, dv, dq = wide[:, 256:320], wide[:, 320:384], torch.empty_like(q)
    ctx.glue_attention_packed_backward(q, k2, v2, a["out"], a["lse"], d, dq, dk, dv, cq, ck, 64)
    assert torch.equal(dq, a["dq"]) and torch.equal(dk, a["dk"]) and torch.equal(dv, a["dv"])


def test_many_sequences_and_too_many():
    ctx = binding.Context()
    klens = [3, 1, 2, 5] * 2048
    q, k, v, d, cq, ck = make(31, [1] * len(klens), klens, 2, 1, 64)
    check(run(ctx, q, k, v, None, cq, ck, 64), ref.attention(q, k, v, cq.tolist(), ck.tolist(), 64), cq, ck)
    qlens = [2, 0, 70, 1, 3] * 20
    q, k, v, d, cq, ck = make(32, qlens, qlens, 4, 2, 128)
    check(run(ctx, q, k, v, d, cq, ck, 128), ref.attention(q, k, v, cq.tolist(), ck.tolist(), 128, dout=d), cq, ck)
    cu = torch.zeros(65538, dtype=torch.int32, device="cuda")
    with pytest.raises(binding.AgzoError):
        ctx.glue_attention_packed(q, k, v, torch.empty_like(q), cu, cu, 128)


def test_refusals():
    ctx = binding.Context()
    q, k, v, d, cq, ck = make(19, [8], [8], 4, 2, 64)
    out = torch.full_like(q, MARK)
    bad = [dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(head_dim=32)]
    for kw in bad:
        with pytest.raises(binding.AgzoError):
            ctx.glue_attention_packed(q, k, v, out, cq, ck, **{"head_dim": 64, **kw})
    with pytest.raises(binding.AgzoError):
        ctx.glue_attention_packed(q[:, :192], k, v, out[:, :192], cq, ck, 64)             # three heads on two
    for bad_out in (q, k.new_empty(0)):
        with pytest.raises((binding.AgzoError, ValueError)):
            ctx.glue_attention_packed(q, k, v, bad_out, cq, ck, 64)
    with pytest.raises(ValueError):
        ctx.glue_attention_packed(q, k, v[:4], out, cq, ck, 64)
    with pytest.raises(ValueError):
        ctx.glue_attention_packed(q, k, v, out, cq, ck[:1], 64)
    with pytest.raises(TypeError):
        ctx.glue_attention_packed(q, k, v, out, cq.long(), ck, 64)
    with pytest.raises(TypeError):
        ctx.glue_attention_packed(q.half(), k, v, out, cq, ck, 64)
    with pytest.raises(ValueError):
        ctx.glue_attention_packed(q, k, v, out, cq.cpu(), ck, 64)
    lse, dq, dk, dv = torch.empty(8, 4, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    with pytest.raises(binding.AgzoError):
        ctx.glue_attention_packed_backward(q, k, v, out, None, d, dq, dk, dv, cq, ck, 64)
    with pytest.raises(binding.AgzoError):
        ctx.glue_attention_packed_backward(q, k, v, out, lse, d, dq, dk, dk, cq, ck, 64)
    with pytest.raises(binding.AgzoError):
        ctx.glue_attention_packed_backward(q, k, v, out, lse, d, d, dk, dv, cq, ck, 64)
    assert (out == MARK).all()
