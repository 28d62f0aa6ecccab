"""Rotation of queries and keys in its layouts (agzo_glue_rope, agzo_glue_rope_backward) against the formula in 64 bits."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu

SCALED = {"plain": {}, "linear": dict(scaling=binding.ROPE_LINEAR, factor=4.0), "turns": dict(scaling=binding.ROPE_TURNS, factor=8.0, low=1.0, high=4.0, original=8192.0),
          "dims": dict(scaling=binding.ROPE_DIMS, factor=4.0, low=1.0, high=32.0, original=32768.0, magnitude=1.25)}


def make(n, heads, kv, dim, dtype, seed, far=5000):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k = (torch.randn(n, h * dim, device="cuda", generator=gen).to(dtype) for h in (heads, kv))
    return q, k, torch.randint(-3, far, (n,), device="cuda", generator=gen).int()


def check(got, x, pos, rope, dim, back=False):
    want, off = ref.rotate(x, pos, rope, dim, back)
    assert ((got.double() - want).abs() <= off + ref.HALF[got.dtype] * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 64), (128, 32), (96, 80), (16, 16), (256, 256), (80, 48)])
def test_forward_and_backward(dim, rot, inter, dtype):
    ctx, rope = binding.Context(), binding.make_rope(rot, 1.0e4, interleaved=inter)
    for n, heads, kv in ((1, 1, 1), (37, 6, 2), (1500, 3, 3), (4103, 2, 1)):
        q, k, pos = make(n, heads, kv, dim, dtype, n)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        ctx.glue_rope(rope, q, k, pos, qo, ko, dim)
        check(qo, q, pos, rope, dim)
        check(ko, k, pos, rope, dim)
        ctx.glue_rope_backward(rope, q, k, pos, qo, ko, dim)
        check(qo, q, pos, rope, dim, True)
        check(ko, k, pos, rope, dim, True)


@pytest.mark.parametrize("scaling", sorted(SCALED))
@pytest.mark.parametrize("inter", [False, True])
def test_scaled_for_long_contexts(scaling, inter):
    ctx, rope = binding.Context(), binding.make_rope(128, 1.0e6, interleaved=inter, **SCALED[scaling])
    q, k, pos = make(300, 4, 2, 128, torch.float32, 5, 200000)
    pos[:4] = torch.tensor([2 ** 31 - 1, -(2 ** 31), 0, 1], device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ctx.glue_rope(rope, q, k, pos, qo, ko)
    check(qo, q, pos, rope, 128)
    check(ko, k, pos, rope, 128)


@pytest.mark.parametrize("scaling", ["turns", "dims"])
def test_frequencies_change_between_both_ends(scaling):
    """what the highest and the lowest frequency become: themselves, and a factor less"""
    rope = binding.make_rope(128, 1.0e6, **SCALED[scaling])
    f, plain = ref.frequencies(rope, "cpu"), ref.frequencies(binding.make_rope(128, 1.0e6), "cpu")
    assert float(f[0]) == float(plain[0]) and math.isclose(float(f[-1]), float(plain[-1]) / rope.factor)
    assert 0 < int(((f < plain) & (f > plain / rope.factor * 1.0000001)).sum()) < 40


def test_the_gradient_is_the_formulas_and_the_differences():
    """d/dx of sum(y * w), by the call and by differences of the call's own results (fp32: steps of 2^-6, exact in x; linear in x)"""
    ctx, rope = binding.Context(), binding.make_rope(32, 1.0e4, interleaved=True, magnitude=1.5)
    q, k, pos = make(5, 2, 1, 48, torch.float32, 9)
    w = torch.randn(5, 96, device="cuda")
    dq, y0, y1 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    ctx.glue_rope_backward(rope, w, None, pos, dq, None, 48)
    h = 2.0 ** -6
    for t, c in ((0, 0), (1, 31), (2, 33), (3, 47), (4, 48 + 5), (4, 95)):
        a, b = q.clone(), q.clone()
        a[t, c] += h
        b[t, c] -= h
        ctx.glue_rope(rope, a, None, pos, y0, None, 48)
        ctx.glue_rope(rope, b, None, pos, y1, None, 48)
        diff = float(((y0.double() - y1.double()) * w.double()).sum()) / float(a[t, c].double() - b[t, c].double())
        # eight roundings of results below 8 (two values, two sides, a product and a sum each), 2^-22, over a step of 2^-5
        assert abs(diff - float(dq[t, c])) < 8 * 2.0 ** -22 * 2 ** 5 * float(w.abs().max())


def test_backward_undoes_forward():
    ctx, rope = binding.Context(), binding.make_rope(64, 1.0e6)
    q, k, pos = make(100, 4, 2, 64, torch.float32, 2)
    y, z = torch.empty_like(q), torch.empty_like(q)
    ctx.glue_rope(rope, q, None, pos, y, None, 64)
    ctx.glue_rope_backward(rope, y, None, pos, z, None, 64)
    assert float((z - q).abs().max()) < 1e-5


def test_in_place_strided_and_one_side():
    ctx, rope = binding.Context(), binding.make_rope(48, 1.0e4)
    wide = torch.randn(70, 5 * 64 + 24, device="cuda").bfloat16()
    q, k = wide[:, :192], wide[:, 200:328]
    pos = torch.arange(70, device="cuda").int()
    qw, kw = torch.empty(70, 192, device="cuda", dtype=torch.bfloat16), torch.empty(70, 128, device="cuda", dtype=torch.bfloat16)
    ctx.glue_rope(rope, q, k, pos, qw, kw, 64)
    only = torch.empty_like(kw)
    ctx.glue_rope(rope, None, k, pos, None, only, 64)
    assert torch.equal(only, kw)
    before = wide.clone()
    ctx.glue_rope(rope, q, k, pos, q, k, 64)
    assert torch.equal(q, qw) and torch.equal(k, kw)
    assert torch.equal(wide[:, 192:200], before[:, 192:200]) and torch.equal(wide[:, 328:], before[:, 328:])


def test_captured_on_another_stream():
    side = torch.cuda.Stream()
    ctx, sctx, rope = binding.Context(), binding.Context(side), binding.make_rope(128, interleaved=True)
    q, k, pos = make(50, 4, 2, 128, torch.bfloat16, 4)
    qo, ko, want = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        sctx.glue_rope(rope, q, k, pos, qo, ko)
    for i in range(3):
        q.copy_(torch.randn_like(q))
        pos += 100
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        ctx.glue_rope(rope, q, None, pos, want, None)
        assert torch.equal(qo, want)


def test_no_tokens():
    ctx, rope = binding.Context(), binding.make_rope(64)
    e, pos = torch.empty(0, 128, device="cuda", dtype=torch.bfloat16), torch.empty(0, device="cuda", dtype=torch.int32)
    ctx.glue_rope(rope, e, e, pos, torch.empty_like(e), torch.empty_like(e), 64)
    ctx.check()


def test_refusals():
    ctx = binding.Context()
    q, k, pos = make(8, 2, 2, 64, torch.bfloat16, 1)
    o = torch.empty_like(q)
    for rope in (binding.make_rope(8), binding.make_rope(24), binding.make_rope(80), binding.make_rope(0), binding.make_rope(64, theta=1.0), binding.make_rope(64, theta=math.inf),
                 binding.make_rope(64, magnitude=math.nan), binding.make_rope(64, scaling=4, factor=2.0), binding.make_rope(64, scaling=binding.ROPE_LINEAR, factor=0.0),
                 binding.make_rope(64, scaling=binding.ROPE_TURNS, factor=2.0, low=4.0, high=4.0, original=100.0), binding.make_rope(64, scaling=binding.ROPE_DIMS, factor=2.0)):
        with pytest.raises(binding.AgzoError):
            ctx.glue_rope(rope, q, None, pos, o, None, 64)
    rope = binding.make_rope(64)
    with pytest.raises(binding.AgzoError):
        ctx.glue_rope(rope, q[:7], None, pos[:7], q[1:], None, 64)              # overlapping
    with pytest.raises(binding.AgzoError):
        ctx.glue_rope(rope, q, k, pos, o, o, 64)
    for args, error in (((q.float(), None, pos, o, None), TypeError), ((q, k.float(), pos, o, torch.empty_like(k)), TypeError), ((q, None, pos.long(), o, None), TypeError),
                        ((q, None, pos[:7], o, None), ValueError), ((q, None, pos, o[:7], None), ValueError), ((None, None, pos, None, None), ValueError), ((q.cpu(), None, pos, o, None), ValueError),
                        ((q, k[:7], pos, o, torch.empty_like(k)), ValueError)):
        with pytest.raises(error):
            ctx.glue_rope(rope, *args, 64)
    with pytest.raises(ValueError):
        ctx.glue_rope(rope, q, None, pos, o, None, 48)
    with pytest.raises(binding.AgzoError):
        ctx.glue_rope(binding.make_rope(32), torch.empty(8, 72, device="cuda").bfloat16(), None, pos, torch.empty(8, 72, device="cuda").bfloat16(), None, 72)
