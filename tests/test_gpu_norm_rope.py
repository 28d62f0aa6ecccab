"""Norms of queries and keys for each head with the rotation by the position, and the gradient, against 64-bit forms; refusals."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
EPS, THETA = 1e-6, 1.0e6


def make(seed, n, heads, kv, dim, far, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    wide = lambda w, c: (rnd(n, w + pad) * c).bfloat16()[:, :w]
    q, k, dq, dk = wide(heads * dim, 0.6), wide(kv * dim, 2.0), wide(heads * dim, 1.0), wide(kv * dim, 0.1)
    pos = torch.randint(-3 if far > 10 else 0, far, (n,), device="cuda", generator=gen).int()
    return q, k, dq, dk, pos, 1 + 0.2 * rnd(dim), 1 + 0.2 * rnd(dim)


def close(got, want, off):
    err = (got.double() - want).abs()
    bad = ~(err <= off)
    assert not bad.any(), (int(bad.sum()), float(err[bad].max()), bad.nonzero()[:3].tolist())


@pytest.mark.parametrize("n,heads,kv,dim,far,pad", [
    (1, 1, 1, 64, 1, 0), (1, 16, 8, 128, 32768, 0), (3, 3, 1, 128, 2 ** 31 - 1, 8), (77, 14, 2, 64, 500, 40), (2047, 4, 2, 128, 4096, 0),
    (2048, 5, 5, 64, 4096, 0), (2051, 8, 1, 128, 200000, 16), (5, 0, 3, 64, 100, 0), (6, 7, 0, 128, 100, 0)])
def test_forward_and_backward(n, heads, kv, dim, far, pad):
    q, k, dqo, dko, pos, qg, kg = make(n, n, heads, kv, dim, far, pad)
    qg = None if n == 77 else qg
    ctx = binding.Context()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    none = lambda t: t if t.shape[1] else None
    ctx.glue_qk_norm_rope(none(q), none(k), pos, none(qo), none(ko), dim, qg, kg, EPS, THETA)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    gq, gk = torch.full((dim,), 7.0, device="cuda"), torch.full((dim,), 7.0, device="cuda")
    ctx.glue_qk_norm_rope_backward(none(q), none(k), pos, none(dqo), none(dko), none(dq), none(dk), dim, qg, kg, gq, gk, EPS, THETA)
    for x, y, dy, dx, gain, dgain in ((q, qo, dqo, dq, qg, gq), (k, ko, dko, dk, kg, gk)):
        if not x.shape[1]:
            assert torch.equal(dgain, torch.zeros_like(dgain))
            continue
        xr = x.double().requires_grad_()
        g = (torch.ones(dim, device="cuda", dtype=torch.float64) if gain is None else gain.double()).requires_grad_()
        want = ref.norm_rope(xr, g, pos, dim, EPS, THETA)
        # fp32 steps (1e-6 of a pair's length, and of the far angles' 2 pi turns) and half a step of bf16
        length = want.view(n, -1, 2, dim // 2).square().sum(2, keepdim=True).sqrt().expand(-1, -1, 2, -1).reshape(n, -1)
        close(y, want.detach(), (ref.HALF * want.abs() + 2e-6 * length).detach())
        want.backward(dy.double())
        size = xr.grad.view(n, -1, dim).square().mean(-1, keepdim=True).sqrt().expand(-1, -1, dim).reshape(n, -1)
        # (what the mean takes out of dx is of the size of dy's rows over x's)
        scale = (dy.double().view(n, -1, dim).norm(dim=-1, keepdim=True) / x.double().view(n, -1, dim).norm(dim=-1, keepdim=True)).expand(-1, -1, dim).reshape(n, -1)
        close(dx, xr.grad, ref.HALF * xr.grad.abs() + 4e-6 * (size + scale))
        unit = (x.double().view(n, -1, dim) / (x.double().view(n, -1, dim).square().mean(-1, keepdim=True) + EPS).sqrt()).abs()
        terms = (dy.double().view(n, -1, dim).abs() + dy.double().view(n, -1, dim).roll(dim // 2, -1).abs()) * unit
        # the gain's gradient: fp32 sums of up to n heads / 16 terms a thread
        close(dgain, g.grad, 1e-5 * terms.sum((0, 1)))


def test_in_place_and_repeatable():
    q, k, dqo, dko, pos, qg, kg = make(5, 300, 6, 2, 128, 1000)
    ctx = binding.Context()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ctx.glue_qk_norm_rope(q, k, pos, qo, ko, 128, qg, kg)
    q2, k2 = q.clone(), k.clone()
    ctx.glue_qk_norm_rope(q2, k2, pos, q2, k2, 128, qg, kg)
    assert torch.equal(qo, q2) and torch.equal(ko, k2)
    outs = []
    for dq, dk in ((torch.empty_like(q), torch.empty_like(k)), (dqo.clone(), dko.clone())):
        gq, gk = torch.empty(128, device="cuda"), torch.empty(128, device="cuda")
        ctx.glue_qk_norm_rope_backward(q, k, pos, dqo if not outs else dq, dko if not outs else dk, dq, dk, 128, qg, kg, gq, gk)
        outs.append((dq, dk, gq, gk))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_no_tokens_and_zero_rows():
    ctx = binding.Context()
    e = torch.empty(0, 128, device="cuda", dtype=torch.bfloat16)
    pos = torch.empty(0, device="cuda", dtype=torch.int32)
    g = torch.full((128,), 3.0, device="cuda")
    ctx.glue_qk_norm_rope(e, e, pos, e, e)
    ctx.glue_qk_norm_rope_backward(e, e, pos, e, e, e, e, dq_gain=g)
    assert torch.equal(g, torch.zeros_like(g))
    # heads of zeros: normalised to zeros, gradients scaled by eps^-1/2
    z, d = torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16), torch.ones(4, 128, device="cuda", dtype=torch.bfloat16)
    pos, y, dz = torch.zeros(4, device="cuda", dtype=torch.int32), torch.empty_like(z), torch.empty_like(z)
    ctx.glue_qk_norm_rope(z, None, pos, y, None)
    ctx.glue_qk_norm_rope_backward(z, None, pos, d, None, dz, None)
    assert torch.equal(y, z) and torch.equal(dz, torch.full_like(dz, 1000.0))


def test_refusals():
    q, k, _, _, pos, qg, kg = make(1, 8, 2, 1, 128, 10)
    ctx = binding.Context()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(q, k, pos, qo, qo[:, :128])                     # k_out inside q_out
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(q, k, pos, qo, q[:, 128:])                      # k_out inside q
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(q, k, pos, qo, ko, eps=-1.0)
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(q, k, pos, qo, ko, rope_theta=1.0)
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(q, k, pos, qo, ko, head_dim=32)
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(q, k, None, qo, ko)
    with pytest.raises(TypeError):
        ctx.glue_qk_norm_rope(q.float(), k, pos, qo, ko)
    with pytest.raises(TypeError):
        ctx.glue_qk_norm_rope(q, k, pos.long(), qo, ko)
    with pytest.raises(ValueError):
        ctx.glue_qk_norm_rope(q, k, pos[:5], qo, ko)
    with pytest.raises(ValueError):
        ctx.glue_qk_norm_rope(q, k, pos, qo[:4], ko)
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope_backward(q, k, pos, qo, ko, qo[:, :], q[:, :128])
    rows = torch.empty(8, 260, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(binding.AgzoError):
        ctx.glue_qk_norm_rope(rows[:, :256], k, pos, qo, ko)                  # rows of no multiple of 16 bytes
