"""Sizes at which a launch would pass 2^32 threads, of which the hardware takes the low 32 bits alone."""
import pytest
import torch

from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def test_norms_with_rotation_of_2_26_tokens():
    """(8.6 GB, in place) every token's result is that of a smaller call"""
    ctx = binding.Context()
    some, n = 1 << 20, (1 << 26) + 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(some, 64, device="cuda", generator=gen).to(BF)
    pos, want = torch.arange(some, device="cuda", dtype=I32), torch.empty_like(x)
    ctx.glue_qk_norm_rope(None, x, pos, None, want, 64)
    k = torch.empty(n, 64, device="cuda", dtype=BF)
    parts = [(i, min(i + some, n)) for i in range(0, n, some)]
    for a, b in parts:
        k[a:b] = x[:b - a]
    ctx.glue_qk_norm_rope(None, k, pos.repeat(65)[:n].contiguous(), None, k, 64)
    assert all(torch.equal(k[a:b], want[:b - a]) for a, b in parts)


def test_gradient_of_inputs_of_more_than_2_32_values():
    """(69 GB) an fp32 layer in two pieces of its outputs.  Few rows are counted; the others' gradients are zeros"""
    ctx = binding.Context()
    n, d, v = 1 << 21, 2049, 300
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, dx = torch.zeros(n, d, device="cuda"), torch.empty(n, d, device="cuda")
    w = torch.randn(v, d, device="cuda", generator=gen) / d ** 0.5
    ids, lse = torch.full((n,), -1, device="cuda", dtype=I32), torch.zeros(n, device="cuda")
    rows = torch.tensor([0, 1, 70000, n // 2, n - 1030, n - 2, n - 1], device="cuda")
    x[rows] = torch.randn(len(rows), d, device="cuda", generator=gen)
    ids[rows] = torch.arange(len(rows), device="cuda", dtype=I32) * 49
    y = x[rows].double() @ w.double().T
    lse[rows] = y.logsumexp(1).float()
    for part in (dx[:4096], dx[n // 2:n // 2 + 4096], dx[-4096:]):
        part.fill_(7.0)
    ctx.ce_backward(binding.make_layer(w, x), w, x, binding.make_loss(ids, binding.LOSS_CE), lse, dx, None)
    p = (y - y.logsumexp(1, keepdim=True)).exp()
    D = p.clone()
    D[torch.arange(len(rows)), ids[rows].long()] -= 1.0
    want = D @ w.double() / len(rows)
    # steps of 2^-24: a logit's, lse's, their difference's and the exponential's to D, and six of the sums and the result
    off = 2.0 ** -24 * ((p * (2 * y.abs() + 2 * y.logsumexp(1, keepdim=True).abs() + 8) + 8 * D.abs()) @ w.double().abs()) / len(rows)
    assert ((dx[rows].double() - want).abs() <= off).all()
    other = torch.ones(n, device="cuda", dtype=torch.bool)
    other[rows] = False
    for a in (0, n // 2, n - 4096):
        assert not dx[a:a + 4096][other[a:a + 4096]].any()
    del x, dx, ctx
    torch.cuda.empty_cache()


def test_more_tiles_than_a_launch_takes_are_refused():
    """65536 sequences of one token with 256 heads: (65536 + 512) 256 workgroups, 2^32 threads and more"""
    ctx = binding.Context()
    n, width = 65536, 256 * 64
    q, k, v, out = (torch.empty(n, width, device="cuda", dtype=BF) for _ in range(4))
    cu = torch.arange(n + 1, device="cuda", dtype=I32)
    out[::1024] = 7.0
    with pytest.raises(binding.AgzoError) as e:
        ctx.glue_attention_packed(q, k, v, out, cu, cu, 64)
    assert e.value.code == binding.EINVAL
    lse = torch.zeros(n, 256, device="cuda")
    with pytest.raises(binding.AgzoError) as e:
        ctx.glue_attention_packed_backward(q, k, v, q, lse, k, out, torch.empty_like(k), torch.empty_like(v), cu, cu, 64)
    assert e.value.code == binding.EINVAL and (out[::1024] == 7.0).all()


def test_an_fp32_loss_of_2_24_tokens_is_refused():
    ctx = binding.Context()
    n = 1 << 24
    w, x, ids = torch.ones(1, 1, device="cuda"), torch.ones(n, 1, device="cuda"), torch.zeros(n, device="cuda", dtype=I32)
    out = torch.full((1,), 7.0, device="cuda", dtype=torch.float64)
    with pytest.raises(binding.AgzoError) as e:
        ctx.ce_forward(binding.make_layer(w, x), w, x, binding.make_loss(ids, binding.LOSS_CE), out)
    assert e.value.code == binding.EINVAL and float(out) == 7.0
    ctx.ce_forward(binding.make_layer(w, x[1:]), w, x[1:], binding.make_loss(ids[1:], binding.LOSS_CE), out)
    assert float(out) == 0.0
