"""What the head's cross-entropy refuses of tensors on the device, before anything is launched; a loss of ids that nothing else holds."""
import gc

import pytest
import torch

from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu


def make(n=32, d=64, v=100, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(n)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(dtype)
    return rnd(v, d) / 8, rnd(n, d), torch.randint(0, v, (n,), device="cuda", generator=gen).int()


def test_tensors_that_are_not_the_layers():
    ctx = binding.Context()
    w, x, ids = make()
    out, lse = torch.full((1,), 7.0, dtype=torch.float64, device="cuda"), torch.full((32,), 7.0, device="cuda")
    dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    layer, loss = binding.make_layer(w, x), binding.make_loss(ids, binding.LOSS_CE)
    wide = torch.cat((ids, ids))
    for bad in (ids.cpu(), ids[:31], wide[::2], wide):
        spec = binding.make_loss(bad, binding.LOSS_CE)
        with pytest.raises(ValueError):
            ctx.ce_forward(layer, w, x, spec, out, lse)
        with pytest.raises(ValueError):
            ctx.ce_backward(layer, w, x, spec, lse, dx, dw)
    for w2, x2, error in ((w[:99], x, ValueError), (w, x[:31], ValueError), (w.cpu(), x, ValueError), (w, x.cpu(), ValueError), (w.float(), x, TypeError), (w, x.float(), TypeError)):
        with pytest.raises(error):
            ctx.ce_forward(layer, w2, x2, loss, out, lse)
        with pytest.raises(error):
            ctx.ce_backward(layer, w2, x2, loss, lse, dx, dw)
    # fp32 inputs beside bf16 weights
    with pytest.raises(TypeError):
        ctx.ce_forward(binding.make_layer(w, x.float()), w, x.float(), loss, out, lse)
    for t in (out, lse, dx, dw):
        assert (t == 7.0).all()


def test_ids_that_only_the_loss_holds():
    ctx = binding.Context()
    w, x, ids = make()
    out, want = (torch.zeros(1, dtype=torch.float64, device="cuda") for _ in range(2))
    ctx.ce_forward(binding.make_layer(w, x), w, x, binding.make_loss(ids, binding.LOSS_CE), want)
    loss = binding.make_loss(ids.clone(), binding.LOSS_CE)
    gc.collect()
    over = [torch.full_like(ids, -1) for _ in range(64)]          # (would take the ids' memory, were it free)
    ctx.ce_forward(binding.make_layer(w, x), w, x, loss, out)
    assert torch.equal(out, want) and len(over) == 64
