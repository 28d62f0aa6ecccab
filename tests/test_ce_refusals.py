"""CPU-only: what the binding of the head's cross-entropy refuses before the library, which sees bare pointers, is called."""
import gc
import weakref

import pytest
import torch

from paper_2601_17261_amd import binding

N, D, V = 6, 16, 40


class Library:
    """Takes the calls in the library's place"""

    def __init__(self):
        self.calls = 0

    def agzo_ce_forward(self, *args):
        self.calls += 1
        return 0

    agzo_ce_backward = agzo_ce_forward


@pytest.fixture
def ctx():
    c = object.__new__(binding.Context)
    c.lib, c.h, c.device = Library(), None, -1          # (what get_device() says of host tensors)
    return c


def tensors(dtype=torch.bfloat16):
    return torch.zeros(V, D, dtype=dtype), torch.zeros(N, D, dtype=dtype), torch.zeros(N, dtype=torch.int32)


def call(ctx, w, x, loss, layer=None):
    layer = layer or binding.make_layer(w, x)
    lse = torch.zeros(layer.n_tokens)
    ctx.ce_forward(layer, w, x, loss, torch.zeros(1, dtype=torch.float64), lse)
    ctx.ce_backward(layer, w, x, loss, lse, torch.empty_like(x), torch.empty_like(w))


def refused(ctx, error, *args, **kw):
    with pytest.raises(error):
        call(ctx, *args, **kw)
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_fits_is_called(ctx, dtype):
    w, x, ids = tensors(dtype)
    call(ctx, w, x, binding.make_loss(ids, binding.LOSS_CE))
    # wide rows; a single row, whose stride says nothing
    wide = torch.zeros(V, D + 8, dtype=dtype)[:, :D]
    call(ctx, wide, x, binding.make_loss(ids, binding.LOSS_CE))
    call(ctx, w, torch.zeros(N, D, dtype=dtype)[::3][:1], binding.make_loss(ids[:1], binding.LOSS_CE))
    assert ctx.lib.calls == 6
    # (no tokens: an error of the library's)
    call(ctx, w, x[:0], binding.make_loss(ids[:0], binding.LOSS_CE))


def test_ids_of_another_length_or_stride(ctx):
    w, x, ids = tensors()
    for bad in (ids[:5], ids[:0], torch.zeros(2 * N, dtype=torch.int32)[::2], torch.zeros(N + 1, dtype=torch.int32)):
        refused(ctx, ValueError, w, x, binding.make_loss(bad, binding.LOSS_CE))


def test_tensors_of_another_device(ctx):
    w, x, ids = tensors()
    ctx.device = 0
    refused(ctx, ValueError, w, x, binding.make_loss(ids, binding.LOSS_CE))


def test_ids_that_nobody_vouches_for(ctx):
    w, x, ids = tensors()
    s = binding.AgzoLossSpec()
    s.kind, s.target = binding.LOSS_CE, ids.data_ptr()
    refused(ctx, ValueError, w, x, s)
    s = binding.make_loss(ids, binding.LOSS_CE)
    s.target = ids.data_ptr() + 4
    refused(ctx, ValueError, w, x, s)


def test_ids_live_as_long_as_the_loss():
    ids = torch.zeros(N, dtype=torch.int32)
    gone = weakref.ref(ids)
    s = binding.make_loss(ids, binding.LOSS_CE)
    del ids
    gc.collect()
    assert gone() is not None
    del s
    gc.collect()
    assert gone() is None


def test_weights_and_inputs_are_the_layers(ctx):
    w, x, ids = tensors()
    loss, layer = binding.make_loss(ids, binding.LOSS_CE), binding.make_layer(w, x)
    wide = torch.zeros(V, 2 * D, dtype=torch.bfloat16)
    for w2, x2, error in ((w[:-1], x, ValueError), (w, x[:-1], ValueError), (wide[:, :D], x, ValueError), (wide, x, ValueError), (w, wide[:N, :D], ValueError),
                          (w.t(), x, ValueError), (wide[:, ::2], x, ValueError), (w.float(), x, TypeError), (w, x.float(), TypeError), (w.view(torch.int16), x, TypeError)):
        refused(ctx, error, w2, x2, loss, layer=layer)
    # the type of a layer is its inputs'
    refused(ctx, TypeError, w, x.float(), loss)
    refused(ctx, TypeError, w.float(), x, loss)
