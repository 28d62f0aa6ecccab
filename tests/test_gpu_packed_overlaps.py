"""Lists of single values (lse, gains and their gradients, positions, offsets, ids, scalars) that overlap a result, or are misaligned, are refused by the
calls on packed batches before anything is launched."""
import pytest
import torch

from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
BF, F32, I32, F64 = torch.bfloat16, torch.float32, torch.int32, torch.float64


class Arena:
    """Memory of which tensors are views at byte offsets; filled with sevens, so that a launch shows"""

    def __init__(self, size=1 << 16):
        self.bytes = torch.full((size,), 7, device="cuda", dtype=torch.uint8)

    def at(self, off, dtype, *shape):
        n = dtype.itemsize
        for d in shape:
            n *= d
        return self.bytes[off:off + n].view(dtype).view(*shape)

    def untouched(self):
        return bool((self.bytes == 7).all())


def refused(arena, f, *args, **kw):
    with pytest.raises(binding.AgzoError) as e:
        f(*args, **kw)
    assert e.value.code == binding.EINVAL
    torch.cuda.synchronize()
    assert arena is None or arena.untouched()


def misaligned(t):
    """The same address and two bytes"""
    class Off(torch.Tensor):
        def data_ptr(self):
            return super().data_ptr() + 2
    return t.as_subclass(Off)


def test_attention():
    ctx, a = binding.Context(), Arena()
    rnd = lambda *s: torch.randn(*s, device="cuda").to(BF)
    q, k, v, d = rnd(8, 256), rnd(8, 128), rnd(8, 128), rnd(8, 256)
    cu = torch.tensor([0, 3, 8], device="cuda", dtype=I32)
    out, lse = a.at(0, BF, 8, 256), a.at(8192, F32, 8, 4)
    f = lambda **kw: refused(a, ctx.glue_attention_packed, q, k, v, out, cu, cu, 64, **kw)
    f(lse=a.at(4092, F32, 8, 4))                                  # over out's end
    f(lse=a.at(0, F32, 8, 4))
    f(lse=misaligned(lse))
    refused(a, ctx.glue_attention_packed, q, k, v, out, a.at(4096 - 12, I32, 3), cu, 64)
    refused(a, ctx.glue_attention_packed, q, k, v, out, cu, a.at(0, I32, 3), 64)
    f(k_len=a.at(2048, I32, 2))
    refused(None, ctx.glue_attention_packed, q, k, v, out, cu, cu, 64, lse=q.view(-1).view(F32)[:32].view(8, 4))
    dq, dk, dv, g = a.at(0, BF, 8, 256), a.at(4096, BF, 8, 128), a.at(6144, BF, 8, 128), torch.zeros(8, 4, device="cuda")
    o = torch.zeros_like(q)
    b = lambda lse, cq, ck: refused(a, ctx.glue_attention_packed_backward, q, k, v, o, lse, d, dq, dk, dv, cq, ck, 64)
    b(a.at(4096, F32, 8, 4), cu, cu)
    b(g, a.at(6144 + 2048 - 12, I32, 3), cu)
    b(g, cu, a.at(100, I32, 3))


def test_norms_with_rotation():
    ctx, a = binding.Context(), Arena()
    q, k = torch.randn(6, 128, device="cuda").to(BF), torch.randn(6, 64, device="cuda").to(BF)
    pos = torch.zeros(6, device="cuda", dtype=I32)
    gain = lambda off: a.at(off, F32, 64)
    qo, ko = a.at(0, BF, 6, 128), a.at(1536, BF, 6, 64)
    free = gain(4096)
    for kw in (dict(q_gain=gain(1532)), dict(k_gain=gain(1536)), dict(q_gain=misaligned(free)), dict(k_gain=misaligned(free))):
        refused(a, ctx.glue_qk_norm_rope, q, k, pos, qo, ko, 64, **kw)
    refused(a, ctx.glue_qk_norm_rope, q, k, a.at(512, I32, 6), qo, ko, 64)
    g = torch.ones(64, device="cuda")
    b = lambda **kw: refused(a, ctx.glue_qk_norm_rope_backward, q, k, pos, q.clone(), k.clone(), qo, ko, 64, **kw)
    b(dq_gain=free, dk_gain=free)
    b(dq_gain=free, dk_gain=gain(4096 + 252))                      # in part
    b(dq_gain=gain(1400))                                          # in dq and dk
    b(dk_gain=gain(1280))
    b(q_gain=gain(0))
    b(k_gain=g, dq_gain=g)                                         # (its own gain it may be, the other not)
    b(dq_gain=misaligned(free))
    b(dk_gain=misaligned(free))
    refused(a, ctx.glue_qk_norm_rope_backward, q, k, a.at(1536, I32, 6), q.clone(), k.clone(), qo, ko, 64)
    refused(None, ctx.glue_qk_norm_rope_backward, q, k, pos, q.clone(), k.clone(), qo, ko, 64, dq_gain=q.view(-1).view(F32)[:64])


def test_gradients_in_place_of_their_gains():
    ctx = binding.Context()
    q, k, dq, dk = (torch.randn(300, w, device="cuda").to(BF) for w in (256, 128, 256, 128))
    pos = torch.arange(300, device="cuda", dtype=I32)
    gains = [torch.rand(64, device="cuda") + 0.5 for _ in range(2)]
    want, own = [torch.empty(64, device="cuda") for _ in range(2)], [g.clone() for g in gains]
    a = [torch.empty_like(q), torch.empty_like(k)]
    b = [torch.empty_like(q), torch.empty_like(k)]
    ctx.glue_qk_norm_rope_backward(q, k, pos, dq, dk, *a, 64, *gains, *want)
    ctx.glue_qk_norm_rope_backward(q, k, pos, dq, dk, *b, 64, *own, *own)
    assert all(torch.equal(x, y) for x, y in zip(a + want, b + own))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_cross_entropy(dtype):
    ctx, a = binding.Context(), Arena()
    n, d, v = 16, 32, 24
    w, x = torch.randn(v, d, device="cuda").to(dtype), torch.randn(n, d, device="cuda").to(dtype)
    ids = torch.zeros(n, device="cuda", dtype=I32)
    layer, loss = binding.make_layer(w, x), binding.make_loss(ids, binding.LOSS_CE)
    out, lse = a.at(0, F64, 1), a.at(64, F32, n)
    refused(a, ctx.ce_forward, layer, w, x, loss, out, a.at(4, F32, n))                  # lse over the loss
    refused(a, ctx.ce_forward, layer, w, x, binding.make_loss(a.at(120, I32, n), binding.LOSS_CE), out, lse)
    refused(a, ctx.ce_forward, layer, w, x, binding.make_loss(a.at(4, I32, n), binding.LOSS_CE), out, None)
    refused(a, ctx.ce_forward, layer, w, x, loss, misaligned(out), lse)
    refused(None, ctx.ce_forward, layer, w, x, loss, x.view(-1).view(F64)[:1], lse)
    refused(None, ctx.ce_forward, layer, w, x, loss, out, w.view(-1).view(F32)[:n])
    dx, dw = a.at(0, dtype, n, d), a.at(n * d * dtype.itemsize, dtype, v, d)
    end = (n + v) * d * dtype.itemsize
    l = torch.zeros(n, device="cuda")
    refused(a, ctx.ce_backward, layer, w, x, loss, a.at(end - 4, F32, n), dx, dw)
    refused(a, ctx.ce_backward, layer, w, x, binding.make_loss(a.at(64, I32, n), binding.LOSS_CE), l, dx, dw)
    refused(a, ctx.ce_backward, layer, w, x, loss, l, dx, dw, a.at(end - 8, F64, 1))
    refused(a, ctx.ce_backward, layer, w, x, loss, l, dx, dw, misaligned(a.at(end + 64, F64, 1)))
