"""A context that ends while another one's stream is captured: Python lets go of contexts at times of its own (those in a cycle, of an exception's traceback for
one, whenever its collector runs), and the capture goes on."""
import gc

import pytest
import torch

from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu


class Holder:
    """holds a context in a cycle"""

    def __init__(self, ctx):
        self.ctx, self.me = ctx, self


@pytest.mark.parametrize("of", ["default", "other"])
@pytest.mark.parametrize("how", ["close", "collect"])
def test_a_context_ends_while_another_stream_is_captured(of, how):
    x, y = torch.randn(5, 128, device="cuda").bfloat16(), torch.empty(5, 128, device="cuda", dtype=torch.bfloat16)
    own = torch.cuda.Stream() if of == "other" else None
    old, side = binding.Context(own), torch.cuda.Stream()
    ctx = binding.Context(side)
    cu = torch.tensor([0, 2, 5], device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    dq, dk, dv, lse = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(5, 2, device="cuda")
    for c in (old, ctx):                                 # (both have a workspace)
        c.glue_attention_packed(x, x, x, y, cu, cu, 64, lse=lse)
        c.glue_attention_packed_backward(x, x, x, y, lse, x, dq, dk, dv, cu, cu, 64)
    torch.cuda.synchronize()
    want = y.clone()
    held = Holder(old) if how == "collect" else old
    del old
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        if how == "collect":
            del held
            gc.collect()
        else:
            held.close()
        ctx.glue_attention_packed(x, x, x, y, cu, cu, 64)
    for _ in range(3):
        y.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
