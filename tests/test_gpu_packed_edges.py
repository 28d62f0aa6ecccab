"""Packed attention at the ends of its ranges: the smallest scales."""
import pytest
import torch

import packed_reference as ref
from paper_2601_17261_amd import binding
from test_gpu_packed_attention import make, run

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
