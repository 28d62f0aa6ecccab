"""CPU-only checks of the calls on packed batches and of the head's gradient: what is refused before any device is asked."""
import ctypes

import pytest
import torch

from paper_2601_17261_amd import binding


def test_no_context_is_an_error():
    lib = binding.load()
    a, layer, loss = binding.AgzoPackedAttention(), binding.AgzoLayer(), binding.AgzoLossSpec()
    null = None
    assert lib.agzo_glue_attention_packed(null, ctypes.byref(a), null, 0, null) == binding.EINVAL
    assert lib.agzo_glue_attention_packed_backward(null, ctypes.byref(a), null, 0, null, null, 0, null, 0, null, 0, null, 0) == binding.EINVAL
    assert lib.agzo_glue_qk_norm_rope(null, null, 0, null, 0, null, null, 0, null, 0, 0, 0, 0, 128, null, null, 1e-6, 1e6) == binding.EINVAL
    assert lib.agzo_glue_qk_norm_rope_backward(null, null, 0, null, 0, null, null, 0, null, 0, null, 0, null, 0, 0, 0, 0, 128, null, null, null, null, 1e-6, 1e6) == binding.EINVAL
    assert lib.agzo_ce_forward(null, ctypes.byref(layer), null, null, ctypes.byref(loss), null, null) == binding.EINVAL
    assert lib.agzo_ce_backward(null, ctypes.byref(layer), null, null, ctypes.byref(loss), null, null, null, 0, null, 0) == binding.EINVAL


def test_layout_of_the_descriptor():
    # three pointers, three leading dimensions, three lists, two counts; five int32 and a float
    assert ctypes.sizeof(binding.AgzoPackedAttention) == 11 * 8 + 6 * 4
    assert binding.AgzoPackedAttention.k_len.offset == 8 * 8 and binding.AgzoPackedAttention.n_seq.offset == 11 * 8


@pytest.mark.parametrize("t,error", [(torch.zeros(4, 64), TypeError), (torch.zeros(4, 64, dtype=torch.float16), TypeError),
                                     (torch.zeros(4, 64, 2, dtype=torch.bfloat16), ValueError), (torch.zeros(64, 4, dtype=torch.bfloat16).t(), ValueError)])
def test_rows_are_bf16_and_of_one_stride(t, error):
    with pytest.raises(error):
        binding._rows(t, "t")


def test_lists_are_contiguous_and_of_their_length():
    x = torch.zeros(8, dtype=torch.int32)
    assert binding._flat(None, "x", torch.int32, 8) is None
    for t, n, error in ((x, 7, ValueError), (x[::2], 4, ValueError), (x.long(), 8, TypeError)):
        with pytest.raises(error):
            binding._flat(t, "x", torch.int32, n)
