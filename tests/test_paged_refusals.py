"""CPU-only checks of the calls on a cache in pages and of verify_drafts: what is refused before any device is asked."""
import ctypes

import pytest
import torch

from paper_2601_17261_amd import binding


def test_no_context_is_an_error():
    lib, null = binding.load(), None
    r, c = ctypes.byref(binding.AgzoRope()), ctypes.byref(binding.AgzoPagedCache())
    for call in (lib.agzo_glue_rope, lib.agzo_glue_rope_backward):
        assert call(null, r, 1, null, 0, null, 0, null, null, 0, null, 0, 0, 0, 0, 64) == binding.EINVAL
    assert lib.agzo_glue_cache_append(null, c, r, null, 0, null, 0, null, 0, null, 0, 0, null, null, 0, 0, null, null, 0.0) == binding.EINVAL
    assert lib.agzo_glue_attention_paged(null, c, null, 0, null, 0, 1, 1.0, null, 0, 0, null, 0, null) == binding.EINVAL
    assert lib.agzo_glue_cache_keep(null, c, null, 0, null, null) == binding.EINVAL
    assert lib.agzo_verify_drafts(null, 0, null, 0, null, 0, null, null, null, null, 0, 0, 1, null, null, null) == binding.EINVAL


def test_layouts_of_the_descriptors():
    # two pointers, six strides, a count, a list with its leading dimension, a list; five int32
    assert binding.AgzoPagedCache.page_size.offset == 12 * 8 and ctypes.sizeof(binding.AgzoPagedCache) == 12 * 8 + 6 * 4
    assert ctypes.sizeof(binding.AgzoRope) == 9 * 4 and binding.AgzoRope.magnitude.offset == 8 * 4


def test_a_cache_is_described():
    k, v = (torch.zeros(5, 16, 2, 64, dtype=torch.bfloat16) for _ in range(2))
    table, k_len = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = binding.make_cache(k, v.transpose(1, 2).contiguous().transpose(1, 2), table, k_len)
    assert (c.k_page, c.k_row, c.k_head, c.v_page, c.v_row, c.v_head) == (2048, 128, 64, 2048, 64, 1024)
    assert (c.n_pages, c.page_size, c.max_pages, c.n_seq, c.n_kv_heads, c.head_dim, c.ld_table) == (5, 16, 4, 3, 2, 64, 4)
    assert binding.make_cache(k, v, torch.zeros(3, 9, dtype=torch.int32)[:, :4], k_len).ld_table == 9
    for args, error in (((k.float(), v, table, k_len), TypeError), ((k, v[:4], table, k_len), ValueError), ((k, v, table.long(), k_len), TypeError), ((k, v, table, k_len[:2]), ValueError),
                        ((k, v, table[0], k_len), ValueError), ((k[0], v[0], table, k_len), ValueError)):
        with pytest.raises(error):
            binding.make_cache(*args)
