"""The binding's checks of what a caller gives the 8-bit cache calls beside tensors (host only: each fails before the library
is called, and before the tensors' device is looked at)."""
import pytest
import torch

from paper_2602_04361_amd import sparvar as sv


def planes(n=64, H=2, d=64):
    return torch.zeros(1, H, n, d, dtype=torch.bfloat16)


def refused(what, fn, *args, **kw):
    with pytest.raises(sv.SparvarError, match=what):
        fn(*args, **kw)


@pytest.mark.parametrize("extra", [1 << 32, -(1 << 32), 1 << 31, 3 << 40])
def test_numbers_past_32_bits(extra):
    """A position or length that ctypes would cut to its low 32 bits, which are in range here."""
    k, c, x = planes(), sv.Q8Cache.empty(1, 2, 64, 64, 32, device="cpu"), torch.zeros(1, 64, 2, 64, dtype=torch.bfloat16)
    g, i = sv.Geometry([8], [8], 4, 0), torch.zeros(9, dtype=torch.int32)
    refused("32 bits", sv.sparvar_qkv_append, x, x, x, extra, None, torch.empty_like(k), q8=c)
    refused("32 bits", sv.sparvar_kv_quantize, k, k, extra, c)
    refused("32 bits", sv.sparvar_kv_dequantize, c, extra, k, k)
    refused("32 bits", sv.sparvar_dense_attn_q8_fwd, k, c, 64 + extra, torch.empty_like(k))
    refused("32 bits", sv.sparvar_block_sparse_attn_q8_fwd, g, 1 + extra, k, c, torch.empty_like(k), i, i)
    refused("32 bits", sv.sparvar_dense_attn_q8_workspace, 1, 2, 2, 1, 64 + extra, 64)
    refused("32 bits", sv.sparvar_dense_attn_q8_form, 1, 2, 2, 64 + extra, 64, 64, True)
    refused("32 bits", sv.sparvar_block_sparse_attn_q8_form, g, 1, 1 + extra, 2, 2, 64)


def test_rows_of_a_block_sparse_call():
    """row_ptr of too few rows, strided arrays, a short launch order: the kernel would read past them."""
    k, c = planes(), sv.Q8Cache.empty(1, 2, 64, 64, 32, device="cpu")
    g, o = sv.Geometry([8], [8], 4, 0), torch.empty_like(planes())  # 2 planes of 4 tiles
    ptr, ids, order = (torch.zeros(n, dtype=torch.int32) for n in (9, 20, 8))
    call = sv.sparvar_block_sparse_attn_q8_fwd
    refused("row_ptr", call, g, 1, k, c, o, ptr[:8], ids)
    refused("row_ptr", call, g, 1, k, c, o, torch.zeros(18, dtype=torch.int32)[::2], ids)
    refused("contiguous", call, g, 1, k, c, o, ptr, torch.zeros(40, dtype=torch.int32)[::2])
    refused("schedule", call, g, 1, k, c, o, ptr, ids, schedule=order[:7])
    refused("schedule", call, g, 1, k, c, o, ptr, ids, schedule=torch.zeros(16, dtype=torch.int32)[::2])
    refused("int32", call, g, 1, k, c, o, ptr.long(), ids)
    refused("scale 2", call, g, 2, k, c, o, ptr, ids)
    refused("not on a GPU", call, g, 1, k, c, o, ptr, ids, schedule=order)  # these are right


@pytest.mark.parametrize("bad", [dict(block=0), dict(block=-16), dict(block=48), dict(capacity=0), dict(capacity=-5),
                                 dict(B=0), dict(H_kv=0)])
def test_empty_cache_of_bad_sizes(bad):
    """An error of the framework's own, before anything is allocated."""
    refused("scale block|is empty", sv.Q8Cache.empty, **{**dict(B=1, H_kv=2, capacity=64, d=64, block=32, device="cpu"), **bad})
