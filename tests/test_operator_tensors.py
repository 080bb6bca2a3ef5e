"""What the binding of the rotation table, the norm and rotation and the masked attention refuses to read (no GPU): tensors of
another type, too small, of another shape, on another device, or whose rows are one row."""
import numpy as np
import pytest
import torch

import paper_2604_04335_amd as da

BF16 = torch.bfloat16


def rows(n=8, heads=2, dim=64, dtype=BF16):
    return torch.zeros((n, heads, dim), dtype=dtype)


def ids(n, dtype=torch.int32):
    return torch.zeros(n, dtype=dtype)


def masked(q=None, k=None, v=None, out=None, lse=None, mask=None, cu_q=(0, 3, 8), cu_k=None, heads=2, kv_heads=2, dim=64, ctx=None, **kw):
    q, k, v, out = (rows() if x is None else x for x in (q, k, v, out))
    da.dit_attn_masked_varlen_fwd(ctx, q, k, v, list(cu_q), cu_k, heads, kv_heads, dim, 0.125, mask, out, lse, **kw)


def norm(x=None, out=None, n=8, dim=64, table=None, rot=8, ctx=None, **kw):
    side = da.NormHeads(rows() if x is None else x, rows() if out is None else out, **kw)
    da.dit_attn_qk_norm_rope(ctx, side, None, n, dim, da.NORM_RMS, 1e-6, torch.zeros(8 * 8) if table is None else table, rot)


def table(positions=None, values=None, n=8, dims=(16, 16), ctx=None):
    da.dit_attn_rope_table(ctx, torch.zeros((8, 2), dtype=torch.int32) if positions is None else positions, n, da.RopeSpec(dims),
                           torch.zeros((8, 16, 2)) if values is None else values)


def passes(call, *args, **kw):
    """The binding lets the call through: without a context the library refuses it."""
    with pytest.raises(da.DitAttnError) as ei:
        call(*args, **kw)
    assert ei.value.code == -1


def refused(call, *args, **kw):
    with pytest.raises(ValueError):
        call(*args, **kw)


def test_what_fits_passes():
    for call in (masked, norm, table):
        passes(call)
    fused = torch.zeros((9, 6 * 64), dtype=BF16)
    view = fused[:, 128:256].unflatten(1, (2, 64))
    passes(masked, q=view, k=view, v=view)
    passes(norm, x=view, out=view)
    passes(masked, q=rows(20), k=rows(20), v=rows(20), out=rows(20), lse=torch.zeros(8, 2))
    passes(masked, q=rows(dtype=torch.int16), k=rows(dtype=torch.int16))  # bit patterns
    passes(norm, x=rows(dtype=torch.int16))
    passes(masked, q=rows().view(8, 128), out=rows().view(-1), k=rows().view(2, 4, 2, 64), v=rows().view(2, 2, 2, 128))
    passes(norm, x=rows().view(8, 128), n_heads=2)
    passes(norm, x=rows().view(-1), out=rows().view(8, 128), n_heads=2)
    passes(norm, weight=torch.zeros(64), bias=torch.zeros(64))
    passes(masked, k=rows(0), v=rows(0), cu_k=[0, 0, 0])
    passes(masked, q=rows(1), out=rows(1), k=rows(1).expand(1, 2, 64), cu_q=[0, 1])
    passes(masked, q=rows(1, 4), k=rows(9, 2), v=rows(9, 2), out=rows(1, 4), cu_q=[0, 1], cu_k=[0, 9], heads=4)
    passes(masked, q=4096, k=4096, v=4096, out=4096, lse=4096)
    passes(masked, q=rows()[:, :1], k=rows()[:, :1], v=rows()[:, :1], heads=1, kv_heads=1, out=rows(8, 1))
    passes(masked, mask=da.AttnMask(causal=True, prefix=[1, 2], slopes=torch.zeros(2), q_doc=ids(8), k_doc=ids(8)))
    passes(masked, q=fused[:, :128], k=fused[:, :128], v=fused[:, :128], row_strides=(384, 384, 384))
    passes(norm, x=fused[:, :128], out=fused[:, :128], n_heads=2, row_stride=384, out_row_stride=384)
    passes(table, n=2 ** 35)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.int32, torch.uint8])
def test_types(dtype):
    for name in ("q", "k", "v", "out"):
        refused(masked, **{name: rows(dtype=dtype)})
    for name in ("q", "k", "v"):
        refused(masked, **{name: rows(dtype=dtype)}, row_strides=(128, 128, 128))
    refused(norm, x=rows(dtype=dtype))
    refused(norm, out=rows(dtype=dtype))
    refused(norm, x=rows(dtype=dtype), row_stride=128)
    if dtype != torch.float32:
        refused(masked, lse=torch.zeros((8, 2), dtype=dtype))
        refused(da.AttnMask, slopes=torch.zeros(2, dtype=dtype))
        refused(norm, weight=torch.zeros(64, dtype=dtype))
        refused(norm, table=torch.zeros(64, dtype=dtype))
        refused(table, values=torch.zeros((8, 16, 2), dtype=dtype))
    if dtype != torch.int32:
        refused(da.AttnMask, q_doc=ids(8, dtype), k_doc=ids(8))
        refused(table, positions=torch.zeros((8, 2), dtype=dtype))


def test_rows_of_an_expanded_tensor_are_one_row():
    """Their stride is 0, which the library takes for contiguous rows."""
    one = rows(1).expand(8, 2, 64)
    for name in ("q", "k", "v", "out"):
        refused(masked, **{name: one})
    refused(norm, x=one)
    refused(norm, out=one)
    head = rows(8, 1).expand(8, 2, 64)
    refused(masked, k=head)
    refused(norm, x=head)


def test_sizes():
    for name in ("q", "k", "v", "out"):
        for x in (rows(7), rows(8, 1), rows(8, 2, 32), rows(8, 4), rows(4, 2, 128), rows(7).view(7, 128), rows(8).view(4, 256)):
            refused(masked, **{name: x})
    refused(masked, k=rows(8), v=rows(9), cu_k=[0, 4, 9])
    refused(masked, k=rows(9), v=rows(8), cu_k=[0, 4, 9])
    refused(masked, k=rows(8, 2), v=rows(8, 1), kv_heads=1)
    refused(masked, lse=torch.zeros((8, 1)))
    refused(masked, lse=torch.zeros((7, 2)))
    refused(masked, mask=da.AttnMask(slopes=torch.zeros(1)))
    refused(masked, mask=da.AttnMask(q_doc=ids(7), k_doc=ids(8)))
    refused(masked, mask=da.AttnMask(q_doc=ids(8), k_doc=ids(7)))
    refused(masked, k=rows(9), v=rows(9), cu_k=[0, 4, 9], mask=da.AttnMask(q_doc=ids(8), k_doc=ids(8)))
    for x in (rows(7), rows(8, 1), rows(8, 4), rows(8, 2, 128)):
        refused(norm, out=x)
    refused(norm, x=rows(7))
    refused(norm, n=9)
    refused(norm, dim=128, rot=0)
    refused(norm, weight=torch.zeros(63))
    refused(norm, weight=torch.zeros(64), bias=torch.zeros(32))
    refused(norm, table=torch.zeros(63))
    refused(norm, table=torch.zeros(8 * 8), rot=16)
    refused(table, n=9)
    refused(table, positions=torch.zeros((8, 1), dtype=torch.int32))
    refused(table, values=torch.zeros((8, 15, 2)))


def test_devices(monkeypatch):
    """A tensor of the host, whose address the GPU cannot read, and one of another device than the context's."""
    def called(*args):
        raise AssertionError("the library was called")

    class Never:
        dit_attn_masked_varlen_fwd = dit_attn_qk_norm_rope = dit_attn_rope_table = staticmethod(called)

    monkeypatch.setattr(da, "load_library", lambda: Never())
    monkeypatch.setitem(da._CTX_DEVICE, 64, 0)
    for call in (masked, norm, table):
        refused(call, ctx=64)
    for tensor in ("q", "k", "v", "out"):
        others = {x: 4096 for x in ("q", "k", "v", "out") if x != tensor}
        refused(masked, ctx=64, **{tensor: rows()}, **others)
    refused(masked, ctx=64, q=4096, k=4096, v=4096, out=4096, lse=torch.zeros((8, 2)))
    for mask in (dict(slopes=torch.zeros(2)), dict(q_doc=ids(8), k_doc=4096), dict(q_doc=4096, k_doc=ids(8))):
        refused(masked, ctx=64, q=4096, k=4096, v=4096, out=4096, mask=da.AttnMask(**mask))
    for kw in (dict(x=rows(), out=4096), dict(x=4096, out=rows()), dict(x=4096, out=4096, weight=torch.zeros(64)),
               dict(x=4096, out=4096, bias=torch.zeros(64)), dict(x=4096, out=4096, table=torch.zeros(64))):
        refused(norm, ctx=64, n_heads=2, **dict(dict(table=4096), **kw))
    refused(table, ctx=64, positions=4096)
    refused(table, ctx=64, values=4096)


def test_contexts_are_known_by_their_device(monkeypatch):
    class Library:
        def dit_attn_create(self, handle, device):
            handle._obj.value = 4096
            return 0

        def dit_attn_destroy(self, handle):
            pass

    monkeypatch.setattr(da, "load_library", lambda: Library())
    assert da.dit_attn_create(3) == 4096 and da._CTX_DEVICE[4096] == 3
    da.dit_attn_destroy(4096)
    assert 4096 not in da._CTX_DEVICE


def test_boundaries_of_other_types_and_strides():
    passes(masked, cu_q=np.array([0, 3, 8], np.int64))
    passes(masked, cu_q=np.array([0, 9, 3, 9, 8, 9], np.int32)[::2])


def test_structures_by_address_and_filled_in_one_by_one():
    import ctypes

    side = da.NormHeads(4096, 4096, n_heads=2)
    for x in (side, ctypes.byref(side), da.NormHeads.from_buffer_copy(bytes(side))):
        passes(da.dit_attn_qk_norm_rope, None, x, None, 8, 64, da.NORM_RMS, 1e-6)
    passes(da.dit_attn_rope_table, None, 4096, 8, ctypes.byref(da.RopeSpec([16])), 4096)
    passes(masked, mask=da.AttnMask.from_buffer_copy(bytes(da.AttnMask(causal=True))))
