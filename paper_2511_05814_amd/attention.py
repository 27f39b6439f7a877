"""The attention half of a layer on torch tensors: 4-bit products, the 4-bit
paged cache, attention over it and the norms around a block.

Each function checks its tensors, allocates what it returns (unless it is given
`out`) and enqueues one call of the C ABI (include/moe_offload.h, which has the
formulas and layouts) on torch's current stream of the tensors' device, so
`with torch.cuda.stream(moe.compute)` puts it in line with an `OffloadedMoE`.
Nothing synchronises.  Tensors are fp32 or bf16 as a whole call; a tensor used
on another stream than its own has to be made known to torch's allocator
(`record_stream`) as with any torch operator.  ValueError: tensors that do not
fit together; binding.MoeError: what the library refuses (alignment, limits).

A cache's pool is uint8 [pages][kv heads][page_size * head_dim * 9 / 8]
(`kv4_pool`).  A batch of B sequences is three int32 tensors on the device:
`q_start` [B + 1], bounds of the sequences' new tokens in this call's rows;
`kv_len` [B], tokens of each sequence with the new ones; `page_table` [B, n],
its pages in order, -1 where there is none.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice

from . import binding as b

GROUP = 64          # columns of a 4-bit matrix that share a scale
KV_GROUP = 32       # dimensions of a cache entry that share one
_DTYPES = {torch.float32: b.MOE_DTYPE_F32, torch.bfloat16: b.MOE_DTYPE_BF16}


# The checks below are written out for speed: a call's launch takes some 3 us,
# and decode calls are this short.

def _place(t: torch.Tensor, dtype):
    """(device, stream, MOE_DTYPE_* of dtype) of a call on t: its device, which
    must be the current one, and torch's current stream there."""
    device = t.get_device()
    if device < 0 or device != _cuda_getDevice():
        raise ValueError(f"tensors must be on the current GPU, not on {t.device}")
    if dtype not in _DTYPES:
        raise ValueError(f"tensors must be float32 or bfloat16, not {dtype}")
    return device, _cuda_getCurrentRawStream(device), _DTYPES[dtype]


def _bad(name, t, device, dtype, shape):
    raise ValueError(f"{name} must be {dtype} {tuple(shape)} with contiguous rows on device {device}, "
                     f"not {t.dtype} {tuple(t.shape)} of strides {t.stride()} on device {t.get_device()}")


def _rows2(name: str, t: torch.Tensor, device: int, dtype, shape) -> int:
    """Elements between the rows of t, which must be of this device, type and
    shape [rows, columns], each row contiguous."""
    outer, inner = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or (inner != 1 and shape[1] > 1):
        _bad(name, t, device, dtype, shape)
    return outer if shape[0] > 1 else shape[1]


def _rows3(name: str, t: torch.Tensor, device: int, dtype, shape) -> int:
    """The same of shape [tokens, heads, head_dim], a token's heads side by side."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _bad(name, t, device, dtype, shape)
    outer, mid, inner = t.stride()
    if inner != 1 or (mid != shape[2] and shape[1] > 1):
        _bad(name, t, device, dtype, shape)
    return outer if shape[0] > 1 else shape[1] * shape[2]


def _vector(name: str, t: torch.Tensor, device: int, dtype, n: int) -> int:
    """Address of a contiguous vector of n elements."""
    if t.dtype is not dtype or t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
        _bad(name, t, device, dtype, (n,))
    return t.data_ptr()


def q4_matmul(x: torch.Tensor, w: torch.Tensor, n: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows, k] times the 4-bit matrix [n x k] in the bytes w, transposed: [rows, n]."""
    if x.dim() != 2:
        raise ValueError("x must be [rows, k]")
    shape = x.shape
    rows, k = shape
    device, stream, code = _place(x, x.dtype)
    if k % GROUP or k == 0 or n < 1:
        raise ValueError(f"a 4-bit matrix [{n} x {k}]: columns must be a multiple of {GROUP}")
    weights = _vector("w", w, device, torch.uint8, n * k // 2 + n * (k // GROUP) * 3)
    if out is None:
        out, out_stride = x.new_empty((rows, n)), n
    else:
        out_stride = _rows2("out", out, device, x.dtype, (rows, n))
    b.moe_q4_matmul(x.data_ptr(), _rows2("x", x, device, x.dtype, shape), weights, out.data_ptr(), out_stride, rows, n, k,
                    code, stream)
    return out


def kv4_record_bytes(page_size: int, head_dim: int) -> int:
    """Bytes that a page of page_size tokens takes for one kv head."""
    return page_size * head_dim * 9 // 8


def kv4_pool(pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda") -> torch.Tensor:
    """A cache's pages, all entries zero."""
    return torch.zeros((pages, kv_heads, kv4_record_bytes(page_size, head_dim)), dtype=torch.uint8, device=device)


def _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim) -> b.moe_kv4_batch:
    if pool.dim() != 3 or pool.dtype != torch.uint8 or not pool.is_contiguous() or pool.get_device() != device:
        raise ValueError("pool must be a contiguous uint8 [pages, kv heads, record] on the call's device")
    pages, kv_heads, record = pool.shape
    page_size = record * 8 // (9 * head_dim)
    if page_size * head_dim * 9 != record * 8:
        raise ValueError(f"records of {record} bytes are not whole tokens of {head_dim} dimensions")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [sequences, columns]")
    seqs, cols = page_table.shape
    stride = _rows2("page_table", page_table, device, torch.int32, (seqs, cols))
    return b.moe_kv4_batch(pool.data_ptr(), page_table.data_ptr(), _vector("q_start", q_start, device, torch.int32, seqs + 1),
                           _vector("kv_len", kv_len, device, torch.int32, seqs), stride, pages, page_size, kv_heads, head_dim,
                           cols, seqs, tokens)


def kv4_append(q, k, v, cos, sin, pool, page_table, q_start, kv_len, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotate the new tokens' q [tokens, heads, head_dim] and k by their
    positions, store k and v [tokens, kv_heads, head_dim] in the cache and
    return the rotated q.  cos and sin: fp32 [positions, rot_dim / 2]; with
    rot_dim 0 nothing is rotated.  Rows may be slices of a joined projection."""
    if q.dim() != 3 or cos.dim() != 2:
        raise ValueError("q must be [tokens, heads, head_dim], cos and sin [positions, rot_dim / 2]")
    dtype, shape = q.dtype, q.shape
    tokens, heads, head_dim = shape
    device, stream, code = _place(q, dtype)
    batch = _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim)
    kv_shape = (tokens, batch.kv_heads, head_dim)
    positions, half = cos.shape
    _rows2("cos", cos, device, torch.float32, (positions, half))
    _rows2("sin", sin, device, torch.float32, (positions, half))
    if not cos.is_contiguous() or not sin.is_contiguous():
        raise ValueError("cos and sin must be contiguous")
    if out is None:
        out, out_stride = q.new_empty(shape), heads * head_dim
    else:
        out_stride = _rows3("out", out, device, dtype, shape)
    b.moe_kv4_append(batch, q.data_ptr(), _rows3("q", q, device, dtype, shape), k.data_ptr(),
                     _rows3("k", k, device, dtype, kv_shape), v.data_ptr(), _rows3("v", v, device, dtype, kv_shape),
                     cos.data_ptr(), sin.data_ptr(), positions, 2 * half, out.data_ptr(), out_stride, heads, code, stream)
    return out


def kv4_read(pool, page_table, q_start, kv_len, tokens: int, head_dim: int, dtype=torch.float32):
    """The stored keys and values of the batch's new tokens, [tokens, kv_heads,
    head_dim] each (exact in both types).  With q_start the running sums of
    kv_len that is everything the sequences have."""
    device, stream, code = _place(pool, dtype)
    batch = _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim)
    k, v = (pool.new_empty((tokens, batch.kv_heads, head_dim), dtype=dtype) for _ in range(2))
    b.moe_kv4_read(batch, k.data_ptr(), v.data_ptr(), code, stream)
    return k, v


def kv4_attention(q, pool, page_table, q_start, kv_len, scale: float, max_new: Optional[int] = None,
                  max_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the new tokens' q [tokens, heads, head_dim] over their
    sequences' caches, causal; rows that see nothing are zeros.  max_new and
    max_len (the longest run of new tokens, the longest sequence) say how to cut
    the work; without them they are taken from the tensors' shapes.  A workspace
    is allocated unless one is given."""
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, head_dim]")
    dtype, shape = q.dtype, q.shape
    tokens, heads, head_dim = shape
    device, stream, code = _place(q, dtype)
    batch = _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim)
    if max_new is None:
        max_new = max(1, -(-tokens // max(1, batch.seqs)))
    if max_len is None:
        max_len = max(1, batch.table_cols * batch.page_size)
    if out is None:
        out, out_stride = q.new_empty(shape), heads * head_dim
    else:
        out_stride = _rows3("out", out, device, dtype, shape)
    if workspace is None:
        need = b.moe_kv4_attention_workspace_bytes(batch, heads, max_new, max_len)
        if need:
            workspace = q.new_empty((need,), dtype=torch.uint8)
    else:
        need = workspace.numel()
        _vector("workspace", workspace, device, torch.uint8, need)
    b.moe_kv4_attention(batch, q.data_ptr(), _rows3("q", q, device, dtype, shape), out.data_ptr(), out_stride, heads, scale,
                        code, max_new, max_len, workspace.data_ptr() if need else None, need, stream)
    return out


def norm_residual(h, y=None, gate=None, post=None, pre=None, residual_scale: float = 1.0, eps: float = 1e-5,
                  dtype=None, h_out: Optional[torch.Tensor] = None, want_h: bool = True, want_x: bool = True):
    """(h', x): h' = residual_scale h + gate (y post / rms(y)), fp32, and the next
    block's input x = h' pre / rms(h') in y's type (`dtype` without y).  h fp32
    [rows, d], y [rows, d], gate [d] or [rows, d], post and pre [d], fp32; without
    y there is no block's result to add, without post y is taken as it is.
    h_out=h updates the residual stream in place; want_h or want_x False: None
    in the place of h' or x."""
    if h.dim() != 2:
        raise ValueError("h must be [rows, d]")
    shape = h.shape
    rows, d = shape
    if y is not None:
        if dtype is not None and dtype != y.dtype:
            raise ValueError(f"y is {y.dtype}, not {dtype}")
        dtype = y.dtype
    elif dtype is None:
        dtype = torch.float32
    device, stream, code = _place(h, dtype)
    h_stride = _rows2("h", h, device, torch.float32, shape)
    y_ptr, y_stride = (y.data_ptr(), _rows2("y", y, device, dtype, shape)) if y is not None else (None, d)
    gate_ptr, gate_stride = None, 0
    if gate is not None:
        if gate.dim() == 1:
            gate_ptr = _vector("gate", gate, device, torch.float32, d)
        else:
            gate_ptr, gate_stride = gate.data_ptr(), _rows2("gate", gate, device, torch.float32, shape)
    h_out_ptr, h_out_stride, x, x_ptr = None, d, None, None
    if h_out is not None:
        h_out_ptr, h_out_stride = h_out.data_ptr(), _rows2("h_out", h_out, device, torch.float32, shape)
    elif want_h:
        h_out = h.new_empty(shape)
        h_out_ptr = h_out.data_ptr()
    if want_x:
        x = h.new_empty(shape, dtype=dtype)
        x_ptr = x.data_ptr()
    b.moe_norm_residual(h.data_ptr(), h_stride, y_ptr, y_stride, gate_ptr, gate_stride,
                        None if post is None else _vector("post", post, device, torch.float32, d),
                        None if pre is None else _vector("pre", pre, device, torch.float32, d),
                        residual_scale, eps, h_out_ptr, h_out_stride, x_ptr, d, rows, d, code, stream)
    return h_out, x
