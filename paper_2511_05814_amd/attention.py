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

from . import binding as b

GROUP = 64          # columns of a 4-bit matrix that share a scale
KV_GROUP = 32       # dimensions of a cache entry that share one
_DTYPES = {torch.float32: b.MOE_DTYPE_F32, torch.bfloat16: b.MOE_DTYPE_BF16}


def _dtype(t) -> int:
    try:
        return _DTYPES[t]
    except KeyError:
        raise ValueError(f"tensors must be float32 or bfloat16, not {t}") from None


def _stream(t: torch.Tensor) -> int:
    """The current stream of t's device, which must be the current device."""
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    s = torch.cuda.current_stream()
    if t.get_device() != s.device_index:
        raise ValueError(f"tensors are on device {t.get_device()}, the current device is {s.device_index}")
    return s.cuda_stream


def _same(device: int, name: str, t: torch.Tensor, dtype, shape) -> torch.Tensor:
    if t.dtype != dtype or t.get_device() != device or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on device {device}, "
                         f"not {t.dtype} {tuple(t.shape)} on device {t.get_device()}")
    return t


def _rows(name: str, t: torch.Tensor) -> int:
    """Elements between the rows of t [rows][...], each row contiguous."""
    inner = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != inner:
            raise ValueError(f"{name}: rows must be contiguous")
        inner *= size
    return t.stride(0) if t.shape[0] > 1 else inner


def q4_matmul(x: torch.Tensor, w: torch.Tensor, n: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows, k] times the 4-bit matrix [n x k] in the bytes w, transposed: [rows, n]."""
    if x.dim() != 2:
        raise ValueError("x must be [rows, k]")
    rows, k = x.shape
    dtype, stream, device = _dtype(x.dtype), _stream(x), x.get_device()
    if k % GROUP or k == 0 or n < 1:
        raise ValueError(f"a 4-bit matrix [{n} x {k}]: columns must be a multiple of {GROUP}")
    _same(device, "w", w, torch.uint8, (n * k // 2 + n * (k // GROUP) * 3,))
    if not w.is_contiguous():
        raise ValueError("w must be contiguous")
    if out is None:
        out = torch.empty((rows, n), dtype=x.dtype, device=x.device)
    else:
        _same(device, "out", out, x.dtype, (rows, n))
    b.moe_q4_matmul(x.data_ptr(), _rows("x", x), w.data_ptr(), out.data_ptr(), _rows("out", out), rows, n, k, dtype, stream)
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
    seqs = kv_len.shape[0]
    for name, t, dims in (("page_table", page_table, 2), ("q_start", q_start, 1), ("kv_len", kv_len, 1)):
        if t.dtype != torch.int32 or t.dim() != dims or t.get_device() != device or t.stride(-1) != 1:
            raise ValueError(f"{name} must be int32 of {dims} dimension(s), contiguous in the last, on the call's device")
    if page_table.shape[0] != seqs or q_start.shape[0] != seqs + 1:
        raise ValueError(f"{seqs} sequences: page_table {tuple(page_table.shape)}, q_start {tuple(q_start.shape)}")
    cols = page_table.shape[1]
    return b.moe_kv4_batch(pool.data_ptr(), page_table.data_ptr(), q_start.data_ptr(), kv_len.data_ptr(),
                           page_table.stride(0) if seqs > 1 else cols, pages, page_size, kv_heads, head_dim, cols, seqs, tokens)


def kv4_append(q, k, v, cos, sin, pool, page_table, q_start, kv_len, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotate the new tokens' q [tokens, heads, head_dim] and k by their
    positions, store k and v [tokens, kv_heads, head_dim] in the cache and
    return the rotated q.  cos and sin: fp32 [positions, rot_dim / 2]; with
    rot_dim 0 nothing is rotated.  Rows may be slices of a joined projection."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v must be [tokens, heads, head_dim]")
    tokens, heads, head_dim = q.shape
    dtype, stream, device = _dtype(q.dtype), _stream(q), q.get_device()
    batch = _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim)
    shape = (tokens, batch.kv_heads, head_dim)
    _same(device, "k", k, q.dtype, shape)
    _same(device, "v", v, q.dtype, shape)
    if cos.dim() != 2 or not cos.is_contiguous() or not sin.is_contiguous():
        raise ValueError("cos and sin must be contiguous [positions, rot_dim / 2]")
    _same(device, "cos", cos, torch.float32, cos.shape)
    _same(device, "sin", sin, torch.float32, cos.shape)
    if out is None:
        out = torch.empty((tokens, heads, head_dim), dtype=q.dtype, device=q.device)
    else:
        _same(device, "out", out, q.dtype, q.shape)
    b.moe_kv4_append(batch, q.data_ptr(), _rows("q", q), k.data_ptr(), _rows("k", k), v.data_ptr(), _rows("v", v),
                     cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], out.data_ptr(), _rows("out", out),
                     heads, dtype, stream)
    return out


def kv4_read(pool, page_table, q_start, kv_len, tokens: int, head_dim: int, dtype=torch.float32):
    """The stored keys and values of the batch's new tokens, [tokens, kv_heads,
    head_dim] each (exact in both types).  With q_start the running sums of
    kv_len that is everything the sequences have."""
    code, stream, device = _dtype(dtype), _stream(pool), pool.get_device()
    batch = _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim)
    k = torch.empty((tokens, batch.kv_heads, head_dim), dtype=dtype, device=pool.device)
    v = torch.empty_like(k)
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
    tokens, heads, head_dim = q.shape
    dtype, stream, device = _dtype(q.dtype), _stream(q), q.get_device()
    batch = _batch(device, pool, page_table, q_start, kv_len, tokens, head_dim)
    if max_new is None:
        max_new = max(1, -(-tokens // max(1, batch.seqs)))
    if max_len is None:
        max_len = max(1, batch.table_cols * batch.page_size)
    if out is None:
        out = torch.empty((tokens, heads, head_dim), dtype=q.dtype, device=q.device)
    else:
        _same(device, "out", out, q.dtype, q.shape)
    if workspace is None:
        need = b.moe_kv4_attention_workspace_bytes(batch, heads, max_new, max_len)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous on the call's device")
    b.moe_kv4_attention(batch, q.data_ptr(), _rows("q", q), out.data_ptr(), _rows("out", out), heads, scale, dtype,
                        max_new, max_len, workspace.data_ptr() if workspace is not None else None,
                        workspace.numel() * workspace.element_size() if workspace is not None else 0, stream)
    return out


def norm_residual(h, y=None, gate=None, post=None, pre=None, residual_scale: float = 1.0, eps: float = 1e-5,
                  dtype=None, h_out: Optional[torch.Tensor] = None, want_h: bool = True, want_x: bool = True):
    """(h', x): h' = residual_scale h + gate (y post / rms(y)), fp32, and the next
    block's input x = h' pre / rms(h') in y's type (`dtype` without y).  h fp32
    [rows, d], y [rows, d], gate [d] or [rows, d], post and pre [d], fp32; without
    y there is no block's result to add, without post y is taken as it is.
    h_out=h updates the residual stream in place."""
    if h.dim() != 2:
        raise ValueError("h must be [rows, d]")
    rows, d = h.shape
    stream, device = _stream(h), h.get_device()
    _same(device, "h", h, torch.float32, h.shape)
    if y is not None:
        if dtype not in (None, y.dtype):
            raise ValueError(f"y is {y.dtype}, not {dtype}")
        dtype = y.dtype
        _same(device, "y", y, dtype, h.shape)
    dtype = dtype or torch.float32
    code = _dtype(dtype)
    for name, t in (("post", post), ("pre", pre)):
        if t is not None and not _same(device, name, t, torch.float32, (d,)).is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    gate_stride = 0
    if gate is not None:
        _same(device, "gate", gate, torch.float32, (d,) if gate.dim() == 1 else (rows, d))
        if gate.stride(-1) != 1:
            raise ValueError("gate: rows must be contiguous")
        gate_stride = 0 if gate.dim() == 1 else _rows("gate", gate)
    if h_out is not None:
        _same(device, "h_out", h_out, torch.float32, h.shape)
    elif want_h:
        h_out = torch.empty((rows, d), dtype=torch.float32, device=h.device)
    x = torch.empty((rows, d), dtype=dtype, device=h.device) if want_x else None
    b.moe_norm_residual(h.data_ptr(), _rows("h", h), y.data_ptr() if y is not None else None,
                        _rows("y", y) if y is not None else d, gate.data_ptr() if gate is not None else None, gate_stride,
                        post.data_ptr() if post is not None else None, pre.data_ptr() if pre is not None else None,
                        residual_scale, eps, h_out.data_ptr() if h_out is not None else None,
                        _rows("h_out", h_out) if h_out is not None else d, x.data_ptr() if x is not None else None, d,
                        rows, d, code, stream)
    return h_out, x
