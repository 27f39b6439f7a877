"""The attention half of a layer on torch tensors: 4-bit products, the 4-bit
paged cache, attention over it and the norms around a block.

Each function checks its tensors, allocates what it returns (unless it is given
`out`) and enqueues one call of the C ABI (include/moe_offload.h, which has the
formulas and layouts) on torch's current stream of the tensors' device, so
`with torch.cuda.stream(moe.compute)` puts it in line with an `OffloadedMoE`.
Nothing synchronises.  None has a gradient: a tensor that requires one is
refused unless gradients are off.  Tensors are fp32 or bf16 as a whole call; a
tensor used on another stream than its own has to be made known to torch's
allocator (`record_stream`) as with any torch operator.  ValueError: tensors
that do not fit together; binding.MoeError: what the library refuses (alignment,
overlap, limits); torch.OutOfMemoryError: no memory for a result or a workspace.

A cache's pool is uint8 [pages][kv heads][page_size * head_dim * 9 / 8]
(`kv4_pool`).  A batch of B sequences is three int32 tensors on the device:
`q_start` [B + 1], bounds of the sequences' new tokens in this call's rows;
`kv_len` [B], tokens of each sequence with the new ones; `page_table` [B, n],
its pages in order, -1 where there is none.
"""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os
from typing import Optional

import torch
from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice

from . import binding as b

GROUP = 64          # columns of a 4-bit matrix that share a scale
KV_GROUP = 32       # dimensions of a cache entry that share one
OPS_PATH = os.path.join(os.path.dirname(b.LIB_PATH), "_attention_ops.so")
_DTYPES = {torch.float32: b.MOE_DTYPE_F32, torch.bfloat16: b.MOE_DTYPE_BF16}

_module = None


def _ops():
    """The built module (csrc/attention_ops.cpp); raises if it is missing."""
    global _module
    if _module is None:
        b.lib()
        if not os.path.exists(OPS_PATH):
            raise RuntimeError(f"{OPS_PATH} is missing: build it with __graft_entry__.build()")
        loader = importlib.machinery.ExtensionFileLoader("_attention_ops", OPS_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_attention_ops", loader))
        loader.exec_module(module)
        module.set_errors(b.MoeError, torch.OutOfMemoryError)
        _module = module
    return _module


def _stream(t: torch.Tensor) -> int:
    """Torch's current stream on t's device, which must be the current one."""
    device = t.get_device()
    if device < 0 or device != _cuda_getDevice():
        raise ValueError(f"tensors must be on the current GPU, not on {t.device}")
    return _cuda_getCurrentRawStream(device)


def _code(dtype) -> int:
    try:
        return _DTYPES[dtype]
    except KeyError:
        raise ValueError(f"tensors must be float32 or bfloat16, not {dtype}") from None


def q4_matmul(x: torch.Tensor, w: torch.Tensor, n: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows, k] times the 4-bit matrix [n x k] in the bytes w, transposed: [rows, n]."""
    return _ops().q4_matmul(x, w, n, out, _stream(x))


def kv4_record_bytes(page_size: int, head_dim: int) -> int:
    """Bytes that a page of page_size tokens takes for one kv head."""
    return page_size * head_dim * 9 // 8


def kv4_pool(pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda") -> torch.Tensor:
    """A cache's pages, all entries zero."""
    return torch.zeros((pages, kv_heads, kv4_record_bytes(page_size, head_dim)), dtype=torch.uint8, device=device)


def kv4_append(q, k, v, cos, sin, pool, page_table, q_start, kv_len, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotate the new tokens' q [tokens, heads, head_dim] and k by their
    positions, store k and v [tokens, kv_heads, head_dim] in the cache and
    return the rotated q.  cos and sin: fp32 [positions, rot_dim / 2]; with
    rot_dim 0 nothing is rotated.  Rows may be slices of a joined projection."""
    return _ops().kv4_append(q, k, v, cos, sin, pool, page_table, q_start, kv_len, out, _stream(q))


def kv4_read(pool, page_table, q_start, kv_len, tokens: int, head_dim: int, dtype=torch.float32):
    """The stored keys and values of the batch's new tokens, [tokens, kv_heads,
    head_dim] each (exact in both types).  With q_start the running sums of
    kv_len that is everything the sequences have."""
    return _ops().kv4_read(pool, page_table, q_start, kv_len, tokens, head_dim, _code(dtype), _stream(pool))


def kv4_attention(q, pool, page_table, q_start, kv_len, scale: float, max_new: Optional[int] = None,
                  max_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the new tokens' q [tokens, heads, head_dim] over their
    sequences' caches, causal; rows that see nothing are zeros.  max_new and
    max_len (the longest run of new tokens, the longest sequence) say how to cut
    the work; without them they are taken from the tensors' shapes.  A workspace
    is allocated unless one (uint8) is given."""
    return _ops().kv4_attention(q, pool, page_table, q_start, kv_len, scale, max_new, max_len, out, workspace, _stream(q))


def norm_residual(h, y=None, gate=None, post=None, pre=None, residual_scale: float = 1.0, eps: float = 1e-5,
                  dtype=None, h_out: Optional[torch.Tensor] = None, want_h: bool = True, want_x: bool = True):
    """(h', x): h' = residual_scale h + gate (y post / rms(y)), fp32, and the next
    block's input x = h' pre / rms(h') in y's type (`dtype` without y).  h fp32
    [rows, d], y [rows, d], gate [d] or [rows, d], post and pre [d], fp32; without
    y there is no block's result to add, without post y is taken as it is.
    h_out=h updates the residual stream in place; want_h or want_x False: None
    in the place of h' or x."""
    return _ops().norm_residual(h, y, gate, post, pre, residual_scale, eps, -1 if dtype is None else _code(dtype), h_out, want_h,
                                want_x, _stream(h))
