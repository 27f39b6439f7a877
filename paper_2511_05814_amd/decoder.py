"""Whole decoder layers: a 4-bit attention block in front of each MoE layer.

The experts of `OffloadedMoE` fill most of the HBM, so what stands before them
is kept small: the attention projections in 4 bits (groups of 64, the setting of
the paper's measured model, Sec. 5.1) and the keys and values in a paged cache
of 4 bits.  A layer is

  x = h pre / rms(h);  q, k, v = x Wqkv^T;  q, k rotated, k and v appended
  y = attention(q) Wo^T;  h += gate (y post / rms(y));  h += MoE(h)

with h in fp32 and everything between in `dtype`.  All of it runs on the MoE's
compute stream.  Run as a module it takes a few sequences through a small stack:

  python -m paper_2511_05814_amd.decoder --config tiny-stack --sequences 3 --prompt 20 --tokens 8
"""
from __future__ import annotations

from typing import List, Optional

import numpy as np
import torch

from . import attention as at
from . import offload
from . import workload as wl


class Sequences:
    """Pages and lengths of a set of sequences that share one page table in
    every layer, kept on the host; `extend` plans a call's new tokens.  pages,
    page_size and max_pos (the longest that a sequence may get) are those of the
    stack; `DecoderStack.sequences` fills them in."""

    def __init__(self, count: int, pages: int, page_size: int, max_pos: Optional[int] = None):
        self.page_size, self.max_pos, self.count, self.free = page_size, max_pos, pages, list(range(pages))[::-1]
        self.length = [0] * count
        self.pages: List[List[int]] = [[] for _ in range(count)]

    def extend(self, new: List[int]) -> dict:
        """The batch of new[b] more tokens for each sequence b: the page_table,
        q_start and kv_len of the calls, on the device, the longest runs, and
        what the plan was made for (tokens, longest, pages, page_size).  Nothing
        changes where one is refused."""
        if len(new) != len(self.length) or min(new) < 0:
            raise ValueError(f"new tokens for {len(self.length)} sequences wanted, got {new}")
        longest = max(n + l for n, l in zip(new, self.length))
        if self.max_pos is not None and longest > self.max_pos:
            raise ValueError(f"a sequence of {longest} tokens, but positions end at {self.max_pos}")
        need = [max(0, -(-(n + l) // self.page_size) - len(p)) for n, l, p in zip(new, self.length, self.pages)]
        if sum(need) > len(self.free):
            raise RuntimeError(f"{sum(need)} pages needed, {len(self.free)} free")
        for b, m in enumerate(need):
            self.pages[b] += [self.free.pop() for _ in range(m)]
            self.length[b] += new[b]
        table = np.full((len(new), max(1, max(map(len, self.pages)))), -1, dtype=np.int32)
        for b, p in enumerate(self.pages):
            table[b, :len(p)] = p
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        arrays = table, start, np.array(self.length, dtype=np.int32)
        table, start, length = (torch.from_numpy(a).to("cuda") for a in arrays)
        return dict(page_table=table, q_start=start, kv_len=length, max_new=max(1, max(new)), max_len=max(1, longest),
                    tokens=sum(new), longest=longest, pages=self.count, page_size=self.page_size)

    def release(self, b: int) -> None:
        """Sequence b is done: its pages are free again."""
        self.free += self.pages[b]
        self.pages[b], self.length[b] = [], 0


class DecoderStack:
    """Attention blocks with seeded weights N(0, 0.02^2), 4-bit, in front of the
    layers of `moe`.  heads * head_dim need not be d_model; both are multiples
    of 64."""

    def __init__(self, moe: offload.OffloadedMoE, heads: int, kv_heads: int, head_dim: int, pages: int,
                 page_size: int = 16, max_pos: int = 4096, dtype=torch.bfloat16, eps: float = 1e-5):
        cfg = moe.cfg
        self.pages, self.page_size, self.max_pos = pages, page_size, max_pos
        self.moe, self.heads, self.kv_heads, self.head_dim, self.dtype, self.eps = moe, heads, kv_heads, head_dim, dtype, eps
        self.width = (heads + 2 * kv_heads) * head_dim
        rng = np.random.default_rng(np.random.SeedSequence(cfg.seed, spawn_key=(len("attention"),)))

        def matrix(n, k):
            return torch.from_numpy(wl.quantize_q4g64(rng.standard_normal((n, k), dtype=np.float32) * np.float32(wl.WEIGHT_STD))).to("cuda")

        def vector(mean):
            return torch.from_numpy((mean + 0.05 * rng.standard_normal(cfg.d_model)).astype(np.float32)).to("cuda")

        self.layers = [dict(wqkv=matrix(self.width, cfg.d_model), wo=matrix(cfg.d_model, heads * head_dim), pre=vector(1.0),
                            post=vector(1.0), gate=vector(0.5),
                            pool=at.kv4_pool(pages, kv_heads, page_size, head_dim)) for _ in range(cfg.layers)]
        angle = np.arange(max_pos)[:, None] * 10000.0 ** (-np.arange(0, head_dim, 2) / head_dim)
        self.cos, self.sin = (torch.from_numpy(f(angle).astype(np.float32)).to("cuda") for f in (np.cos, np.sin))
        for t in (self.cos, self.sin, *(t for l in self.layers for t in l.values())):
            t.record_stream(moe.compute)   # a stack may be dropped before its steps are done

    def sequences(self, count: int) -> Sequences:
        """A set of sequences over this stack's pages (one set at a time)."""
        return Sequences(count, self.pages, self.page_size, self.max_pos)

    def _check(self, H: torch.Tensor, batch: dict) -> None:
        """H and what a plan of `Sequences.extend` says of itself must fit the
        stack; found on the host, before anything is enqueued."""
        if H.dim() != 2 or H.shape[1] != self.moe.cfg.d_model or H.dtype != torch.float32:
            raise ValueError(f"H must be float32 [tokens, {self.moe.cfg.d_model}], not {H.dtype} {list(H.shape)}")
        if batch.get("tokens", H.shape[0]) != H.shape[0]:
            raise ValueError(f"{H.shape[0]} rows of H for a plan of {batch['tokens']} tokens")
        if batch.get("longest", 0) > self.max_pos:
            raise ValueError(f"a sequence of {batch['longest']} tokens, but positions end at {self.max_pos}")
        if batch.get("page_size", self.page_size) != self.page_size or batch.get("pages", 0) > self.pages:
            raise ValueError(f"a plan for {batch['pages']} pages of {batch['page_size']} tokens, but the stack has "
                             f"{self.pages} of {self.page_size}")

    def attention_block(self, layer: int, h: torch.Tensor, batch: dict) -> None:
        """h [tokens][d_model] (fp32, device), in place, on the current stream."""
        w, n, m = self.layers[layer], self.heads, self.heads + self.kv_heads
        plan = batch["page_table"], batch["q_start"], batch["kv_len"]
        _, x = at.norm_residual(h, pre=w["pre"], eps=self.eps, dtype=self.dtype, want_h=False)
        qkv = at.q4_matmul(x, w["wqkv"], self.width).unflatten(1, (-1, self.head_dim))
        q = at.kv4_append(qkv[:, :n], qkv[:, n:m], qkv[:, m:], self.cos, self.sin, w["pool"], *plan)
        o = at.kv4_attention(q, w["pool"], *plan, self.head_dim ** -0.5, max_new=batch["max_new"], max_len=batch["max_len"])
        y = at.q4_matmul(o.flatten(1), w["wo"], h.shape[1])
        at.norm_residual(h, y, gate=w["gate"], post=w["post"], eps=self.eps, h_out=h, want_x=False)

    def step(self, H: torch.Tensor, batch: dict, snapshots: Optional[torch.Tensor] = None) -> None:
        """The batch's new tokens H [tokens][d_model] (fp32, device; rows may lie
        apart) through all layers, in place.  snapshots (optional, [layers][2][tokens][d_model])
        receives h entering and leaving every attention block.  The work is only
        enqueued, on moe.compute: moe.sync() waits for it."""
        moe = self.moe
        self._check(H, batch)
        for t in (H, batch["page_table"], batch["q_start"], batch["kv_len"], snapshots):
            if t is not None:
                t.record_stream(moe.compute)   # the caller may let go of them before it is done
        moe.compute.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(moe.compute):
            for l in range(moe.L):
                if snapshots is not None:
                    snapshots[l, 0].copy_(H)
                self.attention_block(l, H, batch)
                if snapshots is not None:
                    snapshots[l, 1].copy_(H)
                if H.shape[0] > 1 and moe.desc.max_prefill_tokens >= H.shape[0]:
                    dense = H.contiguous()   # moe_prefill_layer takes rows one behind the other
                    offload.b.moe_prefill_layer(moe.handle, l, dense.data_ptr(), H.shape[0])
                    if dense is not H:
                        H.copy_(dense)
                else:
                    for t in range(H.shape[0]):
                        moe.decode_layer(l, H[t])


def main(argv=None) -> None:
    import argparse
    import time
    p = argparse.ArgumentParser(description="sequences through a stack of 4-bit attention blocks and offloaded MoE layers")
    p.add_argument("--config", default="tiny-stack", choices=sorted(wl.CONFIGS))
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--sequences", type=int, default=3)
    p.add_argument("--prompt", type=int, default=20)
    p.add_argument("--tokens", type=int, default=8)
    a = p.parse_args(argv)
    cfg = wl.CONFIGS[a.config].with_(layers=a.layers)
    head_dim = 64 if cfg.d_model < 2048 else 128
    heads = cfg.d_model // head_dim
    total = a.prompt + a.tokens
    batched = a.sequences * a.prompt if cfg.dtype == "bf16" else 0
    moe = offload.OffloadedMoE(cfg, offload.HostStore(cfg), offload.DeviceGates(cfg), slots=cfg.slots[0],
                               policy=cfg.policies[-1], max_prefill_tokens=batched)
    stack = DecoderStack(moe, heads, max(1, heads // 4), head_dim, pages=a.sequences * -(-total // 16), max_pos=total)
    seqs = stack.sequences(a.sequences)
    states = torch.from_numpy(wl.hidden_states(cfg, a.sequences * total)).to("cuda").view(a.sequences, total, -1)

    def take(first, count):
        H = states[:, first:first + count].reshape(a.sequences * count, -1).contiguous()
        stack.step(H, seqs.extend([count] * a.sequences))
        moe.sync()
        return H

    t0 = time.perf_counter()
    take(0, a.prompt)
    t1 = time.perf_counter()
    for i in range(a.tokens):
        H = take(a.prompt + i, 1)
    t2 = time.perf_counter()
    kept = sum(l["pool"].numel() for l in stack.layers)
    print(f"{cfg.name}: {cfg.layers} layers, {heads} heads of {head_dim}, {a.sequences} sequences")
    print(f"prompt: {a.sequences * a.prompt / (t1 - t0):.1f} tokens/s, decode: {a.sequences * a.tokens / (t2 - t1):.1f} tokens/s")
    print(f"cache: {kept / 1e6:.2f} MB in 4 bits ({kept * 32 // 9 / 1e6:.2f} MB in bf16); last rms {H.square().mean().sqrt().item():.4f}")
    hits = moe.stats()
    print("expert hits / misses:", sum(s["hits"] for s in hits), "/", sum(s["misses"] for s in hits))


if __name__ == "__main__":
    main()
