"""Whole decoder layers: a 4-bit attention block in front of each MoE layer.

The experts of `OffloadedMoE` fill most of the HBM, so what stands before them
is kept small: the attention projections in 4 bits (groups of 64, the setting of
the paper's measured model, Sec. 5.1) and the keys and values in a paged cache
of 4 bits.  A layer is

  x = h pre / rms(h);  q, k, v = x Wqkv^T;  q, k rotated, k and v appended
  y = attention(q) Wo^T;  h += gate (y post / rms(y));  h += MoE(h)

with h in fp32 and everything between in `dtype`.  All of it runs on the MoE's
compute stream.  A step's new tokens may be trees of drafted ones (`drafts`), of
which `keep` keeps what was accepted.  Run as a module it takes a few sequences
through a small stack, with --drafts several tokens a step:

  python -m paper_2511_05814_amd.decoder --config tiny-stack --sequences 3 --prompt 20 --tokens 8
  python -m paper_2511_05814_amd.decoder --config tiny-stack --sequences 3 --prompt 20 --tokens 8 --drafts 6
"""
from __future__ import annotations

from typing import List, Optional

import numpy as np
import torch

from . import attention as at
from . import drafts
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
        self.new = [0] * count        # of the last extension, for `keep`
        self.pages: List[List[int]] = [[] for _ in range(count)]

    def extend(self, new: List[int], parents: Optional[List[List[int]]] = None) -> dict:
        """The batch of new[b] more tokens for each sequence b: the page_table,
        q_start and kv_len of the calls, on the device, the longest runs, and
        what the plan was made for (tokens, longest, pages, page_size).  With
        parents the new tokens of a sequence are a tree: parents[b][i] is an
        earlier one of them that token i follows, -1 for what follows the
        sequence so far.  Nothing changes where one is refused."""
        if len(new) != len(self.length) or min(new) < 0:
            raise ValueError(f"new tokens for {len(self.length)} sequences wanted, got {new}")
        behind = list(new)   # positions that the new tokens take
        if parents is not None:
            if [len(p) for p in parents] != list(new) or max(new) > 1024:
                raise ValueError(f"parents of {new} tokens wanted (at most 1024 of a sequence), got those of {[len(p) for p in parents]}")
            for b, tree in enumerate(parents):
                depth: List[int] = []
                for i, p in enumerate(tree):
                    if not -1 <= p < i:
                        raise ValueError(f"sequence {b}: token {i} cannot follow token {p}")
                    depth.append(depth[p] + 1 if p >= 0 else 1)
                behind[b] = max(depth, default=0)
        longest = max(n + l for n, l in zip(behind, self.length))
        if self.max_pos is not None and longest > self.max_pos:
            raise ValueError(f"a sequence of {longest} tokens, but positions end at {self.max_pos}")
        need = [max(0, -(-(n + l) // self.page_size) - len(p)) for n, l, p in zip(new, self.length, self.pages)]
        if sum(need) > len(self.free):
            raise RuntimeError(f"{sum(need)} pages needed, {len(self.free)} free")
        for b, m in enumerate(need):
            self.pages[b] += [self.free.pop() for _ in range(m)]
            self.length[b] += new[b]
        self.new = list(new)
        table = np.full((len(new), max(1, max(map(len, self.pages)))), -1, dtype=np.int32)
        for b, p in enumerate(self.pages):
            table[b, :len(p)] = p
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        arrays = table, start, np.array(self.length, dtype=np.int32)
        table, start, length = (torch.from_numpy(a).to("cuda") for a in arrays)
        batch = dict(page_table=table, q_start=start, kv_len=length, max_new=max(1, max(new)), max_len=max(1, max(self.length)),
                     tokens=sum(new), longest=longest, pages=self.count, page_size=self.page_size)
        if parents is not None:
            batch["parent"] = torch.tensor([p for tree in parents for p in tree], dtype=torch.int32).to("cuda")
        return batch

    def keep(self, count: List[int]) -> None:
        """Of the last extension's new tokens sequence b has kept count[b]
        (`DecoderStack.keep` does so in the caches); its pages stay its own."""
        if len(count) != len(self.new) or any(not 0 <= c <= n for c, n in zip(count, self.new)):
            raise ValueError(f"of {self.new} new tokens {list(count)} cannot be kept")
        self.length = [l - n + c for l, n, c in zip(self.length, self.new, count)]
        self.new = list(count)

    def release(self, b: int) -> None:
        """Sequence b is done: its pages are free again."""
        self.free += self.pages[b]
        self.pages[b], self.length[b], self.new[b] = [], 0, 0


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
        self._check_plan(batch)

    def _check_plan(self, batch: dict) -> None:
        if batch.get("longest", 0) > self.max_pos:
            raise ValueError(f"a sequence of {batch['longest']} tokens, but positions end at {self.max_pos}")
        if batch.get("page_size", self.page_size) != self.page_size or batch.get("pages", 0) > self.pages:
            raise ValueError(f"a plan for {batch['pages']} pages of {batch['page_size']} tokens, but the stack has "
                             f"{self.pages} of {self.page_size}")

    def attention_block(self, layer: int, h: torch.Tensor, batch: dict, tree=None) -> None:
        """h [tokens][d_model] (fp32, device), in place, on the current stream.
        tree: what `drafts.draft_tree` gives, where the new tokens are trees."""
        w, n, m = self.layers[layer], self.heads, self.heads + self.kv_heads
        plan = batch["page_table"], batch["q_start"], batch["kv_len"]
        _, x = at.norm_residual(h, pre=w["pre"], eps=self.eps, dtype=self.dtype, want_h=False)
        qkv = at.q4_matmul(x, w["wqkv"], self.width).unflatten(1, (-1, self.head_dim))
        sizes = dict(max_new=batch["max_new"], max_len=batch["max_len"])
        if tree is None:
            q = at.kv4_append(qkv[:, :n], qkv[:, n:m], qkv[:, m:], self.cos, self.sin, w["pool"], *plan)
            o = at.kv4_attention(q, w["pool"], *plan, self.head_dim ** -0.5, **sizes)
        else:
            pos, seen = tree
            q = at.kv4_append(qkv[:, :n], qkv[:, n:m], qkv[:, m:], self.cos, self.sin, w["pool"], *plan, pos=pos)
            o = at.kv4_tree_attention(q, w["pool"], *plan, seen, self.head_dim ** -0.5, **sizes)
        y = at.q4_matmul(o.flatten(1), w["wo"], h.shape[1])
        at.norm_residual(h, y, gate=w["gate"], post=w["post"], eps=self.eps, h_out=h, want_x=False)

    def step(self, H: torch.Tensor, batch: dict, snapshots: Optional[torch.Tensor] = None) -> None:
        """The batch's new tokens H [tokens][d_model] (fp32, device; rows may lie
        apart) through all layers, in place; trees where the batch has parents.  snapshots (optional, [layers][2][tokens][d_model])
        receives h entering and leaving every attention block.  The work is only
        enqueued, on moe.compute: moe.sync() waits for it."""
        moe = self.moe
        self._check(H, batch)
        parent = batch.get("parent")
        for t in (H, batch["page_table"], batch["q_start"], batch["kv_len"], snapshots, parent):
            if t is not None:
                t.record_stream(moe.compute)   # the caller may let go of them before it is done
        moe.compute.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(moe.compute):
            tree = None if parent is None else drafts.draft_tree(parent, batch["q_start"], batch["kv_len"], batch["max_new"])
            for l in range(moe.L):
                if snapshots is not None:
                    snapshots[l, 0].copy_(H)
                self.attention_block(l, H, batch, tree)
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


    def keep(self, batch: dict, path: torch.Tensor, count: torch.Tensor) -> None:
        """Keeps what `drafts.verify_drafts` accepted of the batch's new tokens in
        all layers' caches; enqueued on moe.compute, in line with the steps.
        `Sequences.keep` takes the counts, once the host has them."""
        moe = self.moe
        self._check_plan(batch)
        if batch.get("tokens", path.numel()) != path.numel():
            raise ValueError(f"a path of {path.numel()} tokens for a plan of {batch['tokens']}")
        for t in (batch["page_table"], batch["q_start"], batch["kv_len"], path, count):
            t.record_stream(moe.compute)
        moe.compute.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(moe.compute):
            at.kv4_keep([l["pool"] for l in self.layers], batch["page_table"], batch["q_start"], batch["kv_len"], path, count, self.head_dim)


class Speculation:
    """Decoding with drafted tokens for a stack of synthetic weights: an
    embedding, a 4-bit head over `vocab` ids and, as the cheap draft, the head on
    the embedding alone, without any layer."""

    def __init__(self, stack: DecoderStack, vocab: int, nodes: int, width: int = 2, seed: int = 0):
        if vocab < 1 or not 1 <= nodes <= 1024 or width < 1:
            raise ValueError(f"trees of {nodes} tokens (1 .. 1024), {width} behind each, of {vocab} ids cannot be drafted")
        self.stack, self.vocab, self.nodes, self.width = stack, vocab, nodes, width
        d, rng = stack.moe.cfg.d_model, np.random.default_rng(seed)
        self.embedding = torch.from_numpy(rng.standard_normal((vocab, d), dtype=np.float32)).to("cuda")
        self.head = torch.from_numpy(wl.quantize_q4g64(rng.standard_normal((vocab, d), dtype=np.float32) * np.float32(3 * d ** -0.5))).to("cuda")
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden: Optional[torch.Tensor] = None   # of the last step's tokens, behind all layers

    def probabilities(self, h: torch.Tensor) -> torch.Tensor:
        """Of the token behind each row of hidden states, fp32 [rows, vocab]."""
        _, x = at.norm_residual(h, want_h=False, dtype=torch.float32)
        return torch.softmax(at.q4_matmul(x, self.head, self.vocab), 1)

    def draft(self, pending: torch.Tensor):
        """Trees behind the pending tokens [sequences], level by level: (parents of
        a sequence, tokens [sequences, nodes], q [sequences, nodes, vocab])."""
        parents, level = [-1], [0]
        while len(parents) < self.nodes:
            grown = [p for p in level for _ in range(self.width)][:self.nodes - len(parents)]
            level = list(range(len(parents), len(parents) + len(grown)))
            parents += grown
        tokens = pending.new_zeros((len(pending), self.nodes))
        q = torch.zeros((len(pending), self.nodes, self.vocab), device="cuda")
        tokens[:, 0] = pending
        for i in range(self.nodes):
            q[:, i] = self.probabilities(self.embedding[tokens[:, i]])
            mine = [c for c, p in enumerate(parents) if p == i]
            if mine:
                tokens[:, mine] = torch.multinomial(q[:, i], len(mine), replacement=True, generator=self.gen).to(tokens.dtype)
        return parents, tokens, q

    def step(self, seqs: Sequences, pending: torch.Tensor, active: List[int]):
        """One step of the sequences in `active`: (every sequence's pending token
        [sequences], how many tokens each took)."""
        stack, moe = self.stack, self.stack.moe
        parents, tokens, q = self.draft(pending[active])
        batch = seqs.extend([self.nodes if b in active else 0 for b in range(len(pending))],
                            [parents if b in active else [] for b in range(len(pending))])
        H = self.hidden = self.embedding[tokens.flatten()]
        stack.step(H, batch)
        torch.cuda.current_stream().wait_stream(moe.compute)
        u = torch.rand(H.shape[0], generator=self.gen, device="cuda")
        path, kept, after = drafts.verify_drafts(self.probabilities(H), tokens.flatten().int(), batch["parent"], u, batch["q_start"],
                                                 q.flatten(0, 1))
        stack.keep(batch, path, kept)
        taken, ids = torch.stack([kept, after]).tolist()
        seqs.keep(taken)
        if any(n and i < 0 for n, i in zip(taken, ids)):
            raise RuntimeError("probabilities of a next token that are not finite")
        return torch.where(kept > 0, after.long(), pending), taken


def main(argv=None) -> None:
    import argparse
    import time
    p = argparse.ArgumentParser(description="sequences through a stack of 4-bit attention blocks and offloaded MoE layers")
    p.add_argument("--config", default="tiny-stack", choices=sorted(wl.CONFIGS))
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--sequences", type=int, default=3)
    p.add_argument("--prompt", type=int, default=20)
    p.add_argument("--tokens", type=int, default=8)
    p.add_argument("--drafts", type=int, default=0, help="tokens of a step's tree; 0: one token a step")
    p.add_argument("--width", type=int, default=2, help="guesses behind each token of a tree")
    p.add_argument("--vocab", type=int, default=1000)
    a = p.parse_args(argv)
    cfg = wl.CONFIGS[a.config].with_(layers=a.layers)
    head_dim = 64 if cfg.d_model < 2048 else 128
    heads = cfg.d_model // head_dim
    total = a.prompt + a.tokens
    room = total + a.drafts   # a step that begins before the last token may end past it
    batched = a.sequences * max(a.prompt, a.drafts) if cfg.dtype == "bf16" else 0
    moe = offload.OffloadedMoE(cfg, offload.HostStore(cfg), offload.DeviceGates(cfg), slots=cfg.slots[0],
                               policy=cfg.policies[-1], max_prefill_tokens=batched)
    stack = DecoderStack(moe, heads, max(1, heads // 4), head_dim, pages=a.sequences * -(-room // 16), max_pos=room)
    seqs = stack.sequences(a.sequences)
    states = torch.from_numpy(wl.hidden_states(cfg, a.sequences * total)).to("cuda").view(a.sequences, total, -1)

    def take(first, count):
        H = states[:, first:first + count].reshape(a.sequences * count, -1).contiguous()
        stack.step(H, seqs.extend([count] * a.sequences))
        moe.sync()
        return H

    spec = Speculation(stack, a.vocab, a.drafts, a.width) if a.drafts else None
    t0 = time.perf_counter()
    H = take(0, a.prompt)
    t1 = time.perf_counter()
    if a.drafts:
        pending, steps = torch.arange(a.sequences, device="cuda") % a.vocab, 0
        while min(seqs.length) < total:
            active = [b for b, n in enumerate(seqs.length) if n < total]
            pending, taken = spec.step(seqs, pending, active)
            H = spec.hidden
            steps += len(active)
        moe.sync()
        made = sum(seqs.length) - a.sequences * a.prompt
        print(f"trees of {a.drafts}: {made / max(steps, 1):.2f} tokens a step of a sequence")
    else:
        made = a.sequences * a.tokens
        for i in range(a.tokens):
            H = take(a.prompt + i, 1)
    t2 = time.perf_counter()
    kept = sum(l["pool"].numel() for l in stack.layers)
    print(f"{cfg.name}: {cfg.layers} layers, {heads} heads of {head_dim}, {a.sequences} sequences")
    print(f"prompt: {a.sequences * a.prompt / (t1 - t0):.1f} tokens/s, decode: {made / (t2 - t1):.1f} tokens/s")
    print(f"cache: {kept / 1e6:.2f} MB in 4 bits ({kept * 32 // 9 / 1e6:.2f} MB in bf16); last rms {H.square().mean().sqrt().item():.4f}")
    hits = moe.stats()
    print("expert hits / misses:", sum(s["hits"] for s in hits), "/", sum(s["misses"] for s in hits))


if __name__ == "__main__":
    main()
