"""Batches over a 4-bit paged cache for the GPU tests, with the oracle's view of them."""
import numpy as np
import torch

from oracle import attention as oa


def bf16(x):
    """fp32 values that bf16 holds."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).bfloat16().float().numpy()


def device(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.bfloat16() if dtype == "bf16" else t


class Batch:
    """Sequences of old[b] cached and new[b] new tokens, their pages in a
    shuffled order; `pool` is the cache's bytes on the host."""

    def __init__(self, new, old, heads, kv_heads, D, P, seed=0, spare=2, short=0):
        self.new, self.old, self.heads, self.kv_heads, self.D, self.P = new, old, heads, kv_heads, D, P
        self.rng = np.random.default_rng(seed)
        self.len = [n + o - short for n, o in zip(new, old)]
        need = [max(0, -(-n // P)) for n in self.len]
        order = self.rng.permutation(sum(need) + spare)
        self.table = np.full((len(new), max(1, max(need))), -1, dtype=np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens = int(self.q_start[-1])
        self.pool = np.zeros((len(order), kv_heads, P * D * 9 // 8), dtype=np.uint8)

    def fill(self, strong=1.0):
        """Random entries everywhere, unused places too."""
        for page in range(self.pool.shape[0]):
            for h in range(self.kv_heads):
                k = self.rng.standard_normal((self.P, self.D)) * np.exp(strong * self.rng.standard_normal(self.D))
                v = self.rng.standard_normal((self.P, self.D))
                self.pool[page, h] = oa.record(*oa.kv4_quantize(k), *oa.kv4_quantize(v))
        return self

    def args(self):
        t = [torch.from_numpy(a).cuda() for a in (self.pool, self.table, self.q_start, np.array(self.len, dtype=np.int32))]
        return t

    def positions(self):
        return np.concatenate([np.arange(n) + (length - n) for n, length in zip(self.new, self.len)]).astype(np.int64)

    def sequence(self, b):
        """(keys, values, held) of sequence b, [heads, length, D]."""
        return oa.gather(self.pool, self.table[b], max(0, self.len[b]), self.P, self.D)

    def attend(self, q, scale):
        """fp64 outputs and, for each, the error bound's ingredients: sum |q||k|
        at its largest and the largest |v|."""
        out, reach, top = np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape[:2])
        group = self.heads // self.kv_heads
        for b, n in enumerate(self.new):
            k, v, held = self.sequence(b)
            first = self.len[b] - n
            seen = (np.arange(k.shape[1]) <= first + np.arange(n)[:, None]) & held
            for h in range(self.heads):
                rows = slice(self.q_start[b], self.q_start[b] + n)
                out[rows, h] = oa.attention(q[rows, h], k[h // group], v[h // group], seen, scale)
                if k.shape[1] and n:
                    mass = np.abs(q[rows, h]) @ np.abs(k[h // group]).T
                    reach[rows, h] = np.nanmax(np.where(seen, mass, 0), 1) * abs(scale)
                    top[rows, h] = np.nanmax(np.abs(v[h // group]))
        return out, reach, top
