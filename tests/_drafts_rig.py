"""Trees of drafted tokens for the GPU tests, with the oracle's view of them."""
import numpy as np
import torch

from oracle import attention as oa
from oracle import drafts as od


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def parents(rng, n, width=3):
    return [-1] + [int(i - 1 - rng.integers(min(i, width))) for i in range(1, n)] if n else []


def masks(bt, rng, kind):
    """What each new token of a batch sees of its sequence's, [n, n] each."""
    out = []
    for n in bt.new:
        if kind == "tree":
            out.append(od.tree(parents(rng, n), 0, 32)[1])
        elif kind == "causal":
            out.append(np.tri(n, dtype=bool))
        elif kind == "none":
            out.append(np.zeros((n, n), dtype=bool))
        else:
            out.append(rng.random((n, n)) < 0.5)
    return out


def words(bt, seen, count=None, junk=False):
    """The masks as one tensor's rows, `junk` in the bits of tokens that are not there."""
    count = count or max(1, -(-max(bt.new) // 32))
    rows = []
    for n, m in zip(bt.new, seen):
        wide = np.ones((n, 32 * count), dtype=bool) if junk else np.zeros((n, 32 * count), dtype=bool)
        wide[:, :min(n, 32 * count)] = m[:, :32 * count]
        rows.append(od.words_of(wide, count))
    return ints(np.concatenate(rows)) if rows else ints(np.zeros((0, count)))


def attend(bt, q, scale, seen):
    """As Batch.attend: fp64 outputs, the largest sum |q||k|, the largest |v|."""
    out, reach, top = np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape[:2])
    group = bt.heads // bt.kv_heads
    for b, n in enumerate(bt.new):
        k, v, held = bt.sequence(b)
        first, length = bt.len[b] - n, k.shape[1]
        view = np.zeros((n, length), dtype=bool)
        view[:, :max(0, first)] = True
        for j in range(n):
            if 0 <= first + j < length:
                view[:, first + j] = seen[b][:, j]
        view &= held
        for h in range(bt.heads):
            rows = slice(bt.q_start[b], bt.q_start[b] + n)
            out[rows, h] = oa.attention(q[rows, h], k[h // group], v[h // group], view, scale)
            if length and n:
                mass = np.abs(q[rows, h]) @ np.abs(k[h // group]).T
                reach[rows, h] = np.nanmax(np.where(view, mass, 0), 1) * abs(scale)
                top[rows, h] = np.nanmax(np.abs(v[h // group]))
    return out, reach, top
