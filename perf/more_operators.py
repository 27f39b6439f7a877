"""Cases of one step with drafted tokens: the plan of a tree of drafts, rotation and append at positions that are not places,
attention of the tree over the 4-bit paged cache, verification against the target's probabilities, and keeping what was
accepted.

A layer whose experts come over the host link costs nearly the same for one token as for a few, so a step takes a sequence's
pending token and a tree of guesses behind it.  Tree token i (its number in the sequence's new tokens) is stored in place
kv_len - n + i, rotated for position kv_len - n + depth, and sees the cached tokens, its ancestors and itself.  Verification
walks down from the first new token; what is accepted moves to the places right behind the cached tokens.

Layers are those beside the package's own configurations (`workload.CONFIGS`: d_model 256, 2048 and 4096); trees have one to
some hundred tokens; contexts and vocabularies go from a few hundred to 131072.  `draw` spreads over what lies between and around.

Storage, as `attention` documents it: a cache is [pages][kv heads][record] bytes.  A record holds P tokens of one head: key
codes [P][D/2] (dimension c in nibble c % 2 of byte c / 2), value codes [P/4][D/8][4][4] (four tokens' eight dimensions side
by side), key metas [P][D/32] and value metas [P/4][D/32][4], uint16.  A meta is scale code k << 8 | zero z of 32 dimensions,
scale(k) = (8 + k % 8) * 2^(k/8 - 24), value = (q - z) * scale; k = 255 marks a group that reads as NaN.  q_start [B + 1]
bounds the sequences' new tokens, kv_len [B] counts their tokens with the new ones, row b of page_table names their pages.
"""
from __future__ import annotations

import math
import random

import torch

own = False
device = "cuda"

LAYER = dict(heads=32, kv_heads=8, head_dim=128)     # beside d_model 4096
FINE = dict(heads=16, kv_heads=16, head_dim=128)     # beside d_model 2048, every head with keys of its own
TINY = dict(heads=4, kv_heads=2, head_dim=64)        # beside d_model 256


def listed():
    return [
        # one sequence with seven drafts: latency alone
        dict(name="tree-one", op="tree", seqs=1, nodes=8, width=3, ctx=900),
        # 64 sequences of up to 509 drafts: long draws of a cheap draft
        dict(name="tree-batch", op="tree", seqs=64, nodes=509, width=6, ctx=4000),
        # 8 sequences of up to 16 tree tokens in a layer of the largest stack: the plan is there, append and read back
        dict(name="append-tree8", op="append", seqs=8, nodes=16, width=4, ctx=2048, page=16, dtype="bf16", **LAYER),
        # 48 sequences of up to 63, fp32 heads with keys of their own, pages of 64 tokens
        dict(name="append-tree48", op="append", seqs=48, nodes=63, width=4, ctx=129, page=64, dtype="f32", **FINE),
        # one sequence of the smallest stack, a tree of six
        dict(name="attn-one-tiny", op="attn", seqs=1, nodes=6, width=3, ctx=508, page=16, dtype="f32", **TINY),
        # 32 ragged sequences with eight tokens each, the ordinary serving step
        dict(name="attn-tree32", op="attn", seqs=32, nodes=8, width=3, ctx=4095, page=16, dtype="bf16", **LAYER),
        # one very long sequence, 24 tokens: few rows, the cache read by the whole chip
        dict(name="attn-long", op="attn", seqs=1, nodes=24, width=4, ctx=131071, page=64, dtype="bf16", **LAYER),
        # wide trees of up to 64 tokens over eight long sequences
        dict(name="attn-wide8", op="attn", seqs=8, nodes=64, width=8, ctx=16383, page=32, dtype="bf16", **LAYER),
        # one sequence, a chain of five drafts, a small vocabulary of odd size
        dict(name="verify-chain", op="verify", seqs=1, nodes=6, width=1, vocab=32001, dtype="f32", drawn=True),
        # 32 sequences with trees of up to 16, a large vocabulary
        dict(name="verify-tree32", op="verify", seqs=32, nodes=16, width=3, vocab=131072, dtype="bf16", drawn=True),
        # one sequence of the smallest stack, two layers
        dict(name="keep-one", op="keep", layers=2, seqs=1, nodes=8, width=3, ctx=500, page=16, **TINY),
        # all 32 layers of the largest stack, 32 sequences
        dict(name="keep-stack32", op="keep", layers=32, seqs=32, nodes=16, width=3, ctx=1000, page=16, **LAYER),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A power of two or an odd number, either spread over the logarithm."""
    if rng.random() < 0.4:
        return 1 << rng.randint(math.ceil(math.log2(lo)), int(math.log2(hi)))
    return min(_log(rng, lo, hi) | 1, hi)


def draw(rng):
    """A case between and around the listed ones."""
    op, dtype = rng.choice(("tree", "append", "attn", "attn", "verify", "verify", "keep")), rng.choice(("bf16", "bf16", "f32"))
    width = rng.choice((1, 2, 3, 4, 6, 9))
    if op == "tree":
        nodes = _size(rng, 1, 1024)
        return dict(op=op, seqs=_log(rng, 1, max(1, min(256, 16_000_000 // nodes ** 2))), nodes=nodes, width=width, ctx=_size(rng, 64, 4096))
    if op == "verify":
        nodes, vocab = _size(rng, 1, 64), _size(rng, 512, 262144)
        most = max(1, min(64, 67_000_000 // (nodes * vocab)))
        return dict(op=op, seqs=_log(rng, 1, most), nodes=nodes, width=width, vocab=vocab, dtype=dtype, drawn=rng.random() < 0.6)
    kv = rng.choice((1, 2, 4, 8, 16))
    heads = kv * rng.choice((1, 2, 4, 5, 8)) if kv < 16 else kv
    dim, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    shape = dict(heads=heads, kv_heads=kv, head_dim=dim)
    if op == "append":
        nodes = _size(rng, 1, 256)
        seqs = _log(rng, 1, max(1, min(64, int(1.8e7 / (nodes * (heads + 2 * kv) * dim)))))
        return dict(op=op, seqs=seqs, nodes=nodes, width=width, ctx=_size(rng, 1, 4096), page=page, dtype=dtype, **shape)
    if op == "keep":
        layers, nodes, ctx = _log(rng, 1, 48), _size(rng, 1, 64), _size(rng, 1, 2048)
        most = int(min(1.1e9 / (layers * (ctx + nodes + page) * kv * dim), 16384 / (layers * nodes) * 8 / kv * 128 / dim))
        return dict(op=op, layers=layers, seqs=_log(rng, 1, max(1, min(64, most))), nodes=nodes, width=width, ctx=ctx, page=page, **shape)
    nodes = rng.choice((rng.randint(1, 16), _size(rng, 1, 64), _size(rng, 1, 256)))
    seqs, ctx = _log(rng, 1, 64), _size(rng, 1, 131071)
    most = min(1.3e8 / (seqs * kv * dim), 2.5e8 / (seqs * heads * nodes))   # of the listed cases' padded keys and scores
    return dict(op=op, seqs=seqs, nodes=nodes, width=width, ctx=max(1, min(ctx, int(most) - nodes)), page=page, dtype=dtype, **shape)


# -- shapes of a ragged batch, from the case alone (trees that are planned or verified: from the seed too) ------------------

def _lengths(case, seed=None):
    """(new tokens, tokens already cached) of each sequence.  The first has the case's own; of the others some have their
    pending token alone, a tree of another size, or sit this step out."""
    ctx = case.get("ctx", 100)
    rng = random.Random("%s %d %d %d" % (case["op"], case["seqs"], case["nodes"], ctx))
    new, old = [case["nodes"]], [ctx]
    for _ in range(case["seqs"] - 1):
        new.append(rng.choice((0, 1, rng.randint(1, case["nodes"]), case["nodes"], case["nodes"], case["nodes"])))
        old.append(rng.choice((0, rng.randint(0, ctx), rng.randint(ctx // 2, ctx), ctx, ctx)))
    if seed is not None:
        rng = random.Random(seed)
        old = [rng.randint(0, ctx) for _ in old]
    return new, old


def _parents(case, seed=None):
    """The parent of every new token, -1 for a sequence's first.  Tree token i follows one of the `width` before it; with a
    width of 1 that is a chain."""
    rng = random.Random("tree %d %d %s" % (case["nodes"], case["width"], seed))
    return [[-1] + [i - 1 - rng.randrange(min(i, case["width"])) for i in range(1, n)] if n else [] for n in _lengths(case)[0]]


def _depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _pages(case):
    new, old = _lengths(case)
    return [-(-(a + b) // case["page"]) for a, b in zip(new, old)]


def _words(case):
    return -(-case["nodes"] // 32)


def work(case):
    new, old = _lengths(case)
    tokens = sum(new)
    if case["op"] == "tree":    # parents in; positions and bits out
        return {"bytes": 4 * tokens * (2 + _words(case)) + 8 * len(new), "flops": tokens * _words(case)}
    b = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "verify":  # the distributions where each sequence's walk ends; the walk's own entries are few
        rows = 2 if case["drawn"] else 1
        busy = sum(n > 0 for n in new)
        return {"bytes": busy * case["vocab"] * rows * b + 12 * tokens, "flops": busy * case["vocab"] * 2 * rows}
    hq, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    entry = hk * d * 9 // 8     # bytes of a token's keys and values
    if case["op"] == "append":  # queries, keys and values in; rotated queries, the entries and their values out
        return {"bytes": tokens * ((2 * hq + 4 * hk) * d * b + entry + 4 * d), "flops": tokens * (hq + 4 * hk) * d * 6}
    if case["op"] == "keep":    # a third of a tree's depth is accepted: read and written in every layer
        kept = sum(max(_depths(p)) / 3 for p in _parents(case) if p)
        return {"bytes": 2 * case["layers"] * kept * entry + 4 * tokens, "flops": 0}
    seen = sum(n * o for n, o in zip(new, old)) + sum(sum(_depths(p)) + len(p) for p in _parents(case))
    return {"bytes": 2 * tokens * hq * d * b + sum(n and n + o for n, o in zip(new, old)) * entry, "flops": 4 * d * hq * seen}


# -- inputs ------------------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=device)


def _accepted(case, seed):
    """A path down each tree, ended by chance at every step: local numbers, -1 behind the last."""
    rng, path, count = random.Random(seed), [], []
    for parents in _parents(case):
        at, mine = 0, [0] if parents else []
        while parents:
            children = [i for i, p in enumerate(parents) if p == at]
            if not children or rng.random() < 0.25:
                break
            at = rng.choice(children)
            mine.append(at)
        count.append(len(mine))
        path += mine + [-1] * (len(parents) - len(mine))
    return _ints(path), _ints(count)


def prepare(case, seed):
    gen = torch.Generator(device=device).manual_seed(seed * 2 + 1)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=device)

    state = dict(case=dict(case))
    shape = seed if case["op"] in ("tree", "verify") else None
    new, old = _lengths(case, shape)
    tokens = sum(new)
    state["parent"] = _ints([p for ps in _parents(case, shape) for p in ps])
    state["q_start"] = _ints([sum(new[:b]) for b in range(len(new) + 1)])
    state["kv_len"] = _ints([a + b for a, b in zip(new, old)])
    state["max_new"], state["max_len"] = max(new), max(a + b for a, b in zip(new, old))
    if case["op"] == "tree":
        return state
    if case["op"] == "verify":
        # the target's logits, a few far above the others; the draft's are near them
        v, dtype = case["vocab"], _dtype(case)
        z = normal(tokens, v)
        z = z + 0.9 * z * z.abs()
        near = z + 0.5 * normal(tokens, v)
        state["p"], q = torch.softmax(z, 1).to(dtype), torch.softmax(near, 1)
        parent = state["parent"].tolist()
        ids, at = [0] * tokens, 0
        seen = {}
        if case["drawn"]:   # children drawn from the draft's distribution of their parent
            state["q"] = q.to(dtype)
            drawn = torch.multinomial(q, max(case["width"], 1), replacement=True, generator=gen).tolist()
        else:               # or its likeliest tokens in turn
            state["q"] = None
            drawn = torch.topk(q, min(v, max(case["width"], 1)), dim=1).indices.tolist()
        for n in new:
            for i in range(1, n):
                p = at + parent[at + i]
                ids[at + i] = drawn[p][seen.get(p, 0) % len(drawn[p])]
                seen[p] = seen.get(p, 0) + 1
            at += n
        state["tokens"] = _ints(ids)
        state["u"] = torch.rand(tokens, generator=gen, device=device)
        return state

    hq, hk, d, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    need = _pages(case)
    order = torch.randperm(sum(need) + 2, generator=gen, device=device).int().tolist()
    table = torch.full((len(need), max(1, max(need))), -1, dtype=torch.int32)
    for b, m in enumerate(need):
        table[b, :m] = torch.tensor(order[sum(need[:b]):sum(need[:b]) + m], dtype=torch.int32)
    state["page_table"] = table.to(device)
    record = page * d * 9 // 8
    if case["op"] == "keep":
        # bytes of entries as they come; this moves them whole
        state["pools"] = [torch.randint(0, 256, (len(order), hk, record), generator=gen, device=device, dtype=torch.uint8)
                          for _ in range(case["layers"])]
        state["path"], state["count"] = _accepted(case, seed)
        return state
    state["pool"] = torch.zeros((len(order), hk, record), dtype=torch.uint8, device=device)
    state["pos"], state["seen"] = _plain_tree(state)
    if case["op"] == "append":
        # what the joined projection leaves: queries, keys and values side by side
        qkv = normal(tokens, (hq + 2 * hk) * d).to(_dtype(case))
        state["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
        state["k"] = qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        state["v"] = qkv[:, (hq + hk) * d:].unflatten(1, (hk, d))
        angle = torch.arange(state["max_len"], dtype=torch.float64, device=device)[:, None] * (
            10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device=device) / d))
        state["cos"], state["sin"] = angle.cos().float(), angle.sin().float()
        return state
    state["q"] = (normal(tokens, hq, d) * 1.5).to(_dtype(case))
    # a filled cache: keys with a few strong dimensions, a whole page of every head at a time
    strong = torch.exp(0.7 * normal(2, hk, 1, d))
    per = max(1, (1 << 25) // (hk * page * d))
    for p in range(0, len(order), per):
        part = min(per, len(order) - p)
        values = normal(2, part, hk, page, d) * strong[:, None]
        state["pool"][p:p + part] = _records(*_quantize(values[0]), *_quantize(values[1]))
    state["scale"] = d ** -0.5
    return state


# -- plain forms -------------------------------------------------------------------------------------------------------------

def _quantize(x):
    """Codes and metas of x [..., d], fp32."""
    g = x.unflatten(-1, (-1, 32))
    fine = torch.isfinite(g).all(-1)
    g = torch.where(fine[..., None], g, 0.0)
    lo, hi = g.amin(-1).clamp(max=0), g.amax(-1).clamp(min=0)
    # the smallest scale that spans hi - lo in 15 steps: the code just below a fifteenth of it, or the next one
    k = torch.clamp((((hi - lo) * (1 / 15)).view(torch.int32) >> 20) - 848, 0, 254)
    k = torch.clamp(k + (15 * ((k + 848) << 20).view(torch.float32) < hi - lo), max=254)
    s = ((k + 848) << 20).view(torch.float32)
    z = torch.clamp(torch.round(-lo / s), 0, 15)
    q = torch.clamp(torch.round(g / s[..., None]) + z[..., None], 0, 15) * fine[..., None]
    k, z = torch.where(fine, k, 255), torch.where(fine, z, 0.0)
    return q.flatten(-2).to(torch.uint8), k << 8 | z.int()


def _records(kq, km, vq, vm):
    """Records [..., bytes] of whole pages: codes [..., P, d] and metas [..., P, d / 32] of keys and values."""
    vq = vq.unflatten(-2, (-1, 4)).unflatten(-1, (-1, 8)).transpose(-3, -2)
    vm = vm.unflatten(-2, (-1, 4)).transpose(-2, -1)
    parts = [c[..., 0::2] | c[..., 1::2] << 4 for c in (kq, vq)]
    parts += [torch.stack([m & 255, m >> 8], -1).to(torch.uint8) for m in (km, vm)]
    lead = kq.dim() - 2
    return torch.cat([p.flatten(lead) for p in parts], -1)


def _scaled(q, m):
    """Values of codes q [..., d] and metas [..., d / 32, 2], bytes."""
    code = m[..., 1].int()
    s = torch.where(code == 255, math.nan, ((code + 848) << 20).view(torch.float32))
    return ((q.unflatten(-1, (-1, 32)).float() - m[..., 0].float()[..., None]) * s[..., None]).flatten(-2)


def _values(rec, page, d):
    """Keys and values [..., P, d], fp32, of records [..., bytes]."""
    lead = rec.dim() - 1
    kc, vc, km, vm = rec.split([page * d // 2, page * d // 2, page * d // 16, page * d // 16], -1)
    kq = torch.stack([kc & 15, kc >> 4], -1).flatten(lead).unflatten(-1, (page, d))
    vq = torch.stack([vc & 15, vc >> 4], -1).flatten(lead).unflatten(-1, (page // 4, d // 8, 4, 8))
    vq = vq.transpose(-3, -2).reshape(*rec.shape[:-1], page, d)
    vm = vm.unflatten(-1, (page // 4, d // 32, 4, 2)).transpose(-3, -2).reshape(*rec.shape[:-1], page, d // 32, 2)
    return _scaled(kq, km.unflatten(-1, (page, d // 32, 2))), _scaled(vq, vm)


def _places(s):
    """Sequence, number in it and place of every new token."""
    start, tokens = s["q_start"].long(), s["parent"].shape[0]
    at = torch.arange(tokens, device=device)
    seq = torch.searchsorted(start[1:], at, right=True)
    return seq, at - start[seq], s["kv_len"].long()[seq] - start[seq + 1] + at


def _entry_bytes(s, seq, pos):
    """Offsets in a pool of the bytes of places pos: key codes, value codes, key metas, value metas, [tokens, heads, n] each."""
    c = s["case"]
    d, page = c["head_dim"], c["page"]
    rec = s["page_table"][seq, pos // page].long()
    t, heads = (pos % page)[:, None, None], torch.arange(c["kv_heads"], device=device)[None, :, None]
    base = (rec[:, None, None] * c["kv_heads"] + heads) * (page * d * 9 // 8)
    j, g = torch.arange(d // 2, device=device), torch.arange(d // 16, device=device)
    return (base + t * (d // 2) + j, base + page * d // 2 + (t // 4) * (d * 2) + j // 4 * 16 + t % 4 * 4 + j % 4,
            base + page * d + t * (d // 16) + g, base + page * d + page * d // 16 + (t // 4) * (d // 4) + g // 2 * 8 + t % 4 * 2 + g % 2)


def _plain_tree(s):
    seq, i, place = _places(s)
    b, n = s["kv_len"].shape[0], s["max_new"]
    parent = s["parent"].long()
    # who is reached in up to 1, 2, 4 .. steps up: [B, n, n]
    reach = torch.zeros((b, n, n), device=device)
    reach[:, torch.arange(n), torch.arange(n)] = 1
    reach[seq, i, torch.where((parent >= 0) & (parent < i), parent, i)] = 1
    for _ in range((n - 1).bit_length()):
        reach = torch.matmul(reach, reach).clamp_(max=1)
    reach = reach[seq, i]
    pos = place - i + reach.sum(1).long() - 1
    bits = torch.nn.functional.pad(reach, (0, -n % 32)).long().unflatten(1, (-1, 32)) << torch.arange(32, device=device)
    return pos.int(), bits.sum(-1).to(torch.int32)


def _plain_append(s):
    seq, _, place = _places(s)
    pos = s["pos"].long()
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]

    def rotate(x):
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    def both(m):
        return torch.stack([m & 255, m >> 8], -1).flatten(-2).to(torch.uint8)

    kq, km = _quantize(rotate(s["k"]))
    vq, vm = _quantize(s["v"].float())
    flat, at = s["pool"].view(-1), _entry_bytes(s, seq, place)
    bytes_ = torch.cat([kq[..., 0::2] | kq[..., 1::2] << 4, vq[..., 0::2] | vq[..., 1::2] << 4, both(km), both(vm)], -1)
    flat[torch.cat(at, -1)] = bytes_
    q = rotate(s["q"]).to(s["q"].dtype)
    # what the cache now holds for these tokens
    kc, vc, km, vm = (flat[a] for a in at)
    k, v = (_scaled(torch.stack([c & 15, c >> 4], -1).flatten(-2), m.unflatten(-1, (-1, 2))).to(s["k"].dtype) for c, m in ((kc, km), (vc, vm)))
    return {"q": q, "k": k, "v": v}


def _plain_attention(s):
    c = s["case"]
    d, page, hk, n = c["head_dim"], c["page"], c["kv_heads"], s["max_new"]
    seq, i, _ = _places(s)
    table, b = s["page_table"].long(), s["page_table"].shape[0]
    k, v = _values(s["pool"][table.clamp(min=0)], page, d)              # [B, pages, heads, P, d]
    k, v = (x.transpose(2, 3).flatten(1, 2).permute(0, 2, 1, 3) for x in (k, v))  # [B, heads, tokens, d]
    length = s["kv_len"].long()
    at = torch.arange(k.shape[2], device=device)
    held = (at < length[:, None])[:, None, :, None]
    k, v = torch.where(held, k, 0.0), torch.where(held, v, 0.0)
    # queries of each sequence side by side, padded to the most: [B, kv heads, group, new, d]
    q = torch.zeros((b, n, c["heads"], d), device=device)
    q[seq, i] = s["q"].float()
    q = q.unflatten(2, (hk, -1)).permute(0, 2, 3, 1, 4)
    score = torch.matmul(q.flatten(2, 3), k.transpose(2, 3).contiguous()).unflatten(2, (-1, n)) * s["scale"]
    # cached tokens, and of the new ones those whose bits are set
    fresh = at - (length - (s["q_start"][1:] - s["q_start"][:-1]).long())[:, None]
    bits = torch.zeros((b, n, s["seen"].shape[1]), dtype=torch.int32, device=device)
    bits[seq, i] = s["seen"]
    word = (fresh // 32).clamp(0, bits.shape[2] - 1)[:, None, :].expand(-1, n, -1)
    seen = (bits.gather(2, word) >> (fresh % 32)[:, None]) & 1 == 1
    seen = ((fresh < 0)[:, None] | seen) & (at < length[:, None])[:, None]
    score = score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (-1, n)) / torch.where(total == 0, 1.0, total)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, i].to(s["q"].dtype)


def _plain_verify(s):
    """In 64 bits: a decision next to a border must not depend on the order of a sum."""
    seq, i, _ = _places(s)
    b, n, vocab = s["kv_len"].shape[0], s["max_new"], s["p"].shape[1]
    tokens = i.shape[0]
    me = torch.arange(tokens, device=device)
    parent = torch.where(i > 0, me - i + s["parent"].long(), me)
    ids, u, drawn = s["tokens"].long(), s["u"].double().clamp(min=0), s["q"] is not None
    # older siblings of every token, and how many children each has
    sibling = (parent[:, None] == parent[None]) & (me[None] < me[:, None]) & (i > 0) & (i > 0)[:, None]
    rank, children = sibling.sum(1), torch.zeros(tokens, dtype=torch.long, device=device).index_add_(0, parent, (i > 0).long())
    p_id = s["p"][parent, ids].double()
    if drawn:
        # share[t, k] of q is taken from p once k children of t are refused, which leaves left[t, k]
        most = int(children.max()) if tokens else 0
        share, left = torch.zeros((2, tokens, most + 1), dtype=torch.float64, device=device)
        left[:, 0] = 1
        for k in range(1, most + 1):
            share[:, k] = share[:, k - 1] + left[:, k - 1]
            rows = torch.nonzero(children > k)[:, 0]
            left[rows, k] = (s["p"][rows].double() - share[rows, k, None] * s["q"][rows].double()).clamp(min=0).sum(1)
        q_id = s["q"][parent, ids].double()
        good = u * left[parent, rank] * q_id < (p_id - share[parent, rank] * q_id).clamp(min=0)
    else:
        same = sibling & (ids[:, None] == ids[None])
        first = ~same.any(1)
        gone = torch.where(sibling & first[None], p_id[None], 0.0).sum(1)
        good = u * (1 - gone).clamp(min=0) < torch.where(first, p_id, 0.0)
    # the first good child of each token; a token is accepted if it and all above it are that
    best = torch.full((tokens,), tokens, device=device).scatter_reduce_(0, parent, torch.where(good & (i > 0), me, tokens), "amin")
    up, fine, depth = parent, (i == 0) | (best[parent] == me), (i > 0).long()
    for _ in range((n - 1).bit_length()):
        fine, depth, up = fine & fine[up], depth + depth[up], up[up]
    path = torch.full((tokens + 1,), -1, dtype=torch.long, device=device)
    path[torch.where(fine, me - i + depth, tokens)] = i
    path[tokens] = -1
    count = torch.zeros(b, dtype=torch.long, device=device).index_add_(0, seq, fine.long())
    # the next token from what is left where the path ends
    start = s["q_start"].long()[:-1]
    busy = count > 0
    end = (start + path[(start + count - 1).clamp(min=0)]).clamp(min=0, max=max(tokens - 1, 0))
    row = s["p"][end].double()
    if drawn:
        rest = (row - share[end, children[end], None] * s["q"][end].double()).clamp_(min=0)
    else:
        tried = torch.zeros((tokens, vocab), dtype=torch.bool, device=device)
        tried[torch.where(i > 0, parent, me)[i > 0], ids[i > 0]] = True
        rest = torch.where(tried[end], 0.0, row.clamp(min=0))
    total = rest.sum(1, keepdim=True)
    rest = torch.where(total == 0, row.clamp(min=0), rest)
    total = rest.sum(1, keepdim=True)
    at = torch.arange(vocab, device=device)
    over = (rest.cumsum(1) > u[start.clamp(max=tokens - 1)][:, None] * total) & (rest > 0)
    pick = torch.where(over, at, vocab).amin(1)
    pick = torch.where(pick == vocab, torch.where(rest > 0, at, -1).amax(1), pick)
    pick = torch.where(busy & torch.isfinite(total[:, 0]), pick, -1)
    return {"path": path[:tokens].int(), "count": count.int(), "next": pick.int()}


def _plain_keep(s):
    seq, i, place = _places(s)
    inside = i < s["count"].long()[seq]
    moved = torch.where(inside, place - i + s["path"].long(), place)
    to, source = (torch.cat(_entry_bytes(s, seq, at), -1) for at in (place, moved))
    for pool in s["pools"]:
        flat = pool.view(-1)
        flat[to] = flat[source]
    return s["pools"]


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"tree": _plain_tree, "append": _plain_append, "attn": _plain_attention, "verify": _plain_verify, "keep": _plain_keep}[op](s)
    from paper_2511_05814_amd import attention, drafts
    if op == "tree":
        return drafts.draft_tree(s["parent"], s["q_start"], s["kv_len"], s["max_new"])
    if op == "append":
        plan = s["pool"], s["page_table"], s["q_start"], s["kv_len"]
        q = attention.kv4_append(s["q"], s["k"], s["v"], s["cos"], s["sin"], *plan, pos=s["pos"])
        k, v = attention.kv4_read(*plan, q.shape[0], q.shape[2], q.dtype)
        return {"q": q, "k": k, "v": v}
    if op == "attn":
        return attention.kv4_tree_attention(s["q"], s["pool"], s["page_table"], s["q_start"], s["kv_len"], s["seen"], s["scale"],
                                            max_new=s["max_new"], max_len=s["max_len"])
    if op == "verify":
        path, count, after = drafts.verify_drafts(s["p"], s["tokens"], s["parent"], s["u"], s["q_start"], q=s["q"])
        return {"path": path, "count": count, "next": after}
    attention.kv4_keep(s["pools"], s["page_table"], s["q_start"], s["kv_len"], s["path"], s["count"], s["case"]["head_dim"])
    return s["pools"]


# -- the definitions in 64 bits --------------------------------------------------------------------------------------------

def _exact_store(x):
    """Values that a cache holds for x [tokens, heads, d], fp64."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    bottom, top = torch.clamp(g.min(-1).values, max=0.0), torch.clamp(g.max(-1).values, min=0.0)
    steps = torch.tensor([(8 + k % 8) * 2.0 ** (k // 8 - 24) for k in range(255)], dtype=torch.float64, device=x.device)
    s = steps[torch.clamp(torch.searchsorted(15 * steps, top - bottom), max=254)].unsqueeze(-1)
    z = torch.clamp(torch.round(-bottom.unsqueeze(-1) / s), 0, 15)
    return ((torch.clamp(torch.round(g / s) + z, 0, 15) - z) * s).reshape(x.shape)


def _exact_append(case, s):
    new, old = _lengths(case)
    pos = torch.tensor([o + t for o, p in zip(old, _parents(case)) for t in _depths(p)], device=device)
    half = case["head_dim"] // 2
    c, n = s["cos"].double()[pos].unsqueeze(1), s["sin"].double()[pos].unsqueeze(1)
    turned = []
    for x in (s["q"].double(), s["k"].double()):
        y = torch.empty_like(x)
        y[..., :half] = x[..., :half] * c - x[..., half:] * n
        y[..., half:] = x[..., half:] * c + x[..., :half] * n
        turned.append(y)
    return {"q": turned[0], "k": _exact_store(turned[1]), "v": _exact_store(s["v"].double())}


def _exact_attention(case, s):
    d, page, hk = case["head_dim"], case["page"], case["kv_heads"]
    new, old = _lengths(case)
    out, at = torch.zeros(s["q"].shape, dtype=torch.float64, device=device), 0
    code = torch.arange(255, dtype=torch.float64, device=device)
    steps = (8 + code % 8) * 2.0 ** (code // 8 - 24)
    group = case["heads"] // hk
    for b, (n, o, parents) in enumerate(zip(new, old, _parents(case))):
        if n == 0:
            continue
        length = n + o
        seen = torch.zeros((n, length), dtype=torch.bool)
        seen[:, :o] = True
        for i, p in enumerate(parents):
            if p >= 0:
                seen[i] = seen[p]
            seen[i, o + i] = True
        seen = seen.to(device)
        ids = s["page_table"][b, :-(-length // page)].long()
        tok, dim = torch.arange(length, device=device), torch.arange(d, device=device)
        rec = s["pool"][ids].view(len(ids), hk, -1)
        mine, t = (tok // page)[:, None], (tok % page)[:, None]
        for h in range(hk):
            r = rec[:, h]
            kc = r[mine, t * (d // 2) + dim // 2]
            vc = r[mine, page * d // 2 + t // 4 * (2 * d) + dim // 8 * 16 + t % 4 * 4 + dim % 8 // 2]
            km = page * d + (t * (d // 32) + dim // 32) * 2
            vm = page * d * 17 // 16 + ((t // 4 * (d // 32) + dim // 32) * 4 + t % 4) * 2
            kv = [(((raw.long() >> dim % 2 * 4) & 15) - r[mine, m].long()) * steps[r[mine, m + 1].long()] for raw, m in ((kc, km), (vc, vm))]
            q = s["q"][at:at + n, h * group:(h + 1) * group].double()
            w = torch.matmul(q.transpose(0, 1).reshape(-1, d), kv[0].t().contiguous()).view(group, n, length) * s["scale"]
            w.masked_fill_(~seen, -math.inf)
            o_h = torch.matmul(torch.softmax(w, -1).view(-1, length), kv[1]).view(group, n, d)
            out[at:at + n, h * group:(h + 1) * group] = o_h.transpose(0, 1)
        at += n
    return out


def _exact_verify(case, s, seed):
    path, count, after, at = [], [], [], 0
    ids, u = s["tokens"].tolist(), s["u"].double().tolist()
    for parents in _parents(case, seed):
        n = len(parents)
        if n == 0:
            count.append(0)
            after.append(-1)
            continue
        mine = [0]
        while True:
            t = at + mine[-1]
            rest, left, accepted = s["p"][t].double(), 1.0, None
            for c in (i for i, p in enumerate(parents) if p == mine[-1]):
                guess = torch.zeros_like(rest) if s["q"] is None else s["q"][t].double()
                if s["q"] is None:
                    guess[ids[at + c]] = 1
                if u[at + c] * left * float(guess[ids[at + c]]) < float(rest[ids[at + c]]):
                    accepted = c
                    break
                if s["q"] is None:
                    left = max(0.0, left - float(rest[ids[at + c]]))
                    rest = torch.where(guess == 1, 0.0, rest)
                else:
                    rest = torch.clamp(rest - left * guess, min=0.0)
                    left = float(rest.sum())
            if accepted is None:
                break
            mine.append(accepted)
        rest = s["p"][at + mine[-1]].double() if float(rest.sum()) == 0 else rest
        over = torch.nonzero((torch.cumsum(rest, 0) > u[at] * rest.sum()) & (rest > 0))
        after.append(int(over[0]) if len(over) else int(torch.nonzero(rest > 0)[-1]))
        count.append(len(mine))
        path += mine + [-1] * (n - len(mine))
        at += n
    return {"path": _ints(path), "count": _ints(count), "next": _ints(after)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, s)
    if case["op"] == "attn":
        return _exact_attention(case, s)
    if case["op"] == "verify":
        return _exact_verify(case, s, seed)
    new, old = _lengths(case, seed if case["op"] == "tree" else None)
    if case["op"] == "tree":
        pos = [o + t for o, p in zip(old, _parents(case, seed)) for t in _depths(p)]
        rows = []
        for parents in _parents(case, seed):
            mask = []
            for i, p in enumerate(parents):
                mask.append(1 << i | (mask[p] if p >= 0 else 0))
            rows += [[(m >> 32 * w & 0xFFFFFFFF) - ((m >> 32 * w + 31 & 1) << 32) for w in range(_words(case))] for m in mask]
        return _ints(pos), _ints(rows)
    page, d = case["page"], case["head_dim"]
    table, path, count, at = s["page_table"].tolist(), s["path"].tolist(), s["count"].tolist(), 0

    def views(pool, b, place):
        """The four pieces of an entry, all heads."""
        rec, t = pool[table[b][place // page]], place % page
        k, v, km, vm = rec.split([page * d // 2, page * d // 2, page * d // 16, page * d // 16], -1)
        return (k.unflatten(-1, (page, -1))[:, t], v.unflatten(-1, (page // 4, d // 8, 4, 4))[:, t // 4, :, t % 4],
                km.unflatten(-1, (page, -1))[:, t], vm.unflatten(-1, (page // 4, d // 32, 4, 2))[:, t // 4, :, t % 4])

    if case["layers"] * sum(count) > 8000:
        return None
    pools = [p.cpu() for p in s["pools"]]
    for b, (n, o) in enumerate(zip(new, old)):
        for pool in pools:
            for k in range(count[b]):   # ascending: a place is written after it was read
                for to, source in zip(views(pool, b, o + k), views(pool, b, o + path[at + k])):
                    to.copy_(source.clone())
        at += n
    return [p.to(device) for p in pools]
