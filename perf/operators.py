"""Cases of the attention half of a decoder layer: products with 4-bit weights, rotation and append to a 4-bit paged
cache, attention over that cache, and the norms around a block.

The sizes are those of layers beside the package's own MoE configurations (`workload.CONFIGS`: d_model 256, 512, 2048 and
4096): heads of 64 or 128, all heads with keys of their own or four to a key head, contexts from a few tokens to 131072.
`draw` spreads over what lies between and around them.

Storage, as `attention` documents it:

* 4-bit weights [n][k], k a multiple of 64: planes back to back, codes [n][k/2] (column c in nibble c % 2 of byte c / 2),
  fp16 scales [n][k/64], uint8 zero codes [n][k/64]; weight = (q - zero / 16) * scale.
* A cache is [pages][kv heads][record] bytes.  A record holds P tokens of one head: key codes [P][D/2], value codes
  [P/4][D/8][4][4] (four tokens' eight dimensions side by side), key metas [P][D/32] and value metas [P/4][D/32][4], uint16.
  A meta is scale code k << 8 | zero z of 32 dimensions, scale(k) = (8 + k % 8) * 2^(k/8 - 24), value = (q - z) * scale;
  k = 255 stands for a group that held an infinity or a NaN and reads as NaN.
* A batch of B sequences: q_start [B + 1] bounds their new tokens, kv_len [B] counts their tokens with the new ones, row b
  of page_table names their pages in order.  New token i of sequence b has position kv_len[b] - n_b + i.
"""
from __future__ import annotations

import math
import random

import torch

own = False

LAYER = dict(heads=32, kv_heads=8, head_dim=128)     # beside d_model 4096
FINE = dict(heads=16, kv_heads=16, head_dim=128)     # beside d_model 2048, every head with keys of its own
TINY = dict(heads=4, kv_heads=2, head_dim=64)        # beside d_model 256


def listed():
    return [
        # one token through the smallest projection: latency alone
        dict(name="q4-one-tiny", op="q4", rows=1, n=512, k=512, dtype="f32"),
        # one token through the joined query, key and value projection of a d 4096 layer
        dict(name="q4-one-layer", op="q4", rows=1, n=6144, k=4096, dtype="bf16"),
        # 13 sequences decoding together, an odd number of output rows
        dict(name="q4-batch13", op="q4", rows=13, n=4099, k=2048, dtype="f32"),
        # a prompt of ragged length through the joined projection
        dict(name="q4-prompt", op="q4", rows=2037, n=6144, k=4096, dtype="bf16"),
        # 8 sequences decoding together: one new token each
        dict(name="append-decode8", op="append", seqs=8, new=1, ctx=2048, page=16, dtype="bf16", **LAYER),
        # three prompts of ragged lengths into fp32 heads, pages of 64 tokens
        dict(name="append-prompt", op="append", seqs=3, new=4096, ctx=129, page=64, dtype="f32", **FINE),
        # one sequence of the smallest stack after some hundred tokens
        dict(name="attn-one-tiny", op="attn", seqs=1, new=1, ctx=508, page=16, dtype="f32", **TINY),
        # 32 sequences of ragged lengths decoding together, the ordinary serving step
        dict(name="attn-decode32", op="attn", seqs=32, new=1, ctx=4095, page=16, dtype="bf16", **LAYER),
        # one very long sequence: few rows, the cache read by the whole chip
        dict(name="attn-long", op="attn", seqs=1, new=1, ctx=131071, page=64, dtype="bf16", **LAYER),
        # the later parts of four prompts, ragged, over what is already cached
        dict(name="attn-prompt", op="attn", seqs=4, new=2048, ctx=2048, page=32, dtype="bf16", **LAYER),
        # the hand-over between attention and the experts for one token
        dict(name="norm-one", op="norm", rows=1, d=4096, dtype="bf16", per_token_gate=False),
        # the same for a prompt, with a gate of every token's own
        dict(name="norm-prompt", op="norm", rows=4093, d=4096, dtype="bf16", per_token_gate=True),
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
    op, dtype = rng.choice(("q4", "append", "attn", "attn", "norm")), rng.choice(("bf16", "bf16", "f32"))
    if op == "q4":
        n, k = _size(rng, 64, 16384), 64 * _size(rng, 1, 223)
        most = int(min(4096, 5e10 / (n * k)))  # of the listed prompt's products
        rows = rng.randint(1, 16) if rng.random() < 0.5 else _size(rng, 1, max(1, most))
        return dict(op=op, rows=max(1, min(rows, most)), n=n, k=k, dtype=dtype)
    if op == "norm":
        d = 8 * _size(rng, 8, 1024)
        return dict(op=op, rows=_size(rng, 1, min(8192, 16700000 // d)), d=d, dtype=dtype, per_token_gate=rng.random() < 0.5)
    kv = rng.choice((1, 2, 4, 8, 16))
    heads = kv * rng.choice((1, 2, 4, 5, 8)) if kv < 16 else kv
    dim, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    seqs = _log(rng, 1, 64)
    shape = dict(heads=heads, kv_heads=kv, head_dim=dim)
    if op == "append":
        new = rng.choice((1, _size(rng, 1, 4096)))
        new = max(1, min(new, int(2.5e7 / (seqs * (heads + 2 * kv) * dim))))
        return dict(op=op, seqs=seqs, new=new, ctx=_size(rng, 1, 4096), page=page, dtype=dtype, **shape)
    new = rng.choice((1, 1, rng.randint(1, 9), _size(rng, 16, 2048)))
    ctx = _size(rng, 1, 131071)
    most = 1.3e8 / (seqs * kv * dim)                                    # of the listed cases' padded keys
    ctx = max(1, min(ctx, int(most) - new, int(1.0e9 / (seqs * heads * new)) - new))
    new = max(1, min(new, int(2.0e9 / (seqs * heads * (ctx + new)))))
    return dict(op=op, seqs=seqs, new=new, ctx=ctx, page=page, dtype=dtype, **shape)


# -- lengths of a ragged batch, from the case alone -----------------------------------------------------------------------

def _lengths(case):
    """(new tokens, tokens already cached) of each sequence.  The first has the case's own; of the others some have a single
    token, none cached or, in a prompt, none at all."""
    rng = random.Random("%(op)s %(seqs)d %(new)d %(ctx)d %(heads)d" % case)
    new, old = [case["new"]], [case["ctx"]]
    for _ in range(case["seqs"] - 1):
        new.append(1 if case["new"] == 1 else rng.choice((0, 1, rng.randint(1, case["new"]), rng.randint(1, case["new"]))))
        old.append(rng.choice((0, rng.randint(0, case["ctx"]), rng.randint(case["ctx"] // 2, case["ctx"]), case["ctx"])))
    return new, old


def _pages(case):
    new, old = _lengths(case)
    return [-(-(a + b) // case["page"]) for a, b in zip(new, old)]


def _visible(case):
    """Pairs of a new token and a token that it attends to."""
    new, old = _lengths(case)
    return sum(n * o + n * (n + 1) // 2 for n, o in zip(new, old))


def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "q4":
        t, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": n * k // 2 + 3 * (n * k // 64) + t * (n + k) * b, "flops": 2 * t * n * k}
    if case["op"] == "norm":
        t, d = case["rows"], case["d"]
        return {"bytes": t * d * (4 + 4 + 2 * b + (4 if case["per_token_gate"] else 0)) + 12 * d, "flops": 12 * t * d}
    new, old = _lengths(case)
    hq, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    tokens, entry = sum(new), hk * d * 9 // 8   # bytes of a token's keys and values
    if case["op"] == "append":  # queries, keys and values in; rotated queries, the entries and their values out
        return {"bytes": tokens * ((2 * hq + 4 * hk) * d * b + entry + 4 * d), "flops": tokens * (hq + 4 * hk) * d * 6}
    return {"bytes": 2 * tokens * hq * d * b + sum(n and n + o for n, o in zip(new, old)) * entry, "flops": 4 * d * hq * _visible(case)}


# -- inputs ------------------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 2 + 1)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    state = dict(case=dict(case))
    if case["op"] == "q4":
        n, k = case["n"], case["k"]
        w = normal(n, k // 64, 64) * 0.02
        lo, hi = w.amin(2), w.amax(2)
        scale = ((hi - lo) / 15).half()
        zero = torch.clamp(torch.round(-lo / scale.float() * 16), 0, 255)
        q = torch.clamp(torch.round(w / scale.float()[:, :, None] + zero[:, :, None] / 16), 0, 15).to(torch.uint8).view(n, k)
        state["w"] = torch.cat([(q[:, 0::2] | q[:, 1::2] << 4).reshape(-1), scale.view(torch.uint8).reshape(-1),
                                zero.to(torch.uint8).reshape(-1)])
        # a normed hidden state: a few channels far above the others
        state["x"] = (normal(case["rows"], k) * torch.exp(0.5 * normal(k))).to(_dtype(case))
        return state
    if case["op"] == "norm":
        t, d = case["rows"], case["d"]
        state["h"] = normal(t, d) * torch.exp(0.5 * normal(d))
        state["y"] = normal(t, d).to(_dtype(case))
        state["gate"] = 0.5 * normal(t, d) if case["per_token_gate"] else 0.5 * normal(d)
        state["post"], state["pre"] = 1 + 0.1 * normal(d), 1 + 0.1 * normal(d)
        return state

    new, old = _lengths(case)
    hq, hk, d, page, tokens = case["heads"], case["kv_heads"], case["head_dim"], case["page"], sum(new)
    need = _pages(case)
    order = torch.randperm(sum(need) + 2, generator=gen, device="cuda").int().tolist()
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32)
    for b, m in enumerate(need):
        table[b, :m] = torch.tensor(order[sum(need[:b]):sum(need[:b]) + m], dtype=torch.int32)
    state["page_table"] = table.cuda()
    state["q_start"] = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32).cuda()
    state["kv_len"] = torch.tensor([a + b for a, b in zip(new, old)], dtype=torch.int32).cuda()
    state["max_new"], state["max_len"] = max(new), max(a + b for a, b in zip(new, old))
    state["pool"] = torch.zeros((len(order), hk, page * d * 9 // 8), dtype=torch.uint8, device="cuda")
    if case["op"] == "append":
        # what the joined projection leaves: queries, keys and values side by side
        qkv = normal(tokens, (hq + 2 * hk) * d).to(_dtype(case))
        state["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
        state["k"] = qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        state["v"] = qkv[:, (hq + hk) * d:].unflatten(1, (hk, d))
        angle = torch.arange(state["max_len"], dtype=torch.float64, device="cuda")[:, None] * (
            10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d))
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


def _values(rec, page, d):
    """Keys and values [..., P, d], fp32, of records [..., bytes]."""
    lead = rec.dim() - 1
    kc, vc, km, vm = rec.split([page * d // 2, page * d // 2, page * d // 16, page * d // 16], -1)
    kq = torch.stack([kc & 15, kc >> 4], -1).flatten(lead).unflatten(-1, (page, d))
    vq = torch.stack([vc & 15, vc >> 4], -1).flatten(lead).unflatten(-1, (page // 4, d // 8, 4, 8))
    vq = vq.transpose(-3, -2).reshape(*rec.shape[:-1], page, d)
    vm = vm.unflatten(-1, (page // 4, d // 32, 4, 2)).transpose(-3, -2).reshape(*rec.shape[:-1], page, d // 32, 2)
    km = km.unflatten(-1, (page, d // 32, 2))
    out = []
    for q, m in ((kq, km), (vq, vm)):
        code = m[..., 1].int()
        s = torch.where(code == 255, math.nan, ((code + 848) << 20).view(torch.float32))
        q = q.unflatten(-1, (-1, 32))
        out.append(((q.float() - m[..., 0].float()[..., None]) * s[..., None]).flatten(-2))
    return out


def _places(s):
    """Sequence and position of every new token."""
    start, tokens = s["q_start"].long(), s["q"].shape[0]
    at = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(start[1:], at, right=True)
    return seq, s["kv_len"].long()[seq] - start[seq + 1] + at


def _plain_q4(s):
    c = s["case"]
    n, k = c["n"], c["k"]
    codes, scale, zero = s["w"].split([n * k // 2, n * k // 32, n * k // 64])
    q = torch.stack([codes & 15, codes >> 4], -1).view(n, k // 64, 64).float()
    scale, zero = scale.view(torch.float16).float().view(n, -1, 1), zero.float().view(n, -1, 1)
    return (s["x"].float() @ ((q - zero / 16) * scale).view(n, k).t()).to(s["x"].dtype)


def _plain_append(s):
    c, pool = s["case"], s["pool"]
    d, page = c["head_dim"], c["page"]
    seq, pos = _places(s)
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]

    def rotate(x):
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    kq, km = _quantize(rotate(s["k"]))
    vq, vm = _quantize(s["v"].float())
    rec = s["page_table"][seq, pos // page].long()
    t, heads = (pos % page)[:, None, None], torch.arange(c["kv_heads"], device="cuda")[None, :, None]
    base = (rec[:, None, None] * c["kv_heads"] + heads) * (page * d * 9 // 8)
    flat = pool.view(-1)

    def both(m):
        return torch.stack([m & 255, m >> 8], -1).flatten(-2).to(torch.uint8)

    j, g = torch.arange(d // 2, device="cuda"), torch.arange(d // 16, device="cuda")
    at = [(base + t * (d // 2) + j, kq[..., 0::2] | kq[..., 1::2] << 4),
          (base + page * d // 2 + (t // 4) * (d * 2) + j // 4 * 16 + t % 4 * 4 + j % 4, vq[..., 0::2] | vq[..., 1::2] << 4),
          (base + page * d + t * (d // 16) + g, both(km)),
          (base + page * d + page * d // 16 + (t // 4) * (d // 4) + g // 2 * 8 + t % 4 * 2 + g % 2, both(vm))]
    for index, value in at:
        flat[index] = value
    q = rotate(s["q"]).to(s["q"].dtype)
    # what the cache now holds for these tokens
    kc, vc, km, vm = (flat[index] for index, _ in at)
    out = []
    for codes, m in ((kc, km), (vc, vm)):
        m = m.unflatten(-1, (-1, 2))
        code = m[..., 1].int()
        scale = torch.where(code == 255, math.nan, ((code + 848) << 20).view(torch.float32))[..., None]
        x = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 32)).float()
        out.append(((x - m[..., 0].float()[..., None]) * scale).flatten(-2).to(s["k"].dtype))
    return {"q": q, "k": out[0], "v": out[1]}


def _plain_attention(s):
    c = s["case"]
    d, page, hk = c["head_dim"], c["page"], c["kv_heads"]
    seq, pos = _places(s)
    table, b = s["page_table"].long(), s["page_table"].shape[0]
    k, v = _values(s["pool"][table.clamp(min=0)], page, d)              # [B, pages, heads, P, d]
    k, v = (x.transpose(2, 3).flatten(1, 2).permute(0, 2, 1, 3) for x in (k, v))  # [B, heads, tokens, d]
    held = (torch.arange(k.shape[2], device="cuda") < s["kv_len"].long()[:, None])[:, None, :, None]
    k, v = torch.where(held, k, 0.0), torch.where(held, v, 0.0)
    # queries of each sequence side by side, padded to the most: [B, kv heads, group, new, d]
    i = torch.arange(seq.shape[0], device="cuda") - s["q_start"].long()[seq]
    q = torch.zeros((b, s["max_new"], c["heads"], d), device="cuda")
    q[seq, i] = s["q"].float()
    q = q.unflatten(2, (hk, -1)).permute(0, 2, 3, 1, 4)
    score = torch.matmul(q.flatten(2, 3), k.transpose(2, 3).contiguous()).unflatten(2, (-1, s["max_new"])) * s["scale"]
    first = s["kv_len"].long() - (s["q_start"][1:] - s["q_start"][:-1]).long()
    last = first[:, None] + torch.arange(s["max_new"], device="cuda")
    seen = torch.arange(k.shape[2], device="cuda") <= last[:, :, None]
    score = score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (-1, s["max_new"])) / torch.where(total == 0, 1.0, total)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, i].to(s["q"].dtype)


def _plain_norm(s):
    y = s["y"].float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-5) * s["post"]
    h = 0.75 * s["h"] + s["gate"] * y
    x = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-5) * s["pre"]
    return {"h": h, "x": x.to(s["y"].dtype)}


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"q4": _plain_q4, "append": _plain_append, "attn": _plain_attention, "norm": _plain_norm}[op](s)
    from paper_2511_05814_amd import attention
    if op == "q4":
        return attention.q4_matmul(s["x"], s["w"], s["case"]["n"])
    if op == "append":
        q = attention.kv4_append(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["pool"], s["page_table"], s["q_start"], s["kv_len"])
        k, v = attention.kv4_read(s["pool"], s["page_table"], s["q_start"], s["kv_len"], q.shape[0], q.shape[2], q.dtype)
        return {"q": q, "k": k, "v": v}
    if op == "attn":
        return attention.kv4_attention(s["q"], s["pool"], s["page_table"], s["q_start"], s["kv_len"], s["scale"],
                                       max_new=s["max_new"], max_len=s["max_len"])
    h, x = attention.norm_residual(s["h"], s["y"], s["gate"], s["post"], s["pre"], residual_scale=0.75, eps=1e-5)
    return {"h": h, "x": x}


# -- the definitions in 64 bits --------------------------------------------------------------------------------------------

def _exact_store(x):
    """Values that a cache holds for x [tokens, heads, d], fp64."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    bottom, top = torch.clamp(g.min(-1).values, max=0.0), torch.clamp(g.max(-1).values, min=0.0)
    steps = torch.tensor([(8 + k % 8) * 2.0 ** (k // 8 - 24) for k in range(255)], dtype=torch.float64, device=x.device)
    s = steps[torch.clamp(torch.searchsorted(15 * steps, top - bottom), max=254)].unsqueeze(-1)
    z = torch.clamp(torch.round(-bottom.unsqueeze(-1) / s), 0, 15)
    return ((torch.clamp(torch.round(g / s) + z, 0, 15) - z) * s).reshape(x.shape)


def _exact_attention(s):
    c = s["case"]
    d, page, hk = c["head_dim"], c["page"], c["kv_heads"]
    new, old = _lengths(c)
    out, at = [], 0
    code = torch.arange(255, dtype=torch.float64, device="cuda")
    steps = (8 + code % 8) * 2.0 ** (code // 8 - 24)
    for b, (n, o) in enumerate(zip(new, old)):
        if n == 0:
            continue
        length = n + o
        ids = s["page_table"][b, :-(-length // page)].long()
        tok = torch.arange(length, device="cuda")
        rec = s["pool"][ids].view(len(ids), hk, -1)
        mine, t = tok // page, tok % page
        for h in range(hk):
            r = rec[:, h]
            dim = torch.arange(d, device="cuda")
            kc = r[mine[:, None], t[:, None] * (d // 2) + dim // 2]
            vc = r[mine[:, None], page * d // 2 + t[:, None] // 4 * (2 * d) + dim // 8 * 16 + t[:, None] % 4 * 4 + dim % 8 // 2]
            km = page * d + (t[:, None] * (d // 32) + dim // 32) * 2
            vm = page * d * 17 // 16 + ((t[:, None] // 4 * (d // 32) + dim // 32) * 4 + t[:, None] % 4) * 2
            kv = []
            for raw, m in ((kc, km), (vc, vm)):
                q = (raw.long() >> dim % 2 * 4) & 15
                kv.append((q - r[mine[:, None], m].long()) * steps[r[mine[:, None], m + 1].long()])
            group = c["heads"] // hk
            q = s["q"][at:at + n, h * group:(h + 1) * group].double()
            w = torch.matmul(q.transpose(0, 1).reshape(-1, d), kv[0].t().contiguous()).view(group, n, length) * s["scale"]
            w.masked_fill_(tok > o + torch.arange(n, device="cuda")[:, None], -math.inf)
            out.append((at, h * group, torch.matmul(torch.softmax(w, -1).view(-1, length), kv[1]).view(group, n, d)))
        at += n
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for a, h, x in out:
        o[a:a + x.shape[1], h:h + x.shape[0]] = x.transpose(0, 1)
    return o


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "q4":
        n, k = case["n"], case["k"]
        raw = s["w"][:n * k // 2].view(n, k // 2).long()
        col = torch.arange(k, device="cuda")
        q = ((raw[:, col // 2] >> (col % 2 * 4)) & 15).double()
        scale = s["w"][n * k // 2:n * k // 2 + n * k // 32].view(torch.float16).view(n, k // 64).double()
        zero = s["w"][n * k // 2 + n * k // 32:].view(n, k // 64).double()
        w = (q - zero[:, col // 64] / 16) * scale[:, col // 64]
        return torch.matmul(s["x"].double(), w.t().contiguous())
    if case["op"] == "norm":
        y, h = s["y"].double(), s["h"].double()
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["d"] + 1e-5) * s["post"].double()
        h = h * 0.75 + y * s["gate"].double()
        return {"h": h, "x": h / torch.sqrt(h.square().sum(-1, keepdim=True) / case["d"] + 1e-5) * s["pre"].double()}
    if case["op"] == "attn":
        return _exact_attention(s)
    new, old = _lengths(case)
    pos = torch.cat([torch.arange(o, o + n) for n, o in zip(new, old)]).cuda()
    half = case["head_dim"] // 2
    c, n = s["cos"].double()[pos].unsqueeze(1), s["sin"].double()[pos].unsqueeze(1)
    turned = []
    for x in (s["q"].double(), s["k"].double()):
        y = torch.empty_like(x)
        y[..., :half] = x[..., :half] * c - x[..., half:] * n
        y[..., half:] = x[..., half:] * c + x[..., :half] * n
        turned.append(y)
    return {"q": turned[0], "k": _exact_store(turned[1]), "v": _exact_store(s["v"].double())}
