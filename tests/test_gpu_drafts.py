"""Steps with drafted tokens on an MI355X against the fp64 oracle.

Plans, verification and kept entries are whole numbers and bytes: equal.
Verification is fp64 on both sides, so that a decision differs only where a
random number lies within some 1e-14 of a border; inputs whose borders are hit
on purpose are multiples of powers of two, whose sums are exact in any order.
Attention's tolerances are those of test_gpu_attention, derived there."""
import numpy as np
import pytest

from oracle import attention as oa
from oracle import drafts as od

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests._attention_rig import Batch, bf16, device  # noqa: E402
from tests._drafts_rig import attend, ints, masks, parents, words  # noqa: E402
from tests.test_gpu_attention import BF, U, host, tables  # noqa: E402
from tests.test_gpu_attention_edges import change, key_of, mark  # noqa: E402


def at():
    from paper_2511_05814_amd import attention
    return attention


def dr():
    from paper_2511_05814_amd import drafts
    return drafts


def starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


# -- plans -----------------------------------------------------------------------

@pytest.mark.parametrize("new,most", [
    ([1], 1), ([2], 2), ([31, 0, 32, 33, 1], 33), ([64, 65, 0, 63], 65), ([500, 3, 129, 96], 500), ([1024, 1, 1000], 1024),
    ([40, 70, 8], 20),      # trees past the words: the rest has no place
    ([300] * 70 + [0], 300)])
@pytest.mark.parametrize("kind", ["chain", "bushy", "any"])
def test_draft_tree(new, most, kind):
    rng = np.random.default_rng(len(new) + most)
    lists = []
    for n in new:
        if kind == "any":   # also parents that are none: later tokens, itself, far outside
            lists.append([int(rng.choice([i - 1, rng.integers(-3, i + 3), -1, 2 ** 31 - 1, -2 ** 31, rng.integers(0, i + 1)])) for i in range(n)])
        else:
            lists.append(parents(rng, n, 1 if kind == "chain" else 7))
    length = np.array(new) + rng.integers(0, 5000, len(new))
    parent, start = ints([p for l in lists for p in l]), ints(starts(new))
    pos, seen = dr().draft_tree(parent, start, ints(length), most)
    w = -(-most // 32)
    assert pos.dtype == seen.dtype == torch.int32 and list(seen.shape) == [sum(new), w]
    want = [od.tree(l, int(m) - n, w) for l, m, n in zip(lists, length, new)]
    assert np.array_equal(pos.cpu().numpy(), np.concatenate([p for p, _ in want]))
    assert np.array_equal(seen.cpu().numpy(), np.concatenate([od.words_of(s, w) for _, s in want]))


# -- append at positions -----------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,P,heads,kv,rot,new,old", [(64, 16, 4, 2, 64, [5], [14]), (128, 32, 8, 8, 128, [9, 0, 1, 40], [0, 7, 31, 64]),
                                                      (128, 16, 6, 1, 32, [17, 30], [3, 1])])
def test_append_at_positions(D, P, heads, kv, rot, new, old, dtype):
    """Queries and keys as the oracle's in fp32, bit for bit, in their places;
    other bytes as they were; tokens whose position the tables do not have dropped."""
    bt = Batch(new, old, heads, kv, D, P, seed=D + len(new)).fill(0.5)
    rng = np.random.default_rng(4)
    q, k, v = (rng.standard_normal((bt.tokens, n, D)).astype(np.float32) for n in (heads, kv, kv))
    if dtype == "bf16":
        q, k, v = bf16(q), bf16(k), bf16(v)
    cos, sin = tables(60, rot)   # some places lie past the tables
    pos = rng.integers(0, 60, bt.tokens).astype(np.int32)
    pos[rng.random(bt.tokens) < 0.2] = rng.choice([-1, 60, 2 ** 31 - 1, -2 ** 31])
    fine = (pos >= 0) & (pos < 60)
    pool, table, start, length = bt.args()
    c, s = (torch.from_numpy(t).cuda() for t in (cos, sin))
    got = at().kv4_append(*(device(x, dtype) for x in (q, k, v)), c, s, pool, table, start, length, pos=ints(pos))
    turn = np.where(fine, pos, 0)
    want = np.where(fine[:, None, None], oa.rotate(q, cos[turn], sin[turn]), np.float32(0))
    assert np.array_equal(host(got), bf16(want) if dtype == "bf16" else want)
    keys = oa.rotate(k, cos[turn], sin[turn])
    expect = bt.pool.copy()
    place = bt.positions()
    seq = np.repeat(np.arange(len(new)), new)
    for t in np.flatnonzero(fine):
        page = bt.table[seq[t], place[t] // P]
        for h in range(kv):
            rec = [np.array(x) for x in oa.unpack_record(expect[page, h], P, D)]
            for i, x in ((0, keys[t, h]), (2, v[t, h])):
                codes, metas = oa.kv4_quantize(x[None].astype(np.float32))
                rec[i][place[t] % P], rec[i + 1][place[t] % P] = codes[0], metas[0]
            expect[page, h] = oa.record(*rec)
    assert np.array_equal(pool.cpu().numpy(), expect)


def test_append_at_its_places_is_append():
    bt = Batch([20, 3], [9, 40], 4, 2, 64, 16, seed=2)
    q, k, v = (torch.randn((23, n, 64), device="cuda") for n in (4, 2, 2))
    c, s = (torch.from_numpy(t).cuda() for t in tables(64, 64))
    one, two = bt.args(), bt.args()
    a = at().kv4_append(q, k, v, c, s, *one)
    b = at().kv4_append(q, k, v, c, s, *two, pos=ints(bt.positions()))
    assert torch.equal(a, b) and torch.equal(one[0], two[0])


# -- attention of a tree -------------------------------------------------------------

def check_tree(bt, dtype, seen, scale=None, bits=None, q=None, max_new=None, max_len=None):
    D = bt.D
    scale = D ** -0.5 if scale is None else scale
    q = np.random.default_rng(5).standard_normal((bt.tokens, bt.heads, D)) * 2 if q is None else q
    q = bf16(q) if dtype == "bf16" else np.asarray(q, dtype=np.float32)
    pool, table, start, length = bt.args()
    bits = words(bt, seen) if bits is None else bits
    o = host(at().kv4_tree_attention(device(q, dtype), pool, table, start, length, bits, scale, max_new=max_new, max_len=max_len))
    want, reach, top = attend(bt, q.astype(np.float64), scale, seen)
    prob = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    tol = top * (2 * reach * (2.0 ** -22 + 2 * D * U) + 2 * prob + 64 * U)
    tol = tol[..., None] + (BF * np.abs(want) if dtype == "bf16" else 0)
    assert np.array_equal(np.isnan(o), np.isnan(want))
    fine = ~np.isnan(want)
    bad = np.abs(o - want)[fine] > np.broadcast_to(tol, want.shape)[fine]
    assert not bad.any(), (np.abs(o - want)[fine].max(), bad.mean())
    return o, want


SHAPES = [
    (64, 16, 4, 2, [1], [0]),                        # one token that sees itself, or nothing
    (64, 16, 4, 2, [6], [508]),
    (128, 16, 8, 8, [3, 1, 5, 2], [0, 15, 16, 31]),  # around a page's and a step's end
    (64, 32, 5, 1, [7, 4], [127, 128]),              # an odd group, around a workgroup's step
    (128, 64, 8, 2, [15], [700]),                    # several splits
    (128, 16, 32, 8, [8, 0, 8, 3], [600, 9, 77, 0]),
    (128, 16, 20, 1, [3, 2], [37, 500]),             # more heads to a key head than a tile has rows
    (64, 128, 2, 2, [33, 0, 1], [130, 40, 0]),       # bits in two words
    (128, 32, 8, 2, [20, 12], [200, 31]),            # 17 to 63 rows a key head
    (64, 16, 12, 2, [10, 1], [61, 300]),
    (128, 32, 4, 2, [100, 1, 17], [0, 300, 33]),     # from 64 rows a key head on
    (64, 16, 6, 3, [200], [55]),
    (128, 16, 16, 4, [70, 90], [64, 0])]


# how long the caller says that sequences are: by it, and the rows, the kernels
# differ (results are right whatever it is): those of kv4_attention, or for lengths that
# differ, of 16, 32 or (bf16, from 65 rows on) 128 or 256 rows
HINTS = [None, 1000, 1 << 20]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["tree", "any", "none", "causal"])
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("D,P,heads,kv,new,old", SHAPES)
def test_tree_attention(D, P, heads, kv, new, old, hint, kind, dtype):
    bt = Batch(new, old, heads, kv, D, P, seed=D + P).fill(0.5)
    seen = masks(bt, np.random.default_rng(len(new)), kind)
    o, _ = check_tree(bt, dtype, seen, bits=words(bt, seen, junk=True), max_new=max(new), max_len=hint)
    for b, (n, m) in enumerate(zip(new, old)):
        if m == 0 and kind == "none":
            assert (o[bt.q_start[b]:bt.q_start[b] + n] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("D,P,heads,kv,new,old", [
    (64, 16, 8, 2, [7, 3, 0, 12], [3000, 10, 700, 1900]), (128, 16, 4, 1, [9, 1, 20], [40, 2600, 5000]), (128, 32, 16, 2, [3] * 9, [i * 333 for i in range(9)]),
    (64, 16, 4, 4, [40, 2], [1500, 3]), (128, 64, 8, 2, [30, 1, 50, 0, 5], [4000, 900, 64, 7, 0])])
def test_tree_attention_of_unequal_lengths(D, P, heads, kv, new, old, hint, dtype):
    """Sequences that share workgroups and sequences that lie in many."""
    bt = Batch(new, old, heads, kv, D, P, seed=D + P).fill(0.4)
    check_tree(bt, dtype, masks(bt, np.random.default_rng(5), "tree"), max_new=max(new), max_len=hint)


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("new", [2, 13, 40])
@pytest.mark.parametrize("down", [False, True])
def test_scores_that_grow_along_the_cache(new, hint, down):
    """Every reference is passed by far by a later token, or none is."""
    bt = Batch([new, 1], [700, 90], 4, 2, 64, 16, seed=24).fill(0.3)
    for i, pos in enumerate(range(3, 700, 37)):
        change(bt, 0, 699 - pos if down else pos, 0, key_of(2.0 ** (i - 6)))
    q = np.abs(np.random.default_rng(5).standard_normal((bt.tokens, 4, 64)))
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, masks(bt, np.random.default_rng(6), "tree"), q=q, max_new=new, max_len=hint)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("D,P,heads,kv,new,old", SHAPES)
def test_a_chain_is_attention(D, P, heads, kv, new, old, hint, dtype):
    """With every token seeing those before it, what kv4_attention gives, within
    two roundings of the output and the tolerance between orders of sums."""
    bt = Batch(new, old, heads, kv, D, P, seed=9).fill(0.3)
    q = device(np.random.default_rng(1).standard_normal((bt.tokens, heads, D)), dtype)
    args, bits = bt.args(), words(bt, masks(bt, None, "causal"))
    a = host(at().kv4_tree_attention(q, *args, bits, 0.1, max_new=max(new), max_len=hint))
    b = host(at().kv4_attention(q, *args, 0.1))
    top = np.nanmax(np.abs(b), initial=1.0)
    tol = (2 * BF * np.abs(b) + top * 2.0 ** -9) if dtype == "bf16" else top * 2.0 ** -17
    assert (np.abs(a - b) <= tol).all()


@pytest.mark.parametrize("count", [1, 2, 3, 5, 32])
@pytest.mark.parametrize("heads", [2, 8])
def test_more_and_fewer_words_than_tokens(count, heads):
    """Bits past a row's words are not set; more words change nothing."""
    bt = Batch([70, 3], [50, 600], heads, 2, 64, 16, seed=6).fill(0.3)
    seen = masks(bt, np.random.default_rng(2), "any")
    short = [m & (np.arange(m.shape[1]) < 32 * count) for m in seen]
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, short, bits=words(bt, seen, count))


@pytest.mark.parametrize("max_new,max_len", [(1, 1), (1, 1 << 20), (4096, 1), (3, 100), (16, 1 << 20)])
def test_tree_attention_is_right_whatever_the_hints(max_new, max_len):
    bt = Batch([40, 3], [50, 600], 8, 2, 128, 16, seed=6).fill(0.3)
    seen = masks(bt, np.random.default_rng(3), "tree")
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, seen, max_new=max_new, max_len=max_len)


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("new", [[6, 1, 2], [30, 1, 9], [80, 1, 40]])
def test_tokens_without_places_and_missing_pages(new, hint):
    bt = Batch(new, [0, 0, 50], 4, 2, 64, 16, seed=7, short=1).fill(0.3)
    bt.table[2, 0] = -1
    bt.table[2, 2] = 999
    seen = masks(bt, np.random.default_rng(4), "causal")
    hints = dict(max_new=max(new), max_len=hint)
    o, _ = check_tree(bt, "f32", seen, **hints)
    assert (o[0] == 0).all() and (o[new[0]] == 0).all() and (o[-1] != 0).any()
    bt.table[2, :] = -1
    o, _ = check_tree(bt, "bf16", seen, **hints)
    assert (o[new[0] + 1:] == 0).all()
    bt.table[:, :] = 1 << 30
    assert (check_tree(bt, "bf16", seen, **hints)[0] == 0).all()


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("kind", ["tree", "any", "none"])
@pytest.mark.parametrize("heads", [4, 6, 8])
def test_large_blocks_with_holes_and_growing_scores(heads, kind, hint):
    """More rows of a sequence than a block has, pages that are missing in the middle
    of a tile or take all of it, references that many tokens pass."""
    bt = Batch([120, 3, 60], [1500, 0, 90], heads, 2, 128, 16, seed=heads).fill(0.3)
    for i, pos in enumerate(range(7, 1500, 61)):
        change(bt, 0, pos, i % 2, key_of(2.0 ** (i / 3 - 4)))
    for col in (2, 16, 17, 18, 19, 95):
        bt.table[0, col] = -1
    bt.table[2, 1] = 1 << 30
    q = np.abs(np.random.default_rng(5).standard_normal((bt.tokens, heads, 128)))
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, masks(bt, np.random.default_rng(heads), kind), q=q, max_new=120, max_len=hint)


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("D,new", [(64, 3), (64, 50), (128, 9), (128, 25), (128, 130)])
def test_steps_of_any_size(D, new, hint):
    """Groups whose steps lie at both ends of the scale grid, and between them."""
    bt = Batch([new, 2], [150, 33], 4, 2, D, 32, seed=8).fill(0.3)
    rng = np.random.default_rng(new)
    for i, pos in enumerate(rng.permutation(150)[:60]):
        size = [2.0 ** -24, 1e-6, 2.0 ** -17, 300.0, 7600.0, 7700.0, 28000.0][i % 7]
        for h in range(2):
            page = bt.table[0, pos // 32]
            rec = [np.array(x) for x in oa.unpack_record(bt.pool[page, h], 32, D)]
            for part in (0, 2):
                codes, metas = oa.kv4_quantize(rng.uniform(-1, 1, (1, D)) * size)
                rec[part][pos % 32], rec[part + 1][pos % 32] = codes[0], metas[0]
            bt.pool[page, h] = oa.record(*rec)
    q = rng.standard_normal((bt.tokens, 4, D)) * 1e-3
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, masks(bt, rng, "any"), q=q, max_new=new, max_len=hint)


@pytest.mark.parametrize("new", [3, 9, 25, 150])
@pytest.mark.parametrize("part", [0, 2])
@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("D", [64, 128])
def test_marked_entries_reach_only_rows_that_see_them_in_a_tree(new, hint, part, D):
    """A new token and a cached one marked as not stored, and all places behind
    the end."""
    for cached in (False, True):
        bt = Batch([new, 1], [20, 33], 4, 2, D, 32, seed=8).fill(0.3)
        j = new // 2
        change(bt, 0, 5 if cached else 20 + j, 0, mark(part))
        for b_ in range(2):
            tail = bt.len[b_] % 32
            page = bt.table[b_, (bt.len[b_] - 1) // 32]
            for h in range(2 if tail else 0):
                rec = [np.array(x) for x in oa.unpack_record(bt.pool[page, h], 32, D)]
                rec[1][tail:] = rec[3][tail:] = 255 << 8
                bt.pool[page, h] = oa.record(*rec)
        seen = masks(bt, np.random.default_rng(new), "any")
        seen[0][0, j], seen[0][1, j] = True, False
        for dtype in ("f32", "bf16"):
            o, _ = check_tree(bt, dtype, seen, max_new=new, max_len=hint)
            hit = np.isnan(o[:new, :2]).any((1, 2))
            assert hit.all() if cached else np.array_equal(hit, seen[0][:, j])
            assert not np.isnan(o[:, 2:]).any() and not np.isnan(o[new:]).any()


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("new", [2, 12, 70])
def test_infinities_and_far_scores(new, hint):
    """A row of q with an infinity is NaN and alone; a key that takes all the
    weight is missed by rows that do not see it."""
    bt = Batch([new, 2], [40, 30], 4, 2, 64, 16, seed=24).fill(0.3)
    change(bt, 0, 40 + new - 1, 0, key_of(300.0))
    seen = masks(bt, np.random.default_rng(6), "any")
    seen[0][:, new - 1] = np.arange(new) % 2 == 0
    q = np.abs(np.random.default_rng(5).standard_normal((bt.tokens, 4, 64)))
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, seen, q=q, max_new=new, max_len=hint)
    for value in (np.inf, -np.inf, np.nan):
        q[0, 1, 9] = value
        for dtype in ("f32", "bf16"):
            o = host(at().kv4_tree_attention(device(q, dtype), *bt.args(), words(bt, seen), 0.125, max_new=new, max_len=hint))
            assert np.isnan(o[0, 1]).all() and np.isnan(o).sum() == 64
    for scale in (np.nan, np.inf):
        o = host(at().kv4_tree_attention(device(np.ones((bt.tokens, 4, 64)), "bf16"), *bt.args(), words(bt, seen), scale, max_new=new, max_len=hint))
        assert np.isnan(o).all()


@pytest.mark.parametrize("hint", HINTS)
@pytest.mark.parametrize("scale,size", [(1e-20, 1e20), (-1e-30, 1e30), (0.0, 1e25), (1e-36, 1e-10), (1e25, 1e-25)])
def test_scales_and_queries_of_any_size_in_a_tree(scale, size, hint):
    bt = Batch([20, 1, 33], [300, 20, 64], 4, 2, 64, 16, seed=23).fill(0.3)
    q = np.random.default_rng(4).standard_normal((bt.tokens, 4, 64)) * size
    for dtype in ("f32", "bf16"):
        check_tree(bt, dtype, masks(bt, np.random.default_rng(6), "tree"), q=q, scale=scale, max_new=33, max_len=hint)


def test_strided_queries_given_outputs_and_workspaces():
    bt = Batch([12, 5], [900, 40], 8, 2, 64, 32, seed=3).fill(0.3)
    seen = masks(bt, np.random.default_rng(7), "tree")
    bits, args = words(bt, seen), bt.args()
    ws = torch.full((1 << 27,), 255, dtype=torch.uint8, device="cuda")   # NaN, were it read as it is
    for hint in HINTS:
        wide = torch.randn((17, 12, 64), device="cuda")
        want = at().kv4_tree_attention(wide[:, 2:10].contiguous(), *args, bits, 0.125, max_len=hint)
        out = torch.full((17, 12, 64), 7.0, device="cuda")
        got = at().kv4_tree_attention(wide[:, 2:10], *args, bits, 0.125, out=out[:, 1:9], workspace=ws, max_len=hint)
        assert torch.equal(got, want) and (out[:, :1] == 7).all() and (out[:, 9:] == 7).all()
        at().kv4_tree_attention(wide[:, 2:10], *args, bits, 0.125, out=wide[:, 2:10], max_len=hint)
        assert torch.equal(wide[:, 2:10], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [4, 16])
@pytest.mark.parametrize("hint", HINTS)
def test_starts_that_go_back_or_past_the_tokens(hint, heads, dtype):
    """Bounds are cut to the tokens that there are, and to no fewer than none; rows
    of one sequence alone are right whatever the others claim."""
    starts_, tokens, D = [0, 12, 5, 30, 2 ** 31 - 1, 40, 60, -7, 3], 60, 128
    ends = [min(max(e, 0), tokens) for e in starts_]
    spans = [(s, max(s, e)) for s, e in zip(ends, ends[1:])]   # 12, 0, 25, 30, 0, 20, 0 and 3 tokens
    bt = Batch([e - s for s, e in spans], [300, 20, 700, 64, 5, 130, 10, 33], heads, 2, D, 16, seed=31).fill(0.3)
    rng = np.random.default_rng(4)
    q = rng.standard_normal((tokens, heads, D)) * 2
    q = bf16(q) if dtype == "bf16" else q.astype(np.float32)
    seen = rng.random((tokens, 64)) < 0.5
    mine = [seen[s:e, :e - s] for s, e in spans]
    pool, table, _, length = bt.args()
    bits = ints(od.words_of(seen, 2))
    o = host(at().kv4_tree_attention(device(q, dtype), pool, table, ints(starts_), length, bits, D ** -0.5, max_len=hint))
    want, reach, top = attend(bt, np.concatenate([q[s:e] for s, e in spans]).astype(np.float64), D ** -0.5, mine)
    checked = 0
    for b, (s, e) in enumerate(spans):
        got, row = o[s:e], slice(bt.q_start[b], bt.q_start[b + 1])
        prob = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22   # as in check_tree
        tol = top[row] * (2 * reach[row] * (2.0 ** -22 + 2 * D * U) + 2 * prob + 64 * U)
        tol = tol[..., None] + (BF * np.abs(want[row]) if dtype == "bf16" else 0)
        alone = [i for i in range(e - s) if sum(x <= s + i < y for x, y in spans) == 1]
        assert (np.abs(got - want[row]) <= tol)[alone].all(), b
        checked += len(alone)
    assert checked == 2 + 18 + 10


@pytest.mark.parametrize("size", [0.0, 1e-3, 0.05])
@pytest.mark.parametrize("D,heads,new", [(64, 4, [20, 1, 33]), (128, 8, [9, 4, 2]), (128, 4, [40, 70])])
def test_flat_scores(D, heads, new, size):
    """Rows whose weights are all alike: eight weights at the reference add up to
    more than one of them may be in fp32 calls."""
    bt = Batch(new, [700, 90, 1500][:len(new)], heads, 2, D, 32, seed=29).fill(0.3)
    q = np.random.default_rng(4).standard_normal((bt.tokens, heads, D)) * size
    for dtype in ("f32", "bf16"):
        for hint in HINTS:
            check_tree(bt, dtype, masks(bt, np.random.default_rng(6), "tree"), q=q, max_new=max(new), max_len=hint)


def test_flat_scores_take_no_longer():
    """fp32 over 4 x 16048 tokens: all scores equal, beside one token of every 32
    that holds nearly all weight.  No reference moves in either, so that the same
    instructions run; were a row's reference looked for again in every block of the
    flat ones, they would take 1.6 times as long (226 us beside 143)."""
    seqs, new, length, kv, heads, D, P = 4, 48, 16048, 8, 32, 128, 64
    cols = -(-length // P)
    table = torch.arange(seqs * cols, dtype=torch.int32, device="cuda").view(seqs, cols)
    keys = torch.zeros((length, kv, D), device="cuda")
    keys[::32, :, 0] = 15.0
    none = torch.zeros((length, 0), device="cuda")
    pools = []
    for k in (torch.zeros_like(keys), keys):
        pool = at().kv4_pool(seqs * cols, kv, P, D)
        for b in range(seqs):
            at().kv4_append(k, k, torch.zeros_like(k), none, none, pool, table[b:b + 1], ints([0, length]), ints([length]))
        pools.append(pool)
    start, lengths = ints([new * b for b in range(seqs + 1)]), ints([length] * seqs)
    _, seen = dr().draft_tree(ints(([-1] + list(range(new - 1))) * seqs), start, lengths, new)
    q = torch.zeros((seqs * new, heads, D), device="cuda")
    q[:, :, 0] = 1.0
    out, best = torch.empty_like(q), [float("inf")] * 2
    for _ in range(9):
        for i, pool in enumerate(pools):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            for _ in range(10):
                at().kv4_tree_attention(q, pool, table, start, lengths, seen, 1.0, max_new=new, max_len=length, out=out)
            end.record()
            end.synchronize()
            best[i] = min(best[i], begin.elapsed_time(end))
    assert best[0] < 1.25 * best[1], best


def test_more_sequences_than_a_plan_holds():
    bt = Batch([2, 1] * 150, [5, 17] * 150, 2, 1, 64, 16, seed=3).fill(0.3)
    check_tree(bt, "bf16", masks(bt, np.random.default_rng(7), "tree"), max_len=1 << 20)
    bt = Batch([2, 0, 3, 1] * 64, [5, 17, 0, 200] * 64, 2, 1, 64, 16, seed=3).fill(0.3)
    check_tree(bt, "bf16", masks(bt, np.random.default_rng(7), "tree"), max_len=1 << 20)


# -- verification ----------------------------------------------------------------------

def case(rng, new, vocab, dtype, drawn, width=3, sharp=2.0):
    lists = [parents(rng, n, width) for n in new]
    t = sum(new)
    z = rng.standard_normal((t, vocab)) * sharp
    p, q = (np.exp(x - x.max(1, keepdims=True)) for x in (z, z + 0.5 * rng.standard_normal((t, vocab))))
    p, q = (bf16(x / x.sum(1, keepdims=True)) if dtype == "bf16" else (x / x.sum(1, keepdims=True)).astype(np.float32) for x in (p, q))
    ids, at_ = np.zeros(t, dtype=np.int32), 0
    for l in lists:
        for i in range(1, len(l)):
            w = q[at_ + l[i]].astype(np.float64)
            ids[at_ + i] = rng.choice(vocab, p=w / w.sum())
        at_ += len(l)
    return lists, p, (q if drawn else None), ids, rng.random(t).astype(np.float32)


def check_verify(lists, p, q, ids, u, dtype, place=lambda x: x):
    """place: how a matrix lies on the device."""
    new = [len(l) for l in lists]
    start = starts(new)
    P, Q = (None if x is None else place(device(x, dtype)) for x in (p, q))
    path, count, after = dr().verify_drafts(P, ints(ids), ints([x for l in lists for x in l]), torch.from_numpy(u).cuda(), ints(start), q=Q)
    got = path.cpu().numpy(), count.cpu().numpy(), after.cpu().numpy()
    for b, l in enumerate(lists):
        rows = slice(start[b], start[b + 1])
        with np.errstate(all="ignore"):
            w, n = od.verify(p[rows].astype(np.float64), ids[rows], l, u[rows], None if q is None else q[rows].astype(np.float64))
        assert list(got[0][rows]) == w + [-1] * (len(l) - len(w)), b
        assert (got[1][b], got[2][b]) == (len(w), n), b
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("new,vocab,width", [
    ([1], 1, 1), ([4], 2, 2), ([6], 1000, 1), ([1, 0, 5, 9], 777, 3), ([16] * 9, 4099, 3), ([40, 64, 33], 2048, 6), ([64], 33, 63),
    ([8] * 70, 257, 8), ([2, 3], 70001, 2), ([3], 262144, 3), ([1024, 700], 65, 9)])
def test_verify(new, vocab, width, drawn, dtype):
    rng = np.random.default_rng(sum(new) + vocab)
    for sharp in (0.5, 3.0):
        check_verify(*case(rng, new, vocab, dtype, drawn, width, sharp), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,stride,first", [(999, 999, 0), (1000, 1001, 1), (1000, 1013, 3), (1024, 1032, 8), (515, 516, 0)])
def test_verify_rows_of_any_alignment(vocab, stride, first, dtype):
    rng = np.random.default_rng(vocab)

    def place(x):
        wide = torch.full((x.shape[0], stride + 8), float("nan"), dtype=x.dtype, device="cuda")
        flat = wide.view(-1)[first:first + x.shape[0] * stride].view(x.shape[0], stride)
        flat[:, :vocab] = x
        return flat[:, :vocab]

    for drawn in (True, False):
        check_verify(*case(rng, [9, 12], vocab, dtype, drawn), dtype, place)


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_walks_whole_trees(drawn):
    """Nothing refused, everything refused, and random numbers at both ends."""
    rng = np.random.default_rng(3)
    for value in (0.0, 0.5, 1 - 2.0 ** -24, 1.0, -3.0, np.nan, np.inf):
        lists, p, q, ids, u = case(rng, [30, 7, 1], 300, "f32", drawn, 3)
        u[:] = value
        check_verify(lists, p, q, ids, u, "f32")


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_at_borders(drawn):
    """Probabilities in 64ths and random numbers in 16ths: products and sums are
    exact, and many of them equal."""
    rng = np.random.default_rng(8)
    hits = 0
    for _ in range(40):
        lists = [parents(rng, 12, 4) for _ in range(16)]
        t = 192
        p, q = (np.stack([np.bincount(rng.integers(0, 6, 64), minlength=9) for _ in range(t)]).astype(np.float32) / 64 for _ in range(2))
        ids, u = rng.integers(0, 7, t).astype(np.int32), (rng.integers(0, 16, t) / 16).astype(np.float32)
        _, count, _ = check_verify(lists, p, q if drawn else None, ids, u, "f32")
        hits += (count > 2).sum()
    assert hits > 20


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drawn", [True, False])
def test_verify_of_rows_that_are_no_distribution(drawn, dtype):
    """All zeros, negative entries, an infinity, a NaN, sums far from 1; ids
    outside the vocabulary; children of one id."""
    rng = np.random.default_rng(9)
    lists, p, q, ids, u = case(rng, [6] * 12, 90, dtype, drawn, 5)
    for b in range(12):
        r = 6 * b
        if b == 0: p[r] = 0
        if b == 1: p[r, ::2] *= -1
        if b == 2: p[r, 7] = np.inf
        if b == 3: p[r, 80] = np.nan
        if b == 4: p[r:r + 6] *= 8
        if b == 5: p[r:r + 6] /= 8
        if b == 6: ids[r + 1:r + 6] = [-1, 90, 2 ** 31 - 1, -2 ** 31, 91]
        if b == 7: ids[r + 1:r + 6] = 4
        if b == 8: p[r:r + 6], p[r:r + 6, 5] = 0, 1
        if b == 9 and q is not None: q[r:r + 6] = 0
        if b == 10 and q is not None: q[r:r + 6] = p[r:r + 6] * 2
        if b == 11: u[r + 1:r + 6] = 1
    p, q = (x if x is None or dtype == "f32" else bf16(x) for x in (p, q))
    _, _, after = check_verify(lists, p, q, ids, u, dtype)
    assert after[0] == -1


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("vocab", [66000, 140001])
def test_verify_of_more_passes_than_are_shared(vocab, drawn):
    """Workgroups that share a row tell each other the sums of sixteen passes;
    every one works out the rest by itself."""
    rng = np.random.default_rng(vocab)
    lists, p, q, ids, u = case(rng, [25, 2], vocab, "f32", drawn, 1)
    lists[0] = [-1] + [0] * 24
    u[1:25] = 1
    ids[1:25] = rng.choice(200, 24) if drawn else rng.integers(0, vocab, 24)
    p[0, :200], q_ = p[0, :200] + np.float32(1e-3), q
    check_verify(lists, p, q_, ids, u, "f32")


def refusals(count, vocab):
    """A first token whose children are all refused: the draft was sure of ids that
    the target hardly has."""
    p, q = np.full((2, count + 1, vocab), 1 / vocab, dtype=np.float32)
    q[:, :count] = 0.5 / count
    q[:, count:] = 0.5 / (vocab - count)
    return [[-1] + [0] * count], p, q, np.arange(-1, count, dtype=np.int32), np.full(count + 1, 0.75, dtype=np.float32)


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("count", [16, 17, 127, 128, 129, 250])
def test_verify_of_passes_around_the_last_shared_one(count, drawn):
    """In powers of two: T is always the same sum and S a multiple of it, exact."""
    vocab = 66000
    p, q = np.full((count + 1, vocab), 2.0 ** -17, dtype=np.float32), np.zeros((count + 1, vocab), dtype=np.float32)
    q[:, :256] = 2.0 ** -8
    u = np.full(count + 1, 0.75, dtype=np.float32)
    _, kept, after = check_verify([[-1] + [0] * count], p, q if drawn else None, np.arange(-1, count, dtype=np.int32), u, "f32")
    assert kept[0] == 1 and after[0] >= (256 if drawn else count)


@pytest.mark.parametrize("count", [127, 128, 129, 140])
def test_verify_where_refusals_leave_less_than_a_rounding(count):
    """Ids from `count` on, all alike, keep p - S q > 0 in exact numbers, and every
    refusal halves it: S comes within rounding (2^-52 of itself) of p / q long before
    the last one.  Then |p - S q| <= 2^-51 p whatever was rounded where, and the
    sign that its rounding has says whether these ids are drawn from, as in exact
    numbers, or, nothing being left, p itself.  Both draws are of equal weights: the
    least id at which their share passes 3/4, or, where it is 3/4 of them but for
    the sums' rounding, the one in front of it."""
    vocab = 66000
    lists, p, q, ids, u = refusals(count, vocab)
    path, kept, after = dr().verify_drafts(*(torch.from_numpy(p).cuda(), ints(ids), ints(lists[0]), torch.from_numpy(u).cuda(), ints([0, count + 1])),
                                           q=torch.from_numpy(q).cuda())
    assert kept.tolist() == [1] and path.tolist() == [0] + [-1] * count
    left, whole = count + 3 * (vocab - count) // 4, 3 * vocab // 4
    assert after.item() in (left, left - 1, whole, whole - 1)


@pytest.mark.parametrize("count", [1, 16, 17, 60, 128])
def test_verify_shares_its_passes(count):
    """As many sums in the workspace as there were passes and workgroups: one that is
    not told to the others is worked out by each of them."""
    from paper_2511_05814_amd import binding as b
    vocab = 66000
    (parent,), p, q, ids, u = refusals(count, vocab)
    p, q, u = (torch.from_numpy(x).cuda() for x in (p, q, u))
    ids, parent, start, path, one, after = (ints(x) for x in (ids, parent, [0, count + 1], ids, [0], [0]))
    ws = torch.zeros(b.moe_verify_drafts_workspace_bytes(1, vocab), dtype=torch.uint8, device="cuda")
    b.moe_verify_drafts(*(x for t in (p, q) for x in (t.data_ptr(), vocab)), ids.data_ptr(), parent.data_ptr(), u.data_ptr(), start.data_ptr(),
                        1, count + 1, vocab, b.MOE_DTYPE_F32, path.data_ptr(), one.data_ptr(), after.data_ptr(), ws.data_ptr(), ws.numel(),
                        torch.cuda.current_stream().cuda_stream)
    told = int((ws.view(torch.int64) != -1).sum())
    assert one.item() == 1 and told == count * (vocab // 16384)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [60, 5000, 70001])
def test_verify_reads_no_q_of_tokens_without_children(vocab, dtype):
    """A draft has no distribution behind its last tokens: NaN there changes
    nothing, also where all is accepted up to them."""
    rng = np.random.default_rng(vocab)
    for value in (None, 0.0):
        lists, p, q, ids, u = case(rng, [5, 1, 9], vocab, dtype, True)
        if value is not None:
            u[:] = value
        want = check_verify(lists, p, q, ids, u, dtype)
        at_ = 0
        for l in lists:
            q[[at_ + i for i in range(len(l)) if i not in l]] = np.nan
            at_ += len(l)
        got = check_verify(lists, p, q, ids, u, dtype)
        assert all(np.array_equal(a, b) for a, b in zip(want, got)) and min(got[2]) >= 0


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_without_tokens(drawn):
    p = torch.zeros((0, 50), device="cuda")
    e = ints([])
    path, count, after = dr().verify_drafts(p, e, e, p[:, 0], ints([0, 0, 0]), q=p if drawn else None)
    assert path.numel() == 0 and count.tolist() == [0, 0] and after.tolist() == [-1, -1]


# -- keeping -----------------------------------------------------------------------------

@pytest.mark.parametrize("D,P,kv,new,old", [(64, 16, 2, [6], [13]), (128, 16, 8, [8, 0, 1, 16], [0, 3, 40, 15]), (64, 64, 1, [200, 90], [5, 63]),
                                            (128, 1024, 3, [33], [1000])])
@pytest.mark.parametrize("layers", [1, 3, 70])
def test_keep(D, P, kv, new, old, layers):
    if layers == 70 and P == 1024:
        layers = 2
    rng = np.random.default_rng(D + len(new))
    bt = Batch(new, old, kv, kv, D, P, seed=4)
    pools = rng.integers(0, 256, (layers, *bt.pool.shape), dtype=np.uint8)
    path, count = [], []
    for n in new:
        k = int(rng.integers(0, n + 1))
        if n > 100:
            k = n - 30   # several groups of entries
        path += sorted(rng.choice(n, k, replace=False).tolist()) + [-1] * (n - k) if n else []
        count.append(k)
    _, table, start, length = bt.args()
    dev = [torch.from_numpy(x).cuda() for x in pools]
    at().kv4_keep(dev[0] if layers == 1 else dev, table, start, length, ints(path), ints(count), D)
    for i in sorted({0, layers // 2, layers - 1}):
        want = pools[i].copy()
        for b, n in enumerate(new):
            od.keep(want, bt.table[b], old[b], n, path[bt.q_start[b]:], count[b], P, D)
        assert np.array_equal(dev[i].cpu().numpy(), want), i


def test_keep_leaves_what_it_cannot_move():
    """Paths that go back or outside, more kept than there are, pages missing,
    places below 0."""
    rng = np.random.default_rng(1)
    bt = Batch([20, 6, 9, 3], [10, 0, 30, 3], 2, 2, 64, 16, seed=4)
    bt.table[2, 2] = -1
    pool = rng.integers(0, 256, bt.pool.shape, dtype=np.uint8)
    path = [0, 0, 5, 2, -7, 9, 99, 2 ** 31 - 1, 19, 9] + [-2 ** 31] * 10 + [1, 2, 3, 4, 5, 6] + list(range(9)) + [1, 2, 2]
    path[26:35] = [2, 3, 4, 5, 6, 7, 8, -1, 8]
    count, length = [20, 1 << 30, 9, -5], np.array(bt.len)
    length[1] = 4    # two of its tokens have no place
    _, table, start, _ = bt.args()
    dev = torch.from_numpy(pool).cuda()
    at().kv4_keep([dev], table, start, ints(length), ints(path), ints(count), 64)
    want = pool.copy()
    for b, n in enumerate(bt.new):
        od.keep(want, bt.table[b], int(length[b]) - n, n, path[bt.q_start[b]:], count[b], 16, 64)
    assert np.array_equal(dev.cpu().numpy(), want)


# -- together -----------------------------------------------------------------------------

def step(bt, args, x, cos, sin, parent, ids, p, q, u, pools, most):
    """A step as a program makes it: plan, two layers, verification, keeping."""
    table, start, length = args[1:]
    pos, seen = dr().draft_tree(parent, start, length, most)
    out = []
    for pool in pools:
        turned = at().kv4_append(x[:, :bt.heads], x[:, bt.heads:bt.heads + bt.kv_heads], x[:, bt.heads + bt.kv_heads:], cos, sin, pool, table,
                                 start, length, pos=pos)
        out.append(at().kv4_tree_attention(turned, pool, table, start, length, seen, 0.125, max_new=most, max_len=400))
    path, count, after = dr().verify_drafts(p, ids, parent, u, start, q)
    at().kv4_keep(pools, table, start, length, path, count, bt.D)
    return out + [path, count, after]


@pytest.mark.parametrize("most", [5, 40])
def test_a_step_in_a_graph_and_on_another_stream(most):
    """Replays give what eager calls give, eager work between them; two graphs
    of the same tensors do not disturb each other."""
    bt = Batch([most, 1, 3], [300, 20, 0], 4, 2, 64, 16, seed=12).fill(0.3)
    rng = np.random.default_rng(5)
    lists, p, q, ids, u = case(rng, bt.new, 5000, "bf16", True)
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(512, 64))
    args, x = bt.args(), torch.randn((bt.tokens, 8, 64), device="cuda")
    dev = ints([v for l in lists for v in l]), ints(ids), device(p, "bf16"), device(q, "bf16"), torch.from_numpy(u).cuda()
    first = args[0].clone()
    pools = [first.clone(), first.clone()]

    def fresh(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        x.normal_(generator=gen)
        dev[4].uniform_(generator=gen)
        for pool in pools:
            pool.copy_(first)

    def run():
        return step(bt, args, x, cos, sin, *dev, pools, most)

    def snapshot(out):
        return [t.clone() for t in out + pools]

    fresh(0)
    want = snapshot(run())
    side = torch.cuda.Stream()
    fresh(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got + pools, want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out))
    for i in range(3):
        fresh(i)
        eager = snapshot(run())
        for g, out in graphs:
            fresh(i)
            for t in out:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out + pools, eager))


def test_calls_on_two_streams_and_in_a_graph_at_once():
    """Rows that workgroups share and sequences that lie in many: calls that run
    beside each other, on other streams and as replays, give what they give alone."""
    calls = []
    for seed, dtype in ((1, "bf16"), (2, "f32")):
        rng = np.random.default_rng(seed)
        bt = Batch([30, 1, 50], [3000, 40, 900], 8, 2, 128, 16, seed=seed).fill(0.3)
        args, seen = bt.args(), words(bt, masks(bt, rng, "tree"))
        q = device(rng.standard_normal((bt.tokens, 8, 128)), dtype)
        lists, p, d, ids, u = case(rng, [12, 1, 16, 7], 140001, dtype, True)
        rest = ints(ids), ints([x for l in lists for x in l]), torch.from_numpy(u).cuda(), ints(starts([len(l) for l in lists])), device(d, dtype)
        P = device(p, dtype)
        calls.append(lambda args=args, seen=seen, q=q, rest=rest, P=P: [
            at().kv4_tree_attention(q, *args, seen, 0.1, max_new=50, max_len=3050), *dr().verify_drafts(P, *rest)])
    want = [call() for call in calls]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = calls[0]()
    sides = [torch.cuda.Stream() for _ in calls]
    for _ in range(8):
        got = []
        for t in replayed:
            t.zero_()
        for side in sides:
            side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        for side, call in zip(sides, calls):
            with torch.cuda.stream(side):
                got.append(call())
        torch.cuda.synchronize()
        for a, b in zip(got + [replayed], want + [want[0]]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_what_is_kept_is_what_a_chain_would_have_stored():
    """Accepted tokens' entries and outputs are those that the same tokens,
    taken one after another without drafts, have: the keys' bits to the last one."""
    bt = Batch([9], [37], 4, 2, 64, 16, seed=3).fill(0.3)
    parent, path = [-1, 0, 0, 1, 1, 2, 4, 4, 6], [0, 1, 4, 6, 8]
    x = torch.randn((9, 8, 64), device="cuda")
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(64, 64))
    pool, table, start, length = bt.args()
    pos, seen = dr().draft_tree(ints(parent), start, length, 9)
    q = at().kv4_append(x[:, :4], x[:, 4:6], x[:, 6:], cos, sin, pool, table, start, length, pos=pos)
    o = at().kv4_tree_attention(q, pool, table, start, length, seen, 0.125)
    at().kv4_keep(pool, table, start, length, ints(path + [-1] * 4), ints([5]), 64)
    line = torch.from_numpy(bt.pool).cuda()
    y = x[torch.tensor(path, device="cuda")]
    plan = table, ints([0, 5]), ints([42])
    turned = at().kv4_append(y[:, :4], y[:, 4:6], y[:, 6:], cos, sin, line, *plan)
    want = at().kv4_attention(turned, line, *plan, 0.125)
    for a, b in zip(at().kv4_read(pool, *plan, 5, 64), at().kv4_read(line, *plan, 5, 64)):
        assert torch.equal(a, b)
    assert (host(o)[path] - host(want)).__abs__().max() <= 2.0 ** -17 * np.abs(host(want)).max()


def test_python_refusals_of_drafts():
    from paper_2511_05814_amd import binding as b
    a, d = at(), dr()
    bt = Batch([2, 1], [3, 4], 4, 2, 64, 16)
    pool, table, start, length = bt.args()
    q, seen = torch.zeros((3, 4, 64), device="cuda"), ints(np.zeros((3, 1)))
    p, three, u = torch.zeros((3, 50), device="cuda"), ints([0, 0, 0]), torch.zeros(3, device="cuda")
    two = ints([1, 1])
    for call in (lambda: a.kv4_tree_attention(q, pool, table, start, length, seen[:2], 1.0),
                 lambda: a.kv4_tree_attention(q, pool, table, start, length, seen.long(), 1.0),
                 lambda: a.kv4_tree_attention(q, pool, table, start, length, seen.cpu(), 1.0),
                 lambda: a.kv4_tree_attention(q, pool, table, start, length, seen[:, 0], 1.0),
                 lambda: a.kv4_append(q, q[:, :2], q[:, :2], q[0], q[0], pool, table, start, length, pos=three[:2]),
                 lambda: a.kv4_append(q, q[:, :2], q[:, :2], q[0], q[0], pool, table, start, length, pos=three.long()),
                 lambda: a.kv4_keep([], table, start, length, three, two, 64),
                 lambda: a.kv4_keep([pool, pool[:1]], table, start, length, three, two, 64),
                 lambda: a.kv4_keep([pool, pool.cpu()], table, start, length, three, two, 64),
                 lambda: a.kv4_keep(pool, table, start, length, three, three, 64),
                 lambda: a.kv4_keep(pool, table, start, length, three.long(), two, 64),
                 lambda: a.kv4_keep(pool, table, start, length, three, two, 128 * 5),
                 lambda: d.draft_tree(three, start, length, 0), lambda: d.draft_tree(three, start, length, 1025),
                 lambda: d.draft_tree(three.long(), start, length, 2), lambda: d.draft_tree(three, start[:2], length, 2),
                 lambda: d.draft_tree(three.cpu(), start, length, 2), lambda: d.draft_tree(seen, start, length, 2),
                 lambda: d.verify_drafts(p.half(), three, three, u, start), lambda: d.verify_drafts(p, three[:2], three, u, start),
                 lambda: d.verify_drafts(p, three, three, u.double(), start), lambda: d.verify_drafts(p, three, three, u, start, q=p.bfloat16()),
                 lambda: d.verify_drafts(p, three, three, u, start, q=p[:, :49]), lambda: d.verify_drafts(p.t(), three, three, u, start),
                 lambda: d.verify_drafts(p.clone().requires_grad_(), three, three, u, start)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: a.kv4_keep([pool, pool], table, start, length, three, two, 64),
                 lambda: a.kv4_tree_attention(q, pool, table, start, length, ints(np.zeros((3, 33))), 1.0),
                 lambda: a.kv4_tree_attention(q, pool, table, start, length, ints(np.zeros((3, 0))), 1.0),
                 lambda: d.verify_drafts(p[:, :0], three, three, u, start), lambda: d.verify_drafts(p, three, three, u, start[:1])):
        with pytest.raises(b.MoeError):
            call()
