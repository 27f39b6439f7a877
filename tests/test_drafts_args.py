"""What the entry points of drafted tokens refuse, found on the host before any
GPU work."""
import ctypes

import pytest

from tests.test_attention_args import BF16, F32, P, append, attend, b, batch, refused
from tests.test_attention_limits import A, B, C, D, E, apart, overlap

FAR = P + (11 << 30)


def append_at(bt, pos, **kw):
    a = append(bt, **kw)
    return (a[0], pos, *a[1:])


def tree_attend(bt, seen=P, words=1, **kw):
    a = attend(bt, **kw)
    return (*a[:3], seen, words, *a[3:])


def plan(**kw):
    a = dict(parent=A, q_start=B, kv_len=B + 64, seqs=3, tokens=9, words=2, pos=C, seen=D, stream=0)
    a.update(kw)
    return tuple(a.values())


def verify(**kw):
    a = dict(p=A, ps=50, q=B, qs=50, ids=C, parent=C + 64, u=C + 128, q_start=C + 192, seqs=3, tokens=9, vocab=50, dtype=F32, path=D,
             count=D + 64, next=D + 128, ws=None, wsb=0, stream=0)
    a.update(kw)
    return tuple(a.values())


def keep(bt, pools=(E, E + (1 << 20)), path=P, count=P + 64):
    return bt, list(pools), path, count, 0


def test_append_at_refuses():
    for bad in (dict(q=None), dict(max_pos=0), dict(heads=3), dict(rot=24), dict(dtype=2)):
        refused(b.moe_kv4_append_at, *append_at(batch(), FAR, **bad))
    refused(b.moe_kv4_append_at, *append_at(batch(), FAR + 2))
    b.moe_kv4_append_at(*append_at(batch(tokens=0), None))
    base = dict(q=A, k=B, v=C, out=D, cos=E, sin=E + 80 * 32 * 4)
    far = batch(pool=P + (9 << 30))
    apart(b.moe_kv4_append_at, *append_at(far, FAR, **base))
    overlap(b.moe_kv4_append_at, *append_at(far, D + 4, **base))
    overlap(b.moe_kv4_append_at, *append_at(far, P + (9 << 30), **base))


@pytest.mark.parametrize("bad", [dict(seen=None), dict(seen=P + 2), dict(words=0), dict(words=33), dict(words=-1), dict(q=None), dict(heads=5),
                                 dict(max_new=0), dict(dtype=2), dict(max_len=4096)])
def test_tree_attention_refuses(bad):
    refused(b.moe_kv4_tree_attention, *tree_attend(batch(), **bad))


def test_tree_attention_overlaps():
    far = batch(pool=P + (9 << 30), tokens=4)
    apart(b.moe_kv4_tree_attention, *tree_attend(far, seen=C, words=2, q=A, o=B))
    overlap(b.moe_kv4_tree_attention, *tree_attend(far, seen=B + 4 * 256 * 4 - 4, words=2, q=A, o=B))
    need = b.moe_kv4_tree_attention_workspace_bytes(far, 4, F32, 1, 4096)
    overlap(b.moe_kv4_tree_attention, *tree_attend(far, seen=D + need - 4, words=1, q=A, o=B, max_len=4096, ws=D, wsb=need))
    b.moe_kv4_tree_attention(*tree_attend(batch(tokens=0)))


@pytest.mark.parametrize("dtype,max_new,most,groups,rows", [(F32, 1, 251, 512, 16), (BF16, 64, 4031, 256, 256)])
def test_tree_attention_of_more_work_than_an_int_counts(dtype, max_new, most, groups, rows):
    """Kernels that share all steps out number them: (4 tokens / rows + 1) blocks of each
    of 2048 pairs (sequence, kv head), whatever q_start holds, of 2^20 / 64 + 6 steps
    at most, 2^31 / 2048 / 16390 = 63.98.  One block more and the call is cut as
    moe_kv4_attention's is."""
    bt = batch(head_dim=128, kv_heads=8, seqs=256, page_size=1024, table_cols=1024, table_stride=1024, tokens=most)
    need = b.moe_kv4_tree_attention_workspace_bytes(bt, 32, dtype, max_new, 4096)
    assert need == groups * 2 * rows * (128 + 2) * 4 + 257 * 4
    bt.tokens = most + 1
    assert b.moe_kv4_tree_attention_workspace_bytes(bt, 32, dtype, max_new, 4096) == b.moe_kv4_attention_workspace_bytes(bt, 32, max_new, 4096) != need
    bt.table_cols = 1023
    assert b.moe_kv4_tree_attention_workspace_bytes(bt, 32, dtype, max_new, 4096) == need


@pytest.mark.parametrize("bad", [dict(parent=None), dict(parent=A + 1), dict(q_start=None), dict(kv_len=None), dict(pos=None), dict(seen=None),
                                 dict(pos=C + 2), dict(seqs=0), dict(seqs=(1 << 20) + 1), dict(tokens=-1), dict(tokens=(1 << 24) + 1),
                                 dict(words=0), dict(words=33)])
def test_draft_tree_refuses(bad):
    refused(b.moe_draft_tree, *plan(**bad))


def test_draft_tree_overlaps():
    apart(b.moe_draft_tree, *plan())
    for bad in (dict(pos=A), dict(pos=D + 9 * 8 - 4), dict(seen=A + 32), dict(seen=B + 12), dict(pos=B + 64 + 8)):
        overlap(b.moe_draft_tree, *plan(**bad))
    b.moe_draft_tree(*plan(tokens=0, parent=None, pos=None, seen=None))


@pytest.mark.parametrize("bad", [
    dict(p=None), dict(p=A + 2), dict(ps=49), dict(q=B + 1), dict(qs=40), dict(ids=None), dict(parent=None), dict(u=None), dict(u=C + 129),
    dict(q_start=None), dict(seqs=0), dict(tokens=-1), dict(vocab=0), dict(vocab=(1 << 24) + 1, ps=1 << 25, qs=1 << 25), dict(dtype=2),
    dict(path=None), dict(count=None), dict(next=None), dict(next=D + 130), dict(vocab=1 << 20, ps=1 << 20, qs=1 << 20)])
def test_verify_refuses(bad):
    refused(b.moe_verify_drafts, *verify(**bad))


def test_verify_overlaps():
    apart(b.moe_verify_drafts, *verify())
    apart(b.moe_verify_drafts, *verify(q=None))
    apart(b.moe_verify_drafts, *verify(dtype=BF16, p=A + 2, ps=51))
    for bad in (dict(path=A + 400), dict(path=B), dict(count=C), dict(next=C + 64 + 8), dict(count=C + 128), dict(next=C + 192), dict(next=D + 64),
                dict(count=D + 32), dict(next=D)):
        overlap(b.moe_verify_drafts, *verify(**bad))
    large = dict(p=A, q=None, ps=1 << 20, vocab=1 << 20, ws=E, wsb=b.moe_verify_drafts_workspace_bytes(3, 1 << 20))
    assert large["wsb"] > 0
    apart(b.moe_verify_drafts, *verify(**large))
    for bad in (dict(ws=E + 8), dict(wsb=large["wsb"] - 1), dict(ws=None), dict(ws=A + 16), dict(ws=C), dict(next=E + 64), dict(path=E)):
        refused(b.moe_verify_drafts, *verify(**{**large, **bad}))


def test_keep_refuses():
    one = batch(pool=None)
    apart(b.moe_kv4_keep, *keep(one))   # the batch's own pool is not looked at
    for pools in ((), (None,), (E, None), (E + 4,), (E,) * 2, (E, E + (1 << 20), E + 16), (E + 9 * 2 * 16 * 72 - 16, E), [E] * 1025):
        refused(b.moe_kv4_keep, *keep(one, pools))
    apart(b.moe_kv4_keep, *keep(one, (E + 9 * 2 * 16 * 72, E)))
    for bad in (dict(path=None), dict(count=None), dict(path=P + 2), dict(count=P + 1), dict(path=E), dict(count=E + (1 << 20) + 64)):
        refused(b.moe_kv4_keep, *keep(one, **bad))
    for bad in (dict(page_size=8), dict(kv_heads=0), dict(head_dim=32), dict(seqs=0)):
        refused(b.moe_kv4_keep, *keep(batch(**bad)))
    refused(b.moe_kv4_keep, None, [E], P, P, 0)
    b.moe_kv4_keep(*keep(batch(tokens=0), path=None, count=None))


def test_null_pools():
    assert b.lib().moe_kv4_keep(ctypes.byref(batch()), None, 1, P, P, None) == b.MOE_ERR_ARG
