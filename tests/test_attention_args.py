"""What the attention entry points refuse, found on the host before any GPU work."""
import ctypes

import pytest

from paper_2511_05814_amd import binding as b

BUF = ctypes.create_string_buffer(4096 + 256)
P = (ctypes.addressof(BUF) + 255) // 256 * 256     # an aligned address; never dereferenced
F32, BF16 = b.MOE_DTYPE_F32, b.MOE_DTYPE_BF16


def refused(f, *args):
    with pytest.raises(b.MoeError) as e:
        f(*args)
    assert e.value.code == b.MOE_ERR_ARG and b.moe_last_error()


def test_matrix_bytes():
    assert b.moe_q4_matrix_bytes(1, 64) == 32 + 3
    assert b.moe_q4_matrix_bytes(4099, 2048) == 4099 * (1024 + 32 * 3)
    for n, k in ((0, 64), (4, 0), (4, 32), (4, 100), (1 << 40, 1 << 40)):
        assert b.moe_q4_matrix_bytes(n, k) == 0


def q4(**kw):
    a = dict(x=P, x_stride=128, w=P, y=P, y_stride=7, rows=2, n=7, k=128, dtype=BF16, stream=0)
    a.update(kw)
    return tuple(a.values())


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(x=P + 8), dict(x_stride=127), dict(x_stride=130), dict(w=None), dict(w=P + 4), dict(y=None),
    dict(y=P + 1), dict(y_stride=6), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(n=0), dict(k=0), dict(k=96),
    dict(dtype=b.MOE_DTYPE_Q2G16), dict(dtype=9)])
def test_q4_refuses(bad):
    refused(b.moe_q4_matmul, *q4(**bad))


def test_no_rows_is_no_work():
    b.moe_q4_matmul(*q4(rows=0))
    b.moe_kv4_append(*append(batch(tokens=0)))
    b.moe_kv4_read(batch(tokens=0), P, P, F32, 0)
    b.moe_kv4_attention(*attend(batch(tokens=0)))
    b.moe_norm_residual(*norm(rows=0))


def batch(**kw):
    a = dict(pool=P, page_table=P, q_start=P, kv_len=P, table_stride=5, pages=9, page_size=16, kv_heads=2, head_dim=64,
             table_cols=5, seqs=3, tokens=4)
    a.update(kw)
    return b.moe_kv4_batch(*a.values())


def append(bt, **kw):
    a = dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, cos=P, sin=P, max_pos=80, rot=64, out=P + 16, os=256, heads=4,
             dtype=BF16, stream=0)
    a.update(kw)
    return (bt, *a.values())


def attend(bt, **kw):
    a = dict(q=P, qs=256, o=P, os=256, heads=4, scale=0.125, dtype=F32, max_new=1, max_len=1, ws=None, wsb=0, stream=0)
    a.update(kw)
    return (bt, *a.values())


@pytest.mark.parametrize("bad", [
    dict(pool=None), dict(pool=P + 4), dict(page_table=None), dict(q_start=None), dict(kv_len=None), dict(kv_len=P + 2),
    dict(table_stride=4), dict(pages=0), dict(page_size=8), dict(page_size=48), dict(page_size=2048), dict(kv_heads=0),
    dict(head_dim=96), dict(head_dim=256), dict(table_cols=0), dict(table_cols=1 << 27, table_stride=1 << 27),
    dict(seqs=0), dict(tokens=-1)])
def test_batches_refused_everywhere(bad):
    refused(b.moe_kv4_append, *append(batch(**bad)))
    refused(b.moe_kv4_read, batch(**bad), P, P, F32, 0)
    refused(b.moe_kv4_attention, *attend(batch(**bad)))
    assert b.moe_kv4_attention_workspace_bytes(batch(**bad), 4, 1, 4096) == 0


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q=P + 8), dict(qs=255), dict(qs=260), dict(k=None), dict(ks=100), dict(v=P + 2), dict(vs=132),
    dict(cos=None), dict(sin=P + 4), dict(max_pos=0), dict(rot=-16), dict(rot=80), dict(rot=24), dict(out=None),
    dict(out=P), dict(os=200), dict(heads=0), dict(heads=3), dict(dtype=2)])
def test_append_refuses(bad):
    refused(b.moe_kv4_append, *append(batch(), **bad))


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(qs=200), dict(o=P + 4), dict(os=254), dict(heads=5), dict(dtype=2), dict(max_new=0),
    dict(max_len=0), dict(max_len=4096)])   # the last needs a workspace
def test_attention_refuses(bad):
    refused(b.moe_kv4_attention, *attend(batch(), **bad))


def test_attention_workspace():
    need = b.moe_kv4_attention_workspace_bytes(batch(), 4, 1, 4096)
    assert need > 0 and need % (4 * 4 * 66 * 4) == 0   # splits of 16 rows of 64 + 2 floats
    refused(b.moe_kv4_attention, *attend(batch(), max_len=4096, ws=P, wsb=need - 1))
    refused(b.moe_kv4_attention, *attend(batch(), max_len=4096, ws=P + 4, wsb=need))
    refused(b.moe_kv4_read, batch(), None, P, F32, 0)
    assert b.moe_kv4_attention_workspace_bytes(batch(), 3, 1, 4096) == 0


def test_attention_limits():
    # rows that an int could not count
    big = batch(tokens=1 << 24)
    refused(b.moe_kv4_attention, *attend(big, heads=128, qs=128 * 64, os=128 * 64, ws=P, wsb=1 << 60))
    # hints far past the batch do not size the work past its tokens
    small = b.moe_kv4_attention_workspace_bytes(batch(tokens=1), 4, 1 << 24, 1 << 29)
    assert 0 < small <= 1024 * 4 * 66 * 4


def norm(**kw):
    a = dict(h=P, hs=64, y=P, ys=64, gate=P, gs=0, post=P, pre=P, scale=1.0, eps=1e-5, ho=P, hos=64, x=P, xs=64, rows=3,
             d=64, dtype=BF16, stream=0)
    a.update(kw)
    return tuple(a.values())


@pytest.mark.parametrize("bad", [
    dict(h=None), dict(h=P + 4), dict(hs=60), dict(hs=66), dict(y=P + 2), dict(ys=63), dict(y=None), dict(gate=P + 4),
    dict(gs=32), dict(gs=66), dict(post=P + 8), dict(pre=P + 8), dict(ho=None, x=None), dict(ho=P + 4), dict(hos=128),
    dict(xs=128), dict(x=P + 2), dict(rows=-1), dict(d=0), dict(d=60), dict(d=16392), dict(dtype=2)])
def test_norm_refuses(bad):
    refused(b.moe_norm_residual, *norm(**bad))
