"""The attention entry points on an MI355X against the fp64 oracle: 4-bit
products, rotation and append, attention over the 4-bit cache, block norms.

Tolerances, from the arithmetic (u = 2^-24, one fp32 rounding; bf16, with 8
significant bits, rounds to 2^-8 relative: 1 + 2^-8 lies midway between two):
* products: x enters whole and codes exactly, so what is left are fp32 sums,
  64 columns and k / 64 groups deep, of terms up to (16 + q) and (16 + zero)
  times |x|; twice u for matrix-core sums that truncate.
* append: the same fp32 operations as the oracle's in fp32, bit for bit.
* attention: q carries 22 bits (fp32) or all of its 8 (bf16), so a score is off
  by at most reach (2^-22 + D 2u), reach = scale max_j sum |q||k|, and a
  probability by that and its own rounding (2^-22; 2^-11 with one fp16 number);
  an output is a mean of values weighted with them, and sums of up to n terms
  add n u of the largest value in the worst case, 64 u with the 32-token steps
  that the sums go by at these lengths.
* norms: sums of squares in fp32 over trees, a few roundings an element.
"""
import numpy as np
import pytest

from oracle import attention as oa
from paper_2511_05814_amd import binding as b

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests._attention_rig import Batch, bf16, device  # noqa: E402

U = 2.0 ** -24
BF = 2.0 ** -7.99   # a bf16 rounding and the little above it


def ops():
    from paper_2511_05814_amd import attention
    return attention


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


# -- products with 4-bit weights ------------------------------------------------

def matrix(rng, n, k):
    buf = rng.integers(0, 256, b.moe_q4_matrix_bytes(n, k), dtype=np.uint8)
    scale = (0.002 * np.exp(rng.standard_normal(n * k // 64))).astype(np.float16)
    buf[n * k // 2:n * k // 2 + n * k // 32] = scale.view(np.uint8)
    return buf


def check_product(x, buf, n, k, y, dtype):
    want = x @ oa.q4_dequantize(buf, n, k).T
    s = buf[n * k // 2:n * k // 2 + n * k // 32].view(np.float16).astype(np.float64).reshape(n, k // 64)
    z = buf[n * k // 2 + n * k // 32:].reshape(n, k // 64) / 16.0
    mass = np.abs(x) @ np.repeat(s * (32 + 16 + z), 64, 1).T
    err = np.abs(host(y) - want)
    assert (err <= mass * (80 + k // 64) * 2 * U + (BF * np.abs(want) if dtype == "bf16" else 0)).all()
    rel = np.linalg.norm(err) / np.linalg.norm(want)
    assert rel <= (2.5e-3 if dtype == "bf16" else 1e-5), rel
    return rel


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,k", [(1, 1, 64), (1, 17, 64), (1, 512, 512), (2, 33, 192), (3, 130, 4096), (4, 64, 1088),
                                      (5, 48, 576), (13, 259, 2048), (16, 31, 128), (17, 96, 320), (33, 100, 704),
                                      (64, 256, 512), (65, 129, 960), (130, 384, 256), (257, 200, 1024), (300, 513, 64),
                                      (129, 1000, 1472)])
def test_q4_matmul(rows, n, k, dtype):
    rng = np.random.default_rng(rows * 1000 + n + k)
    buf = matrix(rng, n, k)
    x = rng.standard_normal((rows, k)).astype(np.float32) * np.exp(rng.standard_normal(k)).astype(np.float32)
    x = bf16(x) if dtype == "bf16" else x
    y = ops().q4_matmul(device(x, dtype), torch.from_numpy(buf).cuda(), n)
    check_product(x.astype(np.float64), buf, n, k, y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,k", [(1000, 2000, 128), (2000, 2001, 192), (700, 3001, 1088), (700, 3001, 1024), (333, 5003, 576),
                                      (1025, 1929, 64), (100, 16384, 512)])
def test_q4_matmul_many_rows(rows, n, k, dtype):
    """Shapes that go by tiles of 64 and of 128 rows, with their odd ends; rows
    of scales that are and are not multiples of eight groups."""
    rng = np.random.default_rng(n + k)
    buf = matrix(rng, n, k)
    x = rng.standard_normal((rows, k)).astype(np.float32) * np.exp(rng.standard_normal(k)).astype(np.float32)
    x = bf16(x) if dtype == "bf16" else x
    wide = torch.zeros((rows, k + 8), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    wide[:, :k] = device(x, dtype)
    out = torch.full((rows, n + 3), 7.0, dtype=wide.dtype, device="cuda")
    y = ops().q4_matmul(wide[:, :k], torch.from_numpy(buf).cuda(), n, out=out[:, 1:1 + n])
    check_product(x.astype(np.float64), buf, n, k, y, dtype)
    assert (out[:, 0] == 7).all() and (out[:, 1 + n:] == 7).all()


def test_q4_matmul_many_rows_keeps_rows_apart():
    rng = np.random.default_rng(5)
    rows, n, k = 700, 3001, 128
    w = torch.from_numpy(matrix(rng, n, k)).cuda()
    x = rng.standard_normal((rows, k)).astype(np.float32)
    x[3, 70], x[400, 0], x[699, 127] = np.nan, np.inf, -np.inf
    for dtype in ("f32", "bf16"):
        bad = np.isnan(host(ops().q4_matmul(device(x, dtype), w, n)))
        assert bad[[3, 400, 699]].all() and bad.sum() == 3 * n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 3, 9, 40, 150])
def test_q4_matmul_strided(rows, dtype):
    """x a slice of wider rows, y inside a larger tensor whose other columns stay."""
    rng = np.random.default_rng(rows)
    n, k = 70, 192
    buf = matrix(rng, n, k)
    x = bf16(rng.standard_normal((rows, k + 64)))
    wide = device(x, dtype)
    out = torch.full((rows, n + 9), 7.0, dtype=wide.dtype, device="cuda")
    y = ops().q4_matmul(wide[:, 32:32 + k], torch.from_numpy(buf).cuda(), n, out=out[:, 5:5 + n])
    check_product(x[:, 32:32 + k].astype(np.float64), buf, n, k, y, dtype)
    assert (out[:, :5] == 7).all() and (out[:, 5 + n:] == 7).all()


@pytest.mark.parametrize("rows", [2, 20, 200])
def test_q4_matmul_keeps_rows_apart(rows):
    """A row of x that holds a NaN or an infinity is a row of NaN, and only that row."""
    rng = np.random.default_rng(4)
    n, k = 40, 128
    buf = matrix(rng, n, k)
    x = rng.standard_normal((rows, k)).astype(np.float32)
    x[0, 3], x[rows - 1, 100] = np.nan, np.inf
    for dtype in ("f32", "bf16"):
        y = host(ops().q4_matmul(device(x, dtype), torch.from_numpy(buf).cuda(), n))
        assert np.isnan(y[[0, rows - 1]]).all() and np.isfinite(y[1:rows - 1]).all()


def test_q4_matmul_extremes():
    """Codes and zeros at both ends, scale zero, x of very different sizes."""
    n, k = 32, 256
    buf = np.zeros(b.moe_q4_matrix_bytes(n, k), dtype=np.uint8)
    buf[:n * k // 4] = 0xFF
    s = np.full((n, 4), 0.01, dtype=np.float16)
    s[:, 1] = 0
    buf[n * k // 2:n * k // 2 + n * k // 32] = s.reshape(-1).view(np.uint8)
    buf[n * k // 2 + n * k // 32:] = np.tile([0, 255], n * 2)
    x = np.ones((3, k), dtype=np.float32)
    x[1] *= 1e-30
    x[2, ::2] = 1e20
    y = ops().q4_matmul(device(x, "f32"), torch.from_numpy(buf).cuda(), n)
    want = x.astype(np.float64) @ oa.q4_dequantize(buf, n, k).T
    assert (np.abs(host(y) - want) <= 1e-5 * np.abs(want)).all()


# -- rotation and append ---------------------------------------------------------

def tables(positions, rot):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def run_append(bt, rot, dtype, max_pos, joined=True, seed=3):
    """Appends random tokens; returns what the pool must hold and q must be."""
    rng = np.random.default_rng(seed)
    D, hq, hk, T = bt.D, bt.heads, bt.kv_heads, bt.tokens
    qkv = rng.standard_normal((T, (hq + 2 * hk) * D)).astype(np.float32) * np.exp(rng.standard_normal((hq + 2 * hk) * D)).astype(np.float32)
    qkv = bf16(qkv) if dtype == "bf16" else qkv
    dev = device(qkv, dtype)
    parts = dev[:, :hq * D], dev[:, hq * D:(hq + hk) * D], dev[:, (hq + hk) * D:]
    q, k, v = (p.unflatten(1, (-1, D)) for p in parts)
    if not joined:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    cos, sin = tables(max_pos, rot)
    args = bt.args()
    out = ops().kv4_append(q, k, v, torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), *args)
    hq_, hk_, hv_ = np.split(qkv.reshape(T, -1, D), [hq, hq + hk], 1)
    pos = bt.positions()
    placed = (pos >= 0) & (pos < max_pos)
    safe = np.where(placed, pos, 0)
    c, s = cos[safe], sin[safe]
    want_q = np.where(placed[:, None, None], oa.rotate(hq_, c, s), 0)
    kq, km = oa.kv4_quantize(oa.rotate(hk_, c, s))
    vq, vm = oa.kv4_quantize(hv_)
    pool = bt.pool.copy()
    for t in range(T):
        seq = int(np.searchsorted(bt.q_start[1:], t, side="right"))
        col, at = int(pos[t]) // bt.P, int(pos[t]) % bt.P
        if not placed[t] or col >= bt.table.shape[1] or not 0 <= bt.table[seq, col] < pool.shape[0]:
            continue
        for h in range(hk):
            rec = list(oa.unpack_record(pool[bt.table[seq, col], h], bt.P, D))
            for i, new in enumerate((kq, km, vq, vm)):
                rec[i] = np.array(rec[i])
                rec[i][at] = new[t, h]
            pool[bt.table[seq, col], h] = oa.record(*rec)
    return args, out, want_q, pool


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,P,heads,kv,rot,new,old", [
    (64, 16, 4, 2, 64, [1], [0]), (128, 16, 8, 8, 128, [1, 1, 1], [15, 16, 0]), (64, 32, 5, 1, 32, [7, 0, 33], [3, 9, 31]),
    (128, 64, 6, 3, 128, [70], [60]), (128, 16, 4, 4, 0, [3, 2], [14, 100]), (64, 1024, 2, 2, 16, [5, 6], [1020, 3])])
def test_append_stores_the_bits(D, P, heads, kv, rot, new, old, dtype):
    bt = Batch(new, old, heads, kv, D, P).fill()
    args, q, want_q, pool = run_append(bt, rot, dtype, max_pos=2048, joined=len(new) != 2)
    assert np.array_equal(args[0].cpu().numpy(), pool)
    got = q.float().cpu().numpy()
    assert np.array_equal(got, bf16(want_q) if dtype == "bf16" else want_q)
    # and reads back as the values that the bytes stand for
    bt.pool = pool
    k, v = ops().kv4_read(*args, bt.tokens, D, q.dtype)
    for i in range(len(new)):
        rows = slice(bt.q_start[i], bt.q_start[i + 1])
        wk, wv, _ = bt.sequence(i)
        n = new[i]
        assert np.array_equal(host(k)[rows].transpose(1, 0, 2), wk[:, bt.len[i] - n:])
        assert np.array_equal(host(v)[rows].transpose(1, 0, 2), wv[:, bt.len[i] - n:])


def test_append_skips_what_has_no_place():
    """Negative positions, positions past the tables, missing and impossible
    pages and columns past the table: nothing else changes."""
    bt = Batch([9, 4, 40], [0, 30, 0], 2, 1, 64, 16, short=4).fill()
    bt.table[1, 1] = 12345       # no such page: positions 16 .. of sequence 1
    bt.table[2, 1] = -1
    bt.table = np.ascontiguousarray(bt.table[:, :2])
    args, q, want_q, pool = run_append(bt, 64, "f32", max_pos=34)
    assert np.array_equal(args[0].cpu().numpy(), pool)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert (want_q[:4] == 0).all()      # sequence 0 has five tokens of nine
    k, v = ops().kv4_read(*args, bt.tokens, 64)
    assert (k[:4] == 0).all() and (v[9:13] == 0).all() and (k[4:9] != 0).any()


def test_append_marks_groups_that_cannot_be_stored():
    bt = Batch([3], [5], 2, 2, 64, 16)
    args = bt.args()
    q, k, v = (torch.ones((3, 2, 64), device="cuda") for _ in range(3))
    k[0, 1, 3], v[2, 0, 63], v[1, 1, 0] = float("inf"), float("nan"), 3e38
    none = torch.empty((100, 0), device="cuda")
    ops().kv4_append(q, k, v, none, none, *args)
    k, v = (host(t) for t in ops().kv4_read(*args, 3, 64))
    assert np.isnan(k[0, 1, :32]).all() and np.isnan(k).sum() == 32
    assert np.isnan(v[2, 0, 32:]).all() and np.isnan(v).sum() == 32
    assert v[1, 1, 0] == 15 * oa.STEPS[254] and (v[1, 1, 1:32] == 0).all()


# -- attention ---------------------------------------------------------------------

def check_attention(bt, dtype, scale=None, max_new=None, max_len=None, seed=5, q=None):
    D = bt.D
    scale = D ** -0.5 if scale is None else scale
    if q is None:
        q = np.random.default_rng(seed).standard_normal((bt.tokens, bt.heads, D)) * 2
    q = bf16(q) if dtype == "bf16" else np.asarray(q, dtype=np.float32)
    dev = device(q, dtype)
    o = host(ops().kv4_attention(dev, *bt.args(), scale, max_new=max_new, max_len=max_len))
    want, reach, top = bt.attend(q.astype(np.float64), scale)
    score = reach * (2.0 ** -22 + 2 * D * U)
    prob = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    tol = top * (2 * score + 2 * prob + 64 * U)
    tol = tol[..., None] + (BF * np.abs(want) if dtype == "bf16" else 0)
    assert np.array_equal(np.isnan(o), np.isnan(want))
    fine = ~np.isnan(want)
    bad = np.abs(o - want)[fine] > np.broadcast_to(tol, want.shape)[fine]
    assert not bad.any(), (np.abs(o - want)[fine].max(), bad.mean())
    return o, want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,P,heads,kv,new,old", [
    (64, 16, 4, 2, [1], [0]),                      # one token and nothing before it
    (128, 16, 8, 8, [1, 1, 1, 1], [0, 15, 16, 31]),  # around a page's and a step's end
    (64, 32, 5, 1, [1, 1], [127, 128]),            # an odd group, around a workgroup's step
    (128, 64, 8, 2, [1], [700]),                   # several splits
    (128, 16, 20, 1, [1, 1], [37, 500]),           # more heads to a key head than a tile has rows
    (64, 128, 2, 2, [5, 0, 1], [130, 40, 0]),      # a few tokens at a time, one sequence without any
    (128, 32, 4, 2, [100, 1, 17], [0, 300, 33]),   # prompts
    (64, 16, 6, 3, [200], [55]),
    (128, 16, 16, 4, [70, 90], [64, 0])])
def test_attention(D, P, heads, kv, new, old, dtype):
    check_attention(Batch(new, old, heads, kv, D, P, seed=D + P).fill(0.5), dtype)


@pytest.mark.parametrize("max_new,max_len", [(1, 1), (1, 1 << 20), (4096, 1), (3, 100)])
def test_attention_is_right_whatever_the_hints(max_new, max_len):
    bt = Batch([40, 3], [50, 600], 8, 2, 128, 16, seed=6).fill(0.3)
    for dtype in ("f32", "bf16"):
        check_attention(bt, dtype, max_new=max_new, max_len=max_len)


@pytest.mark.parametrize("new", [[6, 1, 2], [80, 1, 40]])
def test_rows_that_see_nothing_are_zeros(new):
    """kv_len smaller than the new tokens, no tokens at all, pages that are missing."""
    bt = Batch(new, [0, 0, 50], 4, 2, 64, 16, seed=7, short=1).fill(0.3)
    bt.table[2, 0] = -1
    bt.table[2, 2] = 999
    o, want = check_attention(bt, "f32")
    assert (o[0] == 0).all() and (o[new[0]] == 0).all() and (o[-1] != 0).any()
    bt.table[2, :] = -1
    o, _ = check_attention(bt, "bf16")
    assert (o[new[0] + 1:] == 0).all()


@pytest.mark.parametrize("new", [1, 9, 150])
@pytest.mark.parametrize("D", [64, 128])
def test_marked_entries_reach_only_rows_that_see_them(new, D):
    """NaN in later tokens, in unused places of a page and behind the end stays out."""
    bt = Batch([new, 1], [20, 33], 4, 2, D, 32, seed=8).fill(0.3)
    last = bt.len[0] - 1
    for pos, value in ((last, True), (last // 2, False)):
        page = bt.table[0, pos // 32]
        rec = [np.array(x) for x in oa.unpack_record(bt.pool[page, 0], 32, D)]
        rec[3 if value else 1][pos % 32, 1] = 255 << 8
        rec[2 if value else 0][pos % 32, 32:64] = 0
        bt.pool[page, 0] = oa.record(*rec)
    for b_ in range(2):    # everything behind the end of each sequence
        tail = bt.len[b_] % 32
        page = bt.table[b_, (bt.len[b_] - 1) // 32]
        if tail:
            for h in range(2):
                rec = [np.array(x) for x in oa.unpack_record(bt.pool[page, h], 32, D)]
                rec[1][tail:] = rec[3][tail:] = 255 << 8
                bt.pool[page, h] = oa.record(*rec)
    for dtype in ("f32", "bf16"):
        o, want = check_attention(bt, dtype)
        assert np.isnan(o[new - 1, :2]).all() and not np.isnan(o[:, 2:]).any()


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_with_scales_from_end_to_end(new, D):
    """Groups whose scale code is any of 0 .. 254: the smallest and the largest
    steps, among zeros and ordinary ones."""
    bt = Batch([new, 1], [90, 250], 4, 2, D, 16, seed=13).fill(0.3)
    rng = np.random.default_rng(13)
    for page in range(bt.pool.shape[0]):
        for h in range(2):
            rec = [np.array(x) for x in oa.unpack_record(bt.pool[page, h], 16, D)]
            for i in (1, 3):    # a sixth of the groups small, large or all zero
                pick = rng.random(rec[i].shape)
                k = np.where(pick < 0.05, rng.integers(0, 10, rec[i].shape), rec[i] >> 8)
                k = np.where(pick > 0.95, rng.integers(244, 255, rec[i].shape) if i == 3 else k, k)
                rec[i] = (k << 8 | (rec[i] & 255)).astype(np.uint16)
                zero = np.repeat((pick > 0.5) & (pick < 0.55), 32, 1)
                rec[i - 1][zero] = 0
                rec[i][(pick > 0.5) & (pick < 0.55)] = 0
            bt.pool[page, h] = oa.record(*rec)
    for dtype in ("f32", "bf16"):
        check_attention(bt, dtype)


def test_attention_scores_far_apart_and_equal():
    """Softmax where one key takes all, where all are alike, and with scales of either sign or none."""
    bt = Batch([1, 30], [400, 300], 4, 2, 64, 16, seed=9).fill(1.5)
    big = np.random.default_rng(1).standard_normal((31, 4, 64)) * 300
    for q in (big, np.zeros((31, 4, 64)), big * 1e-20, big * 1e15 * 2.0 ** -40):
        check_attention(bt, "f32", q=q)
        check_attention(bt, "bf16", q=q)
    check_attention(bt, "f32", scale=0.0)
    check_attention(bt, "f32", scale=-0.3)


def test_attention_of_a_row_with_nan_leaves_the_others():
    for new in (4, 100):
        bt = Batch([new], [50], 4, 2, 64, 16, seed=10).fill(0.3)
        q = np.random.default_rng(2).standard_normal((new, 4, 64)).astype(np.float32)
        q[1, 2, 7] = np.nan
        o = host(ops().kv4_attention(device(q, "f32"), *bt.args(), 0.125))
        assert np.isnan(o[1, 2]).all() and np.isnan(o).sum() == 64


def test_attention_strided_queries_and_given_outputs():
    bt = Batch([3, 40], [20, 30], 4, 2, 128, 16, seed=11).fill(0.3)
    wide = torch.randn((43, 1024), device="cuda")
    q = wide[:, 256:768].unflatten(1, (4, 128))
    out = torch.full((43, 8, 128), 3.0, device="cuda")
    ops().kv4_attention(q, *bt.args(), 0.1, out=out[:, 2:6])
    want, reach, top = bt.attend(host(q), 0.1)
    assert (np.abs(host(out[:, 2:6]) - want) <= (top * (2 * reach * (2.0 ** -22 + 256 * U) + 2.0 ** -21 + 64 * U))[..., None]).all()
    assert (out[:, :2] == 3).all() and (out[:, 6:] == 3).all()


def test_pages_past_four_gigabytes():
    """Entries whose byte offsets pass 32 bits, written, read and attended to."""
    D, P = 128, 1024
    pages = (5 << 30) // (P * D * 9 // 8)
    pool = torch.empty((pages, 1, P * D * 9 // 8), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    new = 1100
    start, length = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, new], [new]))
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn((new, h, D), device="cuda", generator=g) for h in (2, 1, 1))
    none = torch.empty((2048, 0), device="cuda")
    ops().kv4_append(q, k, v, none, none, pool, table, start, length)
    kk, vv = ops().kv4_read(pool, table, start, length, new, D)
    want, _ = oa.kv4_quantize(k.cpu().numpy()), None
    assert np.array_equal(host(kk), oa.kv4_values(*want))
    o = ops().kv4_attention(q[-1:], pool, table, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), length, 0.09)
    s = host(kk)[:, 0]
    for h in range(2):
        p = np.exp(0.09 * (s @ host(q)[-1, h]))
        ref = (p / p.sum()) @ host(vv)[:, 0]
        assert np.abs(host(o)[0, h] - ref).max() <= 1e-5 * np.abs(host(vv)).max()


# -- norms --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", [(1, 8), (3, 64), (5, 504), (2, 512), (7, 520), (1, 1024), (4, 1832), (2, 2048), (3, 2056),
                                    (2, 4096), (1, 5000), (2, 8192), (1, 16384)])
def test_norm_residual(rows, d, dtype):
    rng = np.random.default_rng(d)
    h = rng.standard_normal((rows, d)).astype(np.float32)
    y = rng.standard_normal((rows, d)).astype(np.float32) * 3
    y = bf16(y) if dtype == "bf16" else y
    gate, post, pre = rng.standard_normal((rows, d)).astype(np.float32), *rng.standard_normal((2, d)).astype(np.float32)
    dev = [torch.from_numpy(t).cuda() for t in (h, gate, post, pre)]
    for use in range(6):
        kw = [dict(gate=gate, post=post, pre=pre), dict(gate=gate[0], post=post, pre=pre), dict(post=post), dict(gate=gate[0]),
              dict(pre=pre), dict()][use]
        on = dict(zip(("gate", "post", "pre"), (dev[1], dev[2], dev[3])))
        on = {n: (on[n][0] if n == "gate" and t.ndim == 1 else on[n]) for n, t in kw.items()}
        ho, xo = ops().norm_residual(dev[0], device(y, dtype), residual_scale=0.75, eps=1e-5, **on)
        wh, wx = oa.norm_residual(h, y, residual_scale=0.75, **kw)
        g = np.abs(kw.get("gate", np.float32(1))) * np.abs((wh - 0.75 * h.astype(np.float64)) / np.where(kw.get("gate", 1) == 0, 1, kw.get("gate", 1)))
        tol_h = 24 * U * (np.abs(0.75 * h) + g)
        assert (np.abs(host(ho) - wh) <= tol_h).all()
        inv = np.abs(wx / np.where(wh == 0, 1, wh))
        tol_x = tol_h * inv + 24 * U * np.abs(wx) + (BF * np.abs(wx) if dtype == "bf16" else 0)
        assert (np.abs(host(xo) - wx) <= tol_x).all()


def test_norm_without_a_block_and_in_place():
    h = torch.randn((5, 256), device="cuda")
    keep = host(h)
    none, x = ops().norm_residual(h, dtype=torch.bfloat16, want_h=False)
    wh, wx = oa.norm_residual(keep)
    assert none is None and x.dtype == torch.bfloat16 and (np.abs(host(x) - wx) <= 2 * BF * np.abs(wx)).all()
    y = torch.randn((5, 512), device="cuda")[:, 128:384]
    wh, wx = oa.norm_residual(keep, host(y), gate=np.full(256, 0.5), residual_scale=2.0)
    ho, x = ops().norm_residual(h, y, gate=torch.full((256,), 0.5, device="cuda"), residual_scale=2.0, h_out=h)
    assert ho is h and np.abs(host(h) - wh).max() <= 24 * U * np.abs(wh).max() * 4
    assert np.abs(host(x) - wx).max() <= 1e-5 * np.abs(wx).max()
    assert (host(ops().norm_residual(torch.zeros((2, 64), device="cuda"))[1]) == 0).all()


# -- together ------------------------------------------------------------------------

def test_streams_and_graphs():
    """The calls go to torch's current stream and can be captured; replays give
    what eager calls give, eager work between them."""
    rng = np.random.default_rng(12)
    n, k = 8 * 64, 256
    w = torch.from_numpy(matrix(rng, n, k)).cuda()
    bt = Batch([1, 1], [300, 20], 4, 2, 64, 16, seed=12).fill(0.3)
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(512, 64))
    args, h = bt.args(), torch.randn((2, k), device="cuda")

    def step():
        _, x = ops().norm_residual(h, dtype=torch.bfloat16)
        qkv = ops().q4_matmul(x, w, n).unflatten(1, (8, 64))
        q = ops().kv4_append(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], cos, sin, *args)
        return ops().kv4_attention(q, *args, 0.125, max_new=1, max_len=512)

    want = step().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(step(), want)
        graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o = step()
    for i in range(3):
        h.normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        eager = step().clone()
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager)


def test_python_refusals():
    a = ops()
    x = torch.zeros((2, 128), device="cuda")
    w = torch.zeros(b.moe_q4_matrix_bytes(8, 128), dtype=torch.uint8, device="cuda")
    for call in (lambda: a.q4_matmul(x.half(), w, 8), lambda: a.q4_matmul(x, w, 9), lambda: a.q4_matmul(x.cpu(), w, 8),
                 lambda: a.q4_matmul(x, w.cpu(), 8), lambda: a.q4_matmul(x.t(), w, 8), lambda: a.q4_matmul(x[0], w, 8),
                 lambda: a.q4_matmul(x, w, 8, out=x), lambda: a.norm_residual(x.bfloat16()),
                 lambda: a.norm_residual(x, x[:1]), lambda: a.norm_residual(x, x, gate=x[0, :64])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(b.MoeError):
        a.q4_matmul(torch.zeros((2, 130), device="cuda")[:, 1:129], w, 8)   # not aligned
    bt = Batch([1, 1], [3, 4], 4, 2, 64, 16)
    pool, table, start, length = bt.args()
    q = torch.zeros((2, 4, 64), device="cuda")
    for call in (lambda: a.kv4_attention(q, pool, table, start, length[:1], 1.0),
                 lambda: a.kv4_attention(q, pool, table.long(), start, length, 1.0),
                 lambda: a.kv4_attention(q, pool.cpu(), table, start, length, 1.0),
                 lambda: a.kv4_attention(q, pool[:, :, :-1], table, start, length, 1.0),
                 lambda: a.kv4_append(q, q, q, q[0], q[0], pool, table, start, length)):
        with pytest.raises(ValueError):
            call()
