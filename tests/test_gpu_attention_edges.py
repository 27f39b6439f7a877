"""Edges of the attention entry points on an MI355X: NaN and infinities, extreme
scales, empty tensors, refusals, and the paths that only some shapes take.

Tolerances are those of test_gpu_attention, derived there."""
import numpy as np
import pytest

from oracle import attention as oa
from paper_2511_05814_amd import binding as b

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests._attention_rig import Batch, bf16, device  # noqa: E402
from tests.test_attention_limits import cut  # noqa: E402
from tests.test_gpu_attention import U, check_attention, check_product, host, matrix, ops  # noqa: E402


def change(bt, seq, pos, head, f):
    """Runs f(record's parts, token) on the entry of position pos."""
    page = bt.table[seq, pos // bt.P]
    rec = [np.array(x) for x in oa.unpack_record(bt.pool[page, head], bt.P, bt.D)]
    f(rec, pos % bt.P)
    bt.pool[page, head] = oa.record(*rec)


def mark(part):
    """Marks the second group of a key (part 0) or a value (2) as not stored."""
    def f(rec, at):
        rec[part + 1][at, 1] = 255 << 8
        rec[part][at, 32:64] = 0
    return f


def key_of(value):
    def f(rec, at):
        codes, metas = oa.kv4_quantize(np.full((1, rec[0].shape[1]), value))
        rec[0][at], rec[1][at] = codes[0], metas[0]
    return f


@pytest.mark.parametrize("part", [0, 2])
@pytest.mark.parametrize("max_len", [None, 1 << 20])   # one split and several
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("D", [64, 128])
def test_marks_count_however_small_their_weight(D, new, max_len, part):
    """A marked entry among tokens whose weights come to 0 beside those of one
    key, some 600 powers of two above, that another wave or split has."""
    bt = Batch([new, 1], [100, 40], 4, 2, D, 16, seed=21).fill(0.3)
    change(bt, 0, 40, 0, key_of(30.0))
    change(bt, 0, 5, 0, mark(part))
    q = np.random.default_rng(3).standard_normal((bt.tokens, 4, D)) + 2
    for dtype in ("f32", "bf16"):
        o, want = check_attention(bt, dtype, q=q, max_len=max_len)
        assert np.isnan(o[:new, :2]).any((1, 2)).all()


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("scale", [np.nan, np.inf, -np.inf])
def test_scales_that_are_not_finite_give_nan(scale, new):
    """But zeros to a row that sees nothing."""
    bt = Batch([new, 1], [300, 0], 4, 2, 64, 16, seed=22, short=1).fill(0.3)
    for dtype in (torch.float32, torch.bfloat16):
        o = host(ops().kv4_attention(torch.randn((bt.tokens, 4, 64), device="cuda").to(dtype), *bt.args(), scale))
        assert np.isnan(o[:new]).all() and (o[new] == 0).all()


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("scale,size", [(1e-20, 1e20), (-1e-30, 1e30), (1e-36, 1e36), (0.0, 1e25), (1e-36, 1e-10), (1e25, 1e-25),
                                        (1e30, 1e-34)])
@pytest.mark.parametrize("max_len", [None, 1 << 20])
def test_scales_and_queries_of_any_size(scale, size, new, max_len):
    """Scores are what counts, not how they divide between q and its scale; with
    scale 0 every token weighs the same."""
    bt = Batch([new, 1], [300, 20], 4, 2, 64, 16, seed=23).fill(0.3)
    q = np.random.default_rng(4).standard_normal((bt.tokens, 4, 64)) * size
    for dtype in ("f32", "bf16"):
        check_attention(bt, dtype, q=q, scale=scale, max_len=max_len)


def alike(new, old, value, seed):
    """A batch whose keys are all one value, and its values 1."""
    bt = Batch(new, old, 4, 2, 64, 16, seed=seed)
    bt.pool[:, :] = oa.record(*oa.kv4_quantize(np.full((16, 64), value)), *oa.kv4_quantize(np.ones((16, 64))))
    return bt


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("value", [np.inf, -np.inf])
def test_a_row_with_an_infinity_is_nan(value, new):
    """Also where all of its scores are minus infinity."""
    bt = alike([new, 2], [40, 30], 3.0, 24)
    q = np.random.default_rng(5).standard_normal((bt.tokens, 4, 64)).astype(np.float32)
    q[0, 1, 9] = value
    for dtype in ("f32", "bf16"):
        o = host(ops().kv4_attention(device(q, dtype), *bt.args(), 0.125))
        assert np.isnan(o[0, 1]).all() and np.isnan(o).sum() == 64


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("max_len", [None, 1 << 20])
@pytest.mark.parametrize("size", [-1e37, 1e37])
def test_dot_products_past_fp32(size, new, max_len):
    """One key takes all the weight; where parts of the row are joined by their
    largest dot products, which fp32 does not hold, NaN, and nothing else."""
    bt = alike([new, 2], [400, 30], 300.0, 25)
    change(bt, 0, 5, 0, key_of(100.0 if size < 0 else 900.0))
    def seven(rec, at):
        codes, metas = oa.kv4_quantize(np.full((1, 64), 7.0))
        rec[2][at], rec[3][at] = codes[0], metas[0]
    change(bt, 0, 5, 0, seven)
    q = np.random.default_rng(5).standard_normal((bt.tokens, 4, 64)).astype(np.float32)
    q[0, 1] = size
    for dtype in ("f32", "bf16"):
        o = host(ops().kv4_attention(device(q, dtype), *bt.args(), 0.125, max_len=max_len))
        assert np.isnan(o[0, 1]).all() or (o[0, 1] == 7).all()
        assert np.isnan(o).sum() == np.isnan(o[0, 1]).sum()


def test_tensors_without_rows():
    """Real empty tensors, which have no address."""
    a = ops()
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.zeros((3, 64), dtype=dtype, device="cuda")
        w = torch.zeros(b.moe_q4_matrix_bytes(8, 64), dtype=torch.uint8, device="cuda")
        for empty in (x[:0], torch.empty((0, 64), dtype=dtype, device="cuda")):
            y = a.q4_matmul(empty, w, 8)
            assert y.shape == (0, 8) and y.dtype == dtype
            h = torch.empty((0, 64), device="cuda")
            v = torch.ones(64, device="cuda")
            for gate in (None, v, h):
                ho, xo = a.norm_residual(h, empty, gate=gate, post=v, pre=v)
                assert ho.shape == xo.shape == (0, 64) and xo.dtype == dtype
            assert a.norm_residual(h, pre=v, h_out=h, want_x=False)[0] is h
        bt = Batch([0, 0], [3, 0], 4, 2, 64, 16)
        args = bt.args()
        q, k = (torch.empty((0, n, 64), dtype=dtype, device="cuda") for n in (4, 2))
        cos = torch.ones((8, 32), device="cuda")
        before = args[0].clone()
        q = a.kv4_append(q, k, k, cos, cos, *args)
        o = a.kv4_attention(q, *args, 0.125)
        assert q.shape == o.shape == (0, 4, 64) and torch.equal(args[0], before)
        assert [t.shape for t in a.kv4_read(*args, 0, 64, dtype)] == [(0, 2, 64)] * 2


def test_overlapping_tensors_are_refused():
    a = ops()
    x = torch.randn((40, 64), device="cuda")
    w = torch.zeros(b.moe_q4_matrix_bytes(64, 64), dtype=torch.uint8, device="cuda")
    wide = torch.zeros((40, 160), device="cuda")
    for call in (lambda: a.q4_matmul(x, w, 64, out=x), lambda: a.q4_matmul(x[1:], w, 64, out=x[:-1]),
                 lambda: a.q4_matmul(wide[:, :64], w, 64, out=wide[:, 60:124]),
                 lambda: a.norm_residual(x[1:], h_out=x[:-1])):
        with pytest.raises(b.MoeError, match="overlaps"):
            call()
    wide[:, 64:] = 5
    a.q4_matmul(wide[:, :64], w, 64, out=wide[:, 64:128])
    assert (wide[:, 128:] == 5).all() and (wide[:, :128] == 0).all()


@pytest.mark.parametrize("new", [[3, 1], [90, 2]])
def test_attention_over_its_queries(new):
    """o in q's place, with one split and with several."""
    bt = Batch(new, [300, 20], 4, 2, 64, 16, seed=26).fill(0.3)
    for max_len in (1, 1 << 20):
        for dtype in (torch.float32, torch.bfloat16):
            q = torch.randn((bt.tokens, 4, 64), device="cuda").to(dtype)
            want = ops().kv4_attention(q, *bt.args(), 0.125, max_len=max_len)
            assert torch.equal(ops().kv4_attention(q, *bt.args(), 0.125, max_len=max_len, out=q), want)


def test_more_workgroups_than_a_launch_takes():
    """One long run of new tokens among many sequences: the largest runs'
    blocks for all of them would pass 2^32 threads, so workgroups take several."""
    seqs, new, heads, kv, D, P = 1 << 16, 4096, 64, 8, 64, 16
    pool = torch.zeros((new // P, kv, P * D * 9 // 8), dtype=torch.uint8, device="cuda")
    table = torch.full((seqs, new // P), -1, dtype=torch.int32, device="cuda")
    table[7] = torch.arange(new // P, device="cuda")
    count = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    count[7] = new
    start = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    start[8:] = new
    k = torch.zeros((new, kv, D), device="cuda")
    v = torch.arange(new, device="cuda").float()[:, None, None].expand(new, kv, D) % 8
    none = torch.empty((new, 0), device="cuda")
    q = torch.randn((new, heads, D), device="cuda")
    ops().kv4_append(q, k, v.contiguous(), none, none, pool, table, start, count)
    o = ops().kv4_attention(q, pool, table, start, count, 0.125, max_new=new, max_len=new)
    _, stored = ops().kv4_read(pool, table, start, count, new, D)
    want = stored[:, 0, 0].double().cumsum(0) / torch.arange(1, new + 1, device="cuda")   # alike keys: the mean of the values so far
    assert (o.double() - want[:, None, None]).abs().max() <= 8 * (2.0 ** -21 + 200 * U)


def test_no_memory_is_torchs_error():
    """More than the card has: torch's own class, and the next call works."""
    bt = Batch([1], [1], 4, 2, 64, 16)
    args = bt.args()
    pool = torch.zeros((4, 1024, 16 * 64 * 9 // 8), dtype=torch.uint8, device="cuda")
    assert (1 << 22) * 1024 * 64 * 4 > 2 * torch.cuda.get_device_properties(0).total_memory
    with pytest.raises(torch.OutOfMemoryError):
        ops().kv4_read(pool, *args[1:], 1 << 22, 64)
    assert ops().kv4_read(*args, 1, 64)[0].shape == (1, 2, 64)


def test_tensors_that_require_grad():
    """Refused while gradients are on, rather than answered without one."""
    a = ops()
    x, h = (torch.randn((3, 64), device="cuda", requires_grad=True) for _ in range(2))
    plain, v = torch.randn((3, 64), device="cuda"), torch.ones(64, device="cuda", requires_grad=True)
    w = torch.zeros(b.moe_q4_matrix_bytes(8, 64), dtype=torch.uint8, device="cuda")
    bt = Batch([3], [1], 1, 1, 64, 16).fill(0.3)
    args, cos = bt.args(), torch.ones((8, 32), device="cuda")
    q = x.unflatten(1, (1, 64))
    calls = [lambda: a.q4_matmul(x, w, 8), lambda: a.q4_matmul(plain, w, 64 // 8, out=torch.empty((3, 8), device="cuda", requires_grad=True)),
             lambda: a.norm_residual(h), lambda: a.norm_residual(plain, x), lambda: a.norm_residual(plain, plain, gate=v),
             lambda: a.norm_residual(plain, plain, post=v), lambda: a.norm_residual(plain, pre=v),
             lambda: a.kv4_append(plain[:, None], q, plain[:, None], cos, cos, *args), lambda: a.kv4_attention(q, *args, 0.125)]
    for call in calls:
        with pytest.raises(ValueError, match="requires grad"):
            call()
        with torch.no_grad():
            call()
    assert not a.q4_matmul(x.detach(), w, 8).requires_grad


# -- splits over a long cache and their joins ----------------------------------------

def splits(bt, max_new, max_len):
    return cut(len(bt.new), bt.kv_heads, bt.heads, bt.tokens, max_new, max_len)


@pytest.mark.parametrize("what", ["plain", "marked", "holes", "empty"])
@pytest.mark.parametrize("new", [[1], [3], [100], [150]])   # a block of 16 rows, of 128; the last goes to the other join
@pytest.mark.parametrize("D", [64, 128])
def test_splits_of_a_long_sequence(D, new, what):
    """One sequence cut into many parts: with few rows they are joined by a
    workgroup for 32 dimensions of a row, with many by a few lanes."""
    bt = Batch(new, [3100], 4, 2, D, 16, seed=31).fill(0.3)
    if what == "marked":      # both in parts of their own, of a head each
        change(bt, 0, 700, 0, mark(0))
        change(bt, 0, 2050, 1, mark(2))
    if what == "holes":       # more than a part without a page, and single pages
        bt.table[0, 40:80] = -1
        bt.table[0, [3, 100, 101, 190]] = 1 << 20
    if what == "empty":       # parts behind the end
        bt.table = np.concatenate([bt.table, np.full((1, 800), -1, np.int32)], 1)
    assert splits(bt, new[0], bt.table.shape[1] * bt.P).splits >= 8
    for dtype in ("f32", "bf16"):
        o, want = check_attention(bt, dtype)
        if what == "marked":
            assert np.isnan(o[:, :2]).all() and np.isnan(o[:, 2:, 32:64]).all() and not np.isnan(o[:, 2:, :32]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_of_many_sequences(dtype):
    """From eight sequences on splits are finer: 16, one of them long, short
    ones and ones without new tokens."""
    new = [16, 2, 0, 16, 1, 5, 16, 0, 9, 3, 16, 1, 16, 7, 16, 2]
    old = [30, 3900, 0, 100, 17, 40, 0, 90, 260, 3, 10, 800, 5, 64, 31, 0]
    bt = Batch(new, old, 32, 8, 64, 16, seed=32).fill(0.3)
    s = splits(bt, 16, 3902)
    assert (s.prompt, s.splits) == (1, 5) and splits(bt, 16, 3071).splits < 5
    check_attention(bt, dtype, max_new=16, max_len=3902)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,k", [(9, 100, 8192), (1, 33, 16384), (31, 64, 4096)])
def test_products_of_long_rows(rows, n, k, dtype):
    """Few rows over many groups: the waves' runs of groups, whole and ragged."""
    rng = np.random.default_rng(k + n)
    for kk in (k, k + 64, k + 192):
        buf = matrix(rng, n, kk)
        x = rng.standard_normal((rows, kk)).astype(np.float32)
        x = bf16(x) if dtype == "bf16" else x
        check_product(x.astype(np.float64), buf, n, kk, ops().q4_matmul(device(x, dtype), torch.from_numpy(buf).cuda(), n), dtype)
