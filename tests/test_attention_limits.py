"""Calls of the attention entry points at the edges of what they take, decided on
the host: no rows, operands that overlap, sizes past a launch's."""
import ctypes

import numpy as np
import pytest

from tests.test_attention_args import BF16, F32, P, append, attend, b, batch, norm, q4, refused


def test_operands_without_elements_may_be_null():
    b.moe_q4_matmul(*q4(rows=0, x=None, y=None))
    none = batch(tokens=0)
    b.moe_kv4_append(*append(none, q=None, k=None, v=None, out=None))
    b.moe_kv4_read(none, None, None, F32, 0)
    b.moe_kv4_attention(*attend(none, q=None, o=None))
    b.moe_norm_residual(*norm(rows=0, h=None, y=None, ho=None, x=None))
    b.moe_norm_residual(*norm(rows=0, h=None, y=None, gate=None, gs=64, ho=None, x=None))


def overlap(f, *args):
    refused(f, *args)
    assert "overlaps" in b.moe_last_error()


# places that no operand below reaches from another; nothing is dereferenced
A, B, C, D, E = (P + (i << 30) for i in range(1, 6))


def apart(f, *args):
    """The call gets past the checks, to a launch that fails without a GPU."""
    if pytest.importorskip("torch").cuda.is_available():
        pytest.skip("the operands are not device memory")
    with pytest.raises(b.MoeError) as e:
        f(*args)
    assert e.value.code == b.MOE_ERR_HIP, e.value


def test_products_refuse_overlap():
    base = dict(x=A, w=B, y=C, rows=3, n=128, k=128, x_stride=128, y_stride=128)
    overlap(b.moe_q4_matmul, *q4(**{**base, "y": A}))
    overlap(b.moe_q4_matmul, *q4(**{**base, "y": A + 3 * 256 - 2}))
    overlap(b.moe_q4_matmul, *q4(**{**base, "y": A - 3 * 256 + 2}))
    overlap(b.moe_q4_matmul, *q4(**{**base, "y": B}))
    overlap(b.moe_q4_matmul, *q4(**{**base, "y": B + 128 * 64 + 128 * 2 * 3 - 2}))
    apart(b.moe_q4_matmul, *q4(**base))
    apart(b.moe_q4_matmul, *q4(**{**base, "y": A + 3 * 256}))
    apart(b.moe_q4_matmul, *q4(**{**base, "y": A - 3 * 256}))
    # columns 0 .. 127 and 128 .. 255 of one buffer
    wide = {**base, "x_stride": 256, "y_stride": 256}
    apart(b.moe_q4_matmul, *q4(**{**wide, "y": A + 256}))
    overlap(b.moe_q4_matmul, *q4(**{**wide, "y": A + 254}))
    overlap(b.moe_q4_matmul, *q4(**{**wide, "y": A - 254}))
    apart(b.moe_q4_matmul, *q4(**{**wide, "y": A - 256}))


def test_append_refuses_overlap():
    base = dict(q=A, k=B, v=C, out=D, cos=E, sin=E + 80 * 32 * 4)
    far = batch(pool=P + (9 << 30))
    apart(b.moe_kv4_append, *append(far, **base))
    overlap(b.moe_kv4_append, *append(far, **{**base, "out": A}))
    apart(b.moe_kv4_append, *append(far, **{**base, "out": A, "rot": 0}))
    overlap(b.moe_kv4_append, *append(far, **{**base, "out": A, "rot": 0, "os": 264}))
    overlap(b.moe_kv4_append, *append(far, **{**base, "out": A + 16, "rot": 0}))
    for at in (B, C, E, E + 80 * 32 * 4, P + (9 << 30)):
        overlap(b.moe_kv4_append, *append(far, **{**base, "out": at}))
    for pool in (A, B, C, E):
        overlap(b.moe_kv4_append, *append(batch(pool=pool), **base))
    # queries, keys and values of a joined projection, the rotated ones beside them
    joined = dict(q=A, k=A + 512, v=A + 768, out=A + 1024, qs=768, ks=768, vs=768, os=768)
    apart(b.moe_kv4_append, *append(far, **{**base, **joined}))
    overlap(b.moe_kv4_append, *append(far, **{**base, **joined, "out": A + 1040}))


def test_read_and_attention_refuse_overlap():
    far = batch(pool=P + (9 << 30))
    size = 4 * 2 * 64 * 4
    apart(b.moe_kv4_read, far, A, A + size, F32, 0)
    overlap(b.moe_kv4_read, far, A, A + size - 16, F32, 0)
    overlap(b.moe_kv4_read, far, A, P + (9 << 30), F32, 0)
    base = dict(q=A, o=B)
    apart(b.moe_kv4_attention, *attend(far, **base))
    apart(b.moe_kv4_attention, *attend(far, **{**base, "o": A}))
    overlap(b.moe_kv4_attention, *attend(far, **{**base, "o": A + 16}))
    overlap(b.moe_kv4_attention, *attend(far, **{**base, "o": P + (9 << 30) + 16}))
    need = b.moe_kv4_attention_workspace_bytes(far, 4, 1, 4096)
    for at, bad in ((C, False), (A - need, False), (A - need + 16, True), (B, True), (P + (9 << 30), True)):
        (overlap if bad else apart)(b.moe_kv4_attention, *attend(far, **base, max_len=4096, ws=at, wsb=need))


def test_norm_refuses_overlap():
    base = dict(h=A, y=B, gate=C, gs=64, post=D, pre=D + 256, ho=E, x=E + (1 << 20), dtype=F32)
    apart(b.moe_norm_residual, *norm(**base))
    for ho, ok in ((A, True), (B, True), (C, True), (D, False), (D + 256, False), (A + 16, False), (base["x"], False)):
        (apart if ok else overlap)(b.moe_norm_residual, *norm(**{**base, "ho": ho}))
    for x, ok in ((A, True), (B, True), (C, True), (D, False), (D + 256, False), (B - 16, False)):
        (apart if ok else overlap)(b.moe_norm_residual, *norm(**{**base, "x": x}))
    overlap(b.moe_norm_residual, *norm(**{**base, "ho": A, "hos": 128}))
    overlap(b.moe_norm_residual, *norm(**{**base, "x": A, "dtype": BF16}))   # other elements
    apart(b.moe_norm_residual, *norm(**{**base, "x": D + 256, "rows": 1}))
    overlap(b.moe_norm_residual, *norm(**{**base, "ho": D + 256, "rows": 1}))


def test_overlap_of_rows_by_hand():
    """Against bytes marked one by one: equal and different strides."""
    rng = np.random.default_rng(1)
    seen = [0, 0]
    for _ in range(400):
        rows, k, n = int(rng.integers(1, 6)), 64 * int(rng.integers(1, 3)), int(rng.integers(1, 90))
        xs = k + 8 * int(rng.integers(0, 12))
        ys = n + int(rng.integers(0, 60)) if rng.random() < 0.6 else max(xs, n)
        y = A + 2 * int(rng.integers(-500, 500))
        taken = set()
        for t in range(rows):
            taken.update(range(A + t * xs * 2, A + t * xs * 2 + k * 2))
        bad = any(not taken.isdisjoint(range(y + t * ys * 2, y + t * ys * 2 + n * 2)) for t in range(rows))
        (overlap if bad else apart)(b.moe_q4_matmul, *q4(x=A, w=B, y=y, rows=rows, n=n, k=k, x_stride=xs, y_stride=ys))
        seen[bad] += 1
    assert min(seen) > 50


class Shape(ctypes.Structure):
    _fields_ = [("splits", ctypes.c_int), ("row_blocks", ctypes.c_int), ("prompt", ctypes.c_int)]


def cut(seqs, kv_heads, heads, tokens, max_new, max_len):
    """moe::kv4_attention_shape, the cut of an attention's launch."""
    f = getattr(b.lib(), "_ZN3moe19kv4_attention_shapeEiiiiii")
    f.argtypes, f.restype = [ctypes.c_int] * 6, Shape
    return f(seqs, kv_heads, heads, tokens, max_new, max_len)


MOST = ((1 << 32) - 1) // 256     # workgroups of 256 threads in a launch's dimension


def test_attention_launches_fit():
    """Workgroups of the attention and of its join, whatever the batch and hints."""
    rng = np.random.default_rng(2)

    def power(most):
        return int(min(most, 2 ** (rng.random() * np.log2(most + 1))))

    cases = [(1024, 8, 64, 1023 + 32768, 32768, 40000), (1 << 20, 15, 15, 1 << 20, 1, 1), (1 << 20, 15, 15, 1 << 24, 1 << 24, 1 << 30),
             (1, 1, 4096, 1 << 18, 1 << 18, 1 << 30), (4, 1, 4096, 1 << 18, 1, 1 << 30)]
    for _ in range(3000):
        kv = power(1024)
        heads = kv * power(4096 // kv)
        cases.append((power(min(1 << 20, MOST // kv)), kv, heads, power(min(1 << 24, (1 << 30) // heads)), power((1 << 31) - 1), power((1 << 31) - 1)))
    for seqs, kv, heads, tokens, max_new, max_len in cases:
        s = cut(seqs, kv, heads, tokens, max_new, max_len)
        assert s.splits >= 1 and s.row_blocks >= 1
        assert seqs * kv * s.row_blocks * s.splits <= MOST, (seqs, kv, heads, tokens, max_new, max_len, s.splits, s.row_blocks)
        if s.splits > 1:   # 8 rows a workgroup at least, or a few rows by 4 workgroups each
            assert -(-tokens * heads // 8) <= MOST


def test_sizes_past_a_launch_are_refused():
    refused(b.moe_kv4_attention, *attend(batch(seqs=1 << 20, kv_heads=16), heads=16, qs=1024, os=1024))
    assert b.moe_kv4_attention_workspace_bytes(batch(seqs=1 << 20, kv_heads=16), 16, 1, 4096) == 0
    most = dict(qs=1024 * 64, ks=1024 * 64, vs=1024 * 64, os=1024 * 64, heads=1024, q=A, k=A, v=A, out=C + (1 << 50), cos=B, sin=B)
    refused(b.moe_kv4_append, *append(batch(pool=D, kv_heads=1024, tokens=1 << 18), **most))
    refused(b.moe_kv4_read, batch(pool=D, kv_heads=1024, tokens=1 << 18), A, C + (1 << 50), F32, 0)
    refused(b.moe_q4_matmul, *q4(rows=1 << 20, n=1 << 24, y_stride=1 << 24))
    wide = dict(d=1032, hs=1032, ys=1032, hos=1032, xs=1032, h=A, y=A, gate=None, post=None, pre=None, ho=None, x=C + (1 << 50))
    refused(b.moe_norm_residual, *norm(**wide, rows=1 << 24))
    apart(b.moe_norm_residual, *norm(**wide, rows=(1 << 24) - 1))
    narrow = {**wide, "d": 1024}
    apart(b.moe_norm_residual, *norm(**narrow, rows=1 << 24))
