"""The fp64 attention oracle: its cache format round-trips, its quantiser keeps
to half a step, and its attention agrees with a direct softmax."""
import numpy as np
import pytest

from oracle import attention as oa


@pytest.mark.parametrize("D", [64, 128])
def test_record_round_trip(D):
    rng = np.random.default_rng(1)
    kq, vq = rng.integers(0, 16, (2, 32, D)).astype(np.uint8)
    km, vm = rng.integers(0, 1 << 16, (2, 32, D // 32)).astype(np.uint16)
    rec = oa.record(kq, km, vq, vm)
    assert rec.size == 32 * D * 9 // 8
    for a, b in zip((kq, km, vq, vm), oa.unpack_record(rec, 32, D)):
        assert np.array_equal(a, b)
    # the stated places of one value word and one value meta
    t, o, g = 13, D // 8 - 1, D // 32 - 1
    at = 32 * D // 2 + ((t // 4) * (D // 8) + o) * 16 + t % 4 * 4
    assert list(rec[at:at + 4]) == [vq[t, 8 * o + 2 * i] | vq[t, 8 * o + 2 * i + 1] << 4 for i in range(4)]
    at = 32 * D + 32 * D // 16 + ((t // 4) * (D // 32) + g) * 8 + t % 4 * 2
    assert int(rec[at]) | int(rec[at + 1]) << 8 == vm[t, g]


@pytest.mark.parametrize("scale", [1e-9, 1e-3, 1.0, 37.0, 1e3])
def test_quantiser_keeps_to_half_a_step(scale):
    x = np.random.default_rng(2).standard_normal((50, 128)) * scale
    x[0] = 0
    q, m = oa.kv4_quantize(x)
    s = np.repeat(oa.STEPS[m >> 8], 32, -1)
    # the zero is rounded too, which can push an end of the range half a step out
    assert (np.abs(oa.kv4_values(q, m) - x) <= s * (1 + 1e-9)).all()
    inside = (q > 0) & (q < 15)
    assert (np.abs(oa.kv4_values(q, m) - x)[inside] <= s[inside] * (0.5 + 1e-9)).all()
    assert (oa.kv4_values(q, m)[0] == 0).all()


def test_values_are_exact_in_fp16_and_bf16():
    k, z, q = np.meshgrid(np.arange(255), np.arange(16), np.arange(16), indexing="ij")
    v = (q - z) * oa.STEPS[k]
    assert np.array_equal(v.astype(np.float16).astype(np.float64), v)
    bits = v.astype(np.float32).view(np.uint32)
    assert np.array_equal(v.astype(np.float32).astype(np.float64), v) and not (bits & 0xFFFF).any()


def test_groups_that_cannot_be_stored_and_saturation():
    x = np.zeros((3, 64))
    x[0, 5], x[1, 40], x[2, 0] = np.inf, np.nan, 1e9
    q, m = oa.kv4_quantize(x)
    v = oa.kv4_values(q, m)
    assert np.isnan(v[0, :32]).all() and (v[0, 32:] == 0).all()
    assert np.isnan(v[1, 32:]).all() and (v[1, :32] == 0).all()
    assert v[2, 0] == 15 * oa.STEPS[254]


def test_attention_and_norm_formulas():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 8)), rng.standard_normal((5, 8)), rng.standard_normal((5, 8))
    seen = np.array([[1, 1, 0, 0, 0], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1]], dtype=bool)
    o = oa.attention(q, k, v, seen, 0.3)
    p = np.exp(0.3 * q[2] @ k.T)
    assert np.allclose(o[2], p @ v / p.sum(), atol=1e-14) and (o[1] == 0).all()
    h, x = oa.norm_residual(q, q, gate=2.0, post=np.ones(8), residual_scale=0.5)
    want = 0.5 * q + 2 * q / np.sqrt((q * q).mean(1, keepdims=True) + 1e-5)
    assert np.allclose(h, want) and np.allclose(x, want / np.sqrt((want * want).mean(1, keepdims=True) + 1e-5))


def test_quantize_q4g64_reads_back():
    from paper_2511_05814_amd import workload as wl
    rng = np.random.default_rng(4)
    w = rng.standard_normal((5, 192)).astype(np.float32) * 0.02
    w[2] = 0
    back = oa.q4_dequantize(wl.quantize_q4g64(w), 5, 192)
    g = w.reshape(5, 3, 64)
    step = (g.max(-1) - g.min(-1)) / 15
    # half a step, the zero point's 1/32 of one and the scale's fp16 rounding over 15
    assert (np.abs(back - w) <= np.repeat(step, 64, 1) * (0.5 + 1 / 32 + 15 * 2.0 ** -10) + 1e-12).all()
    assert (back[2] == 0).all()
    with pytest.raises(ValueError):
        wl.quantize_q4g64(w[:, :100])
