"""The attention block in front of the MoE layers, as decoder.DecoderStack runs
them together: prompts, decoding and a sequence that starts late, against the
fp64 oracle layer by layer (each block from the hidden states and the cache
bytes that the GPU had)."""
import numpy as np
import pytest

from oracle import attention as oa
from oracle import stack as ostack
from paper_2511_05814_amd import workload as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests._gpu_rig import Rig, _batch_tol, _say, _tol  # noqa: E402


def block(w, dec, h, batch, pool, exact):
    """fp64 output of an attention block for hidden states h over the cache's
    bytes; checks that it took the new keys and values to a step of their groups
    (and, of those rounded to bf16 before, 2^-6 of the group's span)."""
    table, start, length = (batch[k].cpu().numpy() for k in ("page_table", "q_start", "kv_len"))
    D, n, m = dec.head_dim, dec.heads, dec.heads + dec.kv_heads
    P = pool.shape[2] * 8 // (9 * D)
    _, x = oa.norm_residual(h, pre=w["pre"])
    qkv = (x @ oa.q4_dequantize(w["wqkv"], dec.width, h.shape[1]).T).reshape(len(h), -1, D)
    cos, sin = dec.cos.cpu().numpy().astype(np.float64), dec.sin.cpu().numpy().astype(np.float64)
    out = np.zeros((len(h), n * D))
    for b in range(len(length)):
        rows = np.arange(start[b], start[b + 1])
        if not rows.size:
            continue
        pos = length[b] - rows.size + np.arange(rows.size)
        q = oa.rotate(qkv[rows, :n], cos[pos], sin[pos])
        k = oa.rotate(qkv[rows, n:m], cos[pos], sin[pos])
        kk, vv, held = oa.gather(pool, table[b], length[b], P, D)
        assert held.all()
        for got, want in ((kk[:, pos], k.transpose(1, 0, 2)), (vv[:, pos], qkv[rows, m:].transpose(1, 0, 2))):
            g = want.reshape(*want.shape[:-1], -1, 32)
            span = np.maximum(g.max(-1), 0) - np.minimum(g.min(-1), 0)
            assert (np.abs(got - want) <= np.repeat(span * (1.125 / 15 + (1e-3 if exact else 2.0 ** -6)), 32, -1)).all()
        seen = np.arange(length[b]) <= pos[:, None]
        for i in range(n):
            out[rows, i * D:(i + 1) * D] = oa.attention(q[:, i], kk[i // (n // (m - n))], vv[i // (n // (m - n))], seen, D ** -0.5)
    y = out @ oa.q4_dequantize(w["wo"], h.shape[1], n * D).T
    return oa.norm_residual(h, y, gate=w["gate"], post=w["post"])[0]


@pytest.mark.parametrize("experts,dtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_decoder_stack(experts, dtype):
    from paper_2511_05814_amd import decoder
    cfg = wl.CONFIGS["tiny-stack"].with_(dtype=experts, tokens=60)
    rig = Rig(cfg)
    moe = rig.cache(8, "lfu", max_prefill_tokens=64 if experts == "bf16" else 0)
    dec = decoder.DecoderStack(moe, 6, 2, 64, pages=14, max_pos=64, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    weights = [{k: v.cpu().numpy() for k, v in l.items() if k != "pool"} for l in dec.layers]
    seqs = decoder.Sequences(3, 14, 16)
    states = wl.hidden_states(cfg, 60)
    at, worst = 0, 0.0
    # a block in bf16 rounds x, qkv, o and y, 2^-8 each at most, through a norm of y
    tol = 1e-4 if dtype == "f32" else 4 * 2.0 ** -8
    for new in ([17, 5, 0], [1, 1, 0], [1, 1, 9], [1, 0, 1], [1, 1, 1]):
        n = sum(new)
        H = torch.from_numpy(np.ascontiguousarray(states[at:at + n])).cuda()
        at += n
        batch = seqs.extend(new)
        snaps = torch.empty((cfg.layers, 2, n, cfg.d_model), device="cuda")
        dec.step(H, batch, snapshots=snaps)
        moe.sync()
        s = snaps.cpu().numpy().astype(np.float64)
        after = [s[l + 1, 0] if l + 1 < cfg.layers else H.cpu().numpy().astype(np.float64) for l in range(cfg.layers)]
        for l in range(cfg.layers):
            pool = dec.layers[l]["pool"].cpu().numpy()
            want = block(weights[l], dec, s[l, 0], batch, pool, dtype == "f32")
            err = np.linalg.norm(s[l, 1] - want, axis=1) / np.linalg.norm(want - s[l, 0], axis=1)
            worst = max(worst, err.max())
            assert err.max() <= tol, (new, l, err)
            for t in range(n):   # and the experts behind it
                st = ostack.layer_step(rig.model, l, s[l, 1, t], cfg.top_k)
                y = after[l][t] - s[l, 1, t]
                bound = _batch_tol(cfg) if n > 1 and experts == "bf16" else _tol(cfg)
                if st["certified"]:
                    assert np.linalg.norm(y - st["y"]) <= bound * np.linalg.norm(st["y"]) + 1e-5
    _say(cfg.name, experts, dtype, "worst block", worst)
    seqs.release(0)
    assert len(seqs.free) == 14 - len(seqs.pages[1]) - len(seqs.pages[2]) and seqs.length[0] == 0
    moe.close()
    rig.store.close()


def test_decoder_command(capsys):
    from paper_2511_05814_amd import decoder
    decoder.main(["--config", "tiny-stack", "--sequences", "2", "--prompt", "5", "--tokens", "2"])
    out = capsys.readouterr().out
    assert "tokens/s" in out and "expert hits" in out


def test_sequences_refuse():
    from paper_2511_05814_amd import decoder
    s = decoder.Sequences(2, 3, 16)
    with pytest.raises(ValueError):
        s.extend([1])
    with pytest.raises(RuntimeError):
        s.extend([40, 20])
    assert s.length == [0, 0] and len(s.free) == 3
