"""DecoderStack at its limits on an MI355X."""
import numpy as np
import pytest

from paper_2511_05814_amd import workload as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests._gpu_rig import Rig  # noqa: E402


@pytest.fixture()
def rig():
    r = Rig(wl.CONFIGS["tiny-stack"].with_(dtype="bf16", tokens=40))
    yield r
    r.store.close()


def hidden(rig, first, n):
    return torch.from_numpy(np.ascontiguousarray(wl.hidden_states(rig.cfg, 40)[first:first + n])).cuda()


def test_up_to_max_pos_and_no_further(rig):
    from paper_2511_05814_amd import decoder
    moe = rig.cache(8, "lfu", max_prefill_tokens=40)
    dec = decoder.DecoderStack(moe, 4, 2, 64, pages=4, max_pos=20)
    free, bound = decoder.Sequences(1, 4, 16), decoder.Sequences(1, 4, 16, max_pos=20)
    for n in (19, 1):
        H = hidden(rig, 0, n)
        dec.step(H, bound.extend([n]))
        moe.sync()
        assert torch.isfinite(H).all()
        free.extend([n])
    with pytest.raises(ValueError, match="positions end at 20"):
        bound.extend([1])
    assert bound.length == [20]
    H = hidden(rig, 0, 1)
    before, pools = H.clone(), [l["pool"].clone() for l in dec.layers]
    with pytest.raises(ValueError, match="positions end at 20"):
        dec.step(H, free.extend([1]))
    moe.sync()
    assert torch.equal(H, before) and all(torch.equal(p, l["pool"]) for p, l in zip(pools, dec.layers))
    moe.close()


def test_rows_of_a_wider_tensor(rig):
    """H may have a stride between rows: the same results in place, nothing beside them."""
    from paper_2511_05814_amd import decoder
    moe = rig.cache(8, "lfu", max_prefill_tokens=40)
    dec = decoder.DecoderStack(moe, 4, 2, 64, pages=4, max_pos=40)
    out = []
    for strided in (False, True):
        seqs = decoder.Sequences(2, 4, 16, max_pos=40)
        moe.reset()
        got = []
        for at, new in ((0, [9, 4]), (13, [1, 1]), (15, [1, 0])):
            H = hidden(rig, at, sum(new))
            wide = torch.full((len(H), 2 * H.shape[1]), 3.0, device="cuda")
            if strided:
                wide[:, :H.shape[1]] = H
                H = wide[:, :H.shape[1]]
            snaps = torch.empty((rig.cfg.layers, 2, *H.shape), device="cuda")
            dec.step(H, seqs.extend(new), snapshots=snaps)
            moe.sync()
            got += [H.clone(), snaps]
            assert (wide[:, -H.shape[1]:] == 3).all()
        out.append(got)
    assert all(torch.equal(a, c) for a, c in zip(*out))
    moe.close()


def test_sequences_of_the_stack(rig):
    """A plan of its own sequences runs; one for more or other pages does not. A step of no tokens is no work."""
    from paper_2511_05814_amd import decoder
    moe = rig.cache(8, "lfu", max_prefill_tokens=40)
    dec = decoder.DecoderStack(moe, 4, 2, 64, pages=4, page_size=16, max_pos=40)
    H = hidden(rig, 0, 3)
    before = H.clone()
    for other in (decoder.Sequences(1, 5, 16), decoder.Sequences(1, 4, 32)):
        with pytest.raises(ValueError, match="the stack has 4 of 16"):
            dec.step(H, other.extend([3]))
    seqs = dec.sequences(2)
    dec.step(H[:0], seqs.extend([0, 0]))
    with pytest.raises(ValueError, match="3 rows of H for a plan of 2"):
        dec.step(H, seqs.extend([2, 0]))
    moe.sync()
    assert torch.equal(H, before)
    dec.step(H, seqs.extend([0, 3]))
    moe.sync()
    assert torch.isfinite(H).all() and not torch.equal(H, before)
    moe.close()


def test_a_stack_dropped_before_its_steps_are_done(rig):
    """What it held is not given to tensors of the caller's stream while the steps still read it."""
    from paper_2511_05814_amd import decoder
    results = []
    for drop in (False, True):
        moe = rig.cache(8, "lfu", max_prefill_tokens=40)
        dec = decoder.DecoderStack(moe, 4, 2, 64, pages=4, max_pos=40)
        seqs, H = dec.sequences(1), hidden(rig, 0, 20)
        snaps = torch.zeros((rig.cfg.layers, 2, *H.shape), device="cuda")
        work = torch.randn((4096, 4096), device="cuda")
        work.record_stream(moe.compute)
        sizes = [t.numel() for l in dec.layers for t in l.values() if t.dtype == torch.uint8]
        torch.cuda.synchronize()
        moe.compute.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(moe.compute):
            for _ in range(30):      # some milliseconds ahead of the step
                work = (work @ work).clamp(-1, 1)
        dec.step(H, seqs.extend([20]), snapshots=snaps)
        if drop:
            del dec, snaps
            held = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
            assert len(held) == 2 * len(sizes)
        moe.sync()
        torch.cuda.synchronize()
        results.append(H.clone())
        moe.close()
    assert torch.equal(*results)
