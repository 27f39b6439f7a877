"""Whole steps with drafted tokens through decoder.DecoderStack: a tree's tokens
come out as the same tokens taken one after another, what is kept serves the
steps that follow, and the command that decodes so runs.

Each path of the tree and the chain that it is compared with do the same
operations in fp32 but for the order of the attention's sums: some 2^-17 of the
largest value a layer (test_gpu_attention has the arithmetic), through norms and
experts whose gain stays below 8 over the two layers."""
import numpy as np
import pytest

from paper_2511_05814_amd import workload as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests._gpu_rig import Rig  # noqa: E402

PARENTS = [[-1, 0, 0, 1, 1, 2, 4], [-1], [-1, 0, 1, 1, 0]]
PATHS = [[0, 1, 4, 6], [0], [0, 4]]


def rig_of(heads=4, kv=2):
    from paper_2511_05814_amd import decoder
    cfg = wl.CONFIGS["tiny-stack"].with_(dtype="f32", tokens=40, layers=2)
    rig = Rig(cfg)
    moe = rig.cache(8, "lfu")
    return cfg, moe, decoder.DecoderStack(moe, heads, kv, 64, pages=12, max_pos=64, dtype=torch.float32)


def close(a, b):
    a, b = a.cpu().numpy(), b.cpu().numpy()
    assert np.abs(a - b).max() <= 8 * 2.0 ** -17 * np.abs(b).max(), np.abs(a - b).max() / np.abs(b).max()


def test_a_tree_is_its_paths():
    cfg, moe, stack = rig_of()
    states = torch.from_numpy(wl.hidden_states(cfg, 40)).to("cuda")
    first, drafted, later = states[:17], states[17:30], states[30:33]
    seqs = stack.sequences(3)
    H = first.clone()
    stack.step(H, seqs.extend([9, 3, 5]))
    moe.sync()
    filled = [l["pool"].clone() for l in stack.layers]
    got = drafted.clone()
    batch = seqs.extend([7, 1, 5], PARENTS)
    stack.step(got, batch)
    flat = [p + [-1] * (n - len(p)) for p, n in zip(PATHS, (7, 1, 5))]
    path, count = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (sum(flat, []), [len(p) for p in PATHS]))
    stack.keep(batch, path, count)
    seqs.keep([len(p) for p in PATHS])
    tail = later.clone()
    stack.step(tail, seqs.extend([1, 1, 1]))
    moe.sync()
    # the same tokens in line, over the caches as they were before
    for l, pool in zip(stack.layers, filled):
        l["pool"].copy_(pool)
    seqs.length, seqs.new = [9, 3, 5], [0, 0, 0]
    rows = torch.tensor([p + s for p, s in zip(sum(PATHS, []), [0] * 4 + [7] + [8] * 2)], device="cuda")
    want = drafted[rows]
    stack.step(want, seqs.extend([4, 1, 2]))
    moe.sync()
    close(got[rows], want)
    end = later.clone()
    stack.step(end, seqs.extend([1, 1, 1]))
    moe.sync()
    close(tail, end)


def test_speculation_takes_what_it_keeps():
    from paper_2511_05814_amd import decoder
    cfg, moe, stack = rig_of()
    spec = decoder.Speculation(stack, 100, 5, width=2)
    seqs = stack.sequences(3)
    stack.step(torch.from_numpy(wl.hidden_states(cfg, 6)).to("cuda"), seqs.extend([4, 1, 1]))
    pending = torch.tensor([1, 2, 3], device="cuda")
    for active in ([0, 1, 2], [0, 2], [1]):
        before = list(seqs.length)
        after, taken = spec.step(seqs, pending, active)
        moe.sync()
        for b in range(3):
            assert taken[b] in range(1, 6) if b in active else taken[b] == 0
            assert seqs.length[b] == before[b] + taken[b] and 0 <= int(after[b]) < 100
            assert b in active or after[b] == pending[b]
        pending = after


@pytest.mark.parametrize("tokens,drafts", [("6", "0"), ("6", "5"), ("0", "0"), ("0", "5")])
def test_the_command_shows_what_came_out(tokens, drafts, capsys, monkeypatch):
    """The rms that it prints is that of the last step's hidden states behind all layers."""
    from paper_2511_05814_amd import decoder
    step, states = decoder.DecoderStack.step, []
    monkeypatch.setattr(decoder.DecoderStack, "step", lambda self, H, *a, **k: (states.append((H, H.clone())), step(self, H, *a, **k)))
    decoder.main(["--config", "tiny-stack", "--sequences", "2", "--prompt", "5", "--tokens", tokens, "--drafts", drafts, "--vocab", "200"])
    said = capsys.readouterr().out.split("last rms ")[1].split()[0]
    behind, entering = (f"{x.square().mean().sqrt().item():.4f}" for x in states[-1])
    assert said == behind != entering and np.isfinite(float(said))


def test_the_command_times_steps_alone(monkeypatch):
    """An embedding and a head are made before the clock starts: tokens/s are those of
    the steps."""
    import time
    from paper_2511_05814_amd import decoder
    clock, make, said = time.perf_counter, decoder.Speculation.__init__, []
    monkeypatch.setattr(time, "perf_counter", lambda: (said.append("clock"), clock())[1])
    monkeypatch.setattr(decoder.Speculation, "__init__", lambda self, *a, **k: (said.append("make"), make(self, *a, **k))[1])
    decoder.main(["--config", "tiny-stack", "--sequences", "1", "--prompt", "3", "--tokens", "2", "--drafts", "3", "--vocab", "200"])
    assert said.index("make") < said.index("clock") and said.count("make") == 1


@pytest.mark.parametrize("drafts", ["0", "5"])
def test_the_command(drafts, capsys):
    from paper_2511_05814_amd import decoder
    decoder.main(["--config", "tiny-stack", "--sequences", "2", "--prompt", "5", "--tokens", "6", "--drafts", drafts, "--vocab", "200"])
    out = capsys.readouterr().out
    assert "decode:" in out and ("trees of 5" in out) == (drafts == "5")
