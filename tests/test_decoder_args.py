"""What the decoder's sequences and stacks refuse, on the host."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2511_05814_amd import decoder  # noqa: E402


def stack(**kw):
    """A stack's sizes alone: no GPU, no weights."""
    s = decoder.DecoderStack.__new__(decoder.DecoderStack)
    s.moe = types.SimpleNamespace(L=1, cfg=types.SimpleNamespace(d_model=64))
    s.pages, s.page_size, s.max_pos = 3, 16, 40
    for name, value in kw.items():
        setattr(s, name, value)
    return s


def plan(**kw):
    table, start, length = (torch.zeros(n, dtype=torch.int32) for n in ((1, 3), 2, 1))
    return {**dict(page_table=table, q_start=start, kv_len=length, max_new=2, max_len=40, tokens=2, longest=40, pages=3, page_size=16), **kw}


def test_positions_past_the_tables():
    """A token past max_pos has no rotation and is not stored: neither a plan
    nor a step takes one, and the sequences stay as they were."""
    s = decoder.Sequences(2, 8, 16, max_pos=40)
    s.length, s.pages, s.free = [39, 3], [[7, 6, 5], [4]], [0, 1, 2, 3]
    with pytest.raises(ValueError, match="positions end at 40"):
        s.extend([2, 1])
    assert s.length == [39, 3] and s.free == [0, 1, 2, 3] and s.pages == [[7, 6, 5], [4]]
    with pytest.raises(ValueError, match="positions end at 40"):
        stack().step(torch.zeros((2, 64)), plan(longest=41))


@pytest.mark.parametrize("wrong,says", [(dict(page_size=32), "pages of 32"), (dict(pages=4), "4 pages"), (dict(tokens=3), "plan of 3 tokens"),
                                        (dict(tokens=1), "plan of 1 tokens")])
def test_plans_for_another_stack(wrong, says):
    """Other pages or page sizes name places that this cache does not have; rows
    without a plan would be results of nothing."""
    with pytest.raises(ValueError, match=says):
        stack().step(torch.zeros((2, 64)), plan(**wrong))


@pytest.mark.parametrize("H", [torch.zeros((2, 32)), torch.zeros((2, 64), dtype=torch.bfloat16), torch.zeros(64)])
def test_hidden_states_of_another_shape(H):
    with pytest.raises(ValueError, match="H must be"):
        stack().step(H, plan())


def test_a_stack_makes_its_sequences():
    s = stack().sequences(5)
    assert (len(s.length), sorted(s.free), s.page_size, s.max_pos) == (5, [0, 1, 2], 16, 40)


def test_tensors_of_a_step_are_known_to_its_stream(monkeypatch):
    """Weights, pages, tables, H, plan and snapshots belong to the caller's
    stream and are used on the experts': torch's allocator must know."""
    known = []

    class Stop(Exception):
        pass

    def stop(*a):
        raise Stop

    to, zeros = torch.Tensor.to, torch.zeros
    monkeypatch.setattr(torch.Tensor, "to", lambda t, *a, **k: t if a == ("cuda",) else to(t, *a, **k))
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **k: zeros(*a, **k))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: known.append((t.data_ptr(), s)))
    monkeypatch.setattr(torch.cuda, "current_stream", stop)
    cfg = types.SimpleNamespace(seed=1, d_model=64, layers=2)
    moe = types.SimpleNamespace(cfg=cfg, L=2, compute=types.SimpleNamespace(wait_stream=stop))
    s = decoder.DecoderStack(moe, 2, 1, 64, pages=3, max_pos=40)
    H, snaps, batch = torch.zeros((2, 64)), torch.zeros((2, 2, 2, 64)), plan()
    with pytest.raises(Stop):
        s.step(H, batch, snapshots=snaps)
    with pytest.raises(Stop):
        s.step(H, batch)
    used = [s.cos, s.sin, H, snaps, *(batch[k] for k in ("page_table", "q_start", "kv_len")), *(t for l in s.layers for t in l.values())]
    assert len(used) == 7 + 2 * 6 and all((t.data_ptr(), moe.compute) in known for t in used)


def test_trees_of_new_tokens(monkeypatch):
    """Positions go by depth, places by number; what is kept stays, and a
    sequence that is released has nothing left to keep."""
    move = torch.Tensor.to
    monkeypatch.setattr(torch.Tensor, "to", lambda t, where, *a: t if where == "cuda" else move(t, where, *a))
    s = decoder.Sequences(2, 8, 16, max_pos=20)
    s.extend([14, 0])
    batch = s.extend([7, 1], [[-1, 0, 0, 1, 1, 2, 3], [-1]])   # 21 places, but 18 positions
    assert batch["parent"].tolist() == [-1, 0, 0, 1, 1, 2, 3, -1] and batch["longest"] == 18 and batch["max_len"] == 21
    assert s.length == [21, 1] and len(s.pages[0]) == 2
    s.keep([3, 1])
    assert s.length == [17, 1] and batch["kv_len"].tolist() == [21, 1]
    with pytest.raises(ValueError, match="positions end at 20"):
        s.extend([4, 0], [[-1, 0, 1, 2], []])
    s.extend([2, 3], [[-1, 0], [-1, -1, 1]])
    s.release(0)
    s.keep([0, 2])
    assert s.length == [0, 3]


@pytest.mark.parametrize("parents", [[[-1, 0]], [[-1, 0], [-1]], [[-1, 1], []], [[-1, -2], []], [[0, 0], []]])
def test_trees_that_are_none(parents):
    s = decoder.Sequences(2, 8, 16, max_pos=40)
    with pytest.raises(ValueError, match="parents of|cannot follow"):
        s.extend([2, 0], parents)
    assert s.length == [0, 0] and len(s.free) == 8


@pytest.mark.parametrize("count", [[3, 0], [-1, 0], [1], [1, 1]])
def test_more_kept_than_there_was(count, monkeypatch):
    move = torch.Tensor.to
    monkeypatch.setattr(torch.Tensor, "to", lambda t, where, *a: t if where == "cuda" else move(t, where, *a))
    s = decoder.Sequences(2, 8, 16)
    s.extend([2, 0])
    with pytest.raises(ValueError, match="cannot be kept"):
        s.keep(count)
    assert s.length == [2, 0]


@pytest.mark.parametrize("wrong,says", [(dict(page_size=32), "pages of 32"), (dict(pages=4), "4 pages"), (dict(longest=41), "positions end at 40"),
                                        (dict(tokens=3), "plan of 3"), (dict(tokens=1), "plan of 1")])
def test_keeping_by_a_plan_for_another_stack(wrong, says):
    """Entries would move between places that are not these tokens'."""
    path, count = (torch.zeros(n, dtype=torch.int32) for n in (2, 1))
    with pytest.raises(ValueError, match=says):
        stack().keep(plan(**wrong), path, count)


@pytest.mark.parametrize("vocab,nodes,width", [(0, 4, 2), (9, 0, 2), (9, -1, 2), (9, 1025, 2), (9, 4, 0)])
def test_trees_that_cannot_be_drafted(vocab, nodes, width):
    with pytest.raises(ValueError, match="cannot be drafted"):
        decoder.Speculation(None, vocab, nodes, width)
