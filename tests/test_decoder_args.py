"""What the decoder's sequences and stacks refuse, on the host."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2511_05814_amd import decoder  # noqa: E402


def stack(**kw):
    """A stack's sizes alone: no GPU, no weights."""
    s = decoder.DecoderStack.__new__(decoder.DecoderStack)
    s.moe = types.SimpleNamespace(L=1, cfg=types.SimpleNamespace(d_model=64))
    s.max_pos = 40
    for name, value in kw.items():
        setattr(s, name, value)
    return s


def plan(**kw):
    table, start, length = (torch.zeros(n, dtype=torch.int32) for n in ((1, 3), 2, 1))
    return {**dict(page_table=table, q_start=start, kv_len=length, max_new=2, max_len=40, longest=40), **kw}


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
