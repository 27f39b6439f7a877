"""Calls of the attention entry points at the edges of what they take, decided on
the host: no rows, operands that overlap, sizes past a launch's."""
from tests.test_attention_args import F32, P, append, attend, b, batch, norm, q4


def test_operands_without_elements_may_be_null():
    b.moe_q4_matmul(*q4(rows=0, x=None, y=None))
    none = batch(tokens=0)
    b.moe_kv4_append(*append(none, q=None, k=None, v=None, out=None))
    b.moe_kv4_read(none, None, None, F32, 0)
    b.moe_kv4_attention(*attend(none, q=None, o=None))
    b.moe_norm_residual(*norm(rows=0, h=None, y=None, ho=None, x=None))
    b.moe_norm_residual(*norm(rows=0, h=None, y=None, gate=None, gs=64, ho=None, x=None))
