"""Steps that take several drafted tokens of a sequence at once.

An expert that a layer copies serves every token of a call that chose it, so a
sequence's pending token and a tree of guesses behind it cost the copies of their
distinct experts: fewer than the tokens one after another, more than one alone.
The tree's tokens are a sequence's new tokens, the pending one first; each other
names its parent.  A step is

  pos, seen = draft_tree(parent, q_start, kv_len, max_new)        once
  attention.kv4_append(..., pos=pos), attention.kv4_tree_attention(..., seen, ...)   in every layer
  path, count, next = verify_drafts(p, tokens, parent, u, q_start, q)
  attention.kv4_keep(pools, ..., path, count, head_dim)           once

(`decoder.DecoderStack.step` and `.keep` do the layers).  The functions take
tensors as those of `attention` do: checked, on torch's current stream, without
gradients, nothing synchronises, the same errors.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from .attention import _ops, _stream


def draft_tree(parent, q_start, kv_len, max_new: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """(pos, seen) of trees whose tokens' parents are parent (int32 [tokens],
    numbers within the sequence; -1: none): pos int32 [tokens], the place of the
    sequence's first new token plus the depth; seen int32 [tokens, ceil(max_new /
    32)], whose bit j says that the sequence's new token j is the token itself or
    one of its ancestors.  max_new (at most 1024) is the largest tree's size."""
    return _ops().draft_tree(parent, q_start, kv_len, max_new, _stream(parent))


def verify_drafts(p, tokens, parent, u, q_start, q: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(path, count, next) of trees of drafted tokens (int32 [tokens] ids) against
    the target's probabilities p [tokens, vocabulary] of the token behind each, so
    that what is accepted is distributed as the target's own tokens.  q, of the
    same type: the draft's, which the children of each token were drawn from;
    without it they are the draft's choice.  u: fp32 [tokens] random numbers in
    [0, 1); a sequence's first one draws its next token.  path int32 [tokens]: of each
    sequence the accepted tokens' numbers, then -1; count: how many; next: the
    token behind them.  include/moe_offload.h has the rule (moe_verify_drafts)."""
    return _ops().verify_drafts(p, tokens, parent, u, q_start, q, _stream(p))
