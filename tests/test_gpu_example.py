"""The example that decodes with the cache, the attention and the verification together.

Greedy verification emits the target's own greedy text, however much of a draft is accepted.  The passes
take other routes (one row, a chain, a tree, a prompt), so activations differ by a few bf16 roundings: 2^-8 of
a value each, some ten of them in the two layers, independent, make about 1% of the logits' unit spread, and
a code of the cache that falls the other way about as much.  Where texts part, the two tokens' logits must be
within 0.125, ten times that.
"""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


@pytest.mark.gpu
@pytest.mark.parametrize("tree,B,longest", [(False, 3, 100), (True, 3, 100), (False, 1, 1), (True, 5, 17)])
def test_drafted_text_is_the_greedy_text(tree, B, longest):
    import draft_and_verify as ex
    steps, room = 10, longest + 10 * 9 + 64
    tokens, length = ex.prompts(B, longest, 3)
    plain, drafted = ex.Decoder(B, room), ex.Decoder(B, room)
    plain.prompt(tokens, length)
    drafted.prompt(tokens, length)
    accepted = torch.stack([drafted.step(tree) for _ in range(steps)])
    while min(map(len, plain.texts)) < max(map(len, drafted.texts)):
        plain.plain_step()
    assert int(accepted.sum()) >= steps                           # drafts are taken, or the test shows nothing
    for b in range(B):
        want, got = plain.texts[b], drafted.texts[b]
        assert len(got) == 1 + int((accepted[:, b] + 1).sum())
        part = next((i for i, (x, y) in enumerate(zip(want, got)) if x != y), None)
        if part is not None:
            logits = plain.margins[b][part - 1]                   # the first token comes from the prompt
            assert part > 0 and float(logits[want[part]] - logits[got[part]]) < 0.125, (b, part)
    for pool in (drafted.target.pool, drafted.drafter.pool):
        count, (head, tail) = pool.block_count.tolist(), pool.ring_pos.tolist()
        held = [pool.block_table[b, :count[b]].tolist() for b in range(B)]
        free = [int(pool.free_ring[i % pool.free_ring.numel()]) for i in range(head, tail)]
        assert sorted(sum(held, free)) == list(range(pool.free_ring.numel()))      # no block is lost or held twice
    for b in range(B):
        assert int(drafted.target.pool.seq_len[b]) == int(length[b]) + len(drafted.texts[b]) - 1
