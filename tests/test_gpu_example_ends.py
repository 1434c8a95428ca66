"""The example's requests that end while others go on."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


@pytest.mark.gpu
@pytest.mark.parametrize("tree", [False, True])
def test_a_request_that_has_ended_stays_empty_until_its_place_is_taken(tree):
    """Where a text parts from plain decoding, the two tokens' logits are within 0.125 (as for the example's text)."""
    import draft_and_verify as ex
    tokens, length = ex.prompts(4, 60, 5)
    plain, drafted = ex.Decoder(4, 400), ex.Decoder(4, 400)
    for d in (plain, drafted):
        d.prompt(tokens, length)
    for _ in range(3):
        drafted.step(tree)
    drafted.fork([0, -1, 2, 0])
    for _ in range(3):
        accepted = drafted.step(tree)
        assert int(accepted[1]) == 0 and drafted.texts[1] == []
        for pool in (drafted.target.pool, drafted.drafter.pool):
            assert int(pool.block_count[1]) == 0 and int(pool.seq_len[1]) == 0
        r = drafted.lesson()
        assert not r.weight[1].any() and not r.grad[1].any() and torch.isfinite(r.head).all() and abs(float(r.weight.sum()) - 1) < 1e-5
    drafted.fork([0, 1, 2, 3])                                     # goes on being empty
    drafted.step(tree)
    assert drafted.texts[1] == [] and int(drafted.target.pool.seq_len[1]) == 0
    drafted.fork([0, 2, 2, 3])                                     # and its place is taken
    for _ in range(2):
        drafted.step(tree)
    while min(map(len, plain.texts)) < max(map(len, drafted.texts)):
        plain.plain_step()
    for b, s in enumerate([0, 2, 2, 0]):
        want, got = plain.texts[s], drafted.texts[b]
        assert len(got) > 10
        part = next((i for i, (x, y) in enumerate(zip(want, got)) if x != y), None)
        if part is not None:
            logits = plain.margins[s][part - 1]
            assert part > 0 and float(logits[want[part]] - logits[got[part]]) < 0.125, (b, part)
    for pool in (drafted.target.pool, drafted.drafter.pool):
        count, (head, tail) = pool.block_count.tolist(), pool.ring_pos.tolist()
        held = set(sum([pool.block_table[b, :count[b]].tolist() for b in range(4)], []))
        free = [int(pool.free_ring[i % pool.free_ring.numel()]) for i in range(head, tail)]
        assert len(set(free)) == len(free) and not held & set(free) and len(held) + len(free) == pool.free_ring.numel()
