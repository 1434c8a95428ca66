"""The plain forms that the tests of the calls after a verified step go by, checked by hand (no GPU)."""
import math

import numpy as np
import pytest
import torch

import after_reference as ref
import pass_reference


def test_scores_of_a_row_worked_out_by_hand():
    x = torch.tensor([[[0.0, math.log(3.0), -math.inf, 0.0]]])
    logp, rank, lse, entropy, top_id, top_x, top_p = ref.score(x, 1.0, torch.tensor([[[3, 1, 2, 9]]]), 6)
    assert torch.allclose(logp[0, 0, :2], torch.tensor([math.log(0.2), math.log(0.6)], dtype=torch.float64))
    assert logp[0, 0, 2] == -math.inf and logp[0, 0, 3] == -math.inf and rank.item() == 2
    assert math.isclose(lse.item(), math.log(5.0), rel_tol=1e-7)
    assert math.isclose(entropy.item(), -(0.6 * math.log(0.6) + 0.4 * math.log(0.2)), rel_tol=1e-7)
    assert top_id[0, 0].tolist() == [1, 0, 3, -1, -1, -1]


def test_distillation_worked_out_by_hand():
    x = torch.log(torch.tensor([[[0.5, 0.25, 0.125, 0.125]]], dtype=torch.float64))
    ids, t = torch.tensor([[[1, 3, 1]]]), torch.log(torch.tensor([[[0.5, 0.25, 0.9]]], dtype=torch.float64))
    loss, accept, lse, g = ref.distill(x, ids, t, 1.0, torch.zeros(1, 1, dtype=torch.float64))
    # p = 0.5 and 0.25 (the repeat has no part), r = 0.25; q = 0.25 and 0.125, s = 0.625
    assert math.isclose(loss.item(), 0.5 * math.log(2) + 0.25 * math.log(2) + 0.25 * math.log(0.4), rel_tol=1e-12)
    assert math.isclose(accept.item(), 0.25 + 0.125 + 0.25, rel_tol=1e-12) and abs(lse.item()) < 1e-12
    assert torch.allclose(g[0, 0], torch.tensor([0.5 * 0.6, -0.25, 0.125 * 0.6, -0.125], dtype=torch.float64))
    assert abs(g.sum().item()) < 1e-12


def test_the_gradient_is_the_losss_derivative():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(2, 2, 11, dtype=torch.float64, generator=gen)
    ids = torch.tensor([3, 7, 0]).expand(2, 2, 3)
    t = torch.randn(2, 2, 3, dtype=torch.float64, generator=gen)
    for lse in (None, torch.full((2, 2), 3.0, dtype=torch.float64)):
        g = ref.distill(x, ids, t, 1.7, lse)[3]
        for v in range(11):
            d = torch.zeros_like(x)
            d[..., v] = 1e-5
            diff = (ref.distill(x + d, ids, t, 1.7, lse)[0] - ref.distill(x - d, ids, t, 1.7, lse)[0]) / 2e-5
            assert (diff - g[..., v]).abs().max() < 1e-9


def test_a_fork_worked_out_by_hand():
    # row 0: 20 tokens in blocks 4, 2; row 1: 16 in block 0 (and 7, which it does not need).  Pages of 16.
    got = ref.fork([0, 0, 1], [20, 17, 16], [20, 16], [2, 2], [5, 8], [[4, 2], [0, 7]], [0, 1, 6, 3, 5, 9, 9, 9], 16, [[-1, -1]] * 3)
    # rows 0 and 1 share block 4; block 2 stays with row 0, row 1 takes ring[5]'s 9
    assert got["table"] == [[4, 2], [4, 9], [0, -1]] and got["copy_src"] == [-1, 2, -1] and got["copy_dst"] == [-1, 9, -1]
    assert got["copy_len"] == [0, 1, 0] and got["block_count"] == [2, 2, 1] and got["seq_len"] == [20, 17, 16]
    assert got["ring_pos"] == [6, 9] and got["ring"][8 % 8] == 7


@pytest.mark.parametrize("D", [64, 128])
def test_token_bytes_are_the_caches_layout(D):
    """A token put into an empty cache changes nothing but its own bytes, and all of them."""
    place = ref.token_bytes(D)
    assert sorted(sum(place, [])) == list(range(16 * (D + 8)))         # every byte belongs to one token
    x = np.where(np.arange(D) % 15 == 0, 15.0, 1.0 + np.arange(D) % 14).astype(np.float32)     # codes 0..15, scale 14 / 15
    for slot in (0, 5, 15, 16 + 9):
        cache = np.zeros((1, 1, 32 * (D + 8)), dtype=np.uint8)
        pass_reference.cache_put(cache, 32, D, slot, 0, x, x)
        other = cache.copy().reshape(2, 16 * (D + 8))
        own = other[slot // 16, place[slot % 16]].copy()
        other[slot // 16, place[slot % 16]] = 0
        assert not other.any() and (own != 0).sum() > (D + 8) * 3 // 4
