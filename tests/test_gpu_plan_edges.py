"""dsp_cache_plan at its ends: no token rows, no new tokens, no requests."""
import ctypes as C

import pytest
import torch

import pass_reference as ref
from paper_2510_02358_b200 import binding as dsp

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_a_tree_plan_without_token_rows_needs_no_mask():
    """An empty tensor has no address.  (No requests either: nothing is launched.)"""
    one, z = C.c_void_p(4096), C.c_void_p(0)

    def plan(B, T, mask):
        return dsp.lib().dsp_cache_plan(one, one, one, one, B, T, 16, 8, 4, one, 4, one, one, one, 5, C.c_void_p(8192), C.c_void_p(8192), one, one,
                                        one, one, z, mask, 1, one, z)
    assert plan(0, 0, z) == dsp.DSP_OK
    assert plan(0, 3, z) == plan(2, 3, z) == dsp.DSP_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("T", [0, 5])
def test_plans_without_new_tokens_give_back_what_is_too_much(tree, T):
    seq, count, page = [5, 0, 33, 16], [2, 1, 3, 3], 16
    kw = dict(node_parent=i32([[-1] * 4] * 4), node_depth=i32([[0] * 4] * 4)) if tree else {}
    table = [[1, 2, 9], [3, 9, 9], [4, 5, 6], [7, 8, 0]]
    t, ring = i32(table), i32([9] * 10)
    want = ref.plan(seq, [0] * 4, count, 3, 4, table, [9] * 10, page, T)
    got = dsp.dsp_cache_plan(i32(seq), i32([0] * 4), i32(count), torch.tensor([3, 4], device=DEV), t, ring, page, T, **kw)
    for name in ("row_status", "block_count", "ring_pos", "cu_new", "kv_len", "slot", "position", "token_row"):
        assert getattr(got, name).tolist() == want[name], name
    assert ring.tolist() == want["free_ring"] and (not tree or not got.mask.any())
    got = dsp.dsp_cache_plan(i32(seq), i32([0, 1, 0, 0]), i32(count), torch.tensor([3, 4], device=DEV), t, ring, page, 0, **kw)
    assert got.row_status.tolist() == [0, ref.PLAN_FULL, 0, 0]
