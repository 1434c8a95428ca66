"""Outputs and workspaces that the caller brings: what is too small or lies elsewhere is refused before anything is launched."""
from types import SimpleNamespace

import pytest
import torch

from paper_2510_02358_b200 import binding as dsp

DEV = "cuda"


@pytest.fixture
def no_launch(monkeypatch):
    def refuse(*a):
        raise AssertionError("launched")
    l = dsp.lib()
    for name in ("dsp_cache_plan", "dsp_attn_kv4"):
        monkeypatch.setattr(l, name, refuse)


def _plan_args(B=3, T=7, tree=False):
    i32 = dict(dtype=torch.int32, device=DEV)
    args = (torch.full((B,), 5, **i32), torch.full((B,), 2, **i32), torch.ones(B, **i32), torch.tensor([0, 8], device=DEV),
            torch.zeros((B, 4), **i32), torch.arange(8, **i32), 16, T)
    kw = dict(node_parent=torch.full((B, 40), -1, **i32), node_depth=torch.zeros((B, 40), **i32)) if tree else {}
    return args, kw


@pytest.mark.gpu
@pytest.mark.parametrize("tree", [False, True])
def test_plan_checks_the_outputs_that_it_is_given(no_launch, tree):
    args, kw = _plan_args(tree=tree)
    B, T = 3, 7
    e = lambda *shape, dt=torch.int32, dev=DEV: torch.empty(shape, dtype=dt, device=dev)      # noqa: E731
    good = dict(block_count=e(B), kv_len=e(B), row_status=e(B), cu_new=e(B + 1), ring_pos=e(2, dt=torch.int64), slot=e(T, dt=torch.int64),
                position=e(T), token_row=e(T), mask=e(T, 2) if tree else None)
    bad = [(n, t) for n, x in good.items() if x is not None
           for t in (x[:-1], x.to(torch.int16), x.cpu(), torch.empty(x.shape + (2,), dtype=x.dtype, device=DEV)[..., 0])]
    bad += [(n, None) for n in good if n != "token_row" and (tree or n != "mask")]
    if tree:
        bad += [("mask", e(T, 1)), ("mask", e(T * 2))]
    for name, t in bad:
        with pytest.raises((ValueError, AttributeError)):
            dsp.dsp_cache_plan(*args, **kw, out=SimpleNamespace(**dict(good, **{name: t})))
    for some in (good, dict(good, token_row=None)):
        with pytest.raises(AssertionError, match="launched"):
            dsp.dsp_cache_plan(*args, **kw, out=SimpleNamespace(**some))


@pytest.mark.gpu
def test_attention_counts_the_bytes_of_the_workspace_that_it_is_given(monkeypatch):
    q, cache = torch.zeros((2, 4, 64), device=DEV).bfloat16(), dsp.kv4_cache(4, 2, 64, 16, DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    args = (q, cache, torch.zeros((2, 2), **i32), torch.full((2,), 9, **i32), torch.arange(3, **i32), 1)
    need, seen = dsp.dsp_attn_kv4_workspace_bytes(2, 2, 4, 2, 64, 1), []
    monkeypatch.setattr(dsp.lib(), "dsp_attn_kv4", lambda *a: seen.append(a[24]) or 0)
    dsp.dsp_attn_kv4(*args, workspace=torch.empty(need // 4, dtype=torch.float32, device=DEV))
    assert seen == [need // 4 * 4]
    for ws in (torch.empty(need, dtype=torch.uint8), torch.empty((need, 2), dtype=torch.uint8, device=DEV)[:, 0]):
        with pytest.raises(ValueError):
            dsp.dsp_attn_kv4(*args, workspace=ws)
    assert len(seen) == 1
