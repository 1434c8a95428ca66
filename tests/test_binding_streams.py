"""``stream=``: a call on another stream than torch's current one, with outputs and workspaces of its own."""
import inspect

import numpy as np
import pytest
import torch

from paper_2510_02358_b200 import binding as dsp

DEV = "cuda"


class _Entered(Exception):
    pass


def test_every_call_that_takes_a_stream_runs_under_it(monkeypatch):
    def under(stream):
        raise _Entered(stream)
    monkeypatch.setattr(torch.cuda, "stream", under)
    calls = [f for n, f in vars(dsp).items() if n.startswith("dsp_") and inspect.isfunction(f) and "stream" in inspect.signature(f).parameters]
    assert len(calls) >= 18
    for f in calls:
        with pytest.raises(_Entered) as e:
            f(stream="s")
        assert e.value.args == ("s",)
    with pytest.raises(_Entered):
        dsp.dsp_beam_tree(None, "s")                               # also by its place


def _attention(new, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    Hq, Hkv, D, page, B, width = 8, 2, 128, 32, 3, 40
    k, v = torch.randn(B * width * page, 2 * Hkv, D, generator=g, device=DEV).bfloat16().split(Hkv, 1)
    cache = dsp.kv4_cache(B * width, Hkv, D, page, DEV)
    dsp.dsp_kv4_append(None, k, v, torch.arange(B * width * page, device=DEV), cache)
    q = torch.randn(B * new, Hq, D, generator=g, device=DEV).bfloat16()
    i32 = dict(dtype=torch.int32, device=DEV)
    return (q, cache, torch.arange(B * width, **i32).view(B, width), torch.full((B,), width * page - 3, **i32),
            torch.arange(B + 1, **i32) * new, new)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 40])
def test_memory_of_a_call_on_another_stream_is_not_handed_out_while_it_runs(monkeypatch, new):
    args, seen = _attention(new), []
    inner = dsp.lib().dsp_attn_kv4

    def spy(*a):
        seen.append((a[22], a[23], a[24]))                         # out, workspace, its bytes
        return inner(*a)
    want = dsp.dsp_attn_kv4(*args)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    monkeypatch.setattr(dsp.lib(), "dsp_attn_kv4", spy)
    s = torch.cuda.Stream()
    got = dsp.dsp_attn_kv4(*args, stream=s)
    out, ws, size = seen[0]
    mine = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]     # of the current stream, while s may still run
    assert got.data_ptr() == out
    assert all(t.data_ptr() + size <= ws or ws + size <= t.data_ptr() for t in mine)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 7, 40])
def test_calls_on_several_streams_give_what_calls_in_a_row_give(new):
    cases = [_attention(new, seed) for seed in range(4)]
    want = [dsp.dsp_attn_kv4(*a) for a in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = [[dsp.dsp_attn_kv4(*a, stream=s) for _ in range(6)] for a, s in zip(cases, streams)]
        torch.cuda.synchronize()
        for row, w in zip(got, want):
            assert all(torch.equal(x, w) for x in row)


@pytest.mark.gpu
def test_step_calls_on_another_stream_own_their_memory():
    draft = torch.randn(2, 6, 4096, device=DEV)
    want = dsp.dsp_lattice_build(draft, 8)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    before = torch.cuda.memory_stats()["allocated_bytes.all.current"]
    got = dsp.dsp_lattice_build(draft, 8, stream=s)
    assert torch.cuda.memory_stats()["allocated_bytes.all.current"] > before
    s.synchronize()
    for name in ("cand_id", "cand_logit", "lse64"):
        assert torch.equal(getattr(got, name), getattr(want, name))
    assert np.isfinite(got.lse64.cpu().numpy()).all()


# ---------------------------------------------------------------------------------------- devices
def test_the_tensors_device_has_to_be_the_current_one(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i)
    assert dsp._queue(torch.device("cuda", 0)) == 100
    for dev in (torch.device("cuda", 1), torch.device("cpu")):
        with pytest.raises(ValueError, match="current CUDA device"):
            dsp._queue(dev)


def test_read_refuses_a_cache_in_host_memory(monkeypatch):
    """On whatever stream: the address would go to the kernel."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(dsp, "lib", lambda: pytest.fail("called"))
    cache, slot = dsp.kv4_cache(2, 2, 64, 16, "cpu"), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        dsp.dsp_kv4_read(cache, slot, 64)


@pytest.mark.gpu
def test_calls_refuse_tensors_of_another_device(monkeypatch):
    args = _attention(1)
    q, cache = args[0], args[1]
    plan = [torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(3)] + [torch.tensor([0, 8], device=DEV), args[2], torch.arange(8, dtype=torch.int32, device=DEV)]
    slot = torch.zeros(3, dtype=torch.int64, device=DEV)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (lambda: dsp.dsp_attn_kv4(*args), lambda: dsp.dsp_qk_norm_rope(q, q[:, :2]), lambda: dsp.dsp_kv4_read(cache, slot, 128),
                 lambda: dsp.dsp_kv4_append(None, q[:, :2], q[:, :2], slot, cache), lambda: dsp.dsp_cache_plan(*plan, 32, 3)):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()
