"""Calls after a verified step that are refused: on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2510_02358_b200 import binding as dsp
from paper_2510_02358_b200 import build

BAD, NOT, WS = dsp.DSP_ERR_INVALID_ARG, dsp.DSP_ERR_UNSUPPORTED, dsp.DSP_ERR_WORKSPACE
ONE, TWO = 256, 1 << 20                                     # addresses that are never read


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def score(**kw):
    a = dict(x=ONE, dtype=1, B=2, L=3, V=100, sb=300, sl=100, lens=None, tok=ONE, G=1, T=1.0, K=2, logp=ONE, rank=ONE, top_id=ONE, top_x=ONE,
             top_p=ONE, lse=ONE, ent=None, status=ONE, ws=ONE, n=1 << 20)
    a.update(kw)
    return dsp.lib().dsp_token_logprobs(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(x=ONE + 1), BAD), (dict(lse=None), BAD), (dict(status=None), BAD), (dict(ws=None), BAD), (dict(ws=ONE + 8), BAD),
    (dict(B=-1), BAD), (dict(L=0), BAD), (dict(V=0), BAD), (dict(sl=99), BAD), (dict(sb=299), BAD), (dict(sb=-1), BAD), (dict(G=-1), BAD), (dict(K=-1), BAD),
    (dict(tok=None), BAD), (dict(logp=None), BAD), (dict(G=0, rank=ONE), BAD), (dict(top_id=None), BAD), (dict(top_x=None), BAD), (dict(top_p=None), BAD),
    (dict(T=0.0), BAD), (dict(T=-1.0), BAD), (dict(T=float("nan")), BAD), (dict(T=1e4), BAD), (dict(dtype=2), NOT), (dict(K=33), NOT), (dict(G=1025), NOT),
    (dict(V=(1 << 30) + 1, sl=1 << 31, sb=1 << 33), NOT), (dict(B=1 << 13, L=1 << 12), NOT), (dict(n=16), WS)])
def test_scores(kw, code):
    assert score(**kw) == code


def distill(**kw):
    a = dict(x=ONE, dtype=0, B=2, L=3, V=100, sb=300, sl=100, ids=ONE, val=ONE, tlse=None, count=None, K=4, T=1.0, w=None, loss=ONE, acc=None, lse=None,
             state=None, g=ONE, gb=300, gl=100, status=None)
    a.update(kw)
    return dsp.lib().dsp_distill(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(x=ONE + 2), BAD), (dict(ids=None), BAD), (dict(val=None), BAD), (dict(loss=None), BAD), (dict(state=ONE + 4), BAD),
    (dict(g=ONE + 2), BAD), (dict(gl=99), BAD), (dict(gb=299), BAD), (dict(sl=99), BAD), (dict(sb=299), BAD), (dict(K=0), BAD), (dict(T=1e-9), BAD),
    (dict(B=-1), BAD), (dict(L=0), BAD), (dict(V=0), BAD), (dict(K=257), NOT), (dict(dtype=5), NOT), (dict(B=1 << 13, L=1 << 12), NOT)])
def test_distillation(kw, code):
    assert distill(**kw) == code


def distill_grad(**kw):
    a = dict(x=ONE, dtype=0, B=2, L=3, V=100, sb=300, sl=100, ids=ONE, K=4, state=ONE, T=1.0, up=ONE, g=ONE, gb=300, gl=100)
    a.update(kw)
    return dsp.lib().dsp_distill_grad(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), BAD), (dict(ids=None), BAD), (dict(state=None), BAD), (dict(state=ONE + 8), BAD), (dict(up=None), BAD), (dict(g=None), BAD),
    (dict(gl=99), BAD), (dict(K=0), BAD), (dict(K=257), NOT), (dict(T=float("inf")), BAD), (dict(dtype=-1), NOT)])
def test_distillation_gradient(kw, code):
    assert distill_grad(**kw) == code


def fork(**kw):
    a = dict(src=ONE, keep=None, Bo=2, seq=ONE, count=ONE, pos=ONE, table=ONE, ts=8, Bi=2, page=16, blocks=50, width=8, ring=ONE, new=TWO, ns=8,
             count2=TWO, seq2=TWO, pos2=TWO, c1=TWO, c2=TWO, c3=TWO, status=TWO, ws=ONE, n=1 << 20)
    a.update(kw)
    return dsp.lib().dsp_cache_fork(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(src=None), BAD), (dict(seq=None), BAD), (dict(count=None), BAD), (dict(pos=None), BAD), (dict(table=None), BAD), (dict(ring=None), BAD),
    (dict(new=None), BAD), (dict(count2=None), BAD), (dict(seq2=None), BAD), (dict(pos2=None), BAD), (dict(c1=None), BAD), (dict(c2=None), BAD),
    (dict(c3=None), BAD), (dict(status=None), BAD), (dict(ws=None), BAD), (dict(ws=ONE + 16), BAD), (dict(Bo=-1), BAD), (dict(Bi=-1), BAD),
    (dict(page=0), BAD), (dict(blocks=0), BAD), (dict(width=0), BAD), (dict(ts=7), BAD), (dict(ns=7), BAD), (dict(new=ONE), BAD), (dict(new=ONE + 32), BAD),
    (dict(new=ONE - 32), BAD), (dict(pos2=ONE), BAD), (dict(count2=ONE), BAD), (dict(seq2=ONE), BAD), (dict(Bo=8193), NOT), (dict(Bi=8193), NOT),
    (dict(width=1 << 30, ts=1 << 30, ns=1 << 30), NOT), (dict(n=64), WS)])
def test_forks(kw, code):
    assert fork(**kw) == code


def copy(**kw):
    a = dict(cache=ONE, layers=2, stride=16 * 136 * 2 * 50, blocks=50, page=16, H=2, D=128, src=ONE, dst=ONE, n=None, N=3)
    a.update(kw)
    return dsp.lib().dsp_kv4_copy(*a.values(), None)


def compact(**kw):
    a = dict(cache=ONE, layers=2, stride=16 * 136 * 2 * 50, blocks=50, page=16, H=2, D=128, table=ONE, ts=8, width=8, seq=ONE, node=ONE, length=ONE, B=2, L=4)
    a.update(kw)
    return dsp.lib().dsp_kv4_compact(*a.values(), None)


@pytest.mark.parametrize("call", [copy, compact])
@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), BAD), (dict(cache=ONE + 8), BAD), (dict(layers=0), BAD), (dict(stride=16 * 136 * 2 * 50 - 16), BAD), (dict(stride=16 * 136 * 2 * 50 + 8), BAD),
    (dict(blocks=0), BAD), (dict(page=0), BAD), (dict(page=24), BAD), (dict(H=0), BAD), (dict(D=96), NOT), (dict(layers=70000), NOT), (dict(H=5000), NOT)])
def test_moves(call, kw, code):
    assert call(**kw) == code


def test_moves_of_their_own():
    assert copy(N=-1) == copy(src=None) == copy(dst=None) == BAD and copy(N=(1 << 24) + 1) == NOT and copy(N=0, src=None) == dsp.DSP_OK
    assert compact(B=-1) == compact(L=-1) == compact(ts=7) == compact(width=0) == compact(table=None) == compact(seq=None) == BAD
    assert compact(node=None) == compact(length=None) == BAD and compact(B=0, table=None) == compact(L=0, node=None) == dsp.DSP_OK


def test_empty_batches_and_workspace_sizes():
    assert score(B=0, x=None) == distill(B=0, x=None) == distill_grad(B=0, x=None) == dsp.DSP_OK
    for V in (1, 15, 32003, 152064, 1 << 30):
        for dt in (0, 1):
            assert dsp.dsp_token_logprobs_workspace_bytes(2, 3, V, dt) % 256 == 0
    assert dsp.dsp_cache_fork_workspace_bytes(0, 0, 1) >= 256
    for bad in ((-1, 0, 1), (0, -1, 1), (0, 0, 0)):
        with pytest.raises(dsp.DspError):
            dsp.dsp_cache_fork_workspace_bytes(*bad)
    n = C.c_size_t(0)
    assert dsp.lib().dsp_token_logprobs_workspace_bytes(1, 1, 0, 0, C.byref(n)) == BAD
    assert dsp.lib().dsp_token_logprobs_workspace_bytes(1, 1, 5, 0, None) == BAD


def test_tensors_in_host_memory_are_refused():
    x, t, f = torch.zeros(2, 3, 50), torch.zeros(2, 3, 4, dtype=torch.int32), torch.zeros(2, 3, 4)
    i = torch.zeros(2, dtype=torch.int32)
    cache = torch.zeros(4, 2, 16 * 136, dtype=torch.uint8)
    for call in (lambda: dsp.dsp_token_logprobs(x, t), lambda: dsp.dsp_distill(x, t, f), lambda: dsp.dsp_distill_grad(x, t, torch.zeros(2, 3, 8), torch.zeros(2, 3)),
                 lambda: dsp.dsp_cache_fork(i, None, i, i, torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4, dtype=torch.int32), i, 16, torch.zeros(2, 4, dtype=torch.int32)),
                 lambda: dsp.dsp_kv4_copy(cache, 128, i, i), lambda: dsp.dsp_kv4_compact(cache, 128, t[0], i, t[0], i)):
        with pytest.raises(ValueError):
            call()
