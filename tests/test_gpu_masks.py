"""Masks of any size in the calls on logits: -inf, the type's lowest number, and what programs put there by hand.

A few tokens of a row are allowed, so that most threads, tiles and vocabulary slices hold masked logits alone; the masks' mass is 0 in 64 bits too.
Error of a row's log-sum-exp: after_reference.exponent_error, of the allowed logits."""
import math
from types import SimpleNamespace

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
MASKS = [-math.inf, "lowest", -1e36, -1e30, -1e20, -1e13, -1e11]


def masked(B, L, V, dtype, mask, seed, allowed=6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    at = torch.rand(B, L, V, generator=g, device="cuda").topk(allowed, -1).indices
    x = torch.full((B, L, V), torch.finfo(dtype).min if mask == "lowest" else mask, device="cuda").to(dtype)
    x.scatter_(2, at, (3.0 * torch.randn(B, L, allowed, generator=g, device="cuda")).to(dtype))
    return x, torch.full_like(x, -math.inf).scatter_(2, at, x.gather(2, at))


def look(mine, lse, entropy=None):
    _, _, want, h, _, _, _ = ref.score(mine, 1.0, torch.zeros(mine.shape[:2] + (1,), dtype=torch.int32, device="cuda"), 1)
    err = ref.exponent_error(mine, 1.0, ref.terms(mine.shape[-1]))
    assert ((lse.double() - want).abs() <= err + 2.0 ** -24 * want.abs()).all()
    if entropy is not None:
        assert ((entropy.double() - h).abs() <= err * (2 + math.log2(mine.shape[-1] + 1)) + 2.0 ** -23).all()
    return want, err


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("B,L,V", [(1, 1, 152064), (4, 80, 80000), (2, 3, 32003), (3, 5, 50)])
def test_lattice_and_its_shards(B, L, V, mask, dtype):
    x, mine = masked(B, L, V, dtype, mask, V)
    lat = dsp.dsp_lattice_build(x, 4)
    look(mine, lat.lse, lat.entropy)
    assert not lat.row_status.any()
    assert torch.equal(lat.cand_id.long(), mine.sort(dim=-1, descending=True, stable=True).indices[..., :4])
    half = V // 16 * 8
    parts = [dsp.dsp_lattice_shard(x[..., :half], 0, 4), dsp.dsp_lattice_shard(x[..., half:], half, 4)]
    both = [torch.stack([getattr(p, k) for p in parts]) for k in ("sums", "keys", "status")]
    merged = dsp.dsp_lattice_merge(*both, V, 4)
    look(mine, merged.lse, merged.entropy)
    assert torch.equal(merged.cand_id, lat.cand_id) and not merged.row_status.any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("B,L,V", [(2, 3, 152064), (2, 3, 32003)])
def test_verification_and_unmasking(B, L, V, mask, dtype):
    x, mine = masked(B, L + 1, V, dtype, mask, V)
    d, _ = masked(B, L, V, dtype, mask, V)                         # other logits at other places
    lat = dsp.dsp_lattice_build(d, 4)
    cps = SimpleNamespace(path=lat.cand_id[..., 0].contiguous(), path_slot=torch.zeros(B, L, dtype=torch.int32, device="cuda"),
                          path_len=torch.full((B,), L, dtype=torch.int32, device="cuda"))
    u = torch.full((B, L + 1), 0.5, device="cuda")
    ver = dsp.dsp_verify(x, d, cps, lat, mode=torch.ones(B, dtype=torch.uint8, device="cuda"), u=u, row_status=lat.row_status)
    look(mine, ver.tgt_lse)
    assert not lat.row_status.any() and torch.equal(ver.tgt_argmax.long(), mine.argmax(-1))
    allowed = mine.gather(1, ver.accepted_len[:, None, None].long().expand(-1, 1, V))[:, 0].gather(1, ver.next_token[:, None].long())
    assert torch.isfinite(allowed).all()                           # no masked token is drawn
    tokens, on = torch.zeros(B, L + 1, dtype=torch.int32, device="cuda"), torch.ones(B, L + 1, dtype=torch.uint8, device="cuda")
    r = dsp.dsp_unmask_step(x, tokens, on, 1)
    conf = mine.double().amax(-1) - mine.double().logsumexp(-1)
    err = ref.exponent_error(mine, 1.0, ref.terms(V))
    assert ((r.confidence.double() - conf).abs() <= err + 2.0 ** -24 * conf.abs()).all() and not r.row_status.any()


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("L,V", [(1, 152064), (300, 32000), (3, 32003), (2, 24)])
def test_rows_without_an_allowed_token_are_named(L, V, mask):
    for dtype in (BF, F32):
        x = torch.full((2, L, V), torch.finfo(dtype).min if mask == "lowest" else mask, device="cuda").to(dtype)
        x[1] = 0.0
        lat = dsp.dsp_lattice_build(x, 4)
        assert lat.row_status.tolist() == [dsp.ROW_NONFINITE_INPUT, 0] and ((lat.lse[1] - math.log(V)).abs() < 1e-5).all()
