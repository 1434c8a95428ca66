"""dsp_token_logprobs: outputs that nobody asks for, and calls without a row to read."""
import math
from types import SimpleNamespace

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,V,K,boost", [(1, 152064, 5, 24.0), (300, 32003, 0, 20.0), (40, 50001, 3, 30.0), (3, 15, 2, 30.0), (2, 1000, 0, 18.0)])
def test_scores_do_not_depend_on_whether_a_rank_is_asked_for(L, V, K, boost, dtype):
    """A token with nearly all of the mass: the first one is kept out of the 32-bit sums with a rank and without."""
    g = torch.Generator(device="cuda").manual_seed(int(boost))
    x = (2.0 * torch.randn(1, L, V, generator=g, device="cuda")).clamp(max=6.0)
    tokens = torch.randint(0, V, (1, L, 1), generator=g, device="cuda", dtype=torch.int32)
    tokens[0, 0] = V - 1
    x = x.scatter_(2, tokens.long(), torch.full((1, L, 1), boost, device="cuda")).to(dtype)
    full = dsp.dsp_token_logprobs(x, tokens, K=K)
    out = SimpleNamespace(**{k: None if v is None or k == "rank" else torch.full_like(v, 7) for k, v in vars(full).items()})
    got = dsp.dsp_token_logprobs(x, tokens, K=K, out=out)
    for name in ("logp", "lse", "entropy") + (("top_id", "top_logit", "top_logp") if K else ()):
        assert torch.equal(getattr(got, name), getattr(full, name)), name
    logp, _, _, entropy, _, _, _ = ref.score(x, 1.0, tokens, K)
    err, other = ref.exponent_error(x, 1.0, ref.terms(V)), -torch.expm1(logp[..., 0])
    assert ((got.logp.double() - logp).abs() <= (err * other)[..., None] + 2.0 ** -24 * logp.abs() + 1e-13).all()
    assert ((got.entropy.double() - entropy).abs() <= 2 * err * (entropy + 2 * other) + 2.0 ** -24 * entropy + 1e-13).all()


@pytest.mark.parametrize("B,L,V,K", [(3, 2, 152064, 5), (3, 300, 32003, 0), (1, 1, 152064, 0), (4, 2, 11, 3), (700, 3, 5001, 2)])
def test_a_call_without_a_row_to_read(B, L, V, K):
    """Every length is 0: nothing is left of the outputs' old contents, and what follows in the stream or the graph finds them written."""
    x = torch.full((B, L, V), math.nan, device="cuda").to(BF)
    tokens, lens = torch.zeros(B, L, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    out = dsp.dsp_token_logprobs(x, tokens, K=K, row_len=lens)

    def run():
        for t in vars(out).values():
            if t is not None:
                t.fill_(77)
        dsp.dsp_token_logprobs(x, tokens, K=K, row_len=lens, out=out)
        return {k: t.clone() for k, t in vars(out).items() if t is not None}

    def look(got):
        assert not got["row_status"].any() and (got["lse"] == -math.inf).all() and (got["logp"] == -math.inf).all()
        assert (got["rank"] == -1).all() and not got["entropy"].any() and (K == 0 or (got["top_id"] == -1).all())

    for _ in range(20):
        look(run())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(20):
        for t in got.values():
            t.fill_(55)
        graph.replay()
        look(got)


# as the call takes them: in 32 bits
TEMPERATURES = torch.tensor([1.0, 0.7, 0.5, 0.3, 0.1, 0.05, 0.01, 1e-3, 1.3, 2.0, 3.0, 10.0, 100.0, 1e3]).clamp(min=1.001e-3).tolist()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,L,V", [(2, 3, 152064), (4, 80, 80003), (3, 100, 32003), (3, 5, 50), (2, 2, 13)])
@pytest.mark.parametrize("mask", [-math.inf, "lowest", -1e37, -7e34, -1e30, -1e20, -1e13])
def test_masks_of_any_size_at_any_temperature(B, L, V, dtype, mask):
    """A few tokens of a row are allowed, so most threads, and whole tiles, see masked logits alone."""
    mask = torch.finfo(dtype).min if mask == "lowest" else mask
    g = torch.Generator(device="cuda").manual_seed(V)
    at = torch.rand(B, L, V, generator=g, device="cuda").topk(6, -1).indices
    x = torch.full((B, L, V), mask, device="cuda").to(dtype)
    x.scatter_(2, at, (3.0 * torch.randn(B, L, 6, generator=g, device="cuda")).to(dtype))
    mine = torch.full_like(x, -math.inf).scatter_(2, at, x.gather(2, at))
    tokens = torch.cat([at[..., :2], (at[..., :1] + 1) % V], -1).int()       # the last one is likely to be masked
    for T in TEMPERATURES:
        if mask > -3e9 * T and mask != -math.inf:
            continue                                                         # next to the bound, or no mask at this temperature
        # the masks weigh nothing in 64 bits either: exp(-10^9 / T) = 0
        logp, rank, lse, entropy, _, _, _ = ref.score(mine, T, tokens, 1)
        given = x.double().gather(-1, tokens.long()) / T - lse[..., None]
        err = ref.exponent_error(mine, T, ref.terms(V))
        for K in (0, 5):
            got = dsp.dsp_token_logprobs(x, tokens, K=K, temperature=T)
            assert not got.row_status.any(), T
            assert ((got.lse.double() - lse).abs() <= err + 2.0 ** -24 * lse.abs()).all(), (T, K)
            near = (got.logp.double() == given.float().double()) | ((got.logp.double() - given).abs() <= err[..., None] + 2.0 ** -24 * given.abs())
            assert near.all() and torch.equal(got.rank.long(), rank), (T, K)
            assert ((got.entropy.double() - entropy).abs() <= err * (2 + math.log2(V + 1)) + 2.0 ** -24 * entropy).all(), (T, K)
            if K:
                order = mine.sort(dim=-1, descending=True, stable=True).indices[..., :5]
                assert torch.equal(got.top_id.long(), order), (T, K)


@pytest.mark.parametrize("T", [1.0, 0.3, 0.05, 100.0])
@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("L,V", [(1, 40000), (400, 30000), (3, 11)])
def test_rows_without_an_allowed_token_are_named(L, V, K, T):
    for dtype in (BF, F32):
        for mask in (-math.inf, torch.finfo(dtype).min, -1e30, -1e13):
            if mask > -3e9 * T:
                continue
            x = torch.full((2, L, V), mask, device="cuda").to(dtype)
            x[1] = 0.0
            got = dsp.dsp_token_logprobs(x, torch.zeros(2, L, 1, dtype=torch.int32, device="cuda"), K=K, temperature=T)
            assert got.row_status.tolist() == [dsp.ROW_NONFINITE_INPUT, 0] and got.lse[0].isnan().all()
            assert ((got.lse[1] - math.log(V)).abs() < 1e-5).all()
