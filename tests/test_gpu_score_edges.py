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
