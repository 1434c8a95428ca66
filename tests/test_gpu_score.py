"""dsp_token_logprobs against the definition in 64 bits."""
import math

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rows(B, L, V, dtype, seed, masked=0.0, offset=0, pitch=0):
    """Logits [B, L, V] with a few likely tokens; `offset` elements into a buffer, rows `pitch` elements longer than V apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = 2.0 * torch.randn(B, L, V, generator=g, device="cuda")
    x.scatter_add_(2, torch.randint(0, V, (B, L, 4), generator=g, device="cuda"), 5 + 3 * torch.rand(B, L, 4, generator=g, device="cuda"))
    if masked:
        x.masked_fill_(torch.rand(B, L, V, generator=g, device="cuda") < masked, -math.inf)
        x[..., V // 2] = 1.0                                              # one logit stays
    buf = torch.empty(B * L * (V + pitch) + offset, dtype=dtype, device="cuda")
    out = buf[offset:].view(B, L, V + pitch)[..., :V]
    out.copy_(x)
    return out, g


def tokens_of(g, B, L, G, V):
    t = torch.randint(0, V, (B, L, G), generator=g, device="cuda", dtype=torch.int32)
    if G > 1:
        t[..., -1] = V - 1
    if G > 2:
        t[..., 1] = 0
    return t


def close(got, want, tol, what):
    got, want = got.double(), want.double()
    same = (got == want) | ((got - want).abs() <= tol + 2.0 ** -24 * want.abs())
    assert same.all(), (what, (got - want).abs()[~same].max().item(), int((~same).sum()))


def check(x, T, tokens, K, row_len=None, got=None):
    got = got or dsp.dsp_token_logprobs(x, tokens, K=K, temperature=T, row_len=row_len)
    three = tokens if tokens.dim() == 3 else tokens[..., None]
    logp, rank, lse, entropy, top_id, top_x, top_p = ref.score(x, T, three, K, row_len)
    err = ref.exponent_error(x, T, ref.terms(x.shape[-1]))
    assert torch.equal(got.rank.long(), rank), "rank"
    close(got.lse, lse, err, "lse")
    close(got.logp.view(three.shape), logp, err[..., None], "logp")
    # T / S: every term's error again, times |a| <= log2 V + 1 in the mean
    close(got.entropy, entropy, err * (2 + math.log2(x.shape[-1] + 1)), "entropy")
    if K:
        assert torch.equal(got.top_id.long(), top_id) and torch.equal(got.top_logit.double(), top_x), "alternatives"
        close(got.top_logp, top_p, err[..., None], "top_logp")
    assert not got.row_status.any()
    return got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1, 2, 7, 15, 16, 17, 23, 33, 1000, 12288, 12289, 12303, 32003, 152064, 300001])
def test_sizes(V, dtype):
    x, g = rows(3, 2, V, dtype, V)
    check(x, 1.0, tokens_of(g, 3, 2, 3, V), min(5, 32))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("offset", range(9))
def test_rows_that_start_anywhere(dtype, offset):
    x, g = rows(2, 3, 5003, dtype, offset, offset=offset, pitch=offset % 3)
    t = tokens_of(g, 2, 3, 1, 5003)
    for first in (0, 1, 6, 7, 8, 9, 4994, 4995, 4996, 5001, 5002):       # tokens outside of the whole pieces, and next to them
        t[:, :, 0] = first
        check(x, 1.0, t, 3)


@pytest.mark.parametrize("T", [0.5, 1.0, 3.7])
@pytest.mark.parametrize("B,L,V,dtype,G,K", [(1, 1, 152064, BF, 1, 5), (16, 17, 32000, BF, 1, 20), (64, 8, 4001, F32, 33, 0),
                                             (1, 300, 32000, BF, 2, 32), (2, 1100, 1000, F32, 1, 1)])
def test_shapes_and_temperatures(B, L, V, dtype, G, K, T):
    x, g = rows(B, L, V, dtype, G)
    check(x, T, tokens_of(g, B, L, G, V), K)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("masked", [0.1, 0.9, 1.0])
@pytest.mark.parametrize("V", [20, 999, 32000, 152064])
def test_masked_vocabularies(V, masked, dtype):
    x, g = rows(2, 3, V, dtype, 5, masked=masked)
    t = tokens_of(g, 2, 3, 2, V)
    t[0, 0, 0] = V // 2
    check(x, 0.8, t, 32)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ties_and_zeros_of_both_signs(dtype):
    V = 4099
    x = torch.zeros(1, 4, V, dtype=dtype, device="cuda")
    x[0, 1, ::2] = -0.0
    x[0, 2] = torch.randint(0, 3, (V,), device="cuda").to(dtype)
    tiny = torch.finfo(dtype).smallest_normal / 4                         # below the smallest normal number
    x[0, 3] = tiny * torch.randint(-2, 3, (V,), device="cuda").to(dtype)
    for tok in (0, 1, 5, 2048, 4097, 4098):
        check(x, 1.0, torch.full((1, 4), tok, dtype=torch.int32, device="cuda"), 32)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ragged_rows_and_tokens_outside(dtype):
    x, g = rows(4, 5, 2000, dtype, 2)
    x[1, 3:] = math.nan                                                   # rows that are not read
    n = torch.tensor([5, 3, 0, 7], dtype=torch.int32, device="cuda")
    t = tokens_of(g, 4, 5, 3, 2000)
    t[0, 0], t[3, 1, 0] = torch.tensor([-1, 2000, 7], device="cuda"), 1 << 30
    got = dsp.dsp_token_logprobs(x, t, K=4, row_len=n)
    y = x.clone()
    y[1, 3:] = 0.0
    check(y, 1.0, t, 4, n.clamp(max=5), got)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [16, 100, 6150, 20000, 50257])
def test_many_rows(V, dtype):
    """More rows than CTAs: each takes several in turn, some of them unread."""
    B, L = 23, 41
    x, g = rows(B, L, V, dtype, V, offset=1, pitch=1)
    t = tokens_of(g, B, L, 3, V)
    n = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n[3], n[4:9] = L, 0
    check(x, 1.3, t, 0, n)
    x[3, 7, V // 2], x[5, 1, 0] = math.nan, math.nan                     # one that is read, one that is not
    got = dsp.dsp_token_logprobs(x, t, temperature=1.3, row_len=n)
    assert got.row_status.tolist() == [int(b == 3) for b in range(B)] and got.lse.isnan().sum() == 1 and got.lse[3, 7].isnan()
    check(x[3:4, 8:12], 1.3, t[3:4, 8:12].contiguous(), 2)               # few rows, cut into slices: other sums, the same bounds


def test_a_bad_row_is_named_and_alone():
    x, g = rows(3, 2, 32000, F32, 3)
    t = tokens_of(g, 3, 2, 1, 32000)
    want = dsp.dsp_token_logprobs(x, t, K=2)
    x[1, 0, 77], x[2, 1, 31999] = math.nan, math.inf
    got = dsp.dsp_token_logprobs(x, t, K=2)
    assert got.row_status.tolist() == [0, 1, 1]
    assert got.lse.isnan().tolist() == [[False, False], [True, False], [False, True]]
    assert got.logp[1, 0].isnan().all() and got.entropy[2, 1].isnan()
    keep = torch.tensor([[True, True], [False, True], [True, False]], device="cuda")
    for name in ("lse", "entropy", "rank", "top_id", "top_logp"):
        assert torch.equal(getattr(got, name)[keep], getattr(want, name)[keep]), name
    x[0] = -math.inf
    assert dsp.dsp_token_logprobs(x, t).row_status.tolist() == [1, 1, 1]


def test_far_logits():
    x = torch.full((1, 2, 9000), -9e36, device="cuda")
    x[0, 0, 5], x[0, 1, 8999] = 1e6, 1e6 - 0.5
    x[0, 1, 3] = 1e6
    check(x, 1.0, torch.tensor([[5, 3]], dtype=torch.int32, device="cuda"), 2)


def test_only_what_is_asked_for():
    x, g = rows(2, 2, 1000, BF, 8)
    got = dsp.dsp_token_logprobs(x)
    assert got.logp is None and got.rank is None and got.top_id is None
    full = dsp.dsp_token_logprobs(x, tokens_of(g, 2, 2, 1, 1000)[..., 0], K=3)
    assert torch.equal(got.lse, full.lse) and torch.equal(got.entropy, full.entropy) and full.logp.shape == (2, 2)
    assert dsp.dsp_token_logprobs(x[:0]).lse.shape == (0, 2)


def test_calls_give_the_same_bits_and_agree_with_the_lattice():
    x, g = rows(4, 8, 152064, BF, 9)
    t = tokens_of(g, 4, 8, 1, 152064)
    a, b = (dsp.dsp_token_logprobs(x, t, K=16) for _ in range(2))
    for name in vars(a):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    lat = dsp.dsp_lattice_build(x, 16)
    assert torch.equal(lat.cand_id, a.top_id) and torch.equal(lat.cand_logit, a.top_logit)
    close(lat.lse, a.lse, 2 * ref.exponent_error(x, 1.0, ref.terms(152064)), "lse")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,L,V,K,offset", [(1, 1, 12304, 5, 0), (3, 1, 24577, 32, 1), (1, 3, 50000, 0, 3), (2, 2, 98304, 1, 0), (5, 1, 110001, 20, 5),
                                            (1, 1, 290000, 7, 0), (1, 4, 147459, 0, 2), (8, 1, 32003, 32, 0)])
def test_few_rows(B, L, V, K, offset, dtype):
    """A cluster's rows, of every number of tiles, with rows that are not read beside them; nothing is left of the outputs' old contents."""
    x, g = rows(B, L, V, dtype, seed=V + K, offset=offset, masked=0.2)
    tokens = tokens_of(g, B, L, 4, V)
    tokens[..., 0] = x.argmax(-1).int()
    tokens[0, 0, 0] = V - 1
    check(x, 1.0, tokens, K)
    lens = torch.tensor([0] + [L] * (B - 1) if B > 1 else [max(1, L - 1)], dtype=torch.int32, device="cuda")
    old = dsp.dsp_token_logprobs(x, tokens, K=K)
    for name in vars(old):
        if getattr(old, name) is not None:
            getattr(old, name).fill_(77)
    check(x, 0.7, tokens, K, row_len=lens, got=dsp.dsp_token_logprobs(x, tokens, K=K, temperature=0.7, row_len=lens, out=old))


@pytest.mark.parametrize("L", [1, 2])
@pytest.mark.parametrize("K", [0, 8])
def test_bad_and_flat_rows_of_few(K, L):
    """NaN and +inf are named in their own status word only; a row of one value (no list is long enough for it) has its first tokens on top."""
    B, V = 4, 40000
    x, g = rows(B, L, V, BF, seed=3)
    x[1, L - 1, 39999], x[2, 0, 0] = math.nan, math.inf
    x[3] = 0.25
    tokens = tokens_of(g, B, L, 1, V)
    got = dsp.dsp_token_logprobs(x, tokens, K=K)
    assert got.row_status.tolist() == [0, dsp.ROW_NONFINITE_INPUT, dsp.ROW_NONFINITE_INPUT, 0]
    assert got.lse[1, L - 1].isnan() and got.lse[2, 0].isnan() and got.logp[2, 0].isnan().all()
    good = torch.tensor([0, 3], device="cuda")
    part = type(got)(**{k: None if v is None else v[good].contiguous() for k, v in vars(got).items()})
    check(x[good], 1.0, tokens[good].contiguous(), K, got=part)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,L,V", [(2, 3, 33000), (3, 200, 5001), (2, 2, 11)])
def test_masks_of_the_lowest_number(B, L, V, dtype):
    """Masks of the type's lowest value are finite logits: they weigh nothing, and stand behind all others among the alternatives."""
    x, g = rows(B, L, V, dtype, seed=8)
    x.masked_fill_(torch.rand(B, L, V, generator=g, device="cuda") < 0.5, torch.finfo(dtype).min)
    x[0, 0] = torch.finfo(dtype).min
    x[0, 0, V - 2], x[0, 0, 4] = 1.5, 0.5
    tokens = tokens_of(g, B, L, 2, V)
    got = dsp.dsp_token_logprobs(x, tokens, K=6)
    logp, rank, lse, entropy, top_id, top_x, top_p = ref.score(x, 1.0, tokens, 6)
    err = ref.exponent_error(x.masked_fill(x < -1e30, 0.0), 1.0, ref.terms(V))
    assert not got.row_status.any() and torch.equal(got.rank.long(), rank)
    assert torch.equal(got.top_id.long(), top_id) and torch.equal(got.top_logit.double(), top_x)
    for a, b, tol in ((got.lse, lse, err), (got.logp, logp, err[..., None]), (got.top_logp, top_p, err[..., None]),
                      (got.entropy, entropy, err * (2 + math.log2(V + 1)))):
        close(a, b, tol, "masked")
    x.fill_(torch.finfo(dtype).min)                                       # nothing is left: named, not answered
    assert (dsp.dsp_token_logprobs(x, tokens, K=6).row_status & dsp.ROW_NONFINITE_INPUT).bool().all()


def test_rows_beyond_32_bits():
    V, L = 160001, 14000
    x = torch.empty(1, L, V, dtype=BF, device="cuda")
    small, g = rows(1, 3, V, BF, seed=4)
    x[:, -3:] = small
    tokens = torch.zeros(1, L, 2, dtype=torch.int32, device="cuda")
    tokens[:, -3:] = tokens_of(g, 1, 3, 2, V)
    got = dsp.dsp_token_logprobs(x, tokens, K=4)
    part = type(got)(**{k: v if k == "row_status" else v[:, -3:].contiguous() for k, v in vars(got).items()})
    part.row_status = torch.zeros_like(part.row_status)                   # the other rows are not initialised
    check(x[:, -3:], 1.0, tokens[:, -3:].contiguous(), 4, got=part)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,V,K,boost", [(1, 152064, 5, 24.0), (300, 32003, 0, 20.0), (40, 50001, 3, 30.0), (3, 15, 2, 30.0), (2, 1000, 0, 18.0)])
def test_a_token_with_nearly_all_of_the_mass(L, V, K, boost, dtype):
    """Its log-probability is made of the other tokens' sum, relative to its own exponent: an error of that sum counts times 1 - p, and in the entropy
    times the others' share of it."""
    x, g = rows(1, L, V, dtype, seed=int(boost))
    x = x.clamp(max=6.0)
    tokens = torch.randint(0, V, (1, L, 1), generator=g, device="cuda", dtype=torch.int32)
    tokens[0, 0] = V - 1
    x.scatter_(2, tokens.long(), torch.full((1, L, 1), boost, dtype=dtype, device="cuda"))
    got = dsp.dsp_token_logprobs(x, tokens, K=K)
    logp, rank, _, entropy, _, _, top_p = ref.score(x, 1.0, tokens, K)
    err = ref.exponent_error(x, 1.0, ref.terms(V))
    other = -torch.expm1(logp[..., 0])
    assert (other < 0.2).all()
    close(got.logp, logp, (err * other)[..., None] + 1e-13, "logp")
    close(got.entropy, entropy, 2 * err * (entropy + 2 * other) + 1e-13, "entropy")
    if K:
        close(got.top_logp[..., 0], top_p[..., 0], err * other + 1e-13, "top_logp")


@pytest.mark.parametrize("L,V", [(18, 10000003), (36, 5000000), (500, 40000)])
def test_many_long_rows(L, V):
    """Rows of many slices, with a CTA count beyond three an SM: a ring of three tiles where the finish needs it, of two elsewhere."""
    g = torch.Generator(device="cuda").manual_seed(L)
    x = torch.randn(1, L, V, generator=g, device="cuda", dtype=torch.bfloat16)
    tokens = torch.randint(0, V, (1, L, 1), generator=g, device="cuda", dtype=torch.int32)
    tokens[0, -1] = x[0, -1].argmax().int()
    got = dsp.dsp_token_logprobs(x, tokens, K=3)
    part = type(got)(**{k: v if k == "row_status" else v[:, -3:].contiguous() for k, v in vars(got).items()})
    check(x[:, -3:], 1.0, tokens[:, -3:].contiguous(), 3, got=part)
