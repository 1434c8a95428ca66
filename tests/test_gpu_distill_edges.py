"""dsp_distill where the teacher's list is all that there is, or where nothing was read."""
import math

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# rows of a cluster with and without the gradient, and rows that are streamed for their loss
FORMS = [(2, 500, 5003, F32, True), (2, 500, 5003, F32, False), (3, 7, 40000, BF, True), (3, 7, 40000, BF, False), (4, 80, 80003, BF, False)]


def grammar(B, L, V, dtype, allowed, mask, seed):
    """Logits of which `allowed` tokens a row are not masked."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((B, L, V), mask, device="cuda").to(dtype)
    at = torch.rand(B, L, V, generator=g, device="cuda").topk(allowed, -1).indices
    return x.scatter_(2, at, (3.0 * torch.randn(B, L, allowed, generator=g, device="cuda")).to(dtype)), at


@pytest.mark.parametrize("B,L,V,dtype,grad", FORMS)
@pytest.mark.parametrize("mask", [-math.inf, "lowest", -1e9, -1e4])
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_a_teacher_under_the_drafters_mask(B, L, V, dtype, grad, mask, T):
    """Scores of a masked target as the teacher's list.  Of the drafter equal to it the loss is the difference of the two log-sum-exps: each
    off by the error of its sum, the teacher's rounded to 32 bits (2^-24 of it), the loss rounded too."""
    mask = torch.finfo(dtype).min if mask == "lowest" else mask
    x, at = grammar(B, L, V, dtype, 6, mask, V)
    t = dsp.dsp_token_logprobs(x, K=8, temperature=T)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    r = dsp.dsp_distill(x, t.top_id, t.top_logit, teacher_lse=t.lse, temperature=T, grad=grad, row_status=status)
    mine = torch.full_like(x, -math.inf).scatter_(2, at, x.gather(2, at))
    err = 2 * ref.exponent_error(mine, T, ref.terms(V)) + 2.0 ** -24 * (t.lse.double().abs() + 1)
    assert not status.any()
    assert (r.loss.double().abs() <= err).all(), (r.loss.abs().max().item(), err.max().item())
    assert ((r.accept.double() - 1).abs() <= 2 * err).all()
    g = r.grad if grad else dsp.dsp_distill_grad(x, t.top_id, r.state, torch.ones(B, L, device="cuda"), temperature=T)
    assert (g.double().abs() <= 4 * err[..., None] / T).all()
    # another drafter under the mask: the loss that the allowed tokens alone give.  With every log p_k off by d, which is the same for all,
    # the sum of p (log p - log q) is off by d (1 + itself)
    y = x.scatter(2, at, x.gather(2, at) + torch.randn(B, L, 6, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype))
    got = dsp.dsp_distill(y, t.top_id, t.top_logit, teacher_lse=t.lse, temperature=T, grad=grad).loss.double()
    want = ref.distill(y, at, x.gather(2, at), T)[0]
    yours = torch.full_like(y, -math.inf).scatter_(2, at, y.gather(2, at))
    off = err + 2 * ref.exponent_error(yours, T, ref.terms(V))
    assert ((got - want).abs() <= off * (1 + want) + 2.0 ** -24 * want).all(), (got - want).abs().max().item()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (9, 9), (9, 12), (32, 32), (200, 256)])
def test_a_list_of_the_whole_vocabulary(V, K, dtype):
    B, L = 5, 60
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (3.0 * torch.randn(B, L, V, generator=g, device="cuda")).to(dtype)
    ids = torch.full((B, L, K), -1, dtype=torch.int32, device="cuda")
    val = torch.zeros(B, L, K, device="cuda")
    ids[..., :V], val[..., :V] = torch.arange(V, device="cuda", dtype=torch.int32), x.float()
    lse = x.double().logsumexp(-1).float()
    err = 2 * ref.exponent_error(x, 1.0, ref.terms(V)) + 2.0 ** -24 * (lse.double().abs() + 1)
    for grad in (True, False):
        r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=grad)
        assert (r.loss.double().abs() <= err).all(), r.loss.abs().max().item()


@pytest.mark.parametrize("grad", [True, False])
def test_mass_of_the_teacher_that_the_drafter_has_no_token_for(grad):
    """More than rounding: the loss is infinite, and the gradient is not."""
    x, at = grammar(2, 40, 5003, F32, 6, -math.inf, 3)
    t = dsp.dsp_token_logprobs(x, K=5)                               # a token short of all
    y = torch.full_like(x, -math.inf).scatter_(2, t.top_id.long(), t.top_logit)
    r = dsp.dsp_distill(y, t.top_id, t.top_logit, teacher_lse=t.lse, grad=grad)
    some = 1 - (t.top_logp.double()).exp().sum(-1) > 1e-5
    assert some.any() and (r.loss[some] == math.inf).all() and not r.loss.isnan().any()
    if grad:
        assert torch.isfinite(r.grad).all()


@pytest.mark.parametrize("B,L,V,dtype,offset", [(3, 4, 4099, F32, 1), (2, 3, 40000, BF, 0), (3, 60, 80000, BF, 0)])
def test_the_gradient_of_a_row_that_the_loss_did_not_read(B, L, V, dtype, offset):
    """A row of weight 0 is not read: whatever its logits are (a padded batch's are anything), its loss is 0 and so is the gradient, with any factor."""
    g = torch.Generator(device="cuda").manual_seed(V)
    buf = torch.randn(B * L * V + offset, generator=g, device="cuda").to(dtype)
    x = buf[offset:].view(B, L, V)
    ids = torch.randint(0, V, (B, L, 4), generator=g, device="cuda", dtype=torch.int32)
    val, w = torch.randn(B, L, 4, generator=g, device="cuda"), torch.ones(B, L, device="cuda")
    lse, up = torch.full((B, L), 9.0, device="cuda"), torch.rand(B, L, generator=g, device="cuda") + 0.5
    w[0, 1], w[1] = 0.0, 0.0
    want = dsp.dsp_distill_grad(x, ids, dsp.dsp_distill(x, ids, val, teacher_lse=lse).state, up)
    want[w == 0] = 0.0
    x[0, 1, ::2], x[1, 0], x[1, 1, 5], x[1, 2] = math.nan, math.nan, math.inf, -math.inf
    r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, weight=w)
    assert not r.loss[w == 0].any()
    assert torch.equal(dsp.dsp_distill_grad(x, ids, r.state, up), want)
    y = x.clone()
    assert torch.equal(dsp.dsp_distill_grad(y, ids, r.state, up, grad=y), want)


@pytest.mark.parametrize("B,L,V,dtype,grad", FORMS + [(3, 5, 50, F32, True), (2, 3, 152064, BF, True), (4, 80, 80000, BF, False)])
@pytest.mark.parametrize("mask", [-math.inf, "lowest", -1e37, -7e34, -1e30, -1e20, -1e13])
@pytest.mark.parametrize("tail", [True, False])
def test_masks_of_any_size_at_any_temperature(B, L, V, dtype, grad, mask, tail):
    """Most threads and warps see masked logits alone; the list has some of the allowed tokens, and a masked one that the teacher does not have
    either.  Error of the row's sums as in the other tests: each of loss, accept and gradient has it a few times."""
    mask = torch.finfo(dtype).min if mask == "lowest" else mask
    g = torch.Generator(device="cuda").manual_seed(V)
    x, at = grammar(B, L, V, dtype, 6, mask, V)
    mine = torch.full_like(x, -math.inf).scatter_(2, at, x.gather(2, at))
    free = (at.sort(-1).values[..., :1] + 1) % V
    free = torch.where((free == at).any(-1, keepdim=True), torch.full_like(free, V), free)             # no second slot of an allowed token
    ids = torch.cat([at[..., :3], free], -1).int()
    val = torch.cat([x.gather(2, at[..., :3]).float() + torch.randn(B, L, 3, generator=g, device="cuda"), torch.full((B, L, 1), -math.inf, device="cuda")], -1)
    # in 32 bits, as the call takes them
    for T in torch.tensor([1.0, 0.7, 0.3, 0.05, 1e-2, 2.0, 10.0, 100.0, 1e3]).tolist():
        if mask > -3e9 * T and mask != -math.inf:
            continue
        lse = ((val.double() / T).logsumexp(-1) + 0.25).float() if tail else None
        loss, accept, full, want = ref.distill(mine, ids, val, T, lse)
        err = 2.0 ** -20 + 4 * ref.exponent_error(mine, T, ref.terms(V))
        status = torch.zeros(B, dtype=torch.int32, device="cuda")
        r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, temperature=T, grad=grad, row_status=status)
        got = r.grad if grad else dsp.dsp_distill_grad(x, ids, r.state, torch.ones(B, L, device="cuda"), temperature=T)
        assert not status.any(), T
        # p (log p - x / T + lse): a listed term is in 64 bits, their sum rounded to 32
        size = (val[..., :3].double() - x.gather(2, at[..., :3]).double()).abs().amax(-1) / T + full.abs()
        assert ((r.loss.double() - loss).abs() <= err + 2.0 ** -22 * (loss.abs() + size)).all(), T
        assert ((r.accept.double() - accept).abs() <= err).all() and ((r.lse.double() - full).abs() <= err + 2.0 ** -24 * full.abs()).all(), T
        assert ((got.double() - want).abs() <= 2 * err[..., None] / T + torch.finfo(dtype).eps / 2 * want.abs()).all(), T


@pytest.mark.parametrize("B,L,V,dtype,grad", FORMS)
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e20, -1e30, -1e37])
def test_listed_tokens_that_the_drafter_has_masked(B, L, V, dtype, grad, mask):
    """The teacher's best tokens are masked: the loss is p times the mask, and the gradient -p there, finite everywhere."""
    x, at = grammar(B, L, V, dtype, 6, mask, V)
    x.scatter_(2, at[..., :2], torch.full_like(x[..., :2], mask))
    ids, val = at[..., :3].int(), torch.tensor([1.0, 0.0, 0.5], device="cuda").expand(B, L, 3).contiguous()
    r = dsp.dsp_distill(x, ids, val, grad=grad)
    p = torch.softmax(val.double(), -1)
    want = (p * (p.log() - torch.log_softmax(x.double(), -1).gather(-1, at[..., :3]))).sum(-1)
    assert ((r.loss.double() - want).abs() <= 2.0 ** -20 * want).all()
    got = r.grad if grad else dsp.dsp_distill_grad(x, ids, r.state, torch.ones(B, L, device="cuda"))
    assert torch.isfinite(got).all()
    assert ((got.double().gather(2, at[..., :2]) + p[..., :2]).abs() <= torch.finfo(dtype).eps / 2 * p[..., :2] + 2.0 ** -20).all()


@pytest.mark.parametrize("grad", [True, False])
def test_rows_without_an_allowed_token_are_named(grad):
    for B, L, V, dtype in ((2, 5, 5003, F32), (2, 90, 80003, BF)):
        for T, mask in ((1.0, -math.inf), (0.3, -1e30), (100.0, -1e30), (1.0, -1e13), (2.0, torch.finfo(dtype).min)):
            x = torch.full((B, L, V), mask, device="cuda").to(dtype)
            x[1] = 0.0
            status = torch.zeros(B, dtype=torch.int32, device="cuda")
            ids = torch.zeros(B, L, 1, dtype=torch.int32, device="cuda")
            r = dsp.dsp_distill(x, ids, torch.zeros(B, L, 1, device="cuda"), temperature=T, grad=grad, row_status=status)
            assert status.tolist() == [dsp.ROW_NONFINITE_INPUT, 0] and r.loss[0].isnan().all() and ((r.loss[1] - math.log(V)).abs() < 1e-5).all()
