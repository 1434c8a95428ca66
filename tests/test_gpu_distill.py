"""dsp_distill and dsp_distill_grad against the definition in 64 bits, and the gradient against differences."""
import math

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def problem(B, L, V, K, dtype, T=1.0, tail=True, seed=0, masked=0.0, offset=0, pitch=0):
    """(student logits, teacher's ids, logits, log-sum-exp or None): the student lies near the teacher."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = 2.0 * torch.randn(B, L, V, generator=g, device="cuda")
    t.scatter_add_(2, torch.randint(0, V, (B, L, 3), generator=g, device="cuda"), 4 + 3 * torch.rand(B, L, 3, generator=g, device="cuda"))
    n = min(K, V)
    top = t.topk(n, -1)
    ids = torch.full((B, L, K), -1, dtype=torch.int32, device="cuda")
    val = torch.zeros(B, L, K, device="cuda")
    ids[..., :n], val[..., :n] = top.indices.int(), top.values
    lse = (t.double() / T).logsumexp(-1).float() if tail else None
    x = t + torch.randn(B, L, V, generator=g, device="cuda")
    if masked:
        x.masked_fill_(torch.rand(B, L, V, generator=g, device="cuda") < masked, -math.inf)
        x[..., 0] = 0.5
    buf = torch.empty(B * L * (V + pitch) + offset, dtype=dtype, device="cuda")
    out = buf[offset:].view(B, L, V + pitch)[..., :V]
    out.copy_(x)
    return out, ids, val, lse


def near(got, want, tol, what):
    got, want = got.double(), want.double()
    ok = (got == want) | ((got - want).abs() <= tol)
    assert ok.all(), (what, (got - want).abs()[~ok].max().item(), int((~ok).sum()))


def bounds(x, T, V):
    """Relative error of a row's sum, and of one exponential of it."""
    rel = ref.exponent_error(x, T, ref.terms(V))
    big = x.double().abs().masked_fill(torch.isinf(x), 0.0).amax(-1) / ref.LN2 / T
    return rel, 2.0 ** -24 * (ref.LN2 * 4 * big + 8)


def check(x, ids, val, T, lse=None, count=None, weight=None, grad=True, two=False, run=True):
    B, L, V = x.shape
    loss, accept, full, g = ref.distill(x, ids, val, T, lse, count, weight)
    rel, one = bounds(x, T, V)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    if two:
        r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, teacher_count=count, temperature=T, row_status=status)
        got = dsp.dsp_distill_grad(x, ids, r.state, weight if weight is not None else torch.ones(B, L, device="cuda"), temperature=T)
        if weight is not None:
            loss, accept, full, _ = ref.distill(x, ids, val, T, lse, count)
    else:
        r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, teacher_count=count, weight=weight, temperature=T, grad=grad, row_status=status)
        got = r.grad
    assert not status.any()
    small = 2.0 ** -24
    near(r.lse, full, rel + small * full.abs().masked_fill(full == -math.inf, 0.0), "lse")
    # loss: P lse and r log s, each off by rel, and the list's values rounded to 32 bits
    fin = torch.isfinite(loss)
    near(r.loss, loss, torch.where(fin, 3 * rel + small * (loss.abs() + 2), torch.zeros_like(loss)), "loss")
    near(r.accept, accept, 2 * rel + 4 * small, "accept")
    if got is None:
        return r
    # gradient: q_v and r q_v / s each off by their sum's and their own exponential's error; one rounding to the type
    w = torch.ones_like(rel) if weight is None else weight.double().abs()
    p, use, rest = ref.teacher(val, T, ids, V, lse, count)
    at = ids.long().clamp(0, V - 1)
    logq = torch.log_softmax(x.double() / T, -1)
    inside = torch.zeros_like(logq).scatter_add_(-1, at, use.double()) > 0
    others = logq.masked_fill(inside, -math.inf)
    log_s = torch.logsumexp(others, -1, keepdim=True)
    share = torch.where(log_s > -math.inf, (others - log_s).exp(), torch.zeros_like(logq))
    size = (logq.exp() + rest[..., None] * share).scatter_add(-1, at, torch.where(use, p, torch.zeros_like(p)))
    tol = (2 * rel + one + 4 * small)[..., None] * size * (w / T)[..., None] + torch.finfo(x.dtype).eps / 2 * g.abs() * 1.001 + 1e-37
    if x.dtype == BF:
        tol = tol * (1 + 2.0 ** -8)
    near(got, g, tol, "gradient")
    return r


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,K", [(1, 1), (5, 3), (9, 9), (16, 4), (17, 2), (1000, 8), (20480, 64), (20481, 1), (32003, 33), (152064, 32), (152064, 256),
                                 (262147, 100)])
def test_sizes(V, K, tail, dtype):
    x, ids, val, lse = problem(2, 3, V, K, dtype, tail=tail, seed=V)
    check(x, ids, val, 1.0, lse)
    check(x, ids, val, 1.0, lse, two=True)


@pytest.mark.parametrize("dtype,V", [(BF, 1000003), (F32, 500009)])
def test_rows_beyond_a_cluster(dtype, V):
    x, ids, val, lse = problem(1, 2, V, 16, dtype, seed=3)
    w = torch.tensor([[0.5, 2.0]], device="cuda")
    check(x, ids, val, 1.0, lse, weight=w)
    check(x, ids, val, 1.0, lse, grad=None)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,K,offset", [(64, 5, 0), (65, 33, 3), (100, 100, 1), (6150, 32, 0), (12303, 256, 5), (32003, 1, 0), (75000, 40, 0), (80003, 256, 3)])
def test_many_rows(V, K, offset, tail, dtype):
    """More rows than CTAs fit: the loss streams its rows, the gradient has clusters in turn; unread rows, repeats, gaps and masks among them."""
    B, L = (13, 37) if V < 70000 else (10, 16)
    x, ids, val, lse = problem(B, L, V, K, dtype, 1.5, tail, seed=V + K, masked=0.2, offset=offset, pitch=offset)
    if K > 4:
        ids[2, :, 3], ids[3, 5, :4], ids[4, 6] = ids[2, :, 1], -1, V
        ids[5, 1, :3] = torch.tensor([0, V - 1, 1], dtype=torch.int32, device="cuda")          # outside of whole pieces, or next to them
    w = torch.rand(B, L, device="cuda") - 0.2
    w[0, 3], w[7] = 0.0, 0.0
    check(x, ids, val, 1.5, lse, weight=w)
    check(x, ids, val, 1.5, lse, weight=w, two=True)
    check(x, ids, val, 1.5, lse, weight=w, grad=None)


@pytest.mark.parametrize("T", [0.5, 2.0])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("two", [False, True])
def test_temperatures_weights_and_skipped_rows(T, dtype, two):
    x, ids, val, lse = problem(5, 7, 8005, 20, dtype, T, seed=4)
    w = torch.rand(5, 7, device="cuda") - 0.3
    w[1], w[2, 3] = 0.0, 0.0
    check(x, ids, val, T, lse, weight=w, two=two)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("offset", range(9))
def test_rows_that_start_anywhere(dtype, offset):
    x, ids, val, lse = problem(2, 3, 4099, 12, dtype, seed=offset, offset=offset, pitch=offset % 4)
    r = check(x, ids, val, 1.0, lse)
    buf = torch.full((2 * 3 * 4105 + 16,), 7.0, dtype=dtype, device="cuda")    # the gradient at another start and pitch
    g = buf[3:3 + 6 * 4105].view(2, 3, 4105)[..., :4099]
    dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=g)
    assert torch.equal(g, r.grad)
    outside = buf.clone()
    outside[3:3 + 6 * 4105].view(2, 3, 4105)[..., :4099] = 7.0
    assert (outside == 7.0).all()
    g.fill_(7.0)
    state = dsp.dsp_distill(x, ids, val, teacher_lse=lse).state
    one = torch.ones(2, 3, device="cuda")
    dsp.dsp_distill_grad(x, ids, state, one, grad=g)
    assert torch.equal(g, dsp.dsp_distill_grad(x, ids, state, one))
    outside = buf.clone()
    outside[3:3 + 6 * 4105].view(2, 3, 4105)[..., :4099] = 7.0
    assert (outside == 7.0).all()
    one.zero_()
    dsp.dsp_distill_grad(x, ids, state, one, grad=g)
    assert not g.any() and (outside == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_lists_with_gaps_repeats_and_counts(dtype):
    x, ids, val, lse = problem(4, 4, 3001, 40, dtype, seed=6)
    count = torch.randint(0, 45, (4, 4), dtype=torch.int32, device="cuda")
    count[0, 0], count[0, 1], count[0, 2] = 0, -3, 40
    ids[1, 1, 5], ids[1, 2, 7], ids[1, 3] = -1, 3001, ids[1, 3, :1]
    ids[2, 0, 9], ids[2, 0, 33] = ids[2, 0, 2], ids[2, 0, 2]
    val[3, 0], val[3, 1, 3:] = -math.inf, -math.inf
    for tail in (lse, None):
        for c in (None, count):
            check(x, ids, val, 1.0, tail, c)
            check(x, ids, val, 1.0, tail, c, two=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_masked_logits_of_the_student(dtype):
    x, ids, val, lse = problem(2, 4, 5000, 16, dtype, seed=7, masked=0.5)
    x[0, 0] = -math.inf
    x[0, 0, 7] = 1.0                                                # one token holds everything
    x[0, 1].scatter_(0, ids[0, 1].long(), -math.inf)                # all of the teacher's are masked: loss is infinite
    for tail in (lse, None):
        r = check(x, ids, val, 1.0, tail)
        assert torch.isfinite(r.grad).all() and r.loss[0, 1] == math.inf


@pytest.mark.parametrize("dtype", [BF, F32])
def test_mass_far_apart(dtype):
    """The teacher's tokens 300 above all others, or below: s and r / s at the ends of the number range."""
    x, ids, val, lse = problem(1, 4, 6000, 8, dtype, seed=8)
    x[0, 0].scatter_add_(0, ids[0, 0].long(), torch.full((8,), 300.0, dtype=dtype, device="cuda"))
    x[0, 1].scatter_add_(0, ids[0, 1].long(), torch.full((8,), -300.0, dtype=dtype, device="cuda"))
    lse[0, 2] = val[0, 2].double().logsumexp(-1).float() - 0.01     # more than all of the mass in the list
    check(x, ids, val, 1.0, lse)
    check(x, ids, val, 1.0, lse, two=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_gradient_may_take_the_logits_place(dtype):
    for V in (30011, 32000, 1000003 if dtype == BF else 500009):
        x, ids, val, lse = problem(2, 2, V, 8, dtype, seed=9)
        w = torch.tensor([[1.0, 0.0], [-2.0, 0.25]], device="cuda")
        want = dsp.dsp_distill(x, ids, val, teacher_lse=lse, weight=w, grad=True)
        state = dsp.dsp_distill(x, ids, val, teacher_lse=lse).state
        want2 = dsp.dsp_distill_grad(x, ids, state, w)
        y = x.clone()
        got = dsp.dsp_distill(y, ids, val, teacher_lse=lse, weight=w, grad=y)
        assert torch.equal(y, want.grad) and torch.equal(got.loss, want.loss)
        y = x.clone()
        assert dsp.dsp_distill_grad(y, ids, state, w, grad=y) is y and torch.equal(y, want2)


def test_bad_rows_are_named_and_alone():
    x, ids, val, lse = problem(4, 2, 40000, 8, F32, seed=10)
    w = torch.ones(4, 2, device="cuda")
    w[3, 0] = 0.0
    want = dsp.dsp_distill(x, ids, val, teacher_lse=lse, weight=w, grad=True)
    x[0, 1, 5], x[1, 0, 39999], x[3, 0, 0] = math.nan, math.inf, math.nan     # the last one is in a row that is not read
    val[2, 1, 3] = math.nan
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    got = dsp.dsp_distill(x, ids, val, teacher_lse=lse, weight=w, grad=True, row_status=status)
    assert status.tolist() == [1, 1, 1, 0]
    bad = torch.tensor([[0, 1], [1, 0], [0, 1], [0, 0]], dtype=torch.bool, device="cuda")
    assert got.loss[bad].isnan().all()
    for name in ("loss", "accept", "lse", "grad"):
        assert torch.equal(getattr(got, name)[~bad], getattr(want, name)[~bad]), name


@pytest.mark.parametrize("tail", [True, False])
def test_the_gradient_against_differences(tail):
    """Central differences of the loss in 64 bits at the kernel's gradient: (f(x+h) - f(x-h)) / 2h is off by h^2 |f'''| / 6 < h^2."""
    x, ids, val, lse = problem(1, 2, 37, 5, F32, seed=11, tail=tail)
    g = dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=True).grad
    rel, one = bounds(x, 1.0, 37)
    h = 1e-4
    for v in range(37):
        d = torch.zeros_like(x, dtype=torch.float64)
        d[..., v] = h
        up, down = (ref.distill(x.double() + s * d, ids, val, 1.0, lse)[0] for s in (1, -1))
        assert ((g[..., v].double() - (up - down) / (2 * h)).abs() <= 2 * (2 * rel + one) + h * h + 1e-11).all()


def test_calls_give_the_same_bits():
    x, ids, val, lse = problem(3, 5, 152064, 32, BF, seed=12)
    a, b = (dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=True, state=True) for _ in range(2))
    for name in vars(a):
        assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), name
    alone = dsp.dsp_distill(x[1:2], ids[1:2], val[1:2], teacher_lse=lse[1:2])
    assert alone.loss.shape == (1, 5) and dsp.dsp_distill(x[:0], ids[:0], val[:0], grad=True).loss.shape == (0, 5)


def test_an_autograd_function_over_the_two_calls():
    """The two-call form inside torch's graph: the drafter's head takes the gradient that the formula gives."""
    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, ids, val, lse):
            r = dsp.dsp_distill(logits, ids, val, teacher_lse=lse)
            ctx.save_for_backward(logits, ids, r.state)
            return r.loss

        @staticmethod
        def backward(ctx, up):
            logits, ids, state = ctx.saved_tensors
            return dsp.dsp_distill_grad(logits, ids, state, up.contiguous()), None, None, None

    x, ids, val, lse = problem(2, 3, 2000, 8, F32, seed=13)
    leaf = x.detach().clone().requires_grad_()
    up = torch.rand(2, 3, device="cuda")
    (Distill.apply(leaf, ids, val, lse) * up).sum().backward()
    want = dsp.dsp_distill(x, ids, val, teacher_lse=lse, weight=up, grad=True).grad
    # each is within (2 rel + one + 4 half steps) of q + p (and of r times the others' share, below q + p here): twice that apart
    rel, one = bounds(x, 1.0, 2000)
    assert ((leaf.grad - want).abs().double() <= 2 * (2 * rel + one + 2.0 ** -22)[..., None] * up.double()[..., None]).all()


@pytest.mark.parametrize("B,L,V,dtype,grad", [(3, 20, 32003, F32, True), (3, 20, 32003, BF, False), (1, 16, 152064, BF, True), (4, 64, 80000, BF, False)])
def test_small_losses_are_exact(B, L, V, dtype, grad):
    """A drafter next to its teacher: dloss = (s - r) dS / S for an error dS of the other tokens' sum, the list's own part is formed in 64 bits,
    and the result is rounded to 32."""
    g = torch.Generator(device="cuda").manual_seed(V)
    t = 2.0 * torch.randn(B, L, V, generator=g, device="cuda")
    t.scatter_add_(2, torch.randint(0, V, (B, L, 3), generator=g, device="cuda"), 6 + 3 * torch.rand(B, L, 3, generator=g, device="cuda"))
    top = t.topk(8, -1)
    ids, val, lse = top.indices.int(), top.values, t.double().logsumexp(-1).float()
    x = (t + 0.1 * torch.randn(B, L, V, generator=g, device="cuda")).to(dtype)
    want = ref.distill(x, ids, val, 1.0, lse)[0]
    r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=grad)
    _, use, rest = ref.teacher(val, 1.0, ids, V, lse)
    q = torch.log_softmax(x.double(), -1).gather(-1, ids.long()).exp().sum(-1)
    near(r.loss, want, (1 - q - rest).abs() * bounds(x, 1.0, V)[0] + 2.0 ** -24 * want.abs() + 1e-12, "loss")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,L,V", [(2, 3, 33000), (1, 200, 80000)])
def test_masks_of_the_lowest_number(B, L, V, dtype):
    """Logits of the type's lowest value: no mass and no gradient among the others; in the list a loss that is next to infinite, not NaN."""
    x, ids, val, lse = problem(B, L, V, 8, dtype, seed=12)
    low = torch.finfo(dtype).min
    x.masked_fill_(torch.rand(B, L, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < 0.5, low)
    x.scatter_(-1, ids.long(), torch.ones(B, L, 8, dtype=dtype, device="cuda"))
    masked = x == low
    x0 = x.masked_fill(masked, -math.inf)
    for grad in (True, False):
        a = dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=grad)
        b = dsp.dsp_distill(x0, ids, val, teacher_lse=lse, grad=grad)
        assert torch.equal(a.loss, b.loss) and torch.equal(a.accept, b.accept) and torch.equal(a.lse, b.lse)
        ga, gb = (a.grad, b.grad) if grad else [dsp.dsp_distill_grad(t, ids, r.state, torch.ones(B, L, device="cuda")) for t, r in ((x, a), (x0, b))]
        assert torch.equal(ga, gb) and not ga[masked].any() and torch.isfinite(ga).all()
    x.scatter_(-1, ids[..., :1].long(), torch.full((B, L, 1), low, dtype=dtype, device="cuda"))
    r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=True)
    assert (r.loss > 1e30).all() and torch.isfinite(r.grad).all() and not r.accept.isnan().any()


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("grad", [True, False])
def test_a_bad_log_sum_exp_of_the_teacher_is_named(value, grad):
    for B, L, V, dtype in ((3, 1, 5000, F32), (3, 60, 80000, BF)):
        x, ids, val, lse = problem(B, L, V, 4, dtype, seed=2)
        lse[1, L - 1] = value
        status = torch.zeros(B, dtype=torch.int32, device="cuda")
        dsp.dsp_distill(x, ids, val, teacher_lse=lse, grad=grad, row_status=status)
        assert status.tolist() == [0, dsp.ROW_NONFINITE_INPUT, 0]


@pytest.mark.parametrize("grad", [True, False])
def test_rows_beyond_32_bits(grad):
    """Logits of more than 2^31 elements: the last rows, in place."""
    V, L = 160001, 14000
    x = torch.empty(1, L, V, dtype=BF, device="cuda")
    small, ids_s, val_s, lse_s = problem(1, 3, V, 4, BF, seed=4)
    x[:, -3:] = small
    ids, val, lse, w = (torch.zeros(1, L, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, L, 4, device="cuda"), torch.zeros(1, L, device="cuda"),
                        torch.zeros(1, L, device="cuda"))
    ids[:, -3:], val[:, -3:], lse[:, -3:], w[:, -3:] = ids_s, val_s, lse_s, 1.0
    r = dsp.dsp_distill(x, ids, val, teacher_lse=lse, weight=w, grad=x if grad else None)
    got = x[:, -3:] if grad else dsp.dsp_distill_grad(x, ids, r.state, w, grad=x)[:, -3:]
    want = dsp.dsp_distill(small.clone(), ids_s, val_s, teacher_lse=lse_s, grad=True)
    near(r.loss[:, -3:], want.loss, 1e-5, "loss")
    near(got, want.grad.double(), 2.0 ** -8 * want.grad.double().abs() + 1e-9, "gradient")     # a last bit may differ between the forms
    assert not r.loss[:, :-3].any() and not x[0, 0].any() and not x[0, L - 4].any()
