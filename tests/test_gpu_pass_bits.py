"""Norm, rotation and what enters the 4-bit cache, bit by bit against the definition in elementary fp32 steps.

include/dsp.h fixes the order of every step (a tree of neighbours for the sum of squares, no product fused with
a sum) and the rounding of scale, offset and code.  Each torch operation below is one such step with one
rounding, so nothing is allowed to differ: not a bit of an output, not a byte of the cache.
"""
import pytest
import torch

import pass_reference as ref
from paper_2510_02358_b200 import binding as dsp

gpu = pytest.mark.gpu
DEV = "cuda"


def _angles(rows, rot):
    f = 1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    a = torch.arange(rows, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


def _norm_rope(x, w, eps, positions, cos_sin, interleaved):
    """One fp32 rounding per line and operation; rounded to x's type at the end."""
    dt, x = x.dtype, x.float()
    if w is not None:
        sq = x * x
        while sq.shape[-1] > 1:
            sq = sq[..., 0::2] + sq[..., 1::2]
        mean = sq * (1.0 / x.shape[-1])
        root = (mean + eps).sqrt()
        x = x * (torch.ones_like(root) / root)
        x = x * w.float()
    if cos_sin is not None:
        rot = cos_sin.shape[1]
        c, s = cos_sin[positions.long()][:, None].split(rot // 2, -1)
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
        ac, bs, bc, as_ = a * c, b * s, b * c, a * s
        first, second = ac - bs, bc + as_
        y = torch.stack([first, second], -1).flatten(-2) if interleaved else torch.cat([first, second], -1)
        x = torch.cat([y, x[..., rot:]], -1)
    return x.to(dt)


def _kept(x):
    """Codes, scale and offset of every head of x [T, H, D] (finite numbers)."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    bits = lo.view(torch.int32)
    z = torch.where(bits < 0, (bits + 0xFFFF) & -65536, bits & -65536).view(torch.float32)
    step = (hi - z) / torch.full_like(z, 15.0)
    s = ((step.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    quotient = (x - z) / torch.where(s > 0, s, torch.ones_like(s))
    code = torch.where(s > 0, quotient.round().clamp(max=15.0), torch.zeros_like(x))
    return code.int(), s, z


def _cache_of(keys, values, slot, n_blocks, page):
    """The cache, byte by byte, that holds these heads at these slots and zeros elsewhere."""
    T, H, D = keys.shape
    size = 16 * (D + 8)
    run = (slot // page * H)[:, None] + torch.arange(H, device=DEV)                 # page of the head ...
    run = run * (page // 16) + (slot % page // 16)[:, None]                         # ... and the run in it
    cache = torch.zeros(n_blocks * H * (page // 16) * size, dtype=torch.int32, device=DEV)
    for x, byte_of, off in ((keys, ref.key_byte, 0), (values, ref.value_byte, 4)):
        code, s, z = _kept(x)
        place = torch.tensor([[byte_of(t, ch, D) for ch in range(D)] for t in range(16)], device=DEV)[slot % 16]
        at = run[..., None] * size + place[:, None, :, 0]
        cache.index_add_(0, at.flatten(), (code << place[:, None, :, 1]).int().flatten())
        num = torch.cat([s, z], -1).to(torch.bfloat16).view(torch.uint8).int()       # four bytes
        at = run[..., None] * size + 16 * D + 8 * (slot % 16)[:, None, None] + off + torch.arange(4, device=DEV)
        cache.index_add_(0, at.flatten(), num.flatten())
    return cache.to(torch.uint8).view(n_blocks, H, -1)


FORMS = [(64, 64, False), (64, 32, False), (64, 48, False), (64, 64, True), (64, 16, True), (64, 0, False),
         (128, 128, False), (128, 64, False), (128, 96, False), (128, 128, True), (128, 32, True), (128, 0, False),
         (256, 256, False), (256, 128, False), (256, 48, False), (256, 256, True)]


@gpu
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("D,rot,inter", FORMS)
@pytest.mark.parametrize("T", [30, 1200, 8000])
def test_every_bit_is_that_of_the_elementary_steps(T, D, rot, inter, bf16):
    """Short calls take a head at a time, long ones several, the longest two launches; all forms of the rotation."""
    dt = torch.bfloat16 if bf16 else torch.float32
    Hq, Hkv, page = 23, 5, 32
    g = torch.Generator(device=DEV).manual_seed(T + D + rot)
    x = torch.randn(T, Hq + 2 * Hkv, D, generator=g, device=DEV)
    x[:, Hq:, 3] *= 9.0                                                             # a strong channel
    q, k, v = x.to(dt).split([Hq, Hkv, Hkv], 1)
    wq, wk = ((1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) for _ in range(2))
    pos = torch.randint(0, 9000, (T,), generator=g, device=DEV, dtype=torch.int32)
    cs = _angles(9000, rot) if rot else None
    rope = dict(q_weight=wq, k_weight=wk, eps=1e-5, positions=pos, cos_sin=cs, interleaved=inter)
    want_q, want_k = _norm_rope(q, wq, 1e-5, pos, cs, inter), _norm_rope(k, wk, 1e-5, pos, cs, inter)
    got_q, got_k = dsp.dsp_qk_norm_rope(q, k, **rope)
    assert torch.equal(got_q, want_q) and torch.equal(got_k, want_k)
    got_q, got_k = dsp.dsp_qk_norm_rope(q, k, **dict(rope, q_weight=None))           # rotation alone
    assert torch.equal(got_q, _norm_rope(q, None, 0.0, pos, cs, inter)) and torch.equal(got_k, want_k)
    if D == 256:
        return
    n = -(-T // page) + 2
    slot = torch.randperm(n * page, generator=g, device=DEV)[:T]
    cache = dsp.kv4_cache(n, Hkv, D, page, DEV)
    assert torch.equal(dsp.dsp_kv4_append(q, k, v, slot, cache, **rope), want_q)
    assert torch.equal(cache, _cache_of(want_k, v, slot, n, page))


@gpu
@pytest.mark.parametrize("D,rot,inter,bf16", [(128, 128, False, True), (64, 64, False, True), (128, 128, True, True), (128, 64, False, True),
                                              (128, 0, False, False), (64, 32, False, False)])
def test_a_million_keys_enter_the_cache_as_the_definition_says(D, rot, inter, bf16):
    """A last bit that differs shows in a code of one head in some thousands only."""
    T, Hkv, page = 1 << 17, 8, 64
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator(device=DEV).manual_seed(D + rot)
    k, v = torch.randn(T, 2 * Hkv, D, generator=g, device=DEV).to(dt).split(Hkv, 1)
    w = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) % 16384
    cs = _angles(16384, rot) if rot else None
    part = T // 8
    slot = torch.cat([torch.randperm(part, generator=g, device=DEV) + lo for lo in range(0, T, part)])
    cache = dsp.kv4_cache(T // page, Hkv, D, page, DEV)
    dsp.dsp_kv4_append(None, k, v, slot, cache, k_weight=w, positions=pos, cos_sin=cs, interleaved=inter)
    for lo in range(0, T, part):                                                     # in parts: the steps take a lot of memory
        s = slice(lo, lo + part)
        want = _cache_of(_norm_rope(k[s], w, 1e-6, pos[s], cs, inter), v[s], slot[s] - lo, part // page, page)
        assert torch.equal(cache[lo // page:(lo + part) // page], want)
