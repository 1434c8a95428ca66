"""The model pass's operators on the GPU against their plain 64-bit definitions (tests/pass_reference.py).

Tolerances.  Integers, codes, and whatever is copied: equal.  Norm and rotation: a few fp32 roundings
(16 of 2^-24 of the row's largest value), and in bf16 the rounding of a number that near.  Attention: its
four bf16 roundings (keys, values, weights, output) are independent and 1.7e-3 of a value each in the
mean, so scores of unit spread give a relative error of 3.3e-3 over a case's outputs in the 2-norm; 5e-3
is allowed, and 2% of the largest value for a single output.
"""
import ctypes as C
import os
import re
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import pass_reference as ref
from paper_2510_02358_b200 import binding as dsp

gpu = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------- plan
def _plan_case(seed, B, width, page, max_new, tree=None, tight=False):
    r = np.random.default_rng(seed)
    N = 0 if tree is None else tree[0] * tree[1]
    cap = width * page
    seq = r.integers(0, max(1, cap - max_new), B)
    new = r.integers(0, (N + 2) if N else max_new + 1, B)
    count = np.clip(-(-(seq + r.integers(-page, max_new + 1, B)) // page), 0, width)
    free = int(r.integers(0, 3)) if tight else int(np.maximum(-(-(seq + new) // page) - count, 0).sum()) + 3
    n = int(count.sum()) + free
    ids = r.permutation(n)
    table = r.integers(0, n, (B, width))
    at = 0
    for b in range(B):
        table[b, :count[b]] = ids[at:at + count[b]]
        at += count[b]
    head = int(r.integers(0, 3 * n))
    ring = r.integers(0, n, n)
    for i in range(free):
        ring[(head + i) % n] = ids[at + i]
    parent = depth = None
    if N:
        parent = np.stack([[int(r.integers(-1, i)) if i else -1 for i in range(N)] for _ in range(B)])
        depth = r.integers(0, 9, (B, N))
    return seq, new, count, head, head + free, table, ring, parent, depth


def _check_plan(c, page, T, words=0, repeat=True):
    seq, new, count, head, tail, table, ring, parent, depth = c
    want = ref.plan(seq.tolist(), new.tolist(), count.tolist(), head, tail, table.tolist(), ring.tolist(), page, T,
                    None if parent is None else parent.tolist(), None if depth is None else depth.tolist(), words)
    t, rg = i32(table), i32(ring)
    args = (i32(seq), i32(new), i32(count), torch.tensor([head, tail], device=DEV), t, rg, page, T)
    kw = {} if parent is None else dict(node_parent=i32(parent), node_depth=i32(depth), mask_words=words)
    for _ in range(2 if repeat else 1):                      # a repeated call writes the same
        got = dsp.dsp_cache_plan(*args, **kw)
        torch.cuda.synchronize()
        for name in ("row_status", "block_count", "ring_pos", "cu_new", "kv_len", "slot", "position", "token_row"):
            assert getattr(got, name).tolist() == want[name], name
        if parent is not None:
            assert (got.mask.cpu().numpy().view(np.uint32) == np.array(want["mask"], dtype=np.uint32).reshape(T, words)).all()
        for b in range(len(seq)):
            assert t[b, :want["block_count"][b]].tolist() == want["block_table"][b][:want["block_count"][b]]
        n = len(ring)
        live = [(i % n) for i in range(want["ring_pos"][0], want["ring_pos"][1])]
        assert rg.cpu().numpy()[live].tolist() == [want["free_ring"][i] for i in live]


@gpu
@pytest.mark.parametrize("seed,B,width,page,max_new", [
    (0, 1, 1, 1, 1), (1, 1, 40, 16, 500), (2, 7, 9, 16, 33), (3, 33, 5, 64, 64), (4, 256, 6, 16, 17), (5, 257, 30, 32, 5),
    (6, 1024, 4, 128, 128), (7, 1500, 7, 16, 40), (8, 8192, 3, 16, 3), (9, 5, 6, 7, 20)])
def test_plan_matches_the_definition(seed, B, width, page, max_new):
    c = _plan_case(seed, B, width, page, max_new)
    _check_plan(c, page, int(c[1].sum()) + 3)


@gpu
@pytest.mark.parametrize("seed", range(6))
def test_plan_with_too_few_blocks_or_token_rows(seed):
    c = _plan_case(100 + seed, 40, 6, 16, 30, tight=True)
    _check_plan(c, 16, max(0, int(c[1].sum()) - 50 * (seed % 3)))


@gpu
@pytest.mark.parametrize("seed,B,W,L,page", [(0, 1, 1, 1, 16), (1, 3, 4, 8, 16), (2, 17, 8, 16, 64), (3, 2, 32, 31, 32), (4, 200, 2, 16, 16)])
def test_plan_of_a_tree(seed, B, W, L, page):
    c = _plan_case(200 + seed, B, 70, page, W * L + 1, tree=(W, L))
    _check_plan(c, page, int(c[1].sum()) + 2, words=(W * L + 32) // 32 + seed % 2)


@gpu
def test_plan_reports_bad_rows_and_serves_the_others():
    c = list(_plan_case(300, 8, 6, 16, 30))
    c[0][1], c[1][2], c[2][3], c[2][4] = -1, -5, -1, 7            # negative lengths, counts outside the table
    c[0][5], c[1][5] = 2 ** 31 - 1, 5
    c[1][6] = 6 * 16 + 1                                          # more than the table holds
    _check_plan(c, 16, 500)


@gpu
def test_plan_masks_are_those_of_the_beam_tree():
    beams = i32([[[5, 6, 7, 8], [5, 6, 9, 9], [4, 6, 7, 8]]])
    tree = dsp.dsp_beam_tree(SimpleNamespace(beam_ids=beams, path_len=i32([4])))
    n = int(tree.n_nodes)
    got = dsp.dsp_cache_plan(i32([10]), i32([1 + n]), i32([1]), torch.tensor([0, 4], device=DEV), i32([[3, 0, 0]]),
                             i32([0, 1, 2, 4]), 16, 1 + n, node_parent=tree.node_parent, node_depth=tree.node_depth)
    path = [[0], [0, 1], [0, 1, 2], [0, 1, 2, 3], [0, 1, 2, 3, 4], [0, 1, 2, 5], [0, 1, 2, 5, 6]]
    path += [[0, 7], [0, 7, 8], [0, 7, 8, 9], [0, 7, 8, 9, 10]]
    assert got.mask[:, 0].tolist() == [sum(1 << j for j in p) for p in path]
    assert got.position.tolist() == [10 + len(p) - 1 for p in path]


# ------------------------------------------------------------------------------ norm, rotation, cache
def _angles(rows, rot):
    f = 1e4 ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(rows)[:, None] * f
    return torch.tensor(np.concatenate([np.cos(a), np.sin(a)], 1), dtype=torch.float32, device=DEV)


def _norm_close(got, want, bf16):
    got = ref.to_numpy(got)
    assert (np.isnan(got) == np.isnan(want)).all()
    top = np.nanmax(np.abs(np.where(np.isnan(want), 0, want)), -1, keepdims=True)
    tol = 16 * 2.0 ** -24 * top + 1e-37
    if bf16:                                   # the rounding of some number within the fp32 error of the definition
        r = lambda x: torch.tensor(x).to(torch.bfloat16).double().numpy()      # noqa: E731
        assert (np.isnan(want) | ((r(want - tol) <= got) & (got <= r(want + tol)))).all()
    else:
        assert (np.isnan(want) | (np.abs(got - want) <= tol)).all()


NORM = [(T, Hq, Hkv, D, rot, inter, bf16) for T, Hq, Hkv, D, rot, inter, bf16 in [
    (1, 1, 1, 64, 64, False, True), (1, 40, 8, 128, 128, False, True), (3, 5, 1, 128, 64, True, False),
    (17, 7, 7, 64, 16, False, False), (130, 28, 4, 128, 128, True, True), (33, 6, 2, 256, 240, False, True),
    (9, 3, 3, 256, 256, False, False), (700, 40, 8, 128, 96, False, True), (2000, 15, 3, 64, 32, True, False)]]


@gpu
@pytest.mark.parametrize("T,Hq,Hkv,D,rot,inter,bf16", NORM)
def test_norm_rope_matches_the_definition(T, Hq, Hkv, D, rot, inter, bf16):
    g = torch.Generator(device=DEV).manual_seed(T)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn((T, Hq + Hkv, D), generator=g, device=DEV).to(dt)
    q, k = x[:, :Hq], x[:, Hq:]                                    # strided views of one projection
    wq, wk = (torch.randn(D, generator=g, device=DEV).to(dt) for _ in range(2))
    pos = torch.randint(0, 50, (T,), generator=g, device=DEV, dtype=torch.int32)
    pos[T // 2] = -1 if T > 2 else 3
    pos[T // 3] = 77 if T > 8 else 2                               # beyond the table
    cs = _angles(50, rot)
    a = (ref.to_numpy(pos).astype(int), ref.to_numpy(cs))
    got = dsp.dsp_qk_norm_rope(q, k, q_weight=wq, k_weight=wk, eps=1e-5, positions=pos, cos_sin=cs, interleaved=inter)
    for y, xi, w in zip(got, (q, k), (wq, wk)):
        _norm_close(y, ref.norm_rope(ref.to_numpy(xi), ref.to_numpy(w), 1e-5, *a, inter), bf16)
    got = dsp.dsp_qk_norm_rope(q, k, k_weight=wk)                  # no rotation, no norm of the queries
    assert torch.equal(got[0], q)
    _norm_close(got[1], ref.norm_rope(ref.to_numpy(k), ref.to_numpy(wk), 1e-6, None, None, False), bf16)


@gpu
@pytest.mark.parametrize("bf16", [True, False])
def test_unaligned_and_strided_rows_give_the_same_bits(bf16):
    dt = torch.bfloat16 if bf16 else torch.float32
    T, Hq, Hkv, D = 11, 6, 2, 128
    g = torch.Generator(device=DEV).manual_seed(3)
    flat = torch.randn(T * 2000 + 7, generator=g, device=DEV).to(dt)
    odd = lambda H, off: torch.as_strided(flat, (T, H, D), (2000 - 1, D + 3, 1), off)      # noqa: E731
    q, k, v = odd(Hq, 1), odd(Hkv, 900), odd(Hkv, 1303)
    w = torch.randn(2 * D + 1, generator=g, device=DEV).to(dt)
    cs = _angles(64, D).flatten()
    cs = torch.cat([cs[:1], cs])[1:].view(64, D)                   # rows that start 4 bytes after a boundary
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    slot = torch.arange(T, device=DEV) + 5
    a = dict(q_weight=w[1:D + 1], k_weight=w[D + 1:], positions=pos, cos_sin=cs)
    b = dict(q_weight=w[1:D + 1].clone(), k_weight=w[D + 1:].clone(), positions=pos, cos_sin=cs.clone())
    caches = [dsp.kv4_cache(2, Hkv, D, 16, DEV) for _ in range(2)]
    one = dsp.dsp_kv4_append(q, k, v, slot, caches[0], **a)
    two = dsp.dsp_kv4_append(q.contiguous(), k.contiguous(), v.contiguous(), slot, caches[1], **b)
    assert torch.equal(one, two) and torch.equal(caches[0], caches[1])


@gpu
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("D,rot,inter", [(64, 64, False), (64, 32, False), (64, 64, True), (64, 0, False), (128, 128, False), (128, 64, False),
                                         (128, 128, True), (128, 48, False), (128, 0, False), (256, 256, False), (256, 128, False), (256, 64, True)])
def test_long_calls_give_the_bits_of_short_ones(D, rot, inter, bf16):
    """However a call's length cuts it, rows, codes and what is read back are those of calls of a few tokens."""
    dt = torch.bfloat16 if bf16 else torch.float32
    T, Hq, Hkv, part = 2500, 23, 5, 50
    g = torch.Generator(device=DEV).manual_seed(D + rot + bf16)
    q, k, v = torch.randn(T, Hq + 2 * Hkv, D, generator=g, device=DEV).to(dt).split([Hq, Hkv, Hkv], 1)
    w = torch.randn(D, generator=g, device=DEV).to(dt)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    rope = dict(q_weight=w, k_weight=w, cos_sin=_angles(T, rot) if rot else None, interleaved=inter)
    norm_q, norm_k = dsp.dsp_qk_norm_rope(q, k, positions=pos, **rope)
    few = [dsp.dsp_qk_norm_rope(q[i:i + part], k[i:i + part], positions=pos[i:i + part], **rope) for i in range(0, T, part)]
    assert torch.equal(norm_q, torch.cat([x for x, _ in few])) and torch.equal(norm_k, torch.cat([y for _, y in few]))
    if D == 256:
        return
    slot = torch.randperm(2560, generator=g, device=DEV)[:T]
    caches = [dsp.kv4_cache(40, Hkv, D, 64, DEV) for _ in range(2)]
    one = dsp.dsp_kv4_append(q, k, v, slot, caches[0], positions=pos, **rope)
    for i in range(0, T, part):
        s = slice(i, i + part)
        assert torch.equal(one[s], dsp.dsp_kv4_append(q[s], k[s], v[s], slot[s], caches[1], positions=pos[s], **rope))
    assert torch.equal(one, norm_q) and torch.equal(caches[0], caches[1])


@gpu
@pytest.mark.parametrize("T,Hq,Hkv,D,page,bf16", [(1, 4, 1, 128, 16, True), (1, 1, 1, 64, 16, False), (37, 10, 2, 64, 48, True),
                                                  (61, 5, 5, 128, 32, False), (900, 28, 4, 128, 64, True), (513, 24, 8, 64, 16, True)])
def test_append_stores_what_the_definition_says(T, Hq, Hkv, D, page, bf16):
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator(device=DEV).manual_seed(T + D)
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device=DEV)
    x[:, Hq:, 3] *= 20.0                                           # a strong channel
    x = x.to(dt)
    q, k, v = x.split([Hq, Hkv, Hkv], 1)
    wq, wk = (1 + torch.randn(D, generator=g, device=DEV).to(dt) / 4 for _ in range(2))
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    cs = _angles(T, D)
    n = -(-T // page) + 3
    slot = torch.randperm(n * page, generator=g, device=DEV)[:T]
    if T > 30:
        slot[2], slot[5], slot[9] = -1, n * page, 2 ** 40
        pos[7] = -1
    rope = dict(q_weight=wq, k_weight=wk, positions=pos, cos_sin=cs)
    cache = torch.randint(0, 255, (n, Hkv, page * (D + 8)), generator=g, device=DEV, dtype=torch.uint8)
    want = cache.cpu().numpy().copy()
    got_q = dsp.dsp_kv4_append(q, k, v, slot, cache, **rope)
    q2, k2 = dsp.dsp_qk_norm_rope(q, k, **rope)
    assert torch.equal(got_q, q2)
    keys, values = k2.float().cpu().numpy(), v.float().cpu().numpy()
    sl, ps = slot.tolist(), pos.tolist()
    for t in range(T):
        if 0 <= sl[t] < n * page and ps[t] >= 0:
            for h in range(Hkv):
                ref.cache_put(want, page, D, sl[t], h, keys[t, h], values[t, h])
    assert (cache.cpu().numpy() == want).all()                     # every byte, those of other tokens included
    # without queries, and read back
    again = cache.clone()
    assert dsp.dsp_kv4_append(None, k, v, slot, again, **rope) is None
    assert torch.equal(cache, again)
    for out_dt in (torch.float32, torch.bfloat16):
        rk, rv = dsp.dsp_kv4_read(cache, slot, D, out_dt)
        for t in list(range(min(T, 20))):
            for h in range(Hkv):
                if not 0 <= sl[t] < n * page:
                    assert not rk[t, h].any() and not rv[t, h].any()
                    continue
                for y, r in zip((rk, rv), ref.cache_get(want, page, D, sl[t], h)):
                    assert torch.equal(y[t, h].cpu(), torch.tensor(r.astype(np.float32)).to(out_dt))


@gpu
def test_heads_that_four_bits_cannot_hold_read_as_nan():
    D = 64
    k = torch.randn((8, 1, D), device=DEV)
    v = torch.randn((8, 1, D), device=DEV)
    k[0, 0, 5], k[1, 0, 63], k[2, 0, 0], v[3, 0, 7] = float("nan"), float("inf"), -float("inf"), float("nan")
    k[4, 0, 0], k[4, 0, 1] = 3.4e38, -3.4e38                      # the range itself overflows
    k[5] = 0.0
    k[6] = float("inf")
    k[7] = 1e-40                                                   # below the smallest normal scale
    cache = dsp.kv4_cache(1, 1, D, 16, DEV)
    slot = torch.arange(8, device=DEV)
    dsp.dsp_kv4_append(None, k, v, slot, cache)
    rk, rv = dsp.dsp_kv4_read(cache, slot, D, torch.float32)
    assert rk.isnan().all(-1).squeeze(1).tolist() == [True, True, True, False, True, False, True, False]
    assert rk.isnan().any(-1).squeeze(1).tolist() == rk.isnan().all(-1).squeeze(1).tolist()
    assert rv.isnan().all(-1).squeeze(1).tolist() == [i == 3 for i in range(8)]
    assert not rk[5].any() and (rk[7].abs() <= 1e-40).all()


# -------------------------------------------------------------------------------------- attention
def _cache_of(r, n_blocks, Hkv, D, page):
    """Random codes with scales and offsets that give values of about unit spread."""
    cache = r.integers(0, 256, (n_blocks, Hkv, page // 16, 16 * (D + 8)), dtype=np.uint8)
    s = r.uniform(0.15, 0.3, (n_blocks, Hkv, page // 16, 16, 2))
    z = -7.5 * s + r.normal(size=s.shape) * 0.2
    num = np.stack([s, z], -1).reshape(*s.shape[:-1], 4).astype(np.float32)
    bits = (np.ascontiguousarray(num).view(np.uint32) >> 16).astype(np.uint16)
    cache[..., 16 * D:] = np.ascontiguousarray(bits).view(np.uint8).reshape(*cache.shape[:3], 128)
    return cache.reshape(n_blocks, Hkv, page * (D + 8))


def _attn_case(seed, new, kv, Hq, Hkv, D, page, spread=1.0):
    r = np.random.default_rng(seed)
    B, width = len(new), max(1, max(-(-n // page) for n in kv)) + 1
    n_blocks = B * width + 2
    table = r.permutation(n_blocks)[:B * width].reshape(B, width).astype(np.int32)
    cache = _cache_of(r, n_blocks, Hkv, D, page)
    T = sum(new)
    q = torch.tensor(r.normal(size=(T, Hq, D)) * spread, dtype=torch.bfloat16)
    return r, q, cache, table, np.cumsum([0] + list(new)).tolist()


def _attend(q, cache, table, kv, cu, max_new, mask, **kw):
    return dsp.dsp_attn_kv4(q.to(DEV), torch.tensor(cache, device=DEV), i32(table), i32(kv), i32(cu), max_new, mask=mask, **kw)


def _attn_close(got, want):
    got = ref.to_numpy(got)
    assert (np.isnan(got) == np.isnan(want)).all()
    ok = ~np.isnan(want)
    if not ok.any():
        return
    d = np.where(ok, got - np.where(ok, want, 0), 0)
    w = np.where(ok, want, 0)
    assert np.linalg.norm(d) <= 5e-3 * np.linalg.norm(w) + 1e-30, np.linalg.norm(d) / np.linalg.norm(w)
    assert np.abs(d).max() <= 0.02 * max(4.0, np.abs(w).max())


ATTN = [
    # single tokens: every small length, an empty cache among them
    ([1] * 12, [0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 255, 700], 5, 1, 128, 16, "causal"),
    ([1] * 6, [1, 5, 130, 64, 65, 1000], 8, 8, 64, 32, "causal"),
    ([1], [5000], 40, 8, 128, 64, "causal"),
    ([1, 1, 1], [3000, 17, 2049], 7, 1, 64, 128, "causal"),
    ([1, 1], [333, 4000], 16, 1, 128, 48, "causal"),
    # chains of drafted tokens, requests without new tokens, a block as long as its cache
    ([3, 0, 17, 9, 1], [3, 50, 400, 9, 77], 40, 8, 128, 16, "causal"),
    ([2, 4, 2], [900, 901, 902], 4, 1, 128, 64, "causal"),
    ([33, 31], [33, 1500], 14, 2, 64, 16, "causal"),
    ([5, 4], [3, 0], 6, 2, 128, 16, "causal"),                     # more new tokens than the cache holds
    # prompts
    ([300], [300], 10, 2, 128, 64, "causal"),
    ([129, 260], [513, 800], 4, 4, 64, 32, "causal"),
    ([200], [1337], 8, 1, 128, 128, "causal"),
    # the drafter's block
    ([32, 7, 1], [200, 7, 1], 16, 16, 64, 32, "full"),
    ([16, 16, 64], [1000, 16, 640], 28, 4, 128, 64, "full"),
    # trees
    ([9, 17, 1], [100, 17, 1], 5, 1, 128, 16, "tree"),
    ([65, 40], [700, 1024], 16, 2, 128, 64, "tree"),
    ([130, 3], [400, 3], 6, 3, 64, 16, "tree"),
]


@gpu
@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,mask", ATTN)
@pytest.mark.parametrize("spread", [1.0, 6.0])
def test_attention_matches_the_definition(new, kv, Hq, Hkv, D, page, mask, spread):
    r, q, cache, table, cu = _attn_case(len(new) + sum(kv), new, kv, Hq, Hkv, D, page)
    scale = spread * D ** -0.5
    bits, words, m = None, 0, mask
    if mask == "tree":
        words = -(-max(new) // 32)
        bits = []
        for n in new:
            for i in range(n):                                     # any bits, own one not forced: rows may see only the cached prefix
                bits.append(int.from_bytes(r.bytes(4 * words), "little") & ((1 << n) - 1) if i % 4 else 0)
        m = torch.tensor(np.array([[b >> 32 * w & 0xFFFFFFFF for w in range(words)] for b in bits], dtype=np.uint32).view(np.int32),
                         device=DEV)
    got = _attend(q, cache, table, kv, cu, max(new), m, scale=scale)
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), kv, cu, scale, bits if bits is not None else mask, words)
    if spread > 1.0:
        # sharper scores: a score's own error (keys rounded to bf16: 1.7e-3 of a score's spread of 6) moves its weight by 1% of
        # itself, six times as far as above
        got, want = ref.to_numpy(got), want
        assert np.linalg.norm(got - want) <= 1.5e-2 * np.linalg.norm(want) + 1e-30
    else:
        _attn_close(got, want)


@gpu
@pytest.mark.parametrize("new,Hq,Hkv,D", [(20, 8, 8, 128), (70, 8, 8, 64), (150, 8, 8, 128), (64, 20, 4, 64), (3, 16, 16, 128)])
def test_attention_of_more_requests_than_the_gpu_has_places_for(new, Hq, Hkv, D):
    """Units of many token tiles in a row on one SM, of one and of two tiles of rows; two requests are looked at closely."""
    page, B = 64, 60
    r = np.random.default_rng(new)
    kv = [int(x) for x in r.integers(1400, 2300, B)]
    width = -(-max(kv) // page)
    cache = _cache_of(r, 200, Hkv, D, page)
    table = r.integers(0, 200, (B, width)).astype(np.int32)       # requests may share blocks
    q = torch.tensor(r.normal(size=(B * new, Hq, D)), dtype=torch.bfloat16)
    cu = [new * b for b in range(B + 1)]
    for mask in ("causal", "full"):
        got = _attend(q, cache, table, kv, cu, new, mask)
        for b in (0, B - 1):
            rows = slice(cu[b], cu[b + 1])
            want = ref.attend(ref.to_numpy(q[rows]), cache, page, D, [table[b].tolist()], [kv[b]], [0, new], D ** -0.5, mask)
            _attn_close(got[rows], want)
        assert torch.isfinite(got).all()


@gpu
@pytest.mark.parametrize("new,D", [(1, 128), (1, 64), (4, 128), (9, 64), (9, 128), (40, 128), (40, 64)])
def test_attention_averages_over_long_contexts_without_losing_bits(new, D):
    """Diffuse weights over 20000 tokens: the output is a hundredth of a value, sums of anything larger must not eat into it."""
    Hq, Hkv, page, kv = 3, 1, 64, 20000
    r, q, cache, table, cu = _attn_case(21, [new], [kv], Hq, Hkv, D, page)
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, 0.2 * D ** -0.5, "causal")
    got = ref.to_numpy(_attend(q, cache, table, [kv], cu, new, "causal", scale=0.2 * D ** -0.5))
    assert np.linalg.norm(got - want) <= 5e-3 * np.linalg.norm(want)


@gpu
@pytest.mark.parametrize("new,D", [(1, 128), (5, 64), (10, 64), (40, 128), (200, 64)])
@pytest.mark.parametrize("key_mul,value_mul,some", [(1e-7, 1.0, False), (1e6, 1.0, False), (1.0, 1e-7, False), (1.0, 1e6, False), (1e5, 3e-5, True),
                                                    (1e-6, 1e5, True), (2.0 ** 100, 2.0 ** 100, False), (2.0 ** -90, 2.0 ** -90, True)])
def test_attention_at_the_ends_of_the_number_range(new, D, key_mul, value_mul, some):
    """Keys and values far from 1, of all tokens or of every seventh; the queries bring the scores back to the usual size."""
    Hq, Hkv, page, kv = 4, 2, 32, 700
    r, q, cache, table, cu = _attn_case(31, [new], [kv], Hq, Hkv, D, page)
    runs = cache.reshape(len(cache), Hkv, page // 16, 16 * (D + 8))
    num = runs[..., 16 * D:].copy().view(np.uint16).astype(np.uint32) << 16
    num = num.view(np.float32).reshape(*runs.shape[:3], 16, 4).astype(np.float64)
    which = (np.arange(16) % 7 == 3) if some else np.ones(16, dtype=bool)
    num[..., which, 0:2] *= key_mul
    num[..., which, 2:4] *= value_mul
    bits = (np.ascontiguousarray(num.astype(np.float32)).view(np.uint32) >> 16).astype(np.uint16)
    runs[..., 16 * D:] = np.ascontiguousarray(bits).view(np.uint8).reshape(*runs.shape[:3], 128)
    back = 1.0 / key_mul if not some or key_mul > 1 else 1.0
    q = (q.double() * back).to(torch.bfloat16)
    args = (ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, D ** -0.5, "causal")
    want = ref.attend(*args)
    got = ref.to_numpy(_attend(q, cache, table, [kv], cu, new, "causal"))
    assert np.isfinite(got).all()
    # against each output's own size: columns of a row may be of any
    assert np.linalg.norm(got - want) <= 5e-3 * np.linalg.norm(want)


@gpu
@pytest.mark.parametrize("D,Hq,Hkv,new", [(128, 5, 1, 1), (64, 4, 2, 6), (128, 40, 8, 40), (64, 16, 2, 200)])
def test_attention_ignores_what_it_must_not_see(D, Hq, Hkv, new):
    """Unwritten places of the pages, pages beyond the length, tokens that the mask hides: all NaN, all block numbers wild."""
    page, kv = 32, 203 + new
    r, q, cache, table, cu = _attn_case(5, [new], [kv], Hq, Hkv, D, page)
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, D ** -0.5, "causal")
    clean = cache.copy()
    used = {int(table[0, u // page]) for u in range(kv)}
    for blk in range(len(cache)):
        if blk not in used:
            cache[blk] = 0xFF
    last = table[0, (kv - 1) // page]
    runs = cache[last].reshape(Hkv, page // 16, 16 * (D + 8))
    for tok in range(kv % page, page):
        runs[:, tok // 16, 16 * D + 8 * (tok % 16):16 * D + 8 * (tok % 16) + 8] = 0xFF      # scale and offset NaN
    table = table.copy()
    table[0, -(-kv // page):] = 2 ** 31 - 1
    _attn_close(_attend(q, cache, table, [kv], cu, new, "causal"), want)
    if new > 1:
        # the last new token holds NaN: only the last query sees it
        u = kv - 1
        clean[table[0, u // page]].reshape(Hkv, page // 16, 16 * (D + 8))[:, u % page // 16, 16 * D + 8 * (u % 16):16 * D + 8 * (u % 16) + 4] = 0xFF
        got = ref.to_numpy(_attend(q, clean, table, [kv], cu, new, "causal"))
        assert np.isfinite(got[:-1]).all() and np.isnan(got[-1]).all()
        bits = torch.tensor([[-1 if j < new // 32 else (1 << new % 32) - 1 for j in range(new // 32 + 1)]] * new, dtype=torch.int32, device=DEV)
        bits[:, (new - 1) // 32] &= ~(1 << (new - 1) % 32) if (new - 1) % 32 < 31 else 2 ** 31 - 1
        assert torch.isfinite(_attend(q, clean, table, [kv], cu, new, bits)).all()
    # a value head of NaN reaches every query that sees it, and a wild block number hides its tokens
    got = _attend(q, clean, table, [kv], cu, new, "full")
    assert torch.isfinite(got).all() == (new == 1)
    table[0, 1] = -7
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, D ** -0.5, "causal")
    _attn_close(_attend(q, cache, table, [kv], cu, new, "causal"), want)


@gpu
@pytest.mark.parametrize("new,D", [(1, 128), (24, 64), (40, 128)])
def test_attention_over_a_cache_beyond_four_gigabytes(new, D):
    Hq, Hkv, page, kv = 8, 2, 128, 500
    r, q, cache, table, cu = _attn_case(9, [new], [kv], Hq, Hkv, D, page)
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, D ** -0.5, "causal")
    far = (5 << 30) // cache[0].nbytes
    big = torch.empty((far + len(cache), Hkv, page * (D + 8)), dtype=torch.uint8, device=DEV)
    big[far:] = torch.tensor(cache, device=DEV)
    got = dsp.dsp_attn_kv4(q.to(DEV), big, i32(table + far), i32([kv]), i32(cu), new)
    _attn_close(got, want)
    slot = torch.tensor([(int(table[0, u // page]) + far) * page + u % page for u in range(kv)], device=DEV)
    rk, _ = dsp.dsp_kv4_read(big, slot, D)
    x = torch.randn((kv, Hkv, D), device=DEV).bfloat16()
    dsp.dsp_kv4_append(None, rk, x, slot, big)
    small = torch.tensor(cache, device=DEV)
    dsp.dsp_kv4_append(None, rk, x, slot - far * page, small)
    assert torch.equal(big[far:], small)


@gpu
def test_attention_of_strided_queries_on_another_stream_and_twice_the_same():
    new, kv, Hq, Hkv, D, page = [7, 20], [300, 90], 10, 2, 128, 16
    r, q, cache, table, cu = _attn_case(11, new, kv, Hq, Hkv, D, page)
    wide = torch.randn((sum(new), Hq + 4, D + 8), device=DEV).bfloat16()
    view = wide[:, 2:2 + Hq, :D]
    view.copy_(q.to(DEV))
    args = (torch.tensor(cache, device=DEV), i32(table), i32(kv), i32(cu), 20)
    plain = dsp.dsp_attn_kv4(q.to(DEV), *args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = dsp.dsp_attn_kv4(view, *args)
    s.synchronize()
    assert torch.equal(plain, other)
    for _ in range(5):
        assert torch.equal(plain, dsp.dsp_attn_kv4(q.to(DEV), *args))


@gpu
def test_rows_beyond_the_requests_are_left_alone_and_graphs_replay_with_other_lengths():
    Hq, Hkv, D, page = 10, 2, 128, 16
    r, q, cache, table, cu = _attn_case(12, [4, 9], [60, 200], Hq, Hkv, D, page)
    T = 20
    qd = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device=DEV)
    qd[:13] = q.to(DEV)
    kv, cud = i32([60, 200]), i32(cu)
    out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = dsp.alloc_workspace(dsp.dsp_attn_kv4_workspace_bytes(2, T, Hq, Hkv, D, 10), DEV)
    args = (qd, torch.tensor(cache, device=DEV), i32(table), kv, cud, 10)
    dsp.dsp_attn_kv4(*args, out=out, workspace=ws)
    assert (out[13:] == 7.0).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dsp.dsp_attn_kv4(*args, out=out, workspace=ws)
    for new, lens in (([4, 9], [60, 200]), ([10, 1], [33, 5]), ([0, 10], [60, 10])):
        c = np.cumsum([0] + new).tolist()
        kv.copy_(i32(lens)), cud.copy_(i32(c))
        out.fill_(7.0)
        g.replay()
        n = sum(new)
        want = ref.attend(ref.to_numpy(qd[:n]), cache, page, D, table.tolist(), lens, c, D ** -0.5, "causal")
        _attn_close(out[:n], want)
        assert (out[n:] == 7.0).all()


# --------------------------------------------------------------------------------------- refusals
def test_declared_argument_types_are_those_of_the_header():
    text = open(os.path.join(os.path.dirname(dsp.LIB_PATH), "..", "include", "dsp.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name, kinds in dsp._SIGNATURES.items():
        args = re.search(r"int32_t %s\(([^;]*)\);" % name, text, flags=re.S).group(1).split(",")
        assert len(args) == len(kinds)
        for a, k in zip(args, kinds):
            want = "p" if "*" in a or "dsp_stream_t" in a else next(c for w, c in (("int64_t", "l"), ("int32_t", "i"), ("float", "f"), ("size_t", "z")) if w in a)
            assert k == want, (name, a)


def test_refusals_happen_on_the_host():
    lib, z, one, odd = dsp.lib(), C.c_void_p(0), C.c_void_p(4096), C.c_void_p(4098)
    i64, f = C.c_int64, C.c_float
    bad, unsup, ok = dsp.DSP_ERR_INVALID_ARG, dsp.DSP_ERR_UNSUPPORTED, dsp.DSP_OK

    def plan(B=4, T=9, page=16, n=8, width=4, stride=4, par=z, dep=z, N=0, seq=one, words=0, mask=z, pos2=C.c_void_p(8192)):
        return lib.dsp_cache_plan(seq, one, one, one, B, T, page, n, width, one, i64(stride), one, par, dep, N, C.c_void_p(8192), pos2,
                                  one, one, one, one, z, mask, words, one, z)
    assert plan(B=-1) == plan(T=-1) == plan(page=0) == plan(n=0) == plan(width=0) == plan(stride=3) == plan(seq=z) == bad
    assert plan(par=one) == plan(par=one, dep=one, N=0) == plan(par=one, dep=one, N=32, mask=one, words=1) == plan(pos2=one) == bad
    assert plan(B=8193) == plan(par=one, dep=one, N=1024, mask=one, words=33) == unsup
    assert plan(B=0, T=0, seq=z) == ok

    def norm(q=one, dt=1, T=3, Hq=4, Hkv=2, D=64, st=256, sh=64, eps=1e-6, pos=one, cs=one, rows=8, rot=64, out=one):
        return lib.dsp_qk_norm_rope(q, one, dt, T, Hq, Hkv, D, i64(st), i64(sh), i64(128), i64(64), one, one, f(eps), pos, cs, rows,
                                    rot, 0, out, one, z)
    assert norm(q=z) == norm(T=-1) == norm(Hq=0) == norm(st=255) == norm(sh=63) == norm(eps=-1.0) == norm(eps=float("nan")) == bad
    assert norm(pos=z) == norm(rows=0) == norm(out=odd) == norm(out=z) == bad
    assert norm(dt=2) == norm(D=96) == norm(rot=8) == norm(rot=80) == norm(rot=24) == norm(Hq=5000, st=1 << 20) == norm(T=1 << 25) == unsup
    assert norm(T=0, q=z) == ok

    def append(q=one, k=one, dt=1, T=3, D=64, slot=one, cache=one, n=4, page=16, qo=one, kst=128):
        return lib.dsp_kv4_append(q, k, one, dt, T, 4, 2, D, i64(256 * D // 64), i64(D), i64(kst * D // 64), i64(D), i64(128 * D // 64),
                                  i64(D), z, z, f(0), z, z, 0, 0, 0, slot, cache, n, page, qo, z)
    assert append(k=z) == append(slot=z) == append(cache=z) == append(cache=odd) == append(n=0) == append(page=24) == append(kst=127) == bad
    assert append(q=z) == append(qo=z) == append(qo=odd) == bad and append(D=256) == append(dt=7) == unsup

    def read(cache=one, D=64, T=3, out=one, page=16, dt=0):
        return lib.dsp_kv4_read(cache, 4, page, 2, D, one, T, dt, out, one, z)
    assert read(cache=z) == read(T=-1) == read(out=odd) == read(page=8) == bad and read(D=256) == read(dt=5) == unsup
    assert read(T=0) == ok

    def attn(q=one, dt=1, B=2, T=3, Hq=4, Hkv=2, D=64, st=256, page=16, width=4, max_new=2, scale=0.1, kind=0, bits=z, words=0, ws=1 << 30,
             w=one):
        return lib.dsp_attn_kv4(q, dt, B, T, Hq, Hkv, D, i64(st), i64(64), one, 8, page, one, i64(4), width, one, one, max_new, f(scale),
                                kind, bits, words, one, w, C.c_size_t(ws), z)
    assert attn(q=z) == attn(q=odd) == attn(B=-1) == attn(Hq=3) == attn(st=255) == attn(st=260) == attn(page=24) == attn(width=5) == bad
    assert attn(max_new=0) == attn(scale=float("inf")) == attn(kind=3) == attn(kind=2) == attn(bits=one, words=1) == attn(w=odd) == bad
    assert attn(dt=0) == attn(D=256, st=2048) == attn(B=70000) == unsup and attn(ws=1) == dsp.DSP_ERR_WORKSPACE
    assert attn(B=0) == attn(T=0) == ok
    n = C.c_size_t(0)
    assert lib.dsp_attn_kv4_workspace_bytes(2, 3, 5, 2, 64, 1, C.byref(n)) == bad
    with pytest.raises(dsp.DspError):
        dsp.dsp_attn_kv4_workspace_bytes(2, 3, 4, 2, 96, 1)


@gpu
def test_the_binding_refuses_wrong_tensors():
    q, k = torch.zeros((2, 4, 64), device=DEV).bfloat16(), torch.zeros((2, 2, 64), device=DEV).bfloat16()
    cache, slot = dsp.kv4_cache(2, 2, 64, 16, DEV), torch.zeros(2, dtype=torch.int64, device=DEV)
    with pytest.raises(ValueError):
        dsp.dsp_qk_norm_rope(q, k.float())
    with pytest.raises(ValueError):
        dsp.dsp_qk_norm_rope(q, k, positions=torch.zeros(3, dtype=torch.int32, device=DEV), cos_sin=_angles(4, 64))
    with pytest.raises(ValueError):
        dsp.dsp_kv4_append(q, k, k, slot.int(), cache)
    with pytest.raises(ValueError):
        dsp.dsp_kv4_append(q, k, k, slot, cache[:, :1])
    table, one = torch.zeros((1, 2), dtype=torch.int32, device=DEV), i32([1])
    with pytest.raises(ValueError):
        dsp.dsp_attn_kv4(q, cache, table, one, i32([0, 2]), 2, mask="prefix")
    with pytest.raises(ValueError):
        dsp.dsp_attn_kv4(q, cache, table, one, i32([0]), 2)
    with pytest.raises(dsp.DspError):
        dsp.dsp_attn_kv4(q.float(), cache, table, one, i32([0, 2]), 2)
