"""dsp_attn_kv4 where masks, lengths, weights and numbers are at their ends, against the plain 64-bit definition.

Tolerances (2-norm of the difference over the 2-norm of the output).  The output's own rounding to bf16 makes
1.7e-3.  Up to 32 query rows a key head: weight times value scale is rounded to bf16, another 1.7e-3, so 2.4e-3;
3.5e-3 is allowed.  More rows: queries, keys, weights and values are fp16 (2.8e-4 each at most, small against the
rest), so 1.8e-3; 2.5e-3 is allowed.
"""
import numpy as np
import pytest
import torch

import pass_reference as ref
from paper_2510_02358_b200 import binding as dsp

gpu = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _allowed(rows):
    return 3.5e-3 if rows <= 32 else 2.5e-3


def _off(got, want):
    return np.linalg.norm(ref.to_numpy(got) - want) / np.linalg.norm(want)


def _case(seed, new, kv, Hq, Hkv, D, page, centred=False):
    """Random codes of unit spread, every request with blocks of its own."""
    r = np.random.default_rng(seed)
    B, width = len(new), max(1, max(-(-n // page) for n in kv)) + 1
    n_blocks = B * width + 2
    table = r.permutation(n_blocks)[:B * width].reshape(B, width).astype(np.int32)
    cache = r.integers(0, 256, (n_blocks, Hkv, page // 16, 16 * (D + 8)), dtype=np.uint8)
    s = r.uniform(0.15, 0.3, (n_blocks, Hkv, page // 16, 16, 2))
    z = -7.5 * s + (0.0 if centred else 0.2) * r.normal(size=s.shape)
    cache[..., 16 * D:] = _bytes(np.stack([s, z], -1).reshape(*s.shape[:-1], 4)).reshape(*cache.shape[:3], 128)
    q = torch.tensor(r.normal(size=(sum(new), Hq, D)), dtype=torch.bfloat16)
    return r, q, cache.reshape(n_blocks, Hkv, -1), table, np.cumsum([0] + list(new)).tolist()


def _bytes(numbers):
    """Numbers as bf16 (cut off), byte by byte along a last axis that is twice as long."""
    with np.errstate(over="ignore"):
        bits = (np.ascontiguousarray(numbers, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.ascontiguousarray(bits).view(np.uint8)


def _set(cache, page, D, table, u, key=None, value=None):
    """Scale and offset of a request's token u, of all heads."""
    run = cache[table[u // page]].reshape(cache.shape[1], page // 16, 16 * (D + 8))[:, u % page // 16]
    at = 16 * D + 8 * (u % 16)
    if key is not None:
        run[:, at:at + 4] = _bytes(np.array(key))
    if value is not None:
        run[:, at + 4:at + 8] = _bytes(np.array(value))


def _attend(q, cache, table, kv, cu, max_new, mask="causal", **kw):
    return dsp.dsp_attn_kv4(q.to(DEV), torch.tensor(cache, device=DEV), i32(table), i32(kv), i32(cu), max_new, mask=mask, **kw)


# ------------------------------------------------------------------------------------ weights
@gpu
@pytest.mark.parametrize("new,D", [(1, 128), (12, 64), (30, 128), (40, 128), (70, 64), (150, 128)])
@pytest.mark.parametrize("above", [18, 20, 22, 25])
@pytest.mark.parametrize("place", [0, 5000])
def test_small_weights_beside_a_dominant_token_count(new, D, above, place):
    """One token's weight is 2^above of the others' and its value 0: the output is what the others leave."""
    page, kv = 64, 8192
    r, q, cache, table, cu = _case(above, [new], [kv], 1, 1, D, page, centred=True)
    q = (0.5 + 0.5 * q.float()).to(torch.bfloat16)
    _set(cache, page, D, table[0], place, key=[0.0, above * np.log(2.0) / (0.5 * D * D ** -0.5)], value=[0.0, 0.0])
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, D ** -0.5, "causal")
    assert _off(_attend(q, cache, table, [kv], cu, new), want) <= _allowed(new)


# ------------------------------------------------------------------------------- hidden tokens
NAN = float("nan")
HIDDEN = [([NAN, NAN], [2000.0, 3000.0]), ([NAN, 0.0], [1e4, -3e4]), ([0.2, -1.5], [NAN, 0.0]), ([NAN, NAN], [2.0 ** 40, 1.0]), ([NAN, 0.1], [1e-30, 1e-30])]


@gpu
@pytest.mark.parametrize("new,Hq,Hkv,D", [(2, 4, 1, 128), (20, 1, 1, 64), (40, 2, 2, 128), (200, 4, 2, 64)])
@pytest.mark.parametrize("key,value", HIDDEN)
@pytest.mark.parametrize("tree", [False, True])
def test_a_hidden_token_changes_nothing_whatever_it_holds(new, Hq, Hkv, D, key, value, tree):
    """New token 1 is seen by later rows only (causal), or by none but row 1 (tree): the others have their usual bits."""
    page, kv = 32, 170 + new
    r, q, cache, table, cu = _case(3, [new], [kv], Hq, Hkv, D, page)
    mask = "causal"
    if tree:
        bits = np.zeros((new, new), dtype=bool)
        bits[np.arange(new), np.arange(new)] = True
        bits[:, 0] = True
        words = -(-new // 32)
        packed = np.packbits(np.pad(bits, ((0, 0), (0, 32 * words - new))), axis=1, bitorder="little").view(np.uint32)
        mask = torch.tensor(packed.view(np.int32).copy(), device=DEV)
    before = _attend(q, cache, table, [kv], cu, new, mask)
    assert torch.isfinite(before).all()
    _set(cache, page, D, table[0], kv - new + 1, key=key, value=value)
    after = _attend(q, cache, table, [kv], cu, new, mask)
    blind = [i for i in range(new) if i != 1] if tree else [0]
    assert torch.equal(before[blind], after[blind])
    assert after[1].isnan().all()


@gpu
@pytest.mark.parametrize("new,Hq,Hkv,D", [(2, 4, 1, 128), (20, 1, 1, 64), (40, 2, 2, 128), (200, 4, 2, 64)])
@pytest.mark.parametrize("key,value", [([0.2, -1.5], [2.0 ** 123, 2.0 ** 120]), ([0.2, -1.5], [3.3e38, 3.3e38]), ([0.2, -1.5], [-3.3e38, -3.3e38]),
                                       ([3.3e38, 3.3e38], [0.2, -1.5]), ([2.0 ** 125, -2.0 ** 125], [2.0 ** 123, -2.0 ** 126])])
def test_a_hidden_token_at_the_end_of_the_number_range_reaches_no_other_row(new, Hq, Hkv, D, key, value):
    page, kv = 32, 170 + new
    r, q, cache, table, cu = _case(4, [new], [kv], Hq, Hkv, D, page)
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, D ** -0.5, "causal")
    u = kv - new // 2                                                               # rows of the first half do not see it
    _set(cache, page, D, table[0], u, key=key, value=value)
    got = _attend(q, cache, table, [kv], cu, new)
    rows = slice(0, new - new // 2)
    assert _off(got[rows], want[rows]) <= _allowed(new * Hq // Hkv)


# ------------------------------------------------------------------------- more than is answered
@gpu
@pytest.mark.parametrize("mask", ["causal", "full", "tree"])
@pytest.mark.parametrize("new,max_new,T,Hq,Hkv,D", [([5], 1, 5, 4, 1, 128), ([9, 20], 4, 29, 2, 2, 64), ([9, 20], 20, 16, 2, 1, 128), ([30, 90], 40, 120, 4, 4, 128),
                                                    ([200], 200, 130, 4, 2, 64), ([70, 300], 100, 333, 8, 1, 128)])
def test_requests_with_more_new_tokens_than_are_answered(new, max_new, T, Hq, Hkv, D, mask):
    """The rows that are answered see what they see in a call that answers all; the others are left alone."""
    page, kv = 16, [100 + 3 * n for n in new]
    r, q, cache, table, cu = _case(6, new, kv, Hq, Hkv, D, page)
    bits, words, m = None, 0, mask
    if mask == "tree":
        words = -(-max(new) // 32)
        bits = [int.from_bytes(r.bytes(4 * words), "little") & ((1 << n) - 1) | 1 for n in new for _ in range(n)]
        m = torch.tensor(np.array([[b >> 32 * w & 0xFFFFFFFF for w in range(words)] for b in bits[:T]], dtype=np.uint32).view(np.int32), device=DEV)
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), kv, cu, D ** -0.5, bits if bits is not None else mask, words)
    out = torch.full((T, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    _attend(q[:T], cache, table, kv, cu, max_new, m, out=out)
    answered = np.concatenate([np.arange(n) < max_new for n in new])[:T]
    assert _off(out[torch.tensor(answered, device=DEV)], want[:T][answered]) <= _allowed(max_new * Hq // Hkv)
    assert (out[torch.tensor(~answered, device=DEV)] == 7.0).all()


# ------------------------------------------------------------------------------ queries and scale
SHAPES = [(1, 4, 1, 128), (6, 2, 1, 64), (30, 1, 1, 128), (40, 2, 2, 128), (70, 4, 2, 64), (200, 4, 2, 64)]


@gpu
@pytest.mark.parametrize("new,Hq,Hkv,D", SHAPES)
def test_queries_with_nan_or_infinity_keep_to_their_rows(new, Hq, Hkv, D):
    """A row of NaN that sees something gets NaN, one that sees nothing 0, and the rows beside it what they always get."""
    page, kv = 16, 150 + new
    r, q, cache, table, cu = _case(8, [new], [kv], Hq, Hkv, D, page)
    clean = _attend(q, cache, table, [kv], cu, new)
    odd = [i for i in range(new) if i % 3 == 0]
    for value in (float("nan"), float("inf"), -float("inf")):
        bad = q.clone()
        bad[odd, :, 5] = value
        got = _attend(bad, cache, table, [kv], cu, new)
        assert torch.equal(got[[i for i in range(new) if i % 3]], clean[[i for i in range(new) if i % 3]])
        assert got[odd].isnan().all()                                               # keys of both signs: never -inf alone
        missing = np.full_like(table, -1)
        assert not _attend(bad, cache, missing, [kv], cu, new).any()
        none = torch.zeros((new, -(-new // 32)), dtype=torch.int32, device=DEV)
        assert not _attend(bad, cache, table, [new], cu, new, none).any()


@gpu
@pytest.mark.parametrize("new,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("scale,size", [(0.0, 0.0), (0.0, 1.0), (0.0, 1e-25), (0.125, 0.0), (1e-30, 1e-25), (-0.1, 1.0), (1e-42, 0.0), (3e-4, 300.0)])
def test_scales_and_queries_of_any_size(new, Hq, Hkv, D, scale, size):
    page, kv = 16, 190 + new
    r, q, cache, table, cu = _case(9, [new], [kv], Hq, Hkv, D, page)
    q = (q.float() * size).to(torch.bfloat16)
    table[0, 2] = -1                                                                # tokens that are not there among those that are
    want = ref.attend(ref.to_numpy(q), cache, page, D, table.tolist(), [kv], cu, scale, "causal")
    assert _off(_attend(q, cache, table, [kv], cu, new, scale=scale), want) <= _allowed(new * Hq // Hkv)
