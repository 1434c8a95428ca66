"""Plain 64-bit (and integer) definitions of the model pass's operators, one step at a time.

Written from the formulas in include/dsp.h: numpy in double, Python integers for the bookkeeping, the
4-bit cache read and written byte by byte.  Nothing of the CUDA library is used.
"""
import numpy as np
import torch

NO_BLOCKS, TABLE_FULL, PLAN_FULL, BAD_LENGTH = 64, 128, 256, 512


def plan(seq, new, count, head, tail, table, ring, page, T, parent=None, depth=None, words=0):
    """dsp_cache_plan on Python lists; table and ring are copied, everything is returned."""
    table, ring = [list(r) for r in table], list(ring)
    before, B, width, n = [list(r) for r in table], len(seq), len(table[0]) if table else 0, len(ring)
    N = len(parent[0]) if parent is not None else None
    status, need = [0] * B, [0] * B
    for b in range(B):
        need[b] = -(-(seq[b] + new[b]) // page)
        if seq[b] < 0 or new[b] < 0 or seq[b] + new[b] > 2 ** 31 - 1 or not 0 <= count[b] <= width or (N is not None and new[b] > N + 1):
            status[b] = BAD_LENGTH
        elif need[b] > width:
            status[b] = TABLE_FULL
    run = 0
    for b in range(B):
        if not status[b]:
            run += new[b]
            if new[b] and run > T:
                status[b] = PLAN_FULL
    run = 0
    for b in range(B):
        lack = max(need[b] - count[b], 0)
        if not status[b] and lack:
            run += lack
            if run > tail - head:
                status[b] = NO_BLOCKS
    cu, kv, cnt, slot, pos, row, mask = [0], [], [], [], [], [], []
    h, t = head, tail
    for b in range(B):
        if status[b]:
            cu.append(cu[-1]), kv.append(max(seq[b], 0)), cnt.append(min(max(count[b], 0), width))
            continue
        for e in range(count[b], need[b]):
            table[b][e] = ring[h % n]
            h += 1
        for e in range(need[b], count[b]):
            ring[t % n] = before[b][e]
            t += 1
        cnt.append(need[b]), cu.append(cu[-1] + new[b]), kv.append(seq[b] + new[b])
        paths = {}
        for i in range(new[b]):
            at = seq[b] + i
            slot.append(table[b][at // page] * page + at % page)
            row.append(b)
            if parent is None:
                pos.append(at)
                continue
            pos.append(at if i == 0 else seq[b] + 1 + depth[b][i - 1])
            up = 0
            if i > 0:
                p = parent[b][i - 1]
                up = p + 1 if 0 <= p < i - 1 else 0
            paths[i] = 1 if i == 0 else paths[up] | 1 << i
            mask.append([paths[i] >> 32 * w & 0xFFFFFFFF for w in range(words)])
    pad = T - len(slot)
    return dict(block_count=cnt, ring_pos=[h, t], block_table=table, free_ring=ring, cu_new=cu, kv_len=kv,
                slot=slot + [-1] * pad, position=pos + [-1] * pad, token_row=row + [-1] * pad, row_status=status,
                mask=mask + [[0] * words] * pad if parent is not None else None)


def norm_rope(x, weight, eps, positions, cos_sin, interleaved):
    """x [T, H, D] double."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if cos_sin is not None:
        rot = cos_sin.shape[1]
        y = x.copy()
        for t, p in enumerate(positions):
            if p < 0 or p >= len(cos_sin):
                continue
            for i in range(rot // 2):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
                c, s = cos_sin[p, i], cos_sin[p, rot // 2 + i]
                y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
                y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
        x = y
    if positions is not None:
        for t, p in enumerate(positions):
            if p < 0:
                x[t] = 0.0
            elif cos_sin is not None and p >= len(cos_sin):
                x[t] = np.nan
    return x


def _bf16_bits(x):
    return int(np.float32(x).view(np.uint32))


def bf16_down(x):
    b = _bf16_bits(x)
    b = (b + 0xFFFF) & 0xFFFF0000 if b >> 31 else b & 0xFFFF0000
    return float(np.uint32(b & 0xFFFFFFFF).view(np.float32))


def bf16_up(x):
    return float(np.uint32((_bf16_bits(x) + 0xFFFF) & 0xFFFF0000).view(np.float32))


def quantise(x):
    """Codes, scale, offset of one head (float32 values)."""
    x = np.asarray(x, dtype=np.float32)
    if not np.isfinite(x).all():
        return np.zeros(len(x), dtype=int), np.nan, np.nan
    z = bf16_down(x.min())
    with np.errstate(over="ignore"):
        s = bf16_up(np.float32(np.float32(x.max() - np.float32(z)) / np.float32(15.0)))
    if not (np.isfinite(z) and np.isfinite(s)):
        return np.zeros(len(x), dtype=int), np.nan, np.nan
    if s < 2.0 ** -126:
        return np.zeros(len(x), dtype=int), 0.0, z
    code = np.rint(((x - np.float32(z)).astype(np.float32) / np.float32(s)).astype(np.float32))
    return np.minimum(code, 15).astype(int), s, z


def key_byte(tok, ch, D):
    """(byte within a run, shift) of a key's code."""
    word, nib = ch // 8, [0, 4, 1, 5, 2, 6, 3, 7][ch % 8]
    r, hi = tok % 8, tok // 8
    if D == 128:
        lane, vec = 4 * r + word // 4, 16 * hi * 32 + 4 * (word % 4)
    else:
        lane, vec = 4 * r + word // 2, 8 * hi + 4 * (word % 2)
    return lane * 16 + vec + nib // 2, 4 * (nib % 2)


def value_byte(tok, ch, D):
    word, nib = ch // 8, [0, 4, 1, 5, 2, 6, 3, 7][ch % 8]
    c, odd, hi = tok % 8 // 2, tok % 2, tok // 8
    if D == 128:
        lane, vec = 4 * (word // 2) + c, 512 * hi + 8 * odd + 4 * (word % 2)
    else:
        lane, vec = 4 * word + c, 8 * hi + 4 * odd
    return 8 * D + lane * 16 + vec + nib // 2, 4 * (nib % 2)


def _runs(cache, page):
    n, H, size = cache.shape
    return cache.reshape(n, H, page // 16, size // (page // 16))


def cache_put(cache, page, D, slot, h, key=None, value=None):
    """Write one token's head (float32 values) into a numpy cache."""
    run = _runs(cache, page)[slot // page, h, slot % page // 16]
    tok = slot % 16
    for x, byte_of, off in ((key, key_byte, 0), (value, value_byte, 4)):
        if x is None:
            continue
        code, s, z = quantise(x)
        for ch in range(D):
            at, sh = byte_of(tok, ch, D)
            run[at] = run[at] & (0xF0 if sh == 0 else 0x0F) | int(code[ch]) << sh
        num = np.array([s, z], dtype=np.float32)
        bits = (num.view(np.uint32) >> 16).astype(np.uint16)
        if np.isnan(s):
            bits = np.array([0x7FFF, 0x7FFF], dtype=np.uint16)
        run[16 * D + 8 * tok + off:16 * D + 8 * tok + off + 4] = bits.view(np.uint8)


def cache_get(cache, page, D, slot, h):
    """(key, value) of one token's head in double."""
    run = _runs(cache, page)[slot // page, h, slot % page // 16]
    tok = slot % 16
    num = run[16 * D + 8 * tok:16 * D + 8 * tok + 8].copy().view(np.uint16).astype(np.uint32) << 16
    num = num.view(np.float32).astype(np.float64)
    out = []
    for byte_of, s, z in ((key_byte, num[0], num[1]), (value_byte, num[2], num[3])):
        code = np.array([run[a] >> sh & 15 for a, sh in (byte_of(tok, ch, D) for ch in range(D))], dtype=np.float64)
        out.append(code * s + z)
    return out


def cache_rows(cache, page, D, slots):
    """Keys and values [len(slots), H, D] in double (vectorised over the tokens)."""
    slots = np.asarray(slots)
    runs = _runs(cache, page)[slots // page, :, slots % page // 16]                # [n, H, bytes]
    tok = slots % 16
    out = []
    for byte_of, off in ((key_byte, 0), (value_byte, 4)):
        at = np.array([[byte_of(t, ch, D) for ch in range(D)] for t in range(16)])  # [16, D, 2]
        idx, sh = at[tok, :, 0], at[tok, :, 1]
        code = np.take_along_axis(runs, idx[:, None, :].repeat(runs.shape[1], 1), 2) >> sh[:, None] & 15
        p = 16 * D + 8 * tok[:, None] + off + np.arange(4)
        num = np.take_along_axis(runs, p[:, None, :].repeat(runs.shape[1], 1), 2)
        num = (np.ascontiguousarray(num).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
        out.append(code * num[..., 0:1] + num[..., 1:2])
    return out


def attend(q, cache, page, D, table, kv_len, cu, scale, mask, words=0):
    """q [T, Hq, D] double; mask: "causal", "full" or a list of visible bits (ints) per token.  [T, Hq, D], NaN where no row is."""
    q = np.asarray(q, dtype=np.float64)
    out = np.full(q.shape, np.nan)
    H = cache.shape[1]
    g = q.shape[1] // H
    for b in range(len(kv_len)):
        n = cu[b + 1] - cu[b]
        kv = max(0, min(kv_len[b], len(table[b]) * page))
        toks = [u for u in range(kv) if 0 <= table[b][u // page] < cache.shape[0]]
        k, v = cache_rows(cache, page, D, [table[b][u // page] * page + u % page for u in toks]) if toks else (None, None)
        toks = np.array(toks, dtype=int)
        for i in range(n):
            t = cu[b] + i
            j = toks - (kv - n)
            if mask == "causal":
                see = j <= i
            elif mask == "full":
                see = np.ones(len(toks), dtype=bool)
            else:
                see = np.array([x < 0 or (x < 32 * words and mask[t] >> int(x) & 1 == 1) for x in j], dtype=bool)
            idx = np.nonzero(see)[0]
            for h in range(q.shape[1]):
                if len(idx) == 0:
                    out[t, h] = 0.0
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (k[idx, h // g] @ q[t, h])
                    if (s == -np.inf).all():
                        out[t, h] = 0.0
                        continue
                    p = np.exp(s - s.max())
                    out[t, h] = p @ v[idx, h // g] / p.sum()
    return out


def to_numpy(t):
    return t.detach().to("cpu", torch.float64).numpy()
