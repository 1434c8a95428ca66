"""What follows a verified step, in 64 bits and plain steps (scores of tokens, distillation, forks, moves of the cache)."""
import math

import torch

LN2 = math.log(2.0)


def score(x, T, tokens, K, row_len=None):
    """x [B, L, V]: (logp [B, L, G], rank [B, L], lse, entropy, top_id, top_logit, top_logp [B, L, K]) with 64-bit values."""
    x = x.double()
    B, L, V = x.shape
    z = x / T
    lse = torch.logsumexp(z, -1)
    p = (z - lse[..., None]).exp()
    entropy = -torch.where(p > 0, p * (z - lse[..., None]), torch.zeros_like(p)).sum(-1)
    ok = (tokens >= 0) & (tokens < V)
    at = tokens.long().clamp(0, V - 1)
    logp = torch.where(ok, z.gather(-1, at) - lse[..., None], torch.full_like(lse[..., None], -math.inf))
    x0, t0 = x.gather(-1, at[..., :1]), at[..., :1]
    ids = torch.arange(V, device=x.device)
    rank = torch.where(ok[..., 0], ((x > x0) | ((x == x0) & (ids < t0))).sum(-1), torch.full_like(t0[..., 0], -1))
    v, i = torch.sort(x, dim=-1, descending=True, stable=True)
    n = min(K, V)
    top_id = torch.full((B, L, K), -1, dtype=torch.int64, device=x.device)
    top_x = torch.full((B, L, K), -math.inf, dtype=torch.float64, device=x.device)
    top_id[..., :n], top_x[..., :n] = i[..., :n].masked_fill(v[..., :n] == -math.inf, -1), v[..., :n]
    top_p = top_x / T - lse[..., None]
    if row_len is not None:
        off = torch.arange(L, device=x.device) >= row_len[:, None]
        for t, pad in ((logp, -math.inf), (rank, -1), (lse, -math.inf), (entropy, 0.0), (top_id, -1), (top_x, -math.inf), (top_p, -math.inf)):
            t[off] = pad
    return logp, rank, lse, entropy, top_id, top_x, top_p


def exponent_error(x, T, terms):
    """Bound on the relative error of a sum of `terms` fp32 exponentials a thread, over a row x [..., V] at temperature T.

    An exponent a = x log2(e)/T - c is rounded twice (against |c| and against |a|, whose mean over the softmax is below log2 V plus what
    the reference lies above the row's sum: nothing), an exponential is off by 2^-22, and a sum of n terms in turn by n half steps; c is at
    most |x|max log2(e)/T."""
    big = x.double().abs().masked_fill(torch.isinf(x), 0.0).amax(-1) / LN2 / T
    return 2.0 ** -24 * (LN2 * (2 * big + math.log2(x.shape[-1]) + 1) + 4 + terms)


def terms(V, per_thread=512):
    """Sums that one thread forms in turn: half of its logits, at most those of a row over the CTA's threads."""
    return min(V, V // per_thread + 64)


def teacher(t, T, ids, V, lse=None, count=None):
    """(p, taking part) of the slots, and the mass of the others; 64 bits."""
    K = ids.shape[-1]
    use = (ids >= 0) & (ids < V)
    if count is not None:
        use &= torch.arange(K, device=ids.device) < count[..., None]
    same = (ids[..., :, None] == ids[..., None, :]) & use[..., None, :]
    first = ~(same & (torch.arange(K, device=ids.device)[None, :] < torch.arange(K, device=ids.device)[:, None])).any(-1)
    use = use & first
    z = (t.double() / T).masked_fill(~use, -math.inf)
    if lse is not None:
        p = (z - lse.double()[..., None]).exp()
        return p, use, (1.0 - p.sum(-1)).clamp(min=0.0)
    m = z.amax(-1, keepdim=True)
    e = torch.where(use & (m > -math.inf), (z - m).exp(), torch.zeros_like(z))
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e / total, torch.zeros_like(e)), use, torch.zeros_like(total[..., 0])


def distill(x, ids, t, T, lse=None, count=None, weight=None):
    """(loss, accept, lse, gradient) in 64 bits; x [B, L, V]."""
    x = x.double()
    V = x.shape[-1]
    p, use, r = teacher(t, T, ids, V, lse, count)
    none = (lse is None) & (p.sum(-1) == 0)
    at = ids.long().clamp(0, V - 1)
    logq = torch.log_softmax(x / T, -1)
    q = logq.exp()
    inside = torch.zeros_like(q).scatter_add_(-1, at, use.double()) > 0
    others = logq.masked_fill(inside, -math.inf)
    log_s = torch.logsumexp(others, -1)
    s = log_s.exp()
    if lse is not None:                                 # a rest that rounding alone can leave of a complete list, where s is nothing beside it
        r = r.masked_fill((r <= 2.0 ** -23 * (lse.double().abs() + 4)) & (s < r / 1024), 0.0)
    qk = torch.where(use, q.gather(-1, at), torch.zeros_like(p))
    logk = logq.gather(-1, at)
    loss = torch.where(p > 0, p * (p.log() - logk), torch.zeros_like(p)).sum(-1) + torch.where(r > 0, r * (r.log() - log_s), torch.zeros_like(r))
    accept = torch.minimum(p, qk).sum(-1) + torch.minimum(r, s)
    # others: q_v - r q_v / s, with q_v / s from the logarithms (s may be far below the smallest number)
    share = torch.where(log_s[..., None] > -math.inf, (others - log_s[..., None]).exp(), torch.zeros_like(others))
    g = q - r[..., None] * share
    g = torch.where(inside, torch.zeros_like(g), torch.where(log_s[..., None] > -math.inf, g, torch.zeros_like(g)))
    g = g.scatter_add(-1, at, torch.where(use, qk - p, torch.zeros_like(p))) / T
    zero = torch.zeros_like(loss)
    loss, accept, g = torch.where(none, zero, loss), torch.where(none, zero, accept), torch.where(none[..., None], torch.zeros_like(g), g)
    full = torch.logsumexp(x / T, -1)
    if weight is not None:
        off = weight == 0
        g = torch.where(off[..., None], torch.zeros_like(g), g * weight.double()[..., None])
        loss, accept, full = loss.masked_fill(off, 0.0), accept.masked_fill(off, 0.0), full.masked_fill(off, -math.inf)
    return loss, accept, full, g


BAD_LENGTH, NO_BLOCKS, BAD_BLOCK = 512, 64, 1024


def fork(src, keep, seq, count, pos, table, ring, page, new_table):
    """The tables after a fork, by lists: arguments as dsp_cache_fork's, as Python lists.  Returns a dict; `table` and `ring` are copies."""
    Bo, width, n_blocks = len(src), len(table[0]) if table else 0, len(ring)
    held = [min(max(c, 0), width) for c in count]
    rows, status = [], [0] * Bo
    for r in range(Bo):
        rows.append([])
        n = 0
        if src[r] == -1:
            keep_r = 0
        elif not 0 <= src[r] < len(seq):
            keep_r, status[r] = 0, BAD_LENGTH
        else:
            keep_r = seq[src[r]] if keep is None else keep[r]
            n = -(-keep_r // page)
            if seq[src[r]] < 0 or keep_r < 0 or keep_r > seq[src[r]] or n > held[src[r]]:
                keep_r, n, status[r] = 0, 0, BAD_LENGTH
            rows[r] = list(table[src[r]][:n]) if n else []
            if any(not 0 <= p < n_blocks for p in rows[r]):
                keep_r, rows[r], status[r] = 0, [], BAD_BLOCK
        rows[r] = (keep_r, rows[r])
    owner = {}
    for r, (k, blocks) in enumerate(rows):
        for e, p in enumerate(blocks):
            owner.setdefault(p, []).append(-1 if (e + 1) * page <= k else r)
    free, taken = min(max(pos[1] - pos[0], 0), n_blocks), 0
    new, ring = [list(t) for t in new_table], list(ring)
    copies, counts, lens = [(-1, -1, 0)] * Bo, [0] * Bo, [0] * Bo
    old_ring = list(ring)
    for r, (k, blocks) in enumerate(rows):
        blocks = list(blocks)
        if blocks and k % page and min(owner[blocks[-1]]) != r:
            if taken >= free:
                status[r], k, blocks = NO_BLOCKS, 0, []
            else:
                fresh = old_ring[(pos[0] + taken) % n_blocks]
                copies[r] = (blocks[-1], fresh, k % page)
                blocks[-1] = fresh
            taken += 1
        new[r][:len(blocks)] = blocks
        counts[r], lens[r] = len(blocks), k
    back, seen = [], set()
    for b in range(len(seq)):
        for p in table[b][:held[b]]:
            if 0 <= p < n_blocks and p not in owner and p not in seen:
                back.append(p)
                seen.add(p)
    for i, p in enumerate(back):
        ring[(pos[1] + i) % n_blocks] = p
    return dict(table=new, block_count=counts, seq_len=lens, ring=ring, ring_pos=[pos[0] + min(taken, free), pos[1] + len(back)],
                copy_src=[c[0] for c in copies], copy_dst=[c[1] for c in copies], copy_len=[c[2] for c in copies], row_status=status)


def token_bytes(D):
    """Bytes of a run's 16 tokens: [16][D + 8], from the layout of the 4-bit cache."""
    out = []
    for t in range(16):
        c, half = (t & 7) >> 1, t >> 3
        key = [t * 64 + 4 * w if D == 128 else (t & 7) * 64 + (w >> 1) * 16 + half * 8 + (w & 1) * 4 for w in range(D // 8)]
        val = [(half * 512 + (w >> 1) * 64 + c * 16 + (t & 1) * 8 + (w & 1) * 4) if D == 128 else (w * 64 + c * 16 + half * 8 + (t & 1) * 4)
               for w in range(D // 8)]
        words = key + [8 * D + w for w in val] + [16 * D + 8 * t, 16 * D + 8 * t + 4]
        out.append([w + i for w in words for i in range(4)])
    return out


def compact(cache, D, table, seq, node, length):
    """cache uint8 [layers, blocks, Hkv, bytes] on the host, moved token by token: a copy."""
    cache = cache.clone()
    page = cache.shape[-1] // (D + 8)
    place = torch.tensor(token_bytes(D))

    def find(b, at):
        if at < 0 or at // page >= len(table[b]) or not 0 <= table[b][at // page] < cache.shape[1]:
            return None
        run, t = at % page // 16, at % 16
        return table[b][at // page], run * 16 * (D + 8) + place[t]

    for b in range(len(seq)):
        for i in range(min(max(length[b], 0), len(node[b]))):
            n = node[b][i]
            if n < 0 or n == i:
                continue
            src, dst = find(b, seq[b] + 1 + n), find(b, seq[b] + 1 + i)
            if src is not None and dst is not None:
                cache[:, dst[0], :, dst[1]] = cache[:, src[0], :, src[1]]
    return cache
