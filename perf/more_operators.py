"""After a verified step: cases for timing and comparison.

What follows a step of draft and verification: tokens are scored under a model's logits (`score`), the
drafter learns from the target's top logits (`distill`: loss and gradient), requests fork, shrink or end
while they share pages of the cache (`fork`, with the pages that have to be copied, in every layer), and
the accepted nodes of a token tree move to their final places in the cache (`compact`).

`run(state)` computes an operator by elementary torch operations in 32 bits (long sums and what lies next
to a border in 64), or, where `own` is true, by the framework's calls.  `exact(case, seed)` is the
definition in 64 bits.

The cache is uint8 [layers, blocks, Hkv, page * (D + 8)]; a page is cut into runs of 16 tokens.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NONE = 1 << 40


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the token that one request has just emitted, with its five best alternatives: latency
        dict(name="score_1", op="score", B=1, L=1, V=152064, dtype="bf16", G=1, K=5, T=1.0, masked=False),
        # the target's rows of sixteen verified chains: accepted tokens and 20 alternatives (a teacher's list)
        dict(name="score_272", op="score", B=16, L=17, V=152064, dtype="bf16", G=1, K=20, T=1.0, masked=False),
        # the lattice's candidates of 64 blocks under cached rows of an fp32 model with an odd vocabulary
        dict(name="score_lattice", op="score", B=64, L=32, V=32003, dtype="f32", G=9, K=0, T=0.7, masked=True),
        # four prompts of up to 512 tokens, every token scored
        dict(name="score_prompt", op="score", B=4, L=512, V=152064, dtype="bf16", G=1, K=0, T=1.0, masked=False),
        # one drafted block learns from its verification
        dict(name="distill_16", op="distill", B=1, L=16, V=152064, dtype="bf16", K=8, T=1.0, tail=True, two=False, skip=0.0),
        # a training step of the drafter: 2048 positions, one of ten without a label
        dict(name="distill_2048", op="distill", B=16, L=128, V=152064, dtype="bf16", K=32, T=1.0, tail=True, two=False, skip=0.1),
        # fp32 logits, odd vocabulary, a stored teacher list without its log-sum-exp, at temperature 2
        dict(name="distill_f32", op="distill", B=3, L=333, V=32003, dtype="f32", K=64, T=2.0, tail=False, two=False, skip=0.0),
        # loss first, the gradient later by factors that come from behind
        dict(name="distill_two", op="distill", B=8, L=64, V=152064, dtype="bf16", K=16, T=1.0, tail=True, two=True, skip=0.0),
        # four requests: one ends, one is sampled twice
        dict(name="fork_4", op="fork", B=4, ctx=500, page=16, layers=2, Hkv=8, D=128),
        # a server's 512 requests after a step, every fourth one ended and another sampled twice instead
        dict(name="fork_512", op="fork", B=512, ctx=8192, page=64, layers=4, Hkv=2, D=128),
        # one verified tree of a small model
        dict(name="compact_1", op="compact", B=1, ctx=700, page=16, beam=4, depth=8, layers=8, Hkv=8, D=64),
        # 64 verified trees of up to 8 x 16 nodes
        dict(name="compact_64", op="compact", B=64, ctx=2000, page=64, beam=8, depth=16, layers=16, Hkv=8, D=128),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "score", "distill", "distill", "fork", "compact"])
    if op in ("score", "distill"):
        V = rng.choice([152064, 32000, 32003, 128256, _spread(rng, 2000, 160000)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 600e6 / (V * (2 if dtype == "bf16" else 4))                         # rows, by their bytes
        rows = _spread(rng, 1, min(2048, most))
        B = _spread(rng, 1, min(64, rows))
        c = dict(op=op, B=B, L=max(1, rows // B), V=V, dtype=dtype)
        if op == "score":
            return dict(c, G=rng.choice([1, 1, 5, 9, 33]), K=rng.choice([0, 0, 1, 5, 20, 32]), T=rng.choice([1.0, 1.0, 0.6, 1.7]),
                        masked=rng.random() < 0.3)
        return dict(c, K=rng.choice([1, 8, 16, 32, 64, 100, 256]), T=rng.choice([1.0, 1.0, 2.0, 0.8]), tail=rng.random() < 0.7,
                    two=rng.random() < 0.3, skip=rng.choice([0.0, 0.1, 0.5]))
    D, Hkv, page = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 128])
    if op == "fork":
        return dict(op=op, B=_spread(rng, 2, 512), ctx=_spread(rng, 50, 8192), page=page, layers=rng.randint(1, 4), Hkv=min(Hkv, 2), D=D)
    return dict(op=op, B=_spread(rng, 1, 64), ctx=_spread(rng, 50, 2000), page=page, beam=rng.randint(2, 8), depth=rng.randint(2, 16),
                layers=_spread(rng, 1, 16), Hkv=Hkv, D=D)


# ----------------------------------------------------------------------------------------- inputs
def _of(c):
    """Lengths and shapes of requests go by the case's values alone, so that its work is known without its inputs."""
    return random.Random("%s" % sorted((k, v) for k, v in c.items() if k != "name"))


def _row_lens(c):
    """Rows that count of each batch row."""
    r = _of(c)
    return [c["L"] if b == 0 or c["L"] == 1 else r.randint(max(1, c["L"] // 2), c["L"]) for b in range(c["B"])]


def _fork_plan(c):
    """(tokens cached, blocks held, row continued, tokens kept) of every request: every fourth row's place is taken by another's fork,
    and a few rows shrink."""
    r = _of(c)
    B, P = c["B"], c["page"]
    seq = [c["ctx"] if b == 0 else r.randint(1, c["ctx"]) for b in range(B)]
    have = [-(-n // P) + r.randint(0, 1) for n in seq]
    src, keep = list(range(B)), list(seq)
    for b in range(B):
        if b % 4 == 3:
            src[b] = -1 if r.random() < 0.3 else r.randrange(B)
            keep[b] = 0 if src[b] < 0 else seq[src[b]]
        if src[b] >= 0 and r.random() < 0.1:
            keep[b] = r.randint(0, seq[src[b]])
    return seq, have, src, keep


def _fork_copies(c):
    """(pages that have to be copied, their tokens, pages held before, pages held after, pages given back), from the plan."""
    seq, have, src, keep = _fork_plan(c)
    P, holder, copies = c["page"], {}, []
    for b, (s, n) in enumerate(zip(src, keep)):
        for e in range(-(-n // P) if s >= 0 else 0):
            key = (s, e)
            whole = (e + 1) * P <= n
            holder[key] = -1 if whole else min(holder.get(key, NONE), b)
    for b, (s, n) in enumerate(zip(src, keep)):
        if s >= 0 and n % P and holder[(s, n // P)] != b:
            copies.append(n % P)
    after = sum(-(-n // P) for s, n in zip(src, keep) if s >= 0)
    return len(copies), copies, sum(have), after, sum(have) - len(holder)


def _trees(c):
    """(cached tokens, new tokens, accepted nodes) of every request: the tree that `beam` paths of `depth` tokens leave, the first path
    first; the accepted nodes follow a path that leaves the first one at some depth."""
    r = _of(c)
    out = []
    for b in range(c["B"]):
        seq, d, w = r.randint(1, c["ctx"]), c["depth"], r.randrange(c["beam"]) if b else c["beam"] - 1
        leave = d if w == 0 else r.randint(0, d - 1) if b else 1
        start = 0 if w == 0 else d + sum(r.randint(1, d) for _ in range(w - 1))      # nodes of the paths before this one
        path = list(range(leave)) + [start + i for i in range(d - leave)]
        out.append((seq, 1 + c["beam"] * d, path[:r.randint(0, d) if b else d]))
    return out


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _teacher_rows(gen, n, V):
    """Logits of n rows in 32 bits: noise with a few likely tokens."""
    x = 2.0 * _rand(gen, n, V)
    few = min(12, V)
    ids = torch.randint(0, V, (n, few), generator=gen, device="cuda")
    x.scatter_add_(1, ids, 4.0 + 3.0 * _rand(gen, n, few).abs())
    return x


def _pool(gen, have, width, spare):
    """A block table with `have` blocks a row, the ring of free blocks, its ends."""
    blocks = sum(have) + spare
    perm = torch.randperm(blocks, generator=gen, device="cuda").int()
    table = torch.zeros((len(have), width), dtype=torch.int32, device="cuda")
    at = torch.arange(width, device="cuda")[None] < _int32(have)[:, None]
    table[at] = perm[:sum(have)]
    head = int(torch.randint(0, blocks, (1,), generator=gen, device="cuda"))
    ring = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(spare, device="cuda")) % blocks] = perm[sum(have):]
    return table, ring, torch.tensor([head, head + spare], dtype=torch.int64, device="cuda")


def _bytes(gen, *shape):
    """Random bytes, eight at a time."""
    n = math.prod(shape)
    w = torch.randint(-(1 << 63), (1 << 63) - 1, (-(-n // 8),), generator=gen, device="cuda", dtype=torch.int64)
    return w.view(torch.uint8)[:n].view(shape)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=c)
    if c["op"] in ("score", "distill"):
        B, L, V, dt = c["B"], c["L"], c["V"], DT[c["dtype"]]
        x = torch.empty((B * L, V), dtype=dt, device="cuda")
        K = min(c["K"], V)
        if c["op"] == "distill":
            s["ids"] = torch.empty((B * L, K), dtype=torch.int32, device="cuda")
            s["top"] = torch.empty((B * L, K), device="cuda")
            s["tlse"] = torch.empty(B * L, device="cuda")
        step = max(1, (1 << 27) // V)
        for lo in range(0, B * L, step):
            n = min(step, B * L - lo)
            t = _teacher_rows(gen, n, V)
            if c["op"] == "distill":
                top = t.topk(K, -1)
                s["ids"][lo:lo + n], s["top"][lo:lo + n] = top.indices.int(), top.values
                s["tlse"][lo:lo + n] = (t / c["T"]).double().logsumexp(-1).float()
                t += 0.8 * _rand(gen, n, V)                                          # the student is near the teacher
            if c.get("masked"):
                t.masked_fill_(torch.rand(n, V, generator=gen, device="cuda") < 0.1, -math.inf)
            x[lo:lo + n] = t.to(dt)
        s["x"] = x.view(B, L, V)
        if c["op"] == "score":
            s["len"] = _int32(_row_lens(c))
            tok = torch.randint(0, V, (B, L, c["G"]), generator=gen, device="cuda").int()
            likely = torch.rand(B, L, generator=gen, device="cuda") < 0.7             # most tokens are ones that the model emitted
            tok[..., 0] = torch.where(likely, s["x"].argmax(-1).int(), tok[..., 0])
            s["tok"] = tok
            return s
        for k, v in (("ids", (B, L, K)), ("top", (B, L, K)), ("tlse", (B, L))):
            s[k] = s[k].view(v)
        r = _of(c)                                                                    # which rows count goes by the case
        on = torch.tensor([1.0 if r.random() >= c["skip"] or i == 0 else 0.0 for i in range(B * L)], device="cuda").view(B, L)
        s["weight"] = on * (0.5 + torch.rand(B, L, generator=gen, device="cuda")) / (B * L)
        return s
    P, H, D, Ly = c["page"], c["Hkv"], c["D"], c["layers"]
    if c["op"] == "fork":
        seq, have, src, keep = _fork_plan(c)
        width = -(-c["ctx"] // P) + 3
        s["table"], s["ring"], s["pos"] = _pool(gen, have, width, _fork_copies(c)[0] + 7)
        s.update(seq=_int32(seq), have=_int32(have), src=_int32(src), keep=_int32(keep))
        s["new_table"] = torch.zeros_like(s["table"])                                # the step's other table
    else:
        trees = _trees(c)
        width = -(-(c["ctx"] + 1 + c["beam"] * c["depth"]) // P) + 1
        s["table"], s["ring"], _ = _pool(gen, [-(-(seq + new) // P) for seq, new, _ in trees], width, 3)
        s["seq"] = _int32([seq for seq, _, _ in trees])
        s["len"] = _int32([len(p) for _, _, p in trees])
        s["node"] = _int32([p + [-1] * (c["depth"] - len(p)) for _, _, p in trees])
    s["cache"] = _bytes(gen, Ly, s["ring"].numel(), H, P * (D + 8))
    return s


# ------------------------------------------------------------------------------------ plain forms
def _best(x, K):
    """The K best of each row, the lowest id first among equals: values and ids."""
    b = x.float().view(torch.int32).long()
    b = torch.where(b == -(1 << 31), torch.zeros_like(b), b)                         # -0 as +0
    order = torch.where(b < 0, -(1 << 31) - b, b)                                     # grows with the value
    key = (order << 32) + (0x7FFFFFFF - torch.arange(x.shape[-1], device=x.device))
    ids = 0x7FFFFFFF - (key.topk(K, -1).values & 0x7FFFFFFF)
    return x.gather(-1, ids), ids


def _plain_score(s):
    c = s["case"]
    B, L, V, K, G = c["B"], c["L"], c["V"], min(c["K"], c["V"]), c["G"]
    rows, toks = s["x"].flatten(0, 1), s["tok"].flatten(0, 1).long()
    out = []
    step = max(1, (1 << 28) // V)
    for lo in range(0, B * L, step):
        x, tok = rows[lo:lo + step].float(), toks[lo:lo + step]
        z = x / c["T"]
        top = z.amax(-1, keepdim=True)
        e = (z - top).exp()
        total = e.sum(-1, keepdim=True, dtype=torch.float64)
        lse = top.double() + total.log()
        mean = torch.where(e > 0, e * (z - top), torch.zeros_like(e)).sum(-1, keepdim=True, dtype=torch.float64) / total
        entropy = total.log() - mean
        mine = x.gather(-1, tok)
        t0, x0 = tok[:, :1], mine[:, :1]
        rank = ((x > x0) | ((x == x0) & (torch.arange(V, device=x.device) < t0))).sum(-1)
        r = [((mine / c["T"]).double() - lse).float(), rank.int(), lse[:, 0].float(), entropy[:, 0].float()]
        if K:
            v, i = _best(x, K)
            none = v == -math.inf
            r += [torch.where(none, torch.full_like(i, -1), i).int(), v, ((v / c["T"]).double() - lse).float()]
        out.append(r)
    off = (torch.arange(L, device="cuda") >= s["len"][:, None])
    out = [torch.cat(t).unflatten(0, (B, L)) for t in zip(*out)]
    for t, pad in zip(out, [-math.inf, -1, -math.inf, 0.0, -1, -math.inf, -math.inf]):
        t[off] = pad
    return out


def _plain_teacher(s, rows):
    """Probabilities of the teacher's tokens and what is left for the others, in 64 bits: near 1 the rest is a small difference."""
    c = s["case"]
    t = s["top"].flatten(0, 1)[rows].double() / c["T"]
    if c["tail"]:
        p = (t - s["tlse"].flatten()[rows].double()[:, None]).exp()
        return p, (1.0 - p.sum(-1)).clamp(min=0.0)
    e = (t - t.amax(-1, keepdim=True)).exp()
    return e / e.sum(-1, keepdim=True), torch.zeros_like(t[:, 0])


def _plain_distill(s):
    c = s["case"]
    B, L, V = c["B"], c["L"], c["V"]
    x, ids, w = s["x"].flatten(0, 1), s["ids"].flatten(0, 1).long(), s["weight"].flatten()
    loss, accept, lse = (torch.empty(B * L, device=x.device) for _ in range(3))
    grad = torch.empty_like(x)
    step = max(1, (1 << 28) // V)
    for lo in range(0, B * L, step):
        rows = torch.arange(lo, min(B * L, lo + step), device=x.device)
        z = x[rows].float() / c["T"]
        top = z.amax(-1, keepdim=True)
        e = (z - top).exp()
        rest = e.scatter(-1, ids[rows], 0.0).sum(-1, dtype=torch.float64)
        mine = e.gather(-1, ids[rows]).double()
        total = rest + mine.sum(-1)
        log_total = total.log() + top[:, 0].double()
        q, tail = mine / total[:, None], rest / total
        p, r = _plain_teacher(s, rows)
        own_log = z.gather(-1, ids[rows]).double() - log_total[:, None]
        kl = torch.where(p > 0, p * (p.log() - own_log), torch.zeros_like(p)).sum(-1)
        kl = kl + torch.where(r > 0, r * (r.log() - tail.log()), torch.zeros_like(r))
        f = w[rows] / c["T"]
        g = e * ((1.0 - r / tail) / total * f).float()[:, None]
        grad[rows] = g.scatter(-1, ids[rows], ((q - p) * f[:, None]).float()).to(x.dtype)
        loss[rows], accept[rows], lse[rows] = kl.float(), (torch.minimum(p, q).sum(-1) + torch.minimum(r, tail)).float(), log_total.float()
    if not c["two"]:                                                                  # rows without weight are not looked at
        off = w == 0
        loss[off], accept[off], lse[off] = 0.0, 0.0, -math.inf
    return [loss.view(B, L), accept.view(B, L), lse.view(B, L), grad.view(B, L, V)]


def _plain_fork(s):
    c = s["case"]
    P, table, blocks = c["page"], s["table"], s["ring"].numel()
    B, W = table.shape
    dev = table.device
    src, keep, have = s["src"].long(), s["keep"].long(), s["have"].long()
    on = src >= 0
    n, full = torch.where(on, (keep + P - 1) // P, 0), keep // P
    e, r = torch.arange(W, device=dev)[None], torch.arange(B, device=dev)[:, None]
    mine = table[src.clamp(min=0)].long()
    held = e < n[:, None]
    # who has a page: -1 if somebody has all of it, else the lowest row that has a part of it
    holder = torch.full((blocks,), NONE, dtype=torch.int64, device=dev)
    holder.scatter_reduce_(0, mine[held], torch.where(e < full[:, None], -1, r)[held], "amin")
    last = mine.gather(1, full.clamp(max=W - 1)[:, None])[:, 0]
    need = on & (n > full) & (holder[last] != r[:, 0])
    fresh = s["ring"].long()[(s["pos"][0] + need.cumsum(0) - 1) % blocks]
    out = torch.where(need[:, None] & (e == full[:, None]), fresh[:, None], mine)
    new_table = torch.where(held, out.int(), s["new_table"])
    minus = torch.full_like(last, -1)
    copy_src, copy_dst = torch.where(need, last, minus), torch.where(need, fresh, minus)
    copy_len = torch.where(need, keep - full * P, torch.zeros_like(keep))
    # pages that were held and are not any more, each once
    was = e < have[:, None]
    at = (r * W + e)[was]
    page = table[was].long()
    first = torch.full((blocks,), NONE, dtype=torch.int64, device=dev).scatter_reduce_(0, page, at, "amin")
    back = page[(holder[page] == NONE) & (first[page] == at)]
    ring = s["ring"].clone()
    ring[(s["pos"][1] + torch.arange(len(back), device=dev)) % blocks] = back.int()
    pos = s["pos"] + torch.stack([need.sum(), torch.tensor(len(back), device=dev)])
    # the copied pages' runs that hold tokens, in every layer
    cache = s["cache"].unflatten(-1, (P // 16, -1))
    i = need.nonzero()[:, 0]
    some = (torch.arange(P // 16, device=dev) * 16 < copy_len[i][:, None])[None, :, None, :, None]
    cache[:, copy_dst[i]] = torch.where(some, cache[:, copy_src[i]], cache[:, copy_dst[i]])
    return [new_table, n.int(), torch.where(on, keep, 0).int(), ring, pos, copy_src.int(), copy_dst.int(), copy_len.int(),
            torch.zeros_like(n).int(), s["cache"]]


def _places(D):
    """Bytes of each of a run's 16 tokens, [16, D + 8]: its key's codes, its value's codes, its four numbers."""
    rows = []
    for t in range(16):
        c, half = (t % 8) // 2, t // 8
        if D == 128:
            words = [t * 64 + 4 * w for w in range(16)] + [1024 + half * 512 + (w // 2) * 64 + c * 16 + (t % 2) * 8 + (w % 2) * 4 for w in range(16)]
        else:
            words = [(t % 8) * 64 + (w // 2) * 16 + half * 8 + (w % 2) * 4 for w in range(8)]
            words += [512 + w * 64 + c * 16 + half * 8 + (t % 2) * 4 for w in range(8)]
        words += [16 * D + 8 * t, 16 * D + 8 * t + 4]
        rows.append([w + i for w in words for i in range(4)])
    return torch.tensor(rows, device="cuda")


def _plain_compact(s):
    c = s["case"]
    P, D, H, Ly = c["page"], c["D"], c["Hkv"], c["layers"]
    i = torch.arange(c["depth"], device="cuda")[None]
    there = (i < s["len"][:, None]) & (s["node"] != i)
    b = there.nonzero()[:, 0]
    start = s["seq"].long()[:, None] + 1
    off = _places(D)

    def bytes_of(at):                       # flat places in a layer of all bytes of the tokens at these positions: [tokens, Hkv, D + 8]
        block = s["table"].long()[b, at // P]
        run = (block[:, None] * H + torch.arange(H, device="cuda")) * (P // 16) + ((at % P) // 16)[:, None]
        return run[..., None] * (16 * (D + 8)) + off[at % 16][:, None]

    old, new = bytes_of((start + s["node"])[there]), bytes_of((start + i).expand_as(there)[there])
    for layer in s["cache"].view(Ly, -1):
        layer[new] = layer[old]
    return [s["cache"]]


# ------------------------------------------------------------------------------- the framework's
def _own_run(s):
    from paper_2510_02358_b200 import binding as dsp
    c = s["case"]
    if c["op"] == "score":
        r = dsp.dsp_token_logprobs(s["x"], s["tok"], K=min(c["K"], c["V"]), temperature=c["T"], row_len=s["len"])
        return [r.logp, r.rank, r.lse, r.entropy] + ([r.top_id, r.top_logit, r.top_logp] if c["K"] else [])
    if c["op"] == "distill":
        list_ = dict(teacher_lse=s["tlse"] if c["tail"] else None, temperature=c["T"])
        if c["two"]:
            r = dsp.dsp_distill(s["x"], s["ids"], s["top"], **list_)
            return [r.loss, r.accept, r.lse, dsp.dsp_distill_grad(s["x"], s["ids"], r.state, s["weight"], temperature=c["T"])]
        r = dsp.dsp_distill(s["x"], s["ids"], s["top"], weight=s["weight"], grad=True, **list_)
        return [r.loss, r.accept, r.lse, r.grad]
    if c["op"] == "fork":
        r = dsp.dsp_cache_fork(s["src"], s["keep"], s["seq"], s["have"], s["pos"], s["table"], s["ring"], c["page"], s["new_table"])
        dsp.dsp_kv4_copy(s["cache"], c["D"], r.copy_src, r.copy_dst, r.copy_len)
        return [s["new_table"], r.block_count, r.seq_len, s["ring"], r.ring_pos, r.copy_src, r.copy_dst, r.copy_len, r.row_status, s["cache"]]
    dsp.dsp_kv4_compact(s["cache"], c["D"], s["table"], s["seq"], s["node"], s["len"])
    return [s["cache"]]


PLAIN = {"score": _plain_score, "distill": _plain_distill, "fork": _plain_fork, "compact": _plain_compact}


def run(state):
    return _own_run(state) if own else PLAIN[state["case"]["op"]](state)


# --------------------------------------------------------------------------------- floor and truth
def work(case):
    c = case
    if c["op"] == "score":
        n, es = sum(_row_lens(c)), 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * (c["V"] * es + c["G"] * 4) + c["B"] * c["L"] * (c["G"] * 4 + 12 + 12 * c["K"]), "flops": 4 * n * c["V"]}
    if c["op"] == "distill":
        r = _of(c)
        n = sum(r.random() >= c["skip"] or i == 0 for i in range(c["B"] * c["L"]))
        es, all_rows = 2 if c["dtype"] == "bf16" else 4, c["B"] * c["L"]
        read = all_rows + n if c["two"] else n                                        # twice: the factors come after the loss
        return {"bytes": (read + all_rows) * c["V"] * es + n * c["K"] * 8 + all_rows * 20, "flops": 8 * n * c["V"]}
    if c["op"] == "fork":
        copies, tokens, before, after, back = _fork_copies(c)
        runs = sum(-(-t // 16) for t in tokens)
        return {"bytes": 4 * (before + after + back) + 40 * c["B"] + 2 * runs * 16 * (c["D"] + 8) * c["Hkv"] * c["layers"], "flops": 0}
    moved = sum(sum(n != i for i, n in enumerate(path)) for _, _, path in _trees(c))
    return {"bytes": 2 * moved * (c["D"] + 8) * c["Hkv"] * c["layers"] + c["B"] * (8 + 4 * c["depth"]), "flops": 0}


def _exact_score(case, s):
    c = case
    n_of, K, V = _row_lens(c), min(c["K"], c["V"]), c["V"]
    B, L, G = c["B"], c["L"], c["G"]
    f64 = dict(dtype=torch.float64, device="cuda")
    logp, lse, entropy = torch.full((B, L, G), -math.inf, **f64), torch.full((B, L), -math.inf, **f64), torch.zeros((B, L), **f64)
    rank = torch.full((B, L), -1, dtype=torch.int32, device="cuda")
    top_id = torch.full((B, L, K), -1, dtype=torch.int32, device="cuda")
    top_x, top_p = torch.full((B, L, K), -math.inf, **f64), torch.full((B, L, K), -math.inf, **f64)
    for b in range(B):
        for lo in range(0, n_of[b], 64):
            at = slice(lo, min(n_of[b], lo + 64))
            x = s["x"][b, at].double()
            logs = torch.log_softmax(x / c["T"], -1)
            lse[b, at] = torch.logsumexp(x / c["T"], -1)
            entropy[b, at] = -(logs.exp() * logs.masked_fill(x == -math.inf, 0.0)).sum(-1)
            tok = s["tok"][b, at].long()
            logp[b, at] = logs.gather(-1, tok)
            x0 = x.gather(-1, tok[:, :1])
            before = torch.arange(V, device="cuda") < tok[:, :1]
            rank[b, at] = ((x > x0).sum(-1) + ((x == x0) & before).sum(-1)).int()
            if K:
                v, i = torch.sort(x, dim=-1, descending=True, stable=True)
                v, i = v[:, :K], i[:, :K]
                top_id[b, at], top_x[b, at] = i.int().masked_fill(v == -math.inf, -1), v
                top_p[b, at] = logs.gather(-1, i)
    return [logp, rank, lse, entropy] + ([top_id, top_x, top_p] if K else [])


def _exact_distill(case, s):
    c = case
    B, L, V = c["B"], c["L"], c["V"]
    x, ids = s["x"].view(B * L, V), s["ids"].view(B * L, -1).long()
    f64 = dict(dtype=torch.float64, device="cuda")
    loss, accept, lse = torch.zeros(B * L, **f64), torch.zeros(B * L, **f64), torch.full((B * L,), -math.inf, **f64)
    grad = torch.zeros((B * L, V), **f64)
    w = s["weight"].view(-1).double()
    for lo in range(0, B * L, 64):
        at = slice(lo, min(B * L, lo + 64))
        logs = torch.log_softmax(x[at].double() / c["T"], -1)
        q_all = logs.exp()
        t = s["top"].view(B * L, -1)[at].double() / c["T"]
        logp = t - s["tlse"].view(-1)[at].double()[:, None] if c["tail"] else torch.log_softmax(t, -1)
        p = logp.exp()
        r = (1.0 - p.sum(-1)).clamp(min=0.0) if c["tail"] else torch.zeros_like(p[:, 0])
        inside = torch.zeros_like(q_all, dtype=torch.bool).scatter(-1, ids[at], True)
        tail = q_all.masked_fill(inside, 0.0).sum(-1)
        q = q_all.gather(-1, ids[at])
        loss[at] = (p * (logp - logs.gather(-1, ids[at]))).sum(-1) + torch.special.xlogy(r, r / tail)
        accept[at] = torch.minimum(p, q).sum(-1) + torch.minimum(r, tail)
        lse[at] = torch.logsumexp(x[at].double() / c["T"], -1)
        g = q_all * (1.0 - r / tail)[:, None]
        grad[at] = g.scatter(-1, ids[at], q - p) * (w[at] / c["T"])[:, None]
    if not c["two"]:
        off = w == 0
        loss[off], accept[off], lse[off] = 0.0, 0.0, -math.inf
    return [loss.view(B, L), accept.view(B, L), lse.view(B, L), grad.view(B, L, V)]


def exact(case, seed):
    if case["op"] in ("fork", "compact"):                # whole numbers: tables, lengths and the cache's bytes, moved as they are
        return None
    s = prepare(case, seed)
    return _exact_score(case, s) if case["op"] == "score" else _exact_distill(case, s)
