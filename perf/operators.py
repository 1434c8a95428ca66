"""The target pass around the draft-and-verify step: cases for timing and comparison.

A speculative step runs a model over the block that it drafts or verifies.  The operators here are
that pass's own: the bookkeeping of a paged cache (`plan`), the norm of every query and key head with
its position rotation (`norm_rope`), the same with keys and values stored in 4 bits (`append`, read
back as values), and attention over the 4-bit cache (`attend`).

`run(state)` computes an operator by elementary torch operations in 32 bits, or, where `own` is true,
by the framework's calls.  `exact(case, seed)` is the definition in 64 bits.

The cache is uint8 [blocks, Hkv, page * (D + 8)].  A page is cut into runs of 16 tokens of 16 * (D + 8)
bytes each: the keys' codes, the values' codes, and for every token the four bf16 numbers (key scale,
key offset, value scale, value offset); a value is code * scale + offset, with codes 0 .. 15.
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
TINY = 2.0 ** -126
NO_BLOCKS, TABLE_FULL, PLAN_FULL, BAD_LENGTH = 64, 128, 256, 512


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # eight conversations, each about to verify a chain of drafted tokens: pure latency, once a step
        dict(name="plan_8", op="plan", B=8, ctx=2048, new=17, page=16, nodes=0, beam=0),
        # sixteen requests that verify a beam tree of up to 8 x 16 nodes: positions by depth, visibility bits
        dict(name="plan_tree_16", op="plan", B=16, ctx=4096, new=129, page=64, nodes=128, beam=8),
        # a full server: a thousand requests with long contexts, some of them reading in a prompt
        dict(name="plan_1024", op="plan", B=1024, ctx=32768, new=128, page=64, nodes=0, beam=0),
        # the queries and keys of a verified block of 16 x 17 tokens, 40 query heads on 8 key heads
        dict(name="norm_rope_272", op="norm_rope", T=272, Hq=40, Hkv=8, D=128, rot=128, inter=False, dtype="bf16"),
        # fp32 activations, odd head counts, neighbouring pairs rotated, half of the channels only
        dict(name="norm_rope_f32", op="norm_rope", T=8191, Hq=15, Hkv=3, D=64, rot=32, inter=True, dtype="f32"),
        # one token of one request enters the cache
        dict(name="append_1", op="append", T=1, Hq=40, Hkv=8, D=128, rot=128, inter=False, dtype="bf16", page=16),
        # a prompt's chunk enters the cache
        dict(name="append_8192", op="append", T=8192, Hq=40, Hkv=8, D=128, rot=128, inter=False, dtype="bf16", page=64),
        # one token of one short conversation
        dict(name="attend_1", op="attend", B=1, q=1, kv=500, Hq=40, Hkv=8, D=128, page=16, mask="causal"),
        # plain decoding of 64 requests of up to 16384 tokens
        dict(name="attend_64", op="attend", B=64, q=1, kv=16384, Hq=40, Hkv=8, D=128, page=64, mask="causal"),
        # verification of a beam tree of up to 8 x 8 nodes behind the last kept token
        dict(name="attend_tree", op="attend", B=16, q=65, kv=8192, Hq=40, Hkv=8, D=128, page=64, mask="tree"),
        # the drafter's block, seen from both sides, as many key heads as query heads
        dict(name="attend_draft", op="attend", B=64, q=32, kv=1023, Hq=16, Hkv=16, D=64, page=32, mask="full"),
        # a chunk of a long prompt over what is cached of it
        dict(name="attend_chunk", op="attend", B=2, q=2048, kv=8200, Hq=40, Hkv=8, D=128, page=128, mask="causal"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "norm_rope", "append", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    if op == "plan":
        if rng.random() < 0.3:
            beam, depth = rng.randint(2, 8), rng.randint(3, 16)
            return dict(op=op, B=_spread(rng, 1, 64), ctx=_spread(rng, 100, 32768), new=1 + beam * depth, page=page,
                        nodes=beam * depth, beam=beam)
        return dict(op=op, B=_spread(rng, 1, 1024), ctx=_spread(rng, 100, 32768), new=_spread(rng, 1, 128), page=page,
                    nodes=0, beam=0)
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 5, 7, 8])
    if op in ("norm_rope", "append"):
        c = dict(op=op, T=_spread(rng, 1, 4096), Hq=Hq, Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2]),
                 inter=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f32"]))
        return dict(c, page=page) if op == "append" else c
    mask = rng.choice(["causal", "causal", "causal", "full", "tree"])
    if mask == "causal" and rng.random() < 0.5:
        q, kv, B = 1, _spread(rng, 1, 16384), _spread(rng, 1, 64)              # single tokens
    elif mask == "causal" and rng.random() < 0.4:
        q, kv, B = _spread(rng, 129, 2048), _spread(rng, 2048, 8192), rng.randint(1, 2)   # prompts
    else:
        q, kv, B = _spread(rng, 2, 128), _spread(rng, 128, 8192), _spread(rng, 1, 16)     # blocks
    return dict(op=op, B=B, q=q, kv=max(kv, q), Hq=Hq, Hkv=Hkv, D=D, page=page, mask=mask)


# ----------------------------------------------------------------------------------------- inputs
def _lens(c):
    """Lengths go by the case's values alone, so that its work is known without its inputs: (new tokens, all tokens) of each request."""
    r = random.Random("%s" % sorted((k, v) for k, v in c.items() if k != "name"))
    new, kv = [], []
    for b in range(c["B"]):
        n = c["q"] if b == 0 or c["q"] <= 2 else r.randint(max(1, c["q"] // 2), c["q"])
        new.append(n)
        kv.append(c["kv"] if b == 0 else max(n, r.randint(c["kv"] // 4, c["kv"])))
    return new, kv


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _table(max_pos, rot):
    f = 1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(max_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


def _parents(g, B, beam, nodes):
    """Trees as a beam leaves them: every node's parent is an earlier one (-1: the last kept token), with its depth."""
    depth_of = max(1, nodes // beam)
    par = torch.arange(nodes) - 1
    par = par.expand(B, nodes).clone()
    dep = (torch.arange(nodes) % depth_of).expand(B, nodes).clone()
    r = torch.rand((B, nodes), generator=g)
    for w in range(beam):                      # beam w leaves the first path at a random depth of its own
        lo = w * depth_of
        par[:, lo] = -1 if w == 0 else (r[:, lo] * depth_of).long() - 1
        dep[:, lo:lo + depth_of] = par[:, lo:lo + 1] + 1 + torch.arange(depth_of)
    return par.int(), dep.int()


def _visible(par, n, words):
    """Bits of the tokens that each of a tree's tokens sees: itself and those before it on its path; token 0 is the last kept one."""
    rows = [1]
    for i in range(n - 1):
        rows.append(rows[int(par[i]) + 1] | (2 << i))
    return [[(m >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for m in rows]


def _signed(words):
    return torch.tensor([[w - (1 << 32) if w >= 1 << 31 else w for w in row] for row in words], dtype=torch.int32)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    cpu = torch.Generator()
    cpu.manual_seed(seed)
    s = dict(case=c)
    if c["op"] == "plan":
        B, P = c["B"], c["page"]
        r = random.Random("%s" % sorted((k, v) for k, v in c.items() if k != "name"))
        seq = [r.randint(1, c["ctx"]) for _ in range(B)]
        if c["nodes"]:
            new = [1 + r.randint(c["nodes"] // 2, c["nodes"]) for _ in range(B)]
        else:
            new = [r.randint(0, c["new"]) if b else c["new"] for b in range(B)]
        # what the last step left: room for its own drafted tokens, so that some rows give blocks back
        have = [-(-(q + r.randint(-min(q, 2 * P), c["new"] // 2)) // P) for q in seq]
        width = -(-(c["ctx"] + c["new"]) // P) + 4
        blocks = sum(have) + sum(-(-n // P) + 3 for n in new) + 8
        perm = torch.randperm(blocks, generator=gen, device="cuda").int()
        s["table"] = torch.zeros((B, width), dtype=torch.int32, device="cuda")
        at = torch.arange(width, device="cuda")[None] < torch.tensor(have, device="cuda")[:, None]
        s["table"][at] = perm[:sum(have)]
        head = int(torch.randint(0, blocks, (1,), generator=cpu))
        free = blocks - sum(have)
        s["ring"] = torch.zeros(blocks, dtype=torch.int32, device="cuda")
        s["ring"][(head + torch.arange(free, device="cuda")) % blocks] = perm[sum(have):]
        t = lambda v, dt=torch.int32: torch.tensor(v, dtype=dt, device="cuda")  # noqa: E731
        s.update(seq=t(seq), new=t(new), have=t(have), pos=t([head, head + free], torch.int64), T=sum(new) + 5)
        if c["nodes"]:
            par, dep = _parents(cpu, B, c["beam"], c["nodes"])
            s.update(parent=par.cuda(), depth=dep.cuda(), words=-(-c["new"] // 32))
        return s
    dt = DT[c.get("dtype", "bf16")]
    D, Hq, Hkv = c["D"], c["Hq"], c["Hkv"]
    if c["op"] in ("norm_rope", "append"):
        T = c["T"]
        qkv = _rand(gen, T, Hq + 2 * Hkv, D)                       # one projection's output
        qkv[:, Hq:Hq + Hkv] *= 1.0 + 3.0 * (torch.rand(Hkv, D, generator=gen, device="cuda") < 0.03)
        s["qkv"] = qkv.to(dt)
        s["wq"] = (1.0 + 0.2 * _rand(gen, D)).to(dt)
        s["wk"] = (1.0 + 0.2 * _rand(gen, D)).to(dt)
        s["table"] = _table(16384, c["rot"])
        start = int(torch.randint(0, 16384 - T + 1, (1,), generator=cpu))
        s["positions"] = torch.arange(start, start + T, dtype=torch.int32, device="cuda")
        if c["op"] == "append":
            P = c["page"]
            blocks = -(-T // P) + 9
            s["cache"] = torch.zeros((blocks, Hkv, P * (D + 8)), dtype=torch.uint8, device="cuda")
            perm = torch.randperm(blocks, generator=gen, device="cuda")
            i = torch.arange(T, device="cuda") + (start % P)
            s["slot"] = perm[i // P] * P + i % P
        return s
    B, P = c["B"], c["page"]
    new, kv = _lens(c)
    width = -(-c["kv"] // P) + 1
    used = [-(-n // P) for n in kv]
    blocks = sum(used) + 3
    perm = torch.randperm(blocks, generator=gen, device="cuda").int()
    s["table"] = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    at = torch.arange(width, device="cuda")[None] < torch.tensor(used, device="cuda")[:, None]
    s["table"][at] = perm[:sum(used)]
    gain = 1.0 + 2.0 * (torch.rand(Hkv, 1, D, generator=gen, device="cuda") < 0.03)     # a few strong key channels
    s["cache"] = torch.empty((blocks, Hkv, P * (D + 8)), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (Hkv * P * D))
    for lo in range(0, blocks, step):
        n = min(step, blocks - lo)
        s["cache"][lo:lo + n] = _packed(_rand(gen, n, Hkv, P, D) * gain, _rand(gen, n, Hkv, P, D))
    s["q"] = _rand(gen, sum(new), Hq, D).to(dt)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s["cu"] = torch.tensor([0] + new, device="cuda").cumsum(0).int()
    if c["mask"] == "tree":
        words = -(-c["q"] // 32)
        par, _ = _parents(cpu, B, 8 if c["q"] > 16 else 2, c["q"] - 1) if c["q"] > 2 else (torch.full((B, 2), -1), None)
        s["bits"] = _signed([w for b in range(B) for w in _visible(par[b], new[b], words)]).cuda()
    return s


# ------------------------------------------------------------------------- the 4-bit form, plainly
def _bf16_up(x):
    """The smallest bf16 number that is not below x >= 0."""
    return ((x.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)


def _bf16_down(x):
    """The largest bf16 number that is not above x."""
    b = x.view(torch.int32)
    return torch.where(b < 0, (b + 0xFFFF) & -65536, b & -65536).view(torch.float32)


def _quantised(x):
    """Codes 0 .. 15 with one scale and one offset for a token's head: x [..., D] in 32 bits."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    z = _bf16_down(lo)
    s = _bf16_up((hi - z) / torch.full_like(z, 15.0))      # by a tensor: torch divides by a number through its inverse
    bad = ~(torch.isfinite(x).all(-1, keepdim=True) & torch.isfinite(s) & torch.isfinite(z))
    s = torch.where(s < TINY, torch.zeros_like(s), s)
    code = torch.where(s > 0, (x - z) / s, torch.zeros_like(x)).round().clamp(0, 15)
    nan = torch.full_like(s, math.nan)
    return torch.where(bad, torch.zeros_like(code), code).to(torch.uint8), torch.where(bad, nan, s), torch.where(bad, nan, z)


def _nibbles(code):
    """[..., D] codes to [..., D / 2] bytes: of eight channels, 0 2 4 6 are the low half of a word and 1 3 5 7 its high half."""
    w = code.unflatten(-1, (-1, 4, 2)).transpose(-1, -2).flatten(-2).unflatten(-1, (4, 2))
    return (w[..., 0] | (w[..., 1] << 4)).flatten(-2)


def _codes(b):
    """The inverse of _nibbles."""
    n = torch.stack([b & 15, b >> 4], -1).flatten(-2).unflatten(-1, (-1, 2, 4))
    return n.transpose(-1, -2).flatten(-3)


def _key_order(b, D, into):
    """Bytes of 16 tokens' keys, [..., 16, D / 2], in their place in the cache ([..., 8 * D]), or back."""
    if D == 128:
        return b.flatten(-2) if into else b.unflatten(-1, (16, 64))
    if into:
        return b.unflatten(-2, (2, 8)).unflatten(-1, (4, 8)).movedim(-4, -2).flatten(-4)
    return b.unflatten(-1, (8, 4, 2, 8)).movedim(-2, -4).flatten(-2).flatten(-3, -2)


def _value_order(b, D, into):
    """The same for values: tokens 2c, 2c+1, 2c+8, 2c+9 of an eighth of the channels lie together."""
    n = D // 16
    if into:
        t = b.unflatten(-2, (2, 4, 2)).unflatten(-1, (8, n))              # half, c, pair, r, byte
        t = t.permute(*range(t.dim() - 5), -5, -2, -4, -3, -1) if D == 128 else t.permute(*range(t.dim() - 5), -2, -4, -5, -3, -1)
        return t.flatten(-5)
    if D == 128:
        t = b.unflatten(-1, (2, 8, 4, 2, n))                               # half, r, c, pair, byte
        t = t.permute(*range(t.dim() - 5), -5, -3, -2, -4, -1)
    else:
        t = b.unflatten(-1, (8, 4, 2, 2, n))                               # r, c, half, pair, byte
        t = t.permute(*range(t.dim() - 5), -3, -4, -2, -5, -1)
    return t.flatten(-2).flatten(-4, -2)


def _runs(k, v):
    """Keys and values of runs of 16 tokens, [..., 16, D] in 32 bits, as the cache holds them: [..., 16 * (D + 8)] bytes."""
    D = k.shape[-1]
    kc, ks, kz = _quantised(k)
    vc, vs, vz = _quantised(v)
    par = torch.cat([ks, kz, vs, vz], -1).to(torch.bfloat16).view(torch.uint8).flatten(-2)
    return torch.cat([_key_order(_nibbles(kc), D, True), _value_order(_nibbles(vc), D, True), par], -1)


def _packed(k, v):
    """Whole pages, [..., page, D], as the cache holds them."""
    return _runs(k.unflatten(-2, (-1, 16)), v.unflatten(-2, (-1, 16))).flatten(-2)


def _values(run, D):
    """Keys and values in 32 bits, [..., 16, D] each, of runs of 16 tokens."""
    par = run[..., 16 * D:].unflatten(-1, (16, 8)).contiguous().view(torch.bfloat16).float()
    k = _codes(_key_order(run[..., :8 * D], D, False)).float() * par[..., 0:1] + par[..., 1:2]
    v = _codes(_value_order(run[..., 8 * D:16 * D], D, False)).float() * par[..., 2:3] + par[..., 3:4]
    return k, v


# ------------------------------------------------------------------------------------ plain forms
def _plain_plan(s):
    P, T, table, ring = s["case"]["page"], s["T"], s["table"], s["ring"]
    blocks, width = ring.numel(), table.shape[1]
    seq, new, have = s["seq"].long(), s["new"].long(), s["have"].long()
    zero = torch.zeros_like(seq)
    bad = (seq < 0) | (new < 0) | (have < 0) | (have > width)
    if "parent" in s:
        bad = bad | (new > s["parent"].shape[1] + 1)
    need = (seq + new + P - 1) // P
    full = ~bad & (need > width)
    new = torch.where(bad | full, zero, new)
    over = ~bad & ~full & (new > 0) & (new.cumsum(0) > T)
    new = torch.where(over, zero, new)
    ok = ~(bad | full | over)
    take = torch.where(ok, (need - have).clamp(min=0), zero)
    free = s["pos"][1] - s["pos"][0]
    miss = (take > 0) & (take.cumsum(0) > free)
    take, new, ok = torch.where(miss, zero, take), torch.where(miss, zero, new), ok & ~miss
    drop = torch.where(ok, (have - need).clamp(min=0), zero)
    status = bad * BAD_LENGTH + full * TABLE_FULL + over * PLAN_FULL + miss * NO_BLOCKS
    held = have.clamp(0, width)
    count = held + take - drop
    # new entries come from the ring's head, in the requests' order; what a row no longer needs goes to its tail
    e = torch.arange(width, device=seq.device)[None]
    rank = (take.cumsum(0) - take)[:, None] + e - have[:, None]
    fresh = (e >= have[:, None]) & (e < (have + take)[:, None])
    table2 = torch.where(fresh, ring[((s["pos"][0] + rank) % blocks)], table)
    back = (e >= need[:, None]) & (e < (need + drop)[:, None])
    rank = (drop.cumsum(0) - drop)[:, None] + e - need[:, None]
    ring2 = ring.clone()
    ring2[((s["pos"][1] + rank) % blocks)[back]] = table[back]
    pos2 = s["pos"] + torch.stack([take.sum(), drop.sum()])
    cu = torch.cat([zero[:1], new.cumsum(0)])
    t = torch.arange(T, device=seq.device)
    row = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    there = t < cu[-1]
    row = torch.where(there, row, torch.zeros_like(row))
    i = t - cu[row]
    at = torch.where(there, seq[row] + i, torch.zeros_like(i))
    slot = torch.where(there, table2[row, at // P].long() * P + at % P, torch.full_like(at, -1))
    position = at
    out = [count.int(), pos2, table2, ring2, cu.int(), (seq.clamp(min=0) + new).int(), slot]
    if "parent" in s:
        nodes = s["parent"].shape[1]
        node = (i - 1).clamp(0, nodes - 1)
        position = torch.where(i > 0, seq[row] + 1 + s["depth"][row, node], position)
        # paths as products of the parents' matrix: token j is seen by token i if it is on i's way to the root
        step = torch.zeros((seq.numel(), nodes + 1, nodes + 1), device=seq.device)
        n = torch.arange(nodes, device=seq.device)
        up = torch.where((s["parent"] >= 0) & (s["parent"] < n), s["parent"], torch.full_like(s["parent"], -1)).long()
        step[torch.arange(seq.numel(), device=seq.device)[:, None], n + 1, up + 1] = 1.0
        eye = torch.eye(nodes + 1, device=seq.device)
        reach = step + eye
        for _ in range(max(1, nodes).bit_length()):
            reach = ((reach @ reach) > 0).float()
        bits = torch.nn.functional.pad(reach, (0, 32 * s["words"] - nodes - 1)).long().unflatten(-1, (s["words"], 32))
        word = (bits << torch.arange(32, device=seq.device)).sum(-1)
        word = torch.where(word >= 1 << 31, word - (1 << 32), word).int()
        mask = torch.where(there[:, None], word[row, i.clamp(0, nodes)], torch.zeros_like(word[0, :1]))
        out.append(mask)
    minus = torch.full_like(at, -1)
    return out + [torch.where(there, position, minus).int(), torch.where(there, row, minus).int(), status.int()]


def _plain_norm_rope(x, w, s):
    """x [T, H, D]: x / sqrt(mean x^2 + eps) * w, then the rotation of its first channels; 32 bits in and out."""
    x = x.float()
    sq = x * x
    while sq.shape[-1] > 1:                    # the sum over the channels as a tree of neighbours
        sq = sq[..., 0::2] + sq[..., 1::2]
    x = (x * (1.0 / (sq * (1.0 / x.shape[-1]) + EPS).sqrt())) * w.float()
    rot = s["case"]["rot"]
    cs = s["table"][s["positions"].long()][:, None]
    c, n = cs[..., :rot // 2], cs[..., rot // 2:]
    if s["case"]["inter"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _split(s):
    c = s["case"]
    return s["qkv"].split([c["Hq"], c["Hkv"], c["Hkv"]], 1)


def _plain_append(s):
    """Queries normed and rotated; the keys' and values' 4-bit forms, read back as the values they stand for."""
    q, k, v = _split(s)
    out = [_plain_norm_rope(q, s["wq"], s).to(q.dtype)]
    for x in (_plain_norm_rope(k, s["wk"], s).to(k.dtype).float(), v.float()):
        code, scale, off = _quantised(x)
        out.append((code.float() * scale + off).to(q.dtype))
    return out


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hkv, D, P = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    cu, kv = s["cu"].long(), s["kv_len"].long()
    run = s["cache"][s["table"].long()].unflatten(-1, (P // 16, -1)).transpose(1, 2)     # [B, Hkv, width, P / 16, bytes]
    k, v = (t.flatten(2, 4) for t in _values(run, D))                                    # [B, Hkv, S, D]
    n, nq = k.shape[2], c["q"]
    i = torch.arange(nq, device=cu.device)
    new = cu[1:] - cu[:-1]
    there = i[None] < new[:, None]
    at = (cu[:-1, None] + i).clamp(max=cu[-1] - 1)
    q = s["q"].float()[at].unflatten(2, (Hkv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [B, Hkv, nq * g, D]
    t = torch.arange(n, device=cu.device)
    see = (t < kv[:, None])[:, None].expand(B, nq, n)
    first = (kv - new)[:, None, None]
    if c["mask"] == "causal":
        see = see & (t <= first + i[None, :, None])
    if c["mask"] == "tree":
        j = (t - first).expand(B, nq, n)
        word = s["bits"][at].gather(2, (j // 32).clamp(0, s["bits"].shape[1] - 1))
        see = see & ((j < 0) | (((word >> (j % 32).int()) & 1) != 0))
    see = see & there[:, :, None]
    score = (q @ k.transpose(2, 3)).unflatten(2, (nq, -1)) * (1.0 / math.sqrt(D))
    score.masked_fill_(~see[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = score.sum(-1, keepdim=True)
    v = torch.where((t < kv[:, None])[:, None, :, None], v, torch.zeros_like(v[:1, :1, :1, :1]))   # pages end inside a run
    o = (score.flatten(2, 3) @ v).unflatten(2, (nq, -1)) / torch.where(total == 0, torch.ones_like(total), total)
    return o.permute(0, 2, 1, 3, 4).flatten(2, 3)[there].to(s["q"].dtype)


# ------------------------------------------------------------------------------- the framework's
def _own_run(s):
    from paper_2510_02358_b200 import binding as dsp
    c = s["case"]
    if c["op"] == "plan":
        tree = dict(node_parent=s["parent"], node_depth=s["depth"], mask_words=s["words"]) if "parent" in s else {}
        r = dsp.dsp_cache_plan(s["seq"], s["new"], s["have"], s["pos"], s["table"], s["ring"], c["page"], s["T"], **tree)
        out = [r.block_count, r.ring_pos, s["table"], s["ring"], r.cu_new, r.kv_len, r.slot]
        return out + ([r.mask] if tree else []) + [r.position, r.token_row, r.row_status]
    if c["op"] == "attend":
        mask = s["bits"] if c["mask"] == "tree" else c["mask"]
        return dsp.dsp_attn_kv4(s["q"], s["cache"], s["table"], s["kv_len"], s["cu"], c["q"], mask=mask)
    q, k, v = _split(s)
    rope = dict(q_weight=s["wq"], k_weight=s["wk"], eps=EPS, positions=s["positions"], cos_sin=s["table"], interleaved=c["inter"])
    if c["op"] == "norm_rope":
        return dsp.dsp_qk_norm_rope(q, k, **rope)
    q = dsp.dsp_kv4_append(q, k, v, s["slot"], s["cache"], **rope)
    return (q,) + tuple(dsp.dsp_kv4_read(s["cache"], s["slot"], c["D"], q.dtype))


def run(state):
    if own:
        r = _own_run(state)
        return list(r) if isinstance(r, (list, tuple)) else [r]
    op = state["case"]["op"]
    if op == "plan":
        return _plain_plan(state)
    if op == "attend":
        return [_plain_attend(state)]
    if op == "append":
        return _plain_append(state)
    q, k, _ = _split(state)
    return [_plain_norm_rope(q, state["wq"], state).to(q.dtype), _plain_norm_rope(k, state["wk"], state).to(k.dtype)]


# --------------------------------------------------------------------------------- floor and truth
def work(case):
    c = case
    if c["op"] == "plan":
        r = random.Random("%s" % sorted((k, v) for k, v in c.items() if k != "name"))
        [r.randint(1, c["ctx"]) for _ in range(c["B"])]
        if c["nodes"]:
            total = sum(1 + r.randint(c["nodes"] // 2, c["nodes"]) for _ in range(c["B"]))
        else:
            total = sum(r.randint(0, c["new"]) if b else c["new"] for b in range(c["B"]))
        tree = c["B"] * c["nodes"] * 8 + total * 4 * -(-c["new"] // 32) if c["nodes"] else 0
        return {"bytes": c["B"] * 24 + total * 16 + 8 * (total // c["page"]) + tree, "flops": 0}
    D, Hq, Hkv = c["D"], c["Hq"], c["Hkv"]
    if c["op"] in ("norm_rope", "append"):
        e = 2 if c["dtype"] == "bf16" else 4
        heads = 2 * (Hq + Hkv) * D * e + c["rot"] * 4 + 4
        if c["op"] == "append":     # keys and values come in, leave in 4 bits, are read in 4 bits and leave as values
            heads = (2 * Hq + 2 * Hkv) * D * e + c["rot"] * 4 + 4 + 8 + 2 * Hkv * (D + 8) + 2 * Hkv * D * e
        return {"bytes": c["T"] * heads, "flops": c["T"] * (Hq + Hkv) * D * 8}
    new, kv = _lens(c)
    pairs = 0
    for n, m in zip(new, kv):
        pairs += n * m - (n * (n - 1) // 2 if c["mask"] != "full" else 0)
    return {"bytes": sum(kv) * Hkv * (D + 8) + 2 * sum(new) * Hq * D * 2, "flops": 4 * D * Hq * pairs}


def _byte_of(token, channel, D):
    """Where the codes of a key and of a value lie within a run of 16 tokens: (byte, shift) of the key, byte of the value."""
    word, odd, pair = channel // 8, channel % 2, (channel % 8) // 2
    nib = pair + 4 * odd
    inside, shift = nib // 2, 4 * (nib % 2)
    at = word * 4 + inside                                        # byte of the token's own row
    r, tk, half = at // (D // 16), token % 2, token // 8
    c, low = (token % 8) // 2, at % (D // 16)
    if D == 128:
        return token * 64 + at, shift, 1024 + half * 512 + r * 64 + c * 16 + tk * 8 + low
    return (token % 8) * 64 + (at // 8) * 16 + half * 8 + at % 8, shift, 512 + r * 64 + c * 16 + half * 8 + tk * 4 + low


def _exact_rows(cache, table, n, D, P):
    """Keys and values of a request's first n tokens in 64 bits, [Hkv, n, D], from the cache's bytes one by one."""
    t = torch.arange(n, device="cuda")
    run = table[t // P].long() * (P // 16) + (t % P) // 16
    rows = cache.view(cache.shape[0], cache.shape[1], P // 16, -1).transpose(1, 2).flatten(0, 1)[run]   # [n, Hkv, bytes]
    kb, shift, vb = _byte_of((t % 16)[:, None], torch.arange(D, device="cuda")[None], D)
    rows = rows.transpose(0, 1)
    pick = lambda at: (rows.gather(2, at.expand(rows.shape[0], n, D)).int() >> shift) & 15  # noqa: E731
    p = 16 * D + 8 * (t % 16)
    num = rows.gather(2, (p[:, None] + torch.arange(8, device="cuda")).expand(rows.shape[0], n, 8)).view(torch.bfloat16).double()
    return pick(kb).double() * num[..., 0:1] + num[..., 1:2], pick(vb).double() * num[..., 2:3] + num[..., 3:4]


def _exact_norm_rope(x, w, s):
    c = s["case"]
    x = x.double()
    x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    half = c["rot"] // 2
    first = 2 * torch.arange(half, device="cuda") if c["inter"] else torch.arange(half, device="cuda")
    second = first + (1 if c["inter"] else half)
    cos, sin = s["table"][s["positions"].long()].double()[:, None].chunk(2, -1)
    y = x.clone()
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def _exact_kept(x, dt):
    """What a token's head becomes in 4 bits: x in the type that it is stored from."""
    x = x.to(dt).double()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)

    def rounded(v, up):
        m = torch.frexp(v).mantissa
        unit = torch.where(m == 0, torch.ones_like(v), v / m / 256.0)      # the last place of v's 8 bits: a power of two
        return ((v / unit).ceil() if up else (v / unit).floor()) * unit

    z = rounded(lo, False)
    s = rounded((hi - z) / 15.0, True)
    return ((x - z) / s).round().clamp(0, 15) * s + z


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    if case["op"] in ("norm_rope", "append"):
        q, k, v = _split(s)
        dt = q.dtype
        q, k = _exact_norm_rope(q, s["wq"], s), _exact_norm_rope(k, s["wk"], s)
        return [q, k] if case["op"] == "norm_rope" else [q, _exact_kept(k, dt), _exact_kept(v, dt)]
    c = case
    new, kv = _lens(c)
    D, g, P, out, lo = c["D"], c["Hq"] // c["Hkv"], c["page"], [], 0
    for b, (n, m) in enumerate(zip(new, kv)):
        k, v = _exact_rows(s["cache"], s["table"][b], m, D, P)
        for at in range(0, n, 256):
            rows = torch.arange(at, min(n, at + 256), device="cuda")
            q = s["q"][lo + rows].double().unflatten(1, (c["Hkv"], g))                    # [rows, Hkv, g, D]
            score = torch.einsum("rhgd,hnd->rhgn", q, k) / math.sqrt(D)
            t = torch.arange(m, device="cuda")
            hide = torch.zeros((len(rows), m), dtype=torch.bool, device="cuda")
            if c["mask"] == "causal":
                hide = t[None] > (m - n + rows)[:, None]
            if c["mask"] == "tree":
                j = torch.arange(n, device="cuda")
                hide[:, m - n:] = ((s["bits"][lo + rows][:, j // 32].long() >> (j % 32)) & 1) == 0
            p = score.masked_fill(hide[:, None, None], -math.inf).softmax(-1)
            out.append(torch.einsum("rhgn,hnd->rhgd", p, v).flatten(1, 2))
        lo += n
    return [torch.cat(out)]
