"""Draft-and-verify decoding with a small target and a small drafter, both with random weights.

One step, whose lengths stay on the device (the host reads the emitted tokens, and with a tree whether any
accepted node lies off the first beam): the drafter sees its block of masks from both sides over its cache
("full" attention), its logits become a lattice and a path (or the beams' token tree), the target passes
over the path ("causal") or the tree (the plan's visibility bits) once, the verification accepts a part (a
tree's accepted nodes move behind the last kept token), and the lengths move by it; what was drafted beyond is
written over by the next step.  Between steps a request may fork or end (`fork`), and the drafter may learn from
the target's rows of the last verification (`lesson`).

    dsp_cache_plan -> projections -> dsp_kv4_append -> dsp_attn_kv4 -> ... -> logits
    dsp_lattice_build -> dsp_cps_search (-> dsp_beam_tree) -> dsp_verify / dsp_verify_tree (-> dsp_kv4_compact)
    dsp_cache_fork -> dsp_kv4_copy
    dsp_token_logprobs (the teacher's list) -> dsp_distill (loss and gradient)

The projections are PyTorch matrix products.  Both models lean towards one fixed chain of tokens, which
stands in for what training would have taught them to agree on.

    python examples/draft_and_verify.py [--tree] [--fork] [--learn] [--steps 16] [--batch 4]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from types import SimpleNamespace

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2510_02358_b200 import binding as dsp  # noqa: E402

VOCAB, WIDTH, LAYERS, HQ, HKV, D, PAGE = 2048, 512, 2, 8, 2, 64, 16
MASK = VOCAB - 1                                   # the drafter's mask token


class Pool:
    """The cache of one model's layers and what dsp_cache_plan keeps about it."""

    def __init__(self, B: int, max_tokens: int, dev):
        width = -(-max_tokens // PAGE)
        n = B * width
        i32 = dict(dtype=torch.int32, device=dev)
        self.block_table, self.free_ring = torch.zeros((B, width), **i32), torch.arange(n, **i32)
        self.ring_pos = torch.tensor([0, n], dtype=torch.int64, device=dev)
        self.block_count, self.seq_len = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.cache = dsp.kv4_cache(n, HKV, D, PAGE, dev, LAYERS)
        self.layers = list(self.cache)

    def plan(self, new_len: torch.Tensor, T: int, tree: SimpleNamespace = None) -> SimpleNamespace:
        p = dsp.dsp_cache_plan(self.seq_len, new_len, self.block_count, self.ring_pos, self.block_table, self.free_ring, PAGE, T,
                               node_parent=tree.node_parent if tree else None, node_depth=tree.node_depth if tree else None)
        self.block_count, self.ring_pos = p.block_count, p.ring_pos
        return p

    def fork(self, src: torch.Tensor):
        """Row r continues what row src[r] holds (-1: it ends)."""
        table = torch.empty_like(self.block_table)
        f = dsp.dsp_cache_fork(src, None, self.seq_len, self.block_count, self.ring_pos, self.block_table, self.free_ring, PAGE, table)
        dsp.dsp_kv4_copy(self.cache, D, f.copy_src, f.copy_dst, f.copy_len)
        self.block_table, self.block_count, self.seq_len, self.ring_pos = table, f.block_count, f.seq_len, f.ring_pos
        return f


class Model:
    def __init__(self, seed: int, B: int, max_tokens: int, dev, lean: float):
        g = torch.Generator(device=dev).manual_seed(seed)
        w = lambda *shape: (torch.randn(shape, generator=g, device=dev) / math.sqrt(shape[0])).to(torch.bfloat16)
        self.embed = torch.randn((VOCAB, WIDTH), generator=g, device=dev).to(torch.bfloat16)
        self.head = w(WIDTH, VOCAB).float()
        self.layers = [SimpleNamespace(qkv=w(WIDTH, (HQ + 2 * HKV) * D), out=w(HQ * D, WIDTH), up=w(WIDTH, 2 * WIDTH), down=w(2 * WIDTH, WIDTH),
                                       q_norm=torch.ones(D, device=dev, dtype=torch.bfloat16), k_norm=torch.ones(D, device=dev, dtype=torch.bfloat16))
                       for _ in range(LAYERS)]
        angle = torch.arange(max_tokens, device=dev)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device=dev) / D)
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
        self.pool = Pool(B, max_tokens, dev)
        self.lean = lean

    @staticmethod
    def norm(x: torch.Tensor) -> torch.Tensor:
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)

    def forward(self, tokens: torch.Tensor, new_len: torch.Tensor, mask="causal", tree=None) -> torch.Tensor:
        """The new tokens ``tokens`` [B, n] (the first new_len[b] of each row) over the cache; logits fp32 [B, n, VOCAB]."""
        B, n = tokens.shape
        p = self.pool.plan(new_len, B * n, tree)
        row = p.token_row.clamp_min(0).long()
        place = (torch.arange(B * n, device=tokens.device) - p.cu_new[row]).clamp(0, n - 1)
        x = self.embed[tokens[row, place].long()]
        for w, cache in zip(self.layers, self.pool.layers):
            q, k, v = (self.norm(x) @ w.qkv).view(B * n, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
            q = dsp.dsp_kv4_append(q, k, v, p.slot, cache, q_weight=w.q_norm, k_weight=w.k_norm, positions=p.position, cos_sin=self.cos_sin)
            o = dsp.dsp_attn_kv4(q, cache, self.pool.block_table, p.kv_len, p.cu_new, n, mask=p.mask if tree else mask)
            x = x + o.view(B * n, HQ * D) @ w.out
            x = x + torch.nn.functional.silu(self.norm(x) @ w.up) @ w.down
        at = (p.cu_new[:-1, None] + torch.arange(n, device=tokens.device)).clamp_max(B * n - 1).long()
        self.hidden = self.norm(x)[at].float()
        return self.hidden @ self.head

    def leaning(self, logits: torch.Tensor, to: torch.Tensor) -> torch.Tensor:
        return logits.scatter_add(-1, to[..., None].long(), torch.full(to.shape + (1,), self.lean, device=to.device))


class Decoder:
    """Greedy decoding of B requests, by drafting or (``plain_step``) token by token."""

    def __init__(self, B: int, max_tokens: int, seed: int = 0, L: int = 8, K: int = 4, W: int = 4, dev="cuda"):
        self.L, self.K, self.W, self.B, self.dev = L, K, W, B, dev
        self.target, self.drafter = Model(seed, B, max_tokens, dev, 5.0), Model(seed + 1, B, max_tokens, dev, 5.0)
        g = torch.Generator(device=dev).manual_seed(seed + 2)
        self.chain = torch.randperm(VOCAB - 1, generator=g, device=dev).int()
        self.chain = torch.cat([self.chain, self.chain[:1]])                        # and something for the mask
        self.proxy = -8.0 * torch.rand(1 << 10, generator=g, device=dev)
        self.texts = [[] for _ in range(B)]
        self.margins = [[] for _ in range(B)]                                      # plain_step: the logits, for comparisons
        self.on = torch.ones(B, dtype=torch.bool, device=dev)                      # requests that go on: the places of the others are empty

    def emit(self, tokens: torch.Tensor, count: torch.Tensor):
        count = count * self.on
        self.pending, self.pending_len = tokens, count                             # what the drafter has not seen yet
        self.last = tokens.gather(1, (count - 1).clamp_min(0)[:, None].long())[:, 0]
        for b, (t, c) in enumerate(zip(tokens.tolist(), count.tolist())):
            self.texts[b] += t[:c]

    def prompt(self, tokens: torch.Tensor, new_len: torch.Tensor):
        logits = self.target.leaning(self.target.forward(tokens, new_len), self.chain[tokens.long()])
        self.target.pool.seq_len = self.target.pool.seq_len + new_len
        first = logits[torch.arange(self.B), new_len.long() - 1].argmax(-1).int()
        joined = torch.cat([tokens, first[:, None]], 1).scatter(1, new_len[:, None].long(), first[:, None])
        self.emit(first[:, None], torch.ones_like(new_len))
        self.pending, self.pending_len = joined, new_len + 1

    def plain_step(self):
        tokens = self.last[:, None]
        one = self.on.int()
        logits = self.logits(self.target.forward(tokens, one), tokens)[:, 0]
        self.target.pool.seq_len = self.target.pool.seq_len + one
        for b in range(self.B):
            self.margins[b].append(logits[b])
        self.emit(logits.argmax(-1).int()[:, None], one)

    def logits(self, logits: torch.Tensor, tokens: torch.Tensor) -> torch.Tensor:
        """The target's, with its leaning; zeros for requests that have ended, which no row was computed for."""
        return self.target.leaning(logits.masked_fill(~self.on[:, None, None], 0.0), self.chain[tokens.long()])

    def draft(self):
        n = self.pending.shape[1] + self.L
        at = torch.arange(n, device=self.dev)[None]
        tokens = torch.nn.functional.pad(self.pending, (0, self.L), value=MASK).masked_fill(at >= self.pending_len[:, None], MASK)
        logits = self.drafter.forward(tokens, (self.pending_len + self.L) * self.on, mask="full")
        self.drafter.pool.seq_len = self.drafter.pool.seq_len + self.pending_len   # the masks are not kept
        block = (self.pending_len[:, None] + torch.arange(self.L, device=self.dev)).long()
        guess = [self.chain[self.last.long()]]
        for _ in range(self.L - 1):
            guess.append(self.chain[guess[-1].long()])
        off = ~self.on[:, None, None]                                              # no rows were computed for these
        logits = logits.gather(1, block[..., None].expand(-1, -1, VOCAB)).masked_fill(off, 0.0)
        logits = self.drafter.leaning(logits, torch.stack(guess, 1))
        self.drafted = logits, self.drafter.hidden.gather(1, block[..., None].expand(-1, -1, WIDTH)).masked_fill(off, 0.0)
        lat = dsp.dsp_lattice_build(logits, self.K)
        cps = dsp.dsp_cps_search(lat, self.last, self.proxy, W=self.W, lam=0.9, table_log2=10, V=VOCAB, row_status=lat.row_status)
        return lat, cps

    def step(self, tree: bool = False) -> torch.Tensor:
        """Drafts, verifies, emits; returns the accepted lengths [B]."""
        lat, cps = self.draft()
        pool, last = self.target.pool, self.last[:, None]
        if not tree:
            tokens = torch.cat([last, cps.path.clamp_min(0)], 1)
            logits = self.logits(self.target.forward(tokens, (1 + cps.path_len) * self.on), tokens)
            ver = dsp.dsp_verify(logits, None, cps, None, all_greedy=True, row_status=lat.row_status)
            accepted, path = ver.accepted_len * self.on, cps.path
        else:
            t = dsp.dsp_beam_tree(cps)
            tokens = torch.cat([last, t.node_token.clamp_min(0)], 1)
            logits = self.logits(self.target.forward(tokens, (1 + t.n_nodes) * self.on, tree=t), tokens)
            ver = dsp.dsp_verify_tree(logits, t, self.L)
            accepted = ver.accepted_len * self.on
            path = t.node_token.gather(1, ver.accepted_node.clamp_min(0).long())
            dsp.dsp_kv4_compact(pool.cache, D, pool.block_table, pool.seq_len, ver.accepted_node, accepted)
        self.rows, self.path, self.right = logits[:, :self.L], cps.path, (cps.path == path).int().cumprod(1).sum(1).minimum(accepted)
        pool.seq_len = pool.seq_len + (1 + accepted) * self.on
        new = torch.cat([path.clamp_min(0), path[:, :1]], 1).scatter(1, accepted[:, None].long(), ver.next_token[:, None])
        self.emit(new, accepted + 1)
        return accepted

    def fork(self, src):
        """Request r goes on from where request src[r] is (-1: it ends, and its place stays empty until a later fork takes it)."""
        src_t = torch.tensor(src, dtype=torch.int32, device=self.dev)
        for pool in (self.target.pool, self.drafter.pool):
            pool.fork(src_t)
        at = src_t.clamp_min(0).long()
        self.on = self.on[at] & (src_t >= 0)
        self.last, self.pending, self.pending_len = self.last[at], self.pending[at], self.pending_len[at] * self.on
        self.texts = [list(self.texts[s]) if s >= 0 else [] for s in src]
        self.margins = [list(self.margins[s]) if s >= 0 else [] for s in src]

    def lesson(self, K: int = 16, temperature: float = 1.0) -> SimpleNamespace:
        """What the drafter can learn from the last step: its block against the target's rows of the best path, whose positions count up to
        the first token that the target did not take.  Returns loss and accept [B, L] and the gradient for the drafter's head."""
        logits, hidden = self.drafted
        n = (self.right + 1).clamp_max(self.L).int() * self.on                     # rows that follow accepted tokens
        teacher = dsp.dsp_token_logprobs(self.rows, self.path, K=K, temperature=temperature, row_len=n)
        weight = (torch.arange(self.L, device=self.dev) < n[:, None]).float() / n.sum()
        r = dsp.dsp_distill(logits, teacher.top_id, teacher.top_logit, teacher_lse=teacher.lse, weight=weight, temperature=temperature, grad=True)
        return SimpleNamespace(loss=r.loss, accept=r.accept, weight=weight, teacher=teacher, grad=r.grad,
                               head=hidden.flatten(0, 1).t() @ r.grad.flatten(0, 1))


def prompts(B: int, longest: int, seed: int, dev="cuda"):
    g = torch.Generator(device=dev).manual_seed(seed)
    tokens = torch.randint(0, VOCAB - 1, (B, longest), generator=g, device=dev, dtype=torch.int32)
    length = torch.randint(1, longest + 1, (B,), generator=g, device=dev, dtype=torch.int32)
    length[0] = longest
    return tokens, length


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tree", action="store_true", help="verify the beams' token tree instead of the best path")
    ap.add_argument("--fork", action="store_true", help="halfway, the last request ends and its place goes on from the first one")
    ap.add_argument("--learn", action="store_true", help="after every step the drafter's head learns from the target's rows")
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--batch", type=int, default=4)
    a = ap.parse_args()
    d = Decoder(a.batch, 128 + a.steps * 9 + 64)
    d.prompt(*prompts(a.batch, 100, 7))
    for s in range(a.steps):
        if a.fork and s == a.steps // 2:
            d.fork(list(range(a.batch - 1)) + [0])
        print("step %2d: accepted %s" % (s, d.step(a.tree).tolist()))
        if a.learn:
            r = d.lesson()
            d.drafter.head -= 0.5 * r.head
            print("         loss %.4f, acceptance within %.3f" % (float((r.loss * r.weight).sum()), float((r.accept * r.weight).sum())))
    for b, text in enumerate(d.texts):
        print("request %d: %d tokens in %d steps: %s ..." % (b, len(text), a.steps, text[:12]))


if __name__ == "__main__":
    main()
