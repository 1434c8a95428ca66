"""A whole pass (plan, norm, rotation, store, attention) in one CUDA graph, replayed while its requests' lengths move.

What a replay writes has to be, bit for bit, what the same calls write outside of a graph on the same inputs.
"""
import numpy as np
import pytest
import torch

import pass_reference as ref
from paper_2510_02358_b200 import binding as dsp

DEV = "cuda"


class Pass:
    """One layer's pass over up to T new tokens of B requests; every buffer is made once."""

    def __init__(self, B, T, max_new, nodes, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.Hq, self.Hkv, self.D, self.page, self.width = 8, 2, 64, 16, 24
        self.B, self.T, self.max_new, self.nodes = B, T, max_new, nodes
        n = B * self.width
        i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
        self.seq, self.new = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.count, self.ring_pos = torch.zeros(B, **i32), torch.tensor([0, n], **i64)
        self.table, self.ring = torch.zeros((B, self.width), **i32), torch.randperm(n, generator=g, device=DEV).int()
        self.parent, self.depth = (torch.zeros((B, nodes), **i32) for _ in range(2)) if nodes else (None, None)
        self.cache = dsp.kv4_cache(n, self.Hkv, self.D, self.page, DEV)
        self.x = torch.zeros((T, self.Hq + 2 * self.Hkv, self.D), dtype=torch.bfloat16, device=DEV)
        self.w = (1 + torch.randn(self.D, generator=g, device=DEV) / 8).bfloat16()
        a = torch.arange(1000, device=DEV)[:, None] * 1e4 ** (-torch.arange(0, self.D, 2, device=DEV) / self.D)
        self.cs = torch.cat([a.cos(), a.sin()], 1).float()

    def run(self):
        q, k, v = self.x.split([self.Hq, self.Hkv, self.Hkv], 1)
        p = dsp.dsp_cache_plan(self.seq, self.new, self.count, self.ring_pos, self.table, self.ring, self.page, self.T,
                               node_parent=self.parent, node_depth=self.depth)
        rope = dict(q_weight=self.w, k_weight=self.w, positions=p.position, cos_sin=self.cs)
        normed = dsp.dsp_qk_norm_rope(q, k, **rope)
        stored = dsp.dsp_kv4_append(q, k, v, p.slot, self.cache, **rope)
        out = dsp.dsp_attn_kv4(stored, self.cache, self.table, p.kv_len, p.cu_new, self.max_new, mask=p.mask if self.nodes else "causal")
        return p, normed, stored, dsp.dsp_kv4_read(self.cache, p.slot, self.D), out


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,max_new,nodes", [(3, 12, 4, 0), (2, 90, 60, 0), (4, 60, 17, 16), (1, 5, 5, 0)])
def test_a_recorded_pass_follows_its_lengths(B, T, max_new, nodes):
    r = np.random.default_rng(T)
    graphed, plain = (Pass(B, T, max_new, nodes, 5) for _ in range(2))
    graphed.run()                                                  # first calls are made outside of a graph
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = graphed.run()
    graphed.cache.zero_()
    seq = np.zeros(B, dtype=int)
    for step in range(8):
        new = r.integers(0, max_new + 1, B)
        while new.sum() > T:
            new[r.integers(0, B)] = 0
        if step == 3:
            new[:] = 0
        x = torch.tensor(r.normal(size=plain.x.shape), dtype=torch.bfloat16)
        parent = np.array([[r.integers(-1, i) if i else -1 for i in range(nodes)] for _ in range(B)]) if nodes else None
        for p in (graphed, plain):
            p.seq.copy_(torch.tensor(seq)), p.new.copy_(torch.tensor(new)), p.x.copy_(x)
            if nodes:
                p.parent.copy_(torch.tensor(parent)), p.depth.copy_(torch.tensor(np.maximum(parent, 0)))
        graph.replay()
        want = plain.run()
        torch.cuda.synchronize()
        n = int(new.sum())
        for name in ("block_count", "ring_pos", "cu_new", "kv_len", "slot", "position", "token_row", "row_status"):
            assert torch.equal(getattr(got[0], name), getattr(want[0], name)), name
        assert not want[0].row_status.any() and want[0].cu_new.tolist() == [0] + np.cumsum(new).tolist()
        for a, b in zip((*got[1], got[2], *got[3], got[4][:n]), (*want[1], want[2], *want[3], want[4][:n])):
            assert torch.equal(a, b)
        assert torch.equal(graphed.cache, plain.cache) and torch.isfinite(want[4][:n]).all()
        for p, w in ((graphed, got[0]), (plain, want[0])):
            p.count.copy_(w.block_count), p.ring_pos.copy_(w.ring_pos)
        seq = seq + np.minimum(new, r.integers(0, max_new + 1, B))                  # a part of the new tokens is kept
    held = [plain.table[b, :int(plain.count[b])].tolist() for b in range(B)]
    head, tail = plain.ring_pos.tolist()
    free = [int(plain.ring[i % plain.ring.numel()]) for i in range(head, tail)]
    assert sorted(sum(held, free)) == list(range(plain.ring.numel()))
    if not nodes:                                                  # and the last step's attention is the definition's
        D = plain.D
        want_o = ref.attend(ref.to_numpy(want[2][:n]), plain.cache.cpu().numpy(), plain.page, D, plain.table.tolist(), want[0].kv_len.tolist(),
                            want[0].cu_new.tolist(), D ** -0.5, "causal")
        assert n == 0 or np.linalg.norm(ref.to_numpy(want[4][:n]) - want_o) <= 3.5e-3 * np.linalg.norm(want_o)
