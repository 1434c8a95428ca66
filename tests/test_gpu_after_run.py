"""What follows a verified step, run together: in the example, and recorded in one graph."""
import os
import sys

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [False, True])
def test_forked_requests_go_on_with_the_greedy_text(tree):
    """As for the example's text: where it parts from plain decoding, the two tokens' logits are within 0.125."""
    import draft_and_verify as ex
    tokens, length = ex.prompts(4, 60, 5)
    plain, drafted = ex.Decoder(4, 300), ex.Decoder(4, 300)
    for d in (plain, drafted):
        d.prompt(tokens, length)
    for _ in range(4):
        drafted.step(tree)
    src = [0, 0, 3, 1]
    drafted.fork(src)
    starts = [len(t) for t in drafted.texts]
    for _ in range(4):
        drafted.step(tree)
    while min(map(len, plain.texts)) < max(map(len, drafted.texts)):
        plain.plain_step()
    for b in range(4):
        want, got = plain.texts[src[b]], drafted.texts[b]
        assert len(got) > starts[b]
        part = next((i for i, (x, y) in enumerate(zip(want, got)) if x != y), None)
        if part is not None:
            logits = plain.margins[src[b]][part - 1]
            assert part > 0 and float(logits[want[part]] - logits[got[part]]) < 0.125, (b, part)
    for pool in (drafted.target.pool, drafted.drafter.pool):
        count, (head, tail) = pool.block_count.tolist(), pool.ring_pos.tolist()
        held = [pool.block_table[b, :count[b]].tolist() for b in range(4)]
        free = [int(pool.free_ring[i % pool.free_ring.numel()]) for i in range(head, tail)]
        every = set(sum(held, []))                                 # shared blocks are held by several
        assert len(set(free)) == len(free) and not every & set(free) and len(every) + len(free) == pool.free_ring.numel()
        assert len(every) < len(sum(held, []))                     # rows 0 and 1 share the prompt's blocks


@pytest.mark.parametrize("tree", [False, True])
def test_the_lesson_has_the_formulas_loss_and_gradients(tree):
    import draft_and_verify as ex
    d = ex.Decoder(3, 200)
    d.prompt(*ex.prompts(3, 50, 6))
    for _ in range(2):
        d.step(tree)
        r = d.lesson(K=12, temperature=1.5)
        logits, hidden = d.drafted
        n = (r.weight > 0).sum(1).int()
        rows = torch.arange(d.L, device="cuda") < n[:, None]
        x = d.rows.double()
        top = x.sort(dim=-1, descending=True, stable=True)
        assert torch.equal(r.teacher.top_id[rows].long(), top.indices[..., :12][rows])
        loss, accept, _, grad = ref.distill(logits, r.teacher.top_id, r.teacher.top_logit, 1.5, (x / 1.5).logsumexp(-1), None, r.weight)
        tol = 4 * ref.exponent_error(logits, 1.5, ref.terms(ex.VOCAB)) + 2.0 ** -20      # the teacher's log-sum-exp is in 32 bits: 2^-24 of it
        assert ((r.loss - loss).abs() <= tol).all() and ((r.accept - accept).abs() <= tol).all()
        assert ((r.grad - grad).abs() <= tol[..., None] * r.weight[..., None] + 2.0 ** -23 * grad.abs()).all()
        head = hidden.flatten(0, 1).double().t() @ grad.flatten(0, 1)
        assert ((r.head - head).abs().max() <= 2.0 ** -9 * head.abs().max())               # the product may run in TF32 (2^-11 a factor)
        d.drafter.head -= 0.1 * r.head


def test_a_recorded_run_follows_its_inputs():
    """Compaction, a fork with its copies, scores and a distillation in one graph, replayed while lengths, sources and logits change."""
    g = torch.Generator(device="cuda").manual_seed(1)
    B, L, K, V, H, D, page, width, layers = 4, 6, 8, 5003, 2, 64, 16, 9, 3
    i32 = dict(dtype=torch.int32, device="cuda")
    blocks = B * width + 6
    table = torch.arange(B * width, **i32).view(B, width)
    free_ring, ring_pos = torch.arange(blocks, **i32), torch.tensor([B * width, blocks], device="cuda")
    count, seq = torch.full((B,), 7, **i32), torch.tensor([70, 33, 50, 96], **i32)
    node, length = torch.tensor([[0, 1, 7, 8, -1, -1]] * B, **i32), torch.tensor([4, 2, 3, 0], **i32)
    src, new_table = torch.tensor([0, 0, -1, 3], **i32), torch.zeros(B, width, **i32)
    cache = torch.randint(0, 256, (layers, blocks, H, page * (D + 8)), dtype=torch.uint8, device="cuda", generator=g)
    target, draft = torch.randn(B, L, V, device="cuda", generator=g), torch.randn(B, L, V, device="cuda", generator=g)
    tokens = torch.randint(0, V, (B, L), device="cuda", generator=g, dtype=torch.int32)
    rows = torch.tensor([6, 3, 0, 1], **i32)
    weight = torch.rand(B, L, device="cuda", generator=g)

    def run():
        dsp.dsp_kv4_compact(cache, D, table, seq, node, length)
        f = dsp.dsp_cache_fork(src, None, seq + 1 + length, count, ring_pos, table, free_ring, page, new_table)
        dsp.dsp_kv4_copy(cache, D, f.copy_src, f.copy_dst, f.copy_len)
        t = dsp.dsp_token_logprobs(target, tokens, K=K, row_len=rows)
        r = dsp.dsp_distill(draft, t.top_id, t.top_logit, teacher_lse=t.lse, weight=weight, grad=True)
        return [f.block_count, f.seq_len, f.ring_pos, f.copy_dst, f.row_status, t.logp, t.top_id, t.lse, r.loss, r.grad, new_table, free_ring, cache]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = [t.clone() for t in (cache, free_ring, new_table)]

    def back():
        for t, k in zip((cache, free_ring, new_table), keep):
            t.copy_(k)

    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for step in range(3):
        seq.copy_(torch.randint(0, 100, (B,), device="cuda", generator=g, dtype=torch.int32))
        src.copy_(torch.randint(-1, B, (B,), device="cuda", generator=g, dtype=torch.int32))
        rows.copy_(torch.randint(0, L + 1, (B,), device="cuda", generator=g, dtype=torch.int32))
        target.copy_(torch.randn(B, L, V, device="cuda", generator=g))
        weight[step] = 0.0
        back()
        graph.replay()
        got = [t.clone() for t in out]
        back()
        want = [t.clone() for t in run()]
        for i, (x, y) in enumerate(zip(got, want)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (step, i)


def test_calls_on_other_streams_do_not_disturb_one_another():
    """Two runs of each call under way at once, on streams of their own: workspaces are not shared."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x = [torch.randn(6, 40, 32003, device="cuda", generator=g) for _ in range(2)]
    t = [torch.randint(0, 32003, (6, 40), device="cuda", generator=g, dtype=torch.int32) for _ in range(2)]
    want = [dsp.dsp_token_logprobs(a, b, K=5) for a, b in zip(x, t)]
    lists = [(w.top_id, w.top_logit, w.lse) for w in want]
    want_d = [dsp.dsp_distill(a, i, v, teacher_lse=l, grad=True) for a, (i, v, l) in zip(reversed(x), lists)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got, got_d = [], []
        for k in range(2):
            got.append(dsp.dsp_token_logprobs(x[k], t[k], K=5, stream=streams[k]))
            i, v, l = lists[k]
            got_d.append(dsp.dsp_distill(x[1 - k], i, v, teacher_lse=l, grad=True, stream=streams[k]))
        torch.cuda.synchronize()
        for k in range(2):
            for name in ("logp", "rank", "top_id", "lse", "entropy"):
                assert torch.equal(getattr(got[k], name), getattr(want[k], name)), name
            assert torch.equal(got_d[k].grad, want_d[k].grad) and torch.equal(got_d[k].loss, want_d[k].loss)
