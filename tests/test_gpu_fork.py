"""dsp_cache_fork, dsp_kv4_copy and dsp_kv4_compact against lists and bytes on the host."""
import random

import pytest
import torch

import after_reference as ref
from paper_2510_02358_b200 import binding as dsp

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def pool(r, lens, page, width, spare, extra=1):
    """Tables of rows with their own blocks, the ring of `spare` free ones in the middle of its way round."""
    have = [min(width, -(-n // page) + r.randint(0, extra)) for n in lens]
    n = sum(have) + spare
    blocks = list(range(n))
    r.shuffle(blocks)
    table, at = [], 0
    for h in have:
        table.append(blocks[at:at + h] + [-7] * (width - h))
        at += h
    head = r.randrange(3 * n)
    ring = [-5] * n
    for i, p in enumerate(blocks[at:]):
        ring[(head + i) % n] = p
    return have, table, ring, [head, head + spare]


def run(src, keep, seq, have, pos, table, ring, page, width, out_rows=None):
    Bo = len(src)
    new = [[-9] * width for _ in range(Bo)]
    want = ref.fork(src, keep, seq, have, pos, table, ring, page, new)
    dev_ring, dev_new = i32(ring), i32(new).view(Bo, width)
    args = (i32(src), None if keep is None else i32(keep), i32(seq), i32(have), torch.tensor(pos, device="cuda"), i32(table).view(len(seq), width))
    for _ in range(2):                                                   # a call may be repeated on its inputs
        r = dsp.dsp_cache_fork(*args, dev_ring, page, dev_new)
        got = dict(table=dev_new.tolist(), block_count=r.block_count.tolist(), seq_len=r.seq_len.tolist(), ring=dev_ring.tolist(),
                   ring_pos=r.ring_pos.tolist(), copy_src=r.copy_src.tolist(), copy_dst=r.copy_dst.tolist(), copy_len=r.copy_len.tolist(),
                   row_status=r.row_status.tolist())
        for k in want:
            assert got[k] == want[k], k
    return want


@pytest.mark.parametrize("B,longest,page", [(1, 5, 16), (3, 100, 16), (8, 700, 16), (64, 3000, 16), (300, 5000, 32), (1000, 2000, 128), (5, 40, 1), (2, 9000, 7)])
@pytest.mark.parametrize("seed", range(3))
def test_forks_ends_and_moves(B, longest, page, seed):
    r = random.Random(seed)
    lens = [r.randint(0, longest) for _ in range(B)]
    width = -(-longest // page) + 2
    have, table, ring, pos = pool(r, lens, page, width, r.randint(1, B + 5))
    Bo = r.choice([B, 2 * B + 1, max(1, B // 2)])
    src = [r.choice([-1, r.randrange(B), r.randrange(B)]) for _ in range(Bo)]
    keep = [r.choice([lens[s], r.randint(0, lens[s])]) if s >= 0 else r.randint(-3, 3) for s in src]
    first = run(src, keep, lens, have, pos, table, ring, page, width)
    # rows that share blocks fork again, and shrink into what they share
    lens, have, table, ring, pos = first["seq_len"], first["block_count"], first["table"], first["ring"], first["ring_pos"]
    src = [r.choice([-1, r.randrange(Bo), b % Bo]) for b in range(B)]
    keep = [r.choice([lens[s], r.randint(0, lens[s])]) if s >= 0 else 0 for s in src]
    second = run(src, keep, lens, have, pos, table, ring, page, width)
    # every block is either held or free, none is both or lost
    n = len(ring)
    held = {p for t, c in zip(second["table"], second["block_count"]) for p in t[:c]}
    free = [second["ring"][i % n] for i in range(*second["ring_pos"])]
    lacked = any(s == ref.NO_BLOCKS for s in first["row_status"] + second["row_status"])
    assert len(set(free)) == len(free) and not held & set(free) and (lacked or len(held) + len(free) == n)
    run(src, None, lens, have, pos, table, ring, page, width)


def test_rows_that_cannot_be_served():
    page, width = 16, 6
    table = [[0, 1, 2, -7, -7, -7], [3, 99, 4, -7, -7, -7], [5, -1, 6, -7, -7, -7], [7, 8, -7, -7, -7, -7], [9, -7, -7, -7, -7, -7]]
    seq, have = [40, 40, 40, 40, -4], [3, 3, 3, 2, 9]
    ring, pos = [10, 11] + [0] * 10, [0, 2]
    #      good  bad row  bad row  too long  bad block  before it  few blocks  negative  copies, until the ring is empty
    src = [0, 5, -2, 0, 1, 1, 3, 4, 0, 0, 0, 2]
    keep = [40, 1, 1, 41, 40, 16, 40, 0, 39, 38, 37, 8]
    want = run(src, keep, seq, have, pos, table, ring, page, width)
    assert want["row_status"] == [0, 512, 512, 512, 1024, 0, 512, 512, 0, 0, 64, 0]
    run([0], [-1], seq, have, pos, table, ring, page, width)
    run([-1] * 3, None, seq, have, pos, table, ring, page, width)


def test_the_same_block_in_two_input_rows_returns_once():
    table = [[0, 1, 2], [0, 1, 3], [0, 4, 4]]
    run([-1], None, [48, 48, 48], [3, 3, 3], [3, 3], table, [9] * 8, 16, 3)
    run([1, 1], [20, 33], [48, 48, 48], [3, 3, 3], [3, 5], table, [5, 5, 5, 6, 7, 5, 5, 5], 16, 3)


def test_no_rows_on_one_side():
    run([], None, [17], [2], [0, 1], [[0, 1]], [2, 0, 0], 16, 2)
    got = dsp.dsp_cache_fork(i32([-1, -1]), None, i32([]), i32([]), torch.tensor([4, 6], device="cuda"), i32([]).view(0, 2), i32([0, 1]), 16,
                             torch.zeros(2, 2, dtype=torch.int32, device="cuda"))
    assert got.block_count.tolist() == [0, 0] and got.ring_pos.tolist() == [4, 6]


def random_cache(layers, blocks, H, page, D, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, (layers, blocks, H, page * (D + 8)), dtype=torch.uint8, generator=g)


@pytest.mark.parametrize("layers,H,page,D", [(1, 1, 16, 64), (3, 2, 32, 128), (5, 8, 64, 64), (2, 3, 128, 128), (1, 2, 1024, 128)])
def test_copies(layers, H, page, D):
    blocks = 12
    cache = random_cache(layers, blocks, H, page, D)
    src = [0, -1, 1, 5, 2, 99, 3, 4]
    dst = [7, 8, 9, -1, 10, 6, 11, 12]
    n = [page, page, 1, page, 17, page, 0, 5]
    for lens in (n, None):
        want = cache.clone()
        for i, (s, d) in enumerate(zip(src, dst)):
            if 0 <= s < blocks and 0 <= d < blocks:
                m = page if lens is None else -(-min(lens[i], page) // 16) * 16
                want[:, d, :, :m * (D + 8)] = cache[:, s, :, :m * (D + 8)]
        got = cache.cuda()
        dsp.dsp_kv4_copy(got, D, i32(src), i32(dst), None if lens is None else i32(lens))
        assert torch.equal(got.cpu(), want)
    one = cache[0].cuda()                                            # a layer by itself, and layers with room between them
    dsp.dsp_kv4_copy(one, D, i32(src), i32(dst))
    assert torch.equal(one.cpu(), want[0])
    wide = torch.zeros(layers, 2 * blocks, H, page * (D + 8), dtype=torch.uint8, device="cuda")
    wide[:, :blocks] = cache.cuda()
    dsp.dsp_kv4_copy(wide[:, :blocks], D, i32(src), i32(dst))
    assert torch.equal(wide[:, :blocks].cpu(), want) and not wide[:, blocks:].any()


def test_many_copies_of_few_blocks():
    cache = random_cache(4, 2000, 2, 16, 64, 1)
    src, dst = [i if i % 3 else -1 for i in range(1000)], [1000 + i for i in range(1000)]
    want = cache.clone()
    at = [i for i in range(1000) if i % 3]
    want[:, [1000 + i for i in at]] = cache[:, at]
    got = cache.cuda()
    dsp.dsp_kv4_copy(got, 64, i32(src), i32(dst))
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("layers,H,page,D", [(1, 1, 16, 64), (2, 3, 16, 128), (3, 2, 32, 64), (2, 8, 64, 128), (1, 1, 1024, 64)])
@pytest.mark.parametrize("seed", range(2))
def test_compaction(layers, H, page, D, seed):
    r = random.Random(seed)
    B, L, longest = 6, 70, 400
    seq = [r.randint(0, 150) for _ in range(B)]
    seq[0], seq[1] = 15, 0
    width = -(-longest // page) + 1
    blocks = B * width
    order = list(range(blocks))
    r.shuffle(order)
    table = [order[b * width:(b + 1) * width] for b in range(B)]
    node, length = [], []
    for b in range(B):
        n = r.choice([L, r.randint(0, L)])
        node.append(sorted(r.sample(range(200), n)) + [-1] * (L - n))     # any growing path: sources and targets overlap
        length.append(n)
    node[2][:length[2]] = range(length[2])                                # everything in place
    node[3] = list(range(1, L + 1))                                       # all of them one place on
    length[3], length[4] = L + 5, -2
    table[5][width // 2] = blocks + 3                                     # a block that there is not
    cache = random_cache(layers, blocks, H, page, D, seed)
    want = ref.compact(cache, D, table, seq, node, length)
    got = cache.cuda()
    dsp.dsp_kv4_compact(got, D, i32(table), i32(seq), i32(node), i32(length))
    assert torch.equal(got.cpu(), want) and not torch.equal(want, cache)


def test_compaction_of_a_single_layer_moves_what_the_cache_holds():
    """The values that dsp_kv4_read gives for the accepted nodes before, at their final places after."""
    B, H, D, page, L = 3, 2, 128, 16, 5
    width = 8
    cache = dsp.kv4_cache(B * width, H, D, page, "cuda")
    table = torch.randperm(B * width, device="cuda").int().view(B, width)
    seq, node, length = [3, 40, 15], [[0, 1, 9, 12, 30], [2, 3, 4, 5, 6], [7, -1, -1, -1, -1]], [5, 4, 1]
    at = torch.arange(width * page, device="cuda")
    slot = (table.long()[:, at // page] * page + at % page).flatten()
    k, v = (torch.randn(len(slot), H, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    dsp.dsp_kv4_append(None, k, v, slot, cache)
    before = [t.view(B, -1, H, D).clone() for t in dsp.dsp_kv4_read(cache, slot, D)]
    dsp.dsp_kv4_compact(cache, D, table, i32(seq), i32(node), i32(length))
    after = [t.view(B, -1, H, D) for t in dsp.dsp_kv4_read(cache, slot, D)]
    for x, y in zip(before, after):
        want = x.clone()
        for b in range(B):
            for i in range(length[b]):
                want[b, seq[b] + 1 + i] = x[b, seq[b] + 1 + node[b][i]]
        assert torch.equal(y, want)


@pytest.mark.parametrize("layers", [1, 2])
def test_moves_beyond_32_bits(layers):
    """A cache of more than 2^32 bytes a layer: copies to and from its end, and a tree in its last blocks."""
    D, page, H, blocks = 64, 16, 1, 3800000
    cache = torch.empty(layers, blocks, H, page * (D + 8), dtype=torch.uint8, device="cuda")
    small = random_cache(layers, 4, H, page, D, seed=3).cuda()
    at = torch.tensor([0, 1, blocks - 2, blocks - 1], device="cuda")
    cache[:, at] = small
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    dsp.dsp_kv4_copy(cache, D, ints(0, blocks - 1), ints(blocks - 3, 7), None)
    assert torch.equal(cache[:, blocks - 3], small[:, 0]) and torch.equal(cache[:, 7], small[:, 3])
    table = ints(0, blocks - 2, blocks - 1).view(1, 3)
    seq, node, n = [page + 2], [[0, 9, 10, 20]], [4]
    dsp.dsp_kv4_compact(cache, D, table, ints(*seq), ints(*node[0]).view(1, 4), ints(*n))
    want = ref.compact(small.cpu(), D, [[0, 2, 3]], seq, node, n)
    assert torch.equal(cache[:, at].cpu(), want)
