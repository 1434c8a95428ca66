"""dsp_cache_fork at the sizes where a launch's shared memory comes to its default limit."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

# (rows before, rows after, blocks): a pool of few rows, whose marks lie in shared memory, and many rows, whose sums do.  Each pair in a
# process of its own, since a call that needs more raises the limit for those after it.
SIZES = [((32, 32, 5983), (6111, 6111, 7000)), ((32, 32, 6000), (6112, 6112, 7000)), ((32, 32, 6014), (6143, 50, 7000)), ((16, 16, 6047), (50, 6130, 7000)),
         ((4, 4, 6126), (6143, 6143, 7000)), ((4, 4, 6127), (6144, 6144, 7000))]

CHILD = """
import random, sys
sys.path.insert(0, %r)
sys.path.insert(0, %r)
import test_gpu_fork as t
for at in (1, 4):
    Bi, Bo, blocks = map(int, sys.argv[at:at + 3])
    r = random.Random(blocks + Bi)
    page, width = 16, 4
    lens = [r.randint(0, 14 if Bi > 1000 else 40) for _ in range(Bi)]
    have, table, ring, pos = t.pool(r, lens, page, width, blocks - sum(-(-n // page) for n in lens), 0)
    assert len(ring) == blocks
    src = [r.choice([-1, r.randrange(Bi), min(b, Bi - 1)]) for b in range(Bo)]
    keep = [r.randint(0, lens[s]) if s >= 0 else 0 for s in src]
    t.run(src, keep, lens, have, pos, table, ring, page, width)
    print("served")
"""


@pytest.mark.parametrize("few,many", SIZES)
def test_pools_and_rows_of_any_number(few, many):
    code = CHILD % (os.path.dirname(HERE), HERE)
    p = subprocess.run([sys.executable, "-c", code] + list(map(str, few + many)), capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.count("served") == 2, p.stderr[-2000:]


@pytest.mark.parametrize("blocks", [1, 100, 30000])
def test_no_rows_at_all(blocks):
    """Nothing comes in and nothing goes out: the ring's ends are handed on, however large the pool is."""
    import torch

    from paper_2510_02358_b200 import binding as dsp
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    table, ring, pos = none.view(0, 4), torch.arange(blocks, dtype=torch.int32, device="cuda"), torch.tensor([3, 3 + blocks], device="cuda")
    got = dsp.dsp_cache_fork(none, None, none, none, pos, table, ring, 16, table.clone())
    assert got.ring_pos.tolist() == [3, 3 + blocks] and torch.equal(ring, torch.arange(blocks, dtype=torch.int32, device="cuda"))
