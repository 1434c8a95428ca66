"""Which tables dsp_cache_fork takes beside one another: on the host, nothing is launched."""
import os
import re
import subprocess

import pytest
import torch

from paper_2510_02358_b200 import build

CASES = r"""
#include <cstdint>
#include <cstdio>
#include <vector>
%s
int main() {
    // every pair of small tables in a common piece of memory, against the entries themselves
    static int32_t memory[4096];
    long wrong = 0, shared = 0, apart = 0;
    for (int width = 1; width <= 3; ++width)
        for (int sa = width; sa <= 7; ++sa)
            for (int sb = width; sb <= 7; ++sb)
                for (int na = 0; na <= 4; ++na)
                    for (int nb = 0; nb <= 4; ++nb)
                        for (int off = -40; off <= 40; ++off) {
                            std::vector<int> seen(400, 0);
                            bool both = false;
                            for (int i = 0; i < na; ++i)
                                for (int e = 0; e < width; ++e) seen[200 + off + i * sa + e] = 1;
                            for (int i = 0; i < nb; ++i)
                                for (int e = 0; e < width; ++e) both |= seen[200 + i * sb + e] != 0;
                            wrong += overlap(memory + 200 + off, sa, na, memory + 200, sb, nb, width) != both;
                            (both ? shared : apart)++;
                        }
    std::printf("%%ld %%d\n", wrong, shared > 1000 && apart > 1000);
    return 0;
}
"""


def test_tables_that_share_memory_are_told_from_those_that_do_not(tmp_path):
    """Two halves of a wider tensor lie in each other's gaps and share nothing; the function is taken from the source and run on the host."""
    text = open(os.path.join(build.CSRC, "fork.cu")).read()
    body = re.search(r"^bool overlap\(.*?^}\n", text, flags=re.M | re.S).group(0)
    src, exe = tmp_path / "overlap.cc", tmp_path / "overlap"
    src.write_text(CASES % body)
    subprocess.run(["g++", "-std=c++17", "-O1", str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split() == ["0", "1"]


@pytest.mark.gpu
def test_the_two_tables_may_be_halves_of_one_tensor():
    from paper_2510_02358_b200 import binding as dsp
    i32 = dict(dtype=torch.int32, device="cuda")
    wide = torch.full((3, 2, 4), -9, **i32)
    wide[:, 0] = torch.arange(12, **i32).view(3, 4)
    ring, pos = torch.arange(20, **i32), torch.tensor([12, 20], device="cuda")
    args = (torch.tensor([2, 0, 2], **i32), None, torch.tensor([64, 0, 33], **i32), torch.tensor([4, 0, 3], **i32), pos)
    apart = torch.full((3, 4), -9, **i32)
    want = dsp.dsp_cache_fork(*args, wide[:, 0].contiguous(), ring.clone(), 16, apart)
    got = dsp.dsp_cache_fork(*args, wide[:, 0], ring, 16, wide[:, 1])
    assert torch.equal(wide[:, 1], apart) and got.copy_dst.tolist() == want.copy_dst.tolist() and not got.row_status.any()
    assert torch.equal(wide[:, 0], torch.arange(12, **i32).view(3, 4))
    with pytest.raises(dsp.DspError):
        dsp.dsp_cache_fork(*args, wide[:, 0], ring, 16, wide.view(3, 8)[:, 3:7])
