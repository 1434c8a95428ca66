"""What the kernels' source has to keep to, checked as text (no GPU)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2510_02358_b200", "csrc")


def _after_the_wait():
    """(file, text) from each grid_dependency_wait() to its function's end."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        text = open(path).read()
        for m in re.finditer(r"^ +grid_dependency_wait\(\);", text, flags=re.M):
            yield os.path.basename(path), text[m.end():text.index("\n}\n", m.end())]


def test_kernels_that_start_early_do_not_read_what_is_being_written_as_read_only():
    """Such a kernel runs beside the one before it; a read-only load is defined for data that nobody writes meanwhile."""
    found = list(_after_the_wait())
    assert {name for name, _ in found} >= {"attn.cu", "attn_block.cu", "verify.cu", "cps.cu"}
    for name, body in found:
        assert not re.search(r"__ldg\(|ldg_stream\(|\.nc\b", body), name
