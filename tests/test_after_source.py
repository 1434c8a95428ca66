"""What the source of the calls after a verified step has to keep to, checked as text (no GPU): waits that run out cannot be made to on a GPU."""
import os
import re

from paper_2510_02358_b200 import build


def source(name):
    return open(os.path.join(build.CSRC, name)).read()


def function(text, name):
    at = text.index(name + "(")
    return text[at:text.index("\n}\n", at)]


def test_a_distillation_whose_copies_or_parts_come_too_late_gives_nan():
    """Status words are the caller's choice, so the numbers themselves say it: NaN for the row's sum goes to all of its CTAs (from which loss,
    accept, lse, state and gradient follow), a CTA that misses the others' parts takes nothing of them, a chunk that is read again is NaN."""
    text = source("distill.cu")
    rows, loss, grad, known = (function(text, name) for name in (") distill_kernel", ") distill_loss_kernel", ") distill_grad_kernel", "Known known_of"))
    # every known_of has the look at the waits in it, after the last of them
    assert len(re.findall(r"\bknown_of\(a, ", text)) == 2 and "lost_if(int timed_out) { return timed_out ? CUDART_NAN_F : 0.f; }" in text
    assert re.search(r"known_of\(a, sh\.part, [^;]*, lost_if\(\*static_cast<volatile int \*>\(&sh\.timed_out\)\), lane\);", rows)
    assert re.search(r"known_of\(a, s_part, [^;]*, lost_if\(bars\.timed_out\), lane\);", loss)
    assert rows.index("take(sh.got") < rows.index("known_of(a, ") and loss.index("stream_slice<") < loss.index("known_of(a, ")
    # copies: seen by the whole CTA, and NaN before anything is handed over
    assert re.search(r"take_copies\(sh, parity\);\s*parity \^= 1u;\s*__syncthreads\(\);[^\n]*\n\s*if \(sh\.timed_out\) Sc = CUDART_NAN_F;", rows)
    assert re.search(r"write_pieces<DT>\(g, p, a\.V, q0, q1, buf, a\.s, c_f, chunks > 1 && sh\.timed_out \? CUDART_NAN_F", rows)
    assert re.search(r"sh\.timed_out \? CUDART_NAN_F", grad)
    # a NaN sum of one warp reaches the row's sum, and no rule makes it a number again
    assert "S = lost," in known and "w2 == 0.f && q[i].S < CUDART_INF_F ? 0.f : q[i].S * w2" in known
    assert "S = (S != 0.f ? S * ex2_approx(c - cn) : 0.f) + " in function(text, "void sum_pieces")


def test_kernels_that_start_early_do_not_end_before_the_launch_that_they_depend_on():
    """If no thread of such a kernel waits, nothing orders what the launch before it writes (status words, tickets) before what follows the
    kernel.  So each way out lies behind a wait: of the kernel itself, or of the row's pass that it calls."""
    text = source("score.cu")
    for name in (") score_kernel", ") score_cluster_kernel"):
        body = function(text, name)
        unread = body[body.index("score_nothing("):]
        unread = unread[:unread.index("return;")]
        assert "grid_dependency_wait();" in unread, name
    assert "grid_dependency_wait();" in function(text, "bool score_sums") and "grid_dependency_wait();" in function(source("row_engine.cuh"), "bool row_engine")
    fork = function(source("fork.cu"), ") fork_part_kernel")
    assert "return" not in fork and "grid_dependency_wait();" in fork
