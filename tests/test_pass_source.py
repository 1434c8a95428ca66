"""What the kernels' source has to keep to, checked as text (no GPU)."""
import glob
import os
import re
import subprocess

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


RING = r"""
#include "copy_ring.h"
#include <cstdio>
#include <vector>
using namespace dsp;

// A barrier as the hardware keeps it: the parity of its current phase; a wait for parity p is over once the phase with it has ended.
struct Bar { unsigned phase = 0; bool done(unsigned p) const { return (phase & 1u) != p; } };

// Segments of `iters` iterations one after the other; copy number `fails` (counted over all) comes late, after its wait has run out.
// Returns the number of faults.
template <int S> int walk(const std::vector<int> &iters, int step, long fails) {
    CopyRing<S> order;
    Bar bars[S];
    long fetched = 0, copy_of[S], faults = 0, waits_for_nothing = 0;
    bool out[S] = {}, lost = false;
    for (int n : iters) {
        const int run0 = 3, run_end = run0 + n * step - (step - 1);
        int run = run0, ahead = run0;
        order.restart();
        for (int i = 0; i < S; ++i) faults += out[i];                       // under way into a place that is used otherwise now
        auto fetch = [&](int st) { faults += out[st]; out[st] = true; copy_of[st] = fetched++; };
        auto land = [&](int st) { out[st] = false; bars[st].phase++; };
        for (int i = 0; i < S - 1; ++i, ahead += step)
            if (ahead < run_end && !lost) fetch(i);
        for (; run < run_end && !lost; run += step, ahead += step) {
            const int st = order.stage;
            faults += !out[st];                                             // waits for a copy that nobody has sent
            if (out[st] && copy_of[st] != fails) land(st);
            lost = !bars[st].done(order.parity());
            if (lost) {
                for (int left = order.under_way(run, ahead, run_end, step); left > 0; --left, order.used()) {
                    const int d = order.stage;
                    faults += !out[d] || bars[d].done(order.parity());      // not under way, or taken for landed before it has
                    if (out[d]) land(d);
                    faults += !bars[d].done(order.parity());
                }
                break;
            }
            if (ahead < run_end) fetch(order.before());
            order.used();
        }
    }
    for (int i = 0; i < S; ++i) faults += out[i];
    faults += fails >= 0 && fails < fetched && !lost;
    return (int)faults;
}

int main() {
    long bad = 0;
    const std::vector<std::vector<int>> lines = {{1}, {2, 3}, {7, 1, 9}, {0, 4, 0, 1, 1, 1, 5}, {40, 2, 33}};
    for (const auto &line : lines)
        for (int step : {1, 4, 8})
            for (long fails = -1; fails < 80; ++fails) bad += walk<2>(line, step, fails) + walk<3>(line, step, fails) + walk<4>(line, step, fails);
    std::printf("%ld\n", bad);
    return 0;
}
"""


def test_the_ring_of_copies_waits_for_what_is_under_way_and_for_nothing_else(tmp_path):
    """Whichever copy comes too late: its warp waits for the others that it has sent, each by the parity of that copy, and sends no more."""
    src, exe = tmp_path / "ring.cc", tmp_path / "ring"
    src.write_text(RING)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.strip() == "0"
    text = open(os.path.join(CSRC, "attn.cu")).read()              # the kernel goes by this bookkeeping and has none of its own
    assert "CopyRing<kStages> order" in text and "phases" not in text


def test_tensor_memory_is_given_back_after_the_last_product():
    """Also where a wait ran out: the products commit to a barrier of their own, which is waited for (with a limit) before the CTA ends."""
    text = open(os.path.join(CSRC, "attn_block.cu")).read()
    end = text[text.index("attn_block_kernel(const AttnArgs a) {"):]
    end = end[end.index("product_role<D>("):end.index("tcgen05.dealloc")]
    assert re.search(r"commit_to\(smem_u32\(&s_bars\.ended\), elected\(\)\);.*__syncthreads\(\);.*while \(!bar_test\(smem_u32\(&s_bars\.ended\), 0u\) && clock64\(\) - t0 < kWaitClocks\)",
                     end, flags=re.S)
    assert "bar_init(smem_u32(&s_bars.ended), kProductWarps)" in text
