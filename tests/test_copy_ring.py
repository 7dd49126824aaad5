"""No GPU: the bookkeeping by which a kernel waits for its copies in flight before it ends (csrc/copy_ring.cuh), against barriers in Python's
stead: a barrier's phase completes when a copy into its stage lands, and a wait for a parity passes once the phase of that parity is over."""
import os
import subprocess

import pytest

from paper_2406_17276_b200 import build

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "copy_ring.cuh"
using namespace ot;

// Copies 0 ... issued - 1 go round the ring, each once its stage has been taken; the first `landed` of them have landed.  True if the drain, from
// the copy that the kernel names, passes exactly when all have landed, and waits for every one that has not.
template <uint32_t kStages> bool check(uint32_t issued, uint32_t landed, uint32_t from) {
    std::vector<uint32_t> phases(kStages, 0);
    for (uint32_t i = 0; i < landed; ++i) ++phases[i % kStages];
    uint32_t stuck = 0;
    CopyRing<kStages>::drain(from, issued, [&](uint32_t stage, uint32_t parity) { stuck += (phases[stage] & 1) == parity; });
    return stuck == issued - landed;
}
template <uint32_t kStages> bool all() {
    for (uint32_t issued = 0; issued < 6 * kStages + 3; ++issued)
        for (uint32_t landed = issued > kStages ? issued - kStages : 0; landed <= issued; ++landed) {
            if (!check<kStages>(issued, landed, CopyRing<kStages>::oldest(issued))) return false;
            // a wait that gave up at copy `landed`, before which all had been taken
            if (!check<kStages>(issued, landed, landed)) return false;
        }
    return true;
}
int main() { std::printf("%d\n", all<1>() && all<2>() && all<3>() && all<6>() && all<12>()); }
"""


def test_every_copy_in_flight_is_waited_for(tmp_path):
    src, exe = tmp_path / "ring.cpp", tmp_path / "ring"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-I", build.CSRC, "-o", str(exe), str(src)])
    assert subprocess.check_output([str(exe)]).strip() == b"1"


def _text(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return f.read()


@pytest.mark.parametrize("name,waits", [("kv_attend_few.cuh", 1), ("kv_attend_tiles.cuh", 2)])
def test_the_kernels_drain_by_it(name, waits):
    """Each ring is drained through CopyRing, and copies are counted where they are issued."""
    text = _text(name)
    assert text.count("::drain(") == waits
    for line in text.split("\n"):
        assert "(done - 1 - i)" not in line and "blocks - 1 - s" not in line


def test_copies_that_nobody_has_waited_for_are_drained_whatever_happened():
    """The copying warp of the tile kernel drains without a condition: a reader that gave up leaves copies behind that the copying warp has no
    reason to know of."""
    text = _text("kv_attend_tiles.cuh")
    before = text[:text.index("::drain(")].rstrip().split("\n")[-3:]
    assert not any("if (" in line for line in before)


def test_converting_warps_leave_at_a_wait_that_ran_out():
    """They hand back no further stages: the copying warp may not run ahead of slots that others still read."""
    text = _text("kv_attend_tiles.cuh")
    loop = text[text.index("wait(free_ + stage, phase ^ 1);"):]
    assert loop.split("\n")[1].strip().startswith("if (dead) break;")
