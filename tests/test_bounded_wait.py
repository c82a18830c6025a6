"""The waits of the attention kernels end, run on the host: a unit that never comes, a unit that comes late, and nothing amiss."""
from __future__ import annotations

import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2512_18337_b200" / "csrc"

# A warp with `units` units and `stages` of them loaded ahead, as the streaming kernel runs it: wait, compute, load the next.
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "bounded_wait.h"
using namespace samb200;
int main(int argc, char** argv) {
    const long units = atol(argv[1]), stages = atol(argv[2]), lost = atol(argv[3]);   // lost: this unit never arrives (-1: none)
    long polls = 0, loaded = stages < units ? stages : units, after = 0;
    bool gave_up = false;
    const RingWaits waits{&gave_up};
    for (long it = 0; it < units; ++it) {
        auto ready = [&](long u) { ++polls; return u < loaded && u != lost; };
        const bool late = !waits.unit([&] { return ready(it); });
        if (late) waits.give_up(static_cast<int>(loaded - it), [&](int i) { return ready(it + i); });
        if (loaded < units && !gave_up) { ++loaded; after += lost >= 0 && it >= lost; }
    }
    std::printf("%ld %d %ld %ld %u\n", polls, gave_up, loaded, after, kCachePolls);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("wait")
    (at / "wait.cpp").write_text(PROGRAM)
    subprocess.check_call([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", str(CSRC), "-o", str(at / "wait"), str(at / "wait.cpp")])
    return str(at / "wait")


@pytest.mark.parametrize("stages", [2, 4])
@pytest.mark.parametrize("units,lost", [(1, 0), (1000, 0), (1000, 500), (1000, 999)])
def test_a_lost_unit_costs_one_wait_and_a_drain(program, units, lost, stages):
    polls, gave_up, loaded, after, limit = map(int, subprocess.check_output([program, str(units), str(stages), str(lost)]).split())
    assert gave_up and after == 0 and loaded == min(units, lost + stages)
    assert polls <= (1 + stages) * limit + units           # not a full wait for each of the units that follow


@pytest.mark.parametrize("units", [0, 1, 3, 1000])
def test_units_that_arrive_cost_one_poll(program, units):
    polls, gave_up, loaded, _, _ = map(int, subprocess.check_output([program, str(units), "4", "-1"]).split())
    assert (polls, gave_up, loaded) == (units, 0, units)
