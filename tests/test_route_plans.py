"""The router's gradient in parts that a launch holds, from the plan compiled with the host
compiler (csrc/plan_experts.hpp)."""

import os
import random
import subprocess

import pytest

from layer_plans import AVAILABLE, HIP_INCLUDE, ROOT

pytestmark = pytest.mark.skipif(not AVAILABLE, reason="g++ or the HIP headers not available")

PROGRAM = r"""
#define __HIP_PLATFORM_AMD__
#include "plan_experts.hpp"
#include <cstdio>

int main() {
  long experts;
  int k;
  while (std::scanf("%ld %d", &experts, &k) == 2)
    std::printf("%d %lld\n", occ::route_lanes(experts, k), (long long)occ::route_bwd_part(experts, k));
}
"""


def parts(folder, cases):
    src, exe = folder / "parts.cpp", folder / "parts"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2301_09830_amd", "csrc"), "-I", HIP_INCLUDE,
                    str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], input="\n".join(f"{e} {k}" for e, k in cases), text=True,
                         capture_output=True, check=True).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_launches_stay_within_the_largest_grid(tmp_path):
    """Fewer than 2^32 threads in a launch, blocks of 256 with whole tokens, whatever
    tokens k < 2^30 there are."""
    rng = random.Random(1)
    cases = [(1, 1), (256, 16), (256, 17), (257, 1), (1024, 32)]
    cases += [(e, rng.randint(1, min(32, e))) for e in (rng.randint(1, 1024) for _ in range(300))]
    for (experts, k), (lanes, part) in zip(cases, parts(tmp_path, cases)):
        assert lanes in (16, 64) and lanes >= k
        per = 256 // lanes
        most = ((1 << 30) - 1) // k
        tokens = min(part, most)
        assert part % per == 0 and -(-tokens // per) * 256 < 1 << 32, (experts, k)
