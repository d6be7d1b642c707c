"""The launch before the products of the experts' backward pass (dZ, bias sums, copies), from
the plan compiled with the host compiler."""

import os
import random
import subprocess

import pytest

from experts_plans import case, compile_plans
from layer_plans import AVAILABLE, HIP_INCLUDE, ROOT
from layer_plans import plans as plans_of

pytestmark = pytest.mark.skipif(not AVAILABLE, reason="g++ or the HIP headers not available")

PROGRAM = r"""
#define __HIP_PLATFORM_AMD__
#include "plan_experts.hpp"
#include <cstdio>
using namespace occ;

static void* at(long i) { return (void*)((i + 1) << 44); }

int main() {
  int f32, act, gated, dx, dw, db;
  long experts, tokens, in, out;
  while (std::scanf("%d %d %d %ld %ld %ld %ld %d %d %d", &f32, &act, &gated, &experts, &tokens, &in, &out, &dx, &dw,
                    &db) == 10) {
    const long wide = gated ? 2 * out : out;
    occ_experts_grad_t p{};
    occ_linear_grad_t& a = p.l;
    p.experts = experts, p.stride_w = p.stride_dw = wide * in;
    a.dtype = a.dw_dtype = f32 ? OCC_F32 : OCC_BF16;
    a.act = act;
    a.tokens = tokens, a.in = in, a.out = out;
    a.dY = at(0), a.lddy = out, a.Z = at(1), a.ldz = wide;
    if (dx) a.dX = at(2), a.lddx = in, a.W = at(3), a.ldw = in;
    if (dw) a.dW = at(4), a.lddw = in, a.X = at(5), a.ldx = in;
    if (db) a.dbias = (float*)at(6);
    ExpertsBwdPlan f;
    const int status = check_experts_bwd(&p, gated) ? 2 : plan_experts_bwd(p, gated, f);
    std::printf("%d %lld %d\n", status, (long long)(f.across * f.strips), f.copy_dy + f.copy_w + f.copy_x);
  }
}
"""

COPY_BLOCKS = 8192      # of one operand, at most


def test_launches_stay_within_the_largest_grid(tmp_path):
    """Fewer than 2^32 threads, 256 a block, or the plan refuses."""
    src, exe = tmp_path / "prep.cpp", tmp_path / "prep"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2301_09830_amd", "csrc"), "-I", HIP_INCLUDE,
                    str(src), "-o", str(exe)], check=True)
    # weights of just under 2^31 rows in all, as many rows of tokens as experts or more
    cases = [(0, 1, 0, 127, 127, 1, 1 << 24, 1, 0, 0), (0, 1, 0, 127, 4000, 1, 1 << 24, 1, 0, 0),
             (0, 1, 0, 1023, 1023, 8, 1 << 21, 1, 0, 0), (0, 2, 0, 1023, 3000, 1, 2098000, 0, 1, 1),
             (1, 1, 0, 255, 300, 3, 1 << 23, 1, 1, 0), (0, 4, 1, 63, 900, 1, 1 << 24, 1, 0, 0)]
    rng = random.Random(5)
    for _ in range(2000):
        experts = rng.choice((1, 8, 100, 1024, rng.randint(1, 1024)))
        gated = rng.random() < 0.3
        out = min(1 << 24, ((1 << 31) - 1) // experts // (2 if gated else 1))
        out = rng.choice((out, rng.randint(1, out)))
        cases.append((int(rng.random() < 0.5), 4 if gated else rng.randint(0, 4), int(gated), experts,
                      rng.choice((1, 127, 1024, 1 << 20, 1 << 29)), rng.choice((1, 64, 300)), out,
                      *rng.choice(((1, 0), (0, 1), (1, 1), (0, 0))), 1))
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), text=True,
                         capture_output=True, check=True).stdout
    plans = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert len(plans) == len(cases) and sum(not p[0] for p in plans) > 200
    for c, (status, blocks, copies) in zip(cases, plans):
        assert status or (blocks + copies * COPY_BLOCKS) * 256 < 1 << 32, (c, blocks, copies)


def test_products_beside_bias_sums_stay_within_the_largest_grid(tmp_path):
    """The products' blocks and those of the bias gradient are one launch, 512 threads each."""
    exe = compile_plans(tmp_path)
    # some 3.6 million bias blocks beside 7.3 million tiles of 64, off 16 bytes
    cases = [dict(kind="bwd", dtype="bf16", experts=e, rows=e, n_in=128, out=wide // e, shift=1, pad=1,
                  act=0, dx=False) for e in (14, 100, 512) for wide in (200 << 20, 224 << 20)]
    rng = random.Random(6)
    for _ in range(3000):
        e = rng.choice((1, 16, 64, 500, 1024))
        gated = rng.random() < 0.3
        out = rng.randint(1, (224 << 20) // e // (2 if gated else 1))
        cases.append(dict(kind="bwd", dtype=rng.choice(("bf16", "f32")), experts=e, gated=gated,
                          rows=rng.choice((1, 300, 1 << 20, rng.randint(1, 1 << 29))), shift=rng.choice((0, 1)),
                          n_in=rng.randint(1, 600), out=min(out, 1 << 24), act=4 if gated else rng.randint(0, 4),
                          dx=rng.random() < 0.5, db=rng.random() < 0.8))
    taken = 0
    for c, p in zip(cases, plans_of(exe, [case(**c) for c in cases])):
        taken += not p["status"]
        assert p["status"] or p["blocks"] * 512 < 1 << 32, (c, p)
    assert taken > 300
