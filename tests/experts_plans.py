"""The plan of the experts' layers (csrc/plan_experts.hpp) compiled with the host
compiler: the form and tiles that a call takes, without a GPU."""

import os
import subprocess

from layer_plans import HIP_INCLUDE, ROOT

PROGRAM = r"""
#define __HIP_PLATFORM_AMD__
#include "plan_experts.hpp"
#include <cstdio>
using namespace occ;

static void* at(long i, long bytes) { return (void*)(((i + 1) << 44) + bytes); }

int main() {
  char kind[8];
  int f32, act, gated, dx, dw, db;
  long experts, tokens, in, out, pad, shift;
  while (std::scanf("%7s %d %d %d %ld %ld %ld %ld %ld %ld %d %d %d", kind, &f32, &act, &gated, &experts, &tokens, &in,
                    &out, &pad, &shift, &dx, &dw, &db) == 13) {
    const long wide = gated ? 2 * out : out, s = shift * (f32 ? 4 : 2), step = wide * (in + pad);
    if (kind[0] == 'f') {
      occ_experts_t p{};
      occ_linear_t& a = p.l;
      p.experts = experts, p.stride_w = step;
      a.dtype = f32 ? OCC_F32 : OCC_BF16;
      a.act = act;
      a.tokens = tokens, a.in = in, a.out = out;
      a.X = at(0, s), a.ldx = in + pad, a.W = at(1, s), a.ldw = in + pad;
      a.Y = at(2, s), a.ldy = out + pad, a.Z = at(3, s), a.ldz = wide + pad;
      ExpertsFwdPlan f;
      std::printf("status %d", check_experts_fwd(&p, gated) ? 2 : plan_experts_fwd(p, gated, f));
      std::printf(" form %s tile %d copied %d bytes %zu blocks %lld\n",
                  f.few ? "few" : f.planes ? "planes" : f.direct ? "direct" : "tiled",
                  f.few ? f.few : f.direct ? 64 : kTiles[f.tile].side, (int)(!f.planes && (f.copy_x || f.copy_w)),
                  f.bytes, (long long)f.blocks);
    } else {
      occ_experts_grad_t p{};
      occ_linear_grad_t& a = p.l;
      p.experts = experts, p.stride_w = p.stride_dw = step;
      a.dtype = a.dw_dtype = f32 ? OCC_F32 : OCC_BF16;
      a.act = act;
      a.tokens = tokens, a.in = in, a.out = out;
      a.dY = at(0, s), a.lddy = out + pad, a.Z = at(1, s), a.ldz = wide + pad;
      if (dx) a.dX = at(2, s), a.lddx = in + pad, a.W = at(3, s), a.ldw = in + pad;
      if (dw) a.dW = at(4, s), a.lddw = in + pad, a.X = at(5, s), a.ldx = in + pad;
      if (db) a.dbias = (float*)at(6, 0);
      ExpertsBwdPlan f;
      std::printf("status %d", check_experts_bwd(&p, gated) ? 2 : plan_experts_bwd(p, gated, f));
      std::printf(" form %s tile %d copied %d bytes %zu blocks %lld ldd %lld made %d\n",
                  f.planes ? "planes" : f.direct ? "direct" : "tiled", f.direct ? 64 : kTiles[f.tile].side,
                  (int)(!f.planes && (f.copy_x || f.copy_w || f.copy_dy)), f.bytes,
                  (long long)(f.dx_blocks + f.dw_blocks + (db ? experts * ((wide + 63) / 64) : 0)), (long long)f.ldd,
                  (int)(f.has_dz || f.copy_dy));
    }
  }
}
"""


def compile_plans(folder):
    """The program's path; it reads cases from its input."""
    src, exe = folder / "plans.cpp", folder / "plans"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2301_09830_amd", "csrc"), "-I", HIP_INCLUDE,
                    str(src), "-o", str(exe)], check=True)
    return str(exe)


def case(kind, dtype, experts, rows, n_in, out, act=2, gated=False, pad=0, shift=0, dx=True,
         dw=True, db=True):
    """kind: 'fwd' or 'bwd'; shift: elements off an aligned address."""
    return (f"{kind} {int(dtype == 'f32')} {act} {int(gated)} {experts} {rows} {n_in} {out} {pad} "
            f"{shift} {int(dx)} {int(dw)} {int(db)}")
