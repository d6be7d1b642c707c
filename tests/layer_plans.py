"""The layers' plan (csrc/plan_layers.hpp) compiled with the host compiler: the
form, tiles and parts of K that a call takes, without a GPU."""

import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIP_INCLUDE = "/opt/rocm/include"
AVAILABLE = shutil.which("g++") is not None and os.path.isdir(os.path.join(HIP_INCLUDE, "hip"))

PROGRAM = r"""
#define __HIP_PLATFORM_AMD__
#include "plan_layers.hpp"
#include <cstdio>
using namespace occ;

static void* at(long i, long bytes) { return (void*)(((i + 1) << 44) + bytes); }

static void product(const char* name, const Product& p) {
  std::printf(" %s_blocks %lld %s_splits %d %s_tiles_k %lld", name, (long long)p.blocks(), name, p.splits, name,
              (long long)p.tiles_k);
}

int main() {
  char kind[8];
  int f32, act, gated, dx, dw, db;
  long tokens, in, out, pad, shift;
  while (std::scanf("%7s %d %d %d %ld %ld %ld %ld %ld %d %d %d", kind, &f32, &act, &gated, &tokens, &in, &out, &pad,
                    &shift, &dx, &dw, &db) == 12) {
    const long wide = gated ? 2 * out : out, s = shift * (f32 ? 4 : 2);
    if (kind[0] == 'f') {
      occ_linear_t a{};
      a.dtype = f32 ? OCC_F32 : OCC_BF16;
      a.act = act;
      a.tokens = tokens, a.in = in, a.out = out;
      a.X = at(0, s), a.ldx = in + pad, a.W = at(1, s), a.ldw = in + pad;
      a.Y = at(2, s), a.ldy = out + pad, a.Z = at(3, s), a.ldz = wide + pad;
      FwdPlan f;
      std::printf("status %d", check_fwd(&a, gated) ? 2 : plan_fwd(a, gated, f));
      std::printf(" form %s tile %d bytes %zu", f.few ? "few" : f.planes ? "planes" : f.direct ? "direct" : "tiled",
                  f.few ? 0 : f.direct ? 64 : kTiles[f.prod.tile].side, f.bytes);
      product("x", f.prod.x);
      product("w", f.prod.w);
    } else {
      occ_linear_grad_t a{};
      a.dtype = a.dw_dtype = f32 ? OCC_F32 : OCC_BF16;
      a.act = act;
      a.tokens = tokens, a.in = in, a.out = out;
      a.dY = at(0, s), a.lddy = out + pad, a.Z = at(1, s), a.ldz = wide + pad;
      if (dx) a.dX = at(2, s), a.lddx = in + pad, a.W = at(3, s), a.ldw = in + pad;
      if (dw) a.dW = at(4, s), a.lddw = in + pad, a.X = at(5, s), a.ldx = in + pad;
      if (db) a.dbias = (float*)at(6, 0);
      BwdPlan f;
      std::printf("status %d", check_bwd(&a, gated) ? 2 : plan_bwd(a, gated, f));
      std::printf(" form %s tile %d bytes %zu", f.planes ? "planes" : f.direct ? "direct" : "tiled",
                  f.direct ? 64 : kTiles[f.prod.tile].side, f.bytes);
      product("x", f.prod.x);
      product("w", f.prod.w);
      std::printf(" ldd %lld made %d", (long long)f.ldd, (int)(f.has_dz || f.copy_dy));
    }
    std::printf("\n");
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


def case(kind, dtype, tokens, n_in, out, act=2, gated=False, pad=0, shift=0, dx=True, dw=True,
         db=True):
    """kind: 'fwd' or 'bwd'; shift: elements off an aligned address."""
    return (f"{kind} {int(dtype == 'f32')} {act} {int(gated)} {tokens} {n_in} {out} {pad} {shift} "
            f"{int(dx)} {int(dw)} {int(db)}")


def plans(exe, cases):
    """A dict for each case: status, form, tile, bytes, {x,w}_{blocks,splits,tiles_k}, .."""
    run = subprocess.run([exe], input="\n".join(cases) + "\n", capture_output=True, text=True,
                         check=True)
    out = []
    for line in run.stdout.splitlines():
        w = line.split()
        out.append({k: v if k == "form" else int(v) for k, v in zip(w[::2], w[1::2])})
    assert len(out) == len(cases)
    return out
