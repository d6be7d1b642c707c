// liboptcc C ABI of the stage operators: linear and gated layers, AdamW.
// Argument validation and launch sequencing, on the host (plan_layers.hpp: the
// layers' forms, tiles and workspaces).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>
#include <vector>

#include "host.hpp"
#include "kernels_adamw.hpp"
#include "kernels_layer.hpp"
#include "optcc.h"
#include "plan_layers.hpp"

using namespace occ;

namespace {

struct Spans {
  Span v[12];
  int n = 0;
  void add(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t es, bool w) {
    if (p && rows > 0) v[n++] = span2d(p, rows, cols, ld, es, w);
  }
  bool clash() const {
    for (int i = 0; i < n; ++i)
      for (int j = i + 1; j < n; ++j)
        if ((v[i].writable || v[j].writable) && v[i].lo < v[j].hi && v[j].lo < v[i].hi) return true;
    return false;
  }
};

void set_tiles(GemmArgs& g, const Product& p, char* part) {
  g.tiles_m = (int32_t)p.tiles_m;
  g.tiles_n = (int32_t)p.tiles_n;
  g.tiles_k = (int32_t)p.tiles_k;
  g.splits = p.splits;
  g.k_per_split = p.k_per_split;
  g.part = p.splits > 1 ? (float*)part : nullptr;
}

// Results bypass the caches when the call's operands and results pass
// kStreamBytes, most of what the memory-side cache holds: they would not
// survive there until they are used, but push out operands that other tiles
// still need (8192 x 4096 x 16384 bf16, 470 MB: 861 us with ordinary stores, 807
// with these).  Rows have to start on 64 bytes.
constexpr double kStreamBytes = 192e6;

bool rows_on_lines(const void* p, int64_t ld, int64_t cols, size_t es) {
  return !p || (aligned(p, 64) && (size_t)ld * es % 64 == 0 && (size_t)cols * es % 64 == 0);
}

unsigned join_blocks(const GemmArgs& g) {
  return (unsigned)std::min<int64_t>(div_up((int64_t)g.M * div_up(g.N, 4), 256), 4096);
}

template <class T>
CopyArgs copy_operand(const void* src, int64_t ld, int64_t rows, int64_t cols, char* dst, bool planes) {
  CopyArgs c{};
  c.src = src;
  c.dst = dst;
  c.ld = ld;
  c.rows = rows;
  c.cols = (int32_t)cols;
  const size_t es = planes ? 2 : sizeof(T);
  c.pieces = (int32_t)(piece_ld(cols, es) * (int64_t)es / 16);
  c.plane = planes ? rows * piece_ld(cols, es) : 0;
  c.blocks = (int32_t)std::min<int64_t>(div_up(rows * c.pieces, 256), 8192);
  return c;
}

template <class T, bool GATED>
occ_status_t run_prep(const PrepArgs& p, hipStream_t s) {
  const int blocks = p.dz_blocks + p.copy[0].blocks + p.copy[1].blocks + p.copy[2].blocks;
  if (!blocks) return OCC_OK;
  return launch("layer_prep", s, [&] {
    hipLaunchKernelGGL((k_prep<T, GATED>), dim3((unsigned)blocks), dim3(256), 0, s, p);
  });
}

template <class T, bool GATED>
occ_status_t run_fwd(const occ_linear_t& l, const FwdPlan& f, char* ws, hipStream_t s) {
  FwdEpi e{};
  e.Y = l.Y;
  e.ldy = l.ldy;
  e.Z = l.Z;
  e.ldz = l.ldz;
  e.R = l.R;
  e.ldr = l.ldr;
  e.bias = l.bias;
  e.act = l.act;
  e.out = (int32_t)l.out;
  const int64_t wide = GATED ? 2 * l.out : l.out;
  const double bytes = (double)sizeof(T) * ((double)l.tokens * (double)(l.in + l.out + (l.Z ? wide : 0)) +
                                            (double)wide * (double)l.in);
  e.stream = bytes > kStreamBytes && rows_on_lines(l.Y, l.ldy, l.out, sizeof(T)) &&
             rows_on_lines(l.Z, l.ldz, l.out, sizeof(T));
  if (f.few) {
    SkinnyArgs g{};
    g.X = l.X;
    g.W = l.W;
    g.ldx = l.ldx;
    g.ldw = l.ldw;
    g.tokens = (int32_t)l.tokens;
    g.in = (int32_t)l.in;
    g.fwd = e;
    const dim3 grid((unsigned)div_up(l.out, 16)), block(SK_WAVES * 64);
    if (l.tokens <= kDotTokens) {
      const dim3 rows((unsigned)div_up(GATED ? l.out : div_up(l.out, 2), DOT_WAVES)), waves(DOT_WAVES * 64);
      return launch(GATED ? "gated_few" : "linear_few", s, [&] {
        if (l.tokens == 1) hipLaunchKernelGGL((k_dot<T, 1, GATED>), rows, waves, 0, s, g);
        else if (l.tokens == 2) hipLaunchKernelGGL((k_dot<T, 2, GATED>), rows, waves, 0, s, g);
        else hipLaunchKernelGGL((k_dot<T, 4, GATED>), rows, waves, 0, s, g);
      });
    }
    return launch(GATED ? "gated_few" : "linear_few", s, [&] {
      if (l.tokens <= 16) hipLaunchKernelGGL((k_skinny<T, 1, GATED>), grid, block, 0, s, g);
      else if (l.tokens <= 32) hipLaunchKernelGGL((k_skinny<T, 2, GATED>), grid, block, 0, s, g);
      else hipLaunchKernelGGL((k_skinny<T, 4, GATED>), grid, block, 0, s, g);
    });
  }
  GemmArgs g{};
  g.A = l.X;
  g.lda = l.ldx;
  g.B = l.W;
  g.ldb = l.ldw;
  PrepArgs prep{};
  const int64_t ldp = piece_ld(l.in, f.planes ? 2 : sizeof(T));
  if (f.copy_x) {
    prep.copy[0] = copy_operand<T>(l.X, l.ldx, l.tokens, l.in, ws + f.x_off, f.planes);
    g.A = ws + f.x_off;
    g.lda = ldp;
    g.plane_a = prep.copy[0].plane * 2;
  }
  if (f.copy_w) {
    prep.copy[1] = copy_operand<T>(l.W, l.ldw, wide, l.in, ws + f.w_off, f.planes);
    g.B = ws + f.w_off;
    g.ldb = ldp;
    g.plane_b = prep.copy[1].plane * 2;
  }
  OCC_TRY((run_prep<T, GATED>(prep, s)));
  g.M = (int32_t)l.tokens;
  g.N = (int32_t)l.out;
  g.ka = g.kb = (int32_t)(f.direct ? l.in : ldp);
  g.fwd = e;
  set_tiles(g, f.prod.x, ws + f.part_off);
  constexpr int EP = GATED ? EP_GATED : EP_FWD;
  const dim3 grid((unsigned)f.prod.x.blocks()), block(512);
  auto product = [&](auto operand) {
    using TI = decltype(operand);
    return launch(GATED ? "gated_fwd" : "linear_fwd", s, [&] {
      switch (f.prod.tile) {
        case TILE_256: hipLaunchKernelGGL((k_gemm<TI, T, Form256, EP>), grid, block, 0, s, g); break;
        case TILE_128: hipLaunchKernelGGL((k_gemm<TI, T, Form128, EP>), grid, block, 0, s, g); break;
        default: hipLaunchKernelGGL((k_gemm<TI, T, Form64, EP>), grid, block, 0, s, g); break;
      }
    });
  };
  if (f.direct) {
    OCC_TRY(launch(GATED ? "gated_fwd" : "linear_fwd", s, [&] {
      hipLaunchKernelGGL((k_gemm_direct<T, EP>), grid, block, 0, s, g);
    }));
  } else if (f.planes) {
    g.seg_tiles = (int32_t)(f.prod.x.tiles_k / kPairs);
    OCC_TRY(product(uint16_t{}));
  } else {
    OCC_TRY(product(T{}));
  }
  if (g.splits == 1) return OCC_OK;
  return launch("layer_join", s, [&] {
    hipLaunchKernelGGL((k_gemm_join<T, EP>), dim3(join_blocks(g)), dim3(256), 0, s, g);
  });
}

occ_status_t check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (!need) return OCC_OK;
  return !ws || !aligned(ws, kWsAlign) || ws_bytes < need ? OCC_E_WORKSPACE : OCC_OK;
}

template <bool GATED>
occ_status_t forward(const occ_linear_t* lp, void* ws, size_t ws_bytes, occ_stream_t stream) {
  OCC_TRY(check_fwd(lp, GATED));
  const occ_linear_t& l = *lp;
  if (l.tokens == 0) return OCC_OK;
  if (!l.X || !l.W || !l.Y) return OCC_E_NULL;
  const size_t es = elem_size(l.dtype);
  if (!aligned(l.X, es) || !aligned(l.W, es) || !aligned(l.Y, es) || !aligned(l.R, es) || !aligned(l.Z, es) ||
      !aligned(l.bias, 4))
    return OCC_E_ALIGN;
  FwdPlan f;
  OCC_TRY(plan_fwd(l, GATED, f));
  OCC_TRY(check_ws(ws, ws_bytes, f.bytes));
  const int64_t wide = GATED ? 2 * l.out : l.out;
  Spans sp;
  sp.add(l.X, l.tokens, l.in, l.ldx, es, false);
  sp.add(l.W, wide, l.in, l.ldw, es, false);
  sp.add(l.bias, 1, wide, wide, 4, false);
  sp.add(l.Y, l.tokens, l.out, l.ldy, es, true);
  sp.add(l.Z, l.tokens, wide, l.ldz, es, true);
  if (l.R && (l.R != l.Y || l.ldr != l.ldy)) sp.add(l.R, l.tokens, l.out, l.ldr, es, false);
  if (f.bytes) sp.add(ws, 1, (int64_t)f.bytes, (int64_t)f.bytes, 1, true);
  if (sp.clash()) return OCC_E_ALIAS;
  hipStream_t s = (hipStream_t)stream;
  return l.dtype == OCC_BF16 ? run_fwd<uint16_t, GATED>(l, f, (char*)ws, s) : run_fwd<float, GATED>(l, f, (char*)ws, s);
}

template <class T, bool GATED>
occ_status_t run_bwd(const occ_linear_grad_t& l, const BwdPlan& f, bool accumulate, char* ws, hipStream_t s) {
  const int64_t wide = GATED ? 2 * l.out : l.out;
  const bool act = GATED || l.act != OCC_ACT_NONE;
  PrepArgs prep{};
  if (f.strips) {
    DzArgs& d = prep.dz;
    d.dY = l.dY;
    d.ldy = l.lddy;
    d.Z = act ? l.Z : nullptr;
    d.ldz = l.ldz;
    d.dZ = f.has_dz ? ws + f.dz_off : nullptr;
    d.ldd = f.ldd;
    d.bias_part = f.strip_bias ? (float*)(ws + f.bias_off) : nullptr;
    d.tokens = (int32_t)l.tokens;
    d.out = (int32_t)l.out;
    d.act = l.act;
    d.strip = (int32_t)f.strip;
    d.across = (int32_t)div_up(l.out, DZ_LANES * 4);
    d.plane = f.planes && f.has_dz ? l.tokens * f.ldd : 0;
    prep.dz_blocks = (int32_t)(d.across * f.strips);
  }
  DzSource src{};
  src.dY = l.dY;
  src.ldy = l.lddy;
  src.Z = act ? l.Z : nullptr;
  src.ldz = l.ldz;
  src.out = (int32_t)l.out;
  src.act = l.act;
  src.gated = GATED;
  const void* dz = l.dY;
  int64_t ldd = l.lddy;
  if (f.has_dz || f.copy_dy) {
    dz = ws + f.dz_off;
    ldd = f.ldd;
  }
  CopyArgs copies[3] = {};
  int nc = 0;
  if (f.copy_dy) copies[nc++] = copy_operand<T>(l.dY, l.lddy, l.tokens, l.out, ws + f.dz_off, f.planes);
  if (f.copy_w) copies[nc++] = copy_operand<T>(l.W, l.ldw, wide, l.in, ws + f.w_off, f.planes);
  if (f.copy_x) copies[nc++] = copy_operand<T>(l.X, l.ldx, l.tokens, l.in, ws + f.x_off, f.planes);
  for (int i = 0; i < 3; ++i) prep.copy[i] = copies[i];
  OCC_TRY((run_prep<T, GATED>(prep, s)));

  const double bytes = (double)sizeof(T) * ((double)l.tokens * (double)(2 * l.in + wide) + 2.0 * (double)wide * (double)l.in);
  const bool stream = bytes > kStreamBytes;
  BackwardArgs a{};
  const int64_t ldp = piece_ld(l.in, f.planes ? 2 : sizeof(T));
  const int64_t dz_plane = f.planes ? l.tokens * f.ldd * 2 : 0;
  if (l.dX) {
    GemmArgs& g = a.dx;
    g.A = dz;
    g.lda = ldd;
    g.B = f.copy_w ? ws + f.w_off : l.W;
    g.ldb = f.copy_w ? ldp : l.ldw;
    g.plane_a = dz_plane;
    g.plane_b = wide * ldp * 2;
    g.seg_tiles = (int32_t)(f.prod.x.tiles_k / kPairs);
    g.M = (int32_t)l.tokens;
    g.N = (int32_t)l.in;
    g.ka = (int32_t)(f.has_dz || f.copy_dy ? f.ldd : wide);
    g.kb = (int32_t)wide;
    g.C = l.dX;
    g.ldc = l.lddx;
    g.stream = stream && rows_on_lines(l.dX, l.lddx, l.in, sizeof(T));
    g.dz = src;
    set_tiles(g, f.prod.x, ws + f.dx_part);
    a.dx_blocks = (int32_t)f.prod.x.blocks();
  }
  if (l.dW) {
    GemmArgs& g = a.dw;
    g.A = dz;
    g.lda = ldd;
    g.B = f.copy_x ? ws + f.x_off : l.X;
    g.ldb = f.copy_x ? ldp : l.ldx;
    g.plane_a = dz_plane;
    g.plane_b = l.tokens * ldp * 2;
    g.seg_tiles = (int32_t)(f.prod.w.tiles_k / kPairs);
    g.M = (int32_t)wide;
    g.N = (int32_t)l.in;
    g.ka = g.kb = (int32_t)l.tokens;
    g.C = l.dW;
    g.ldc = l.lddw;
    g.c_f32 = l.dw_dtype == OCC_F32;
    g.accumulate = accumulate;
    g.stream = stream && rows_on_lines(l.dW, l.lddw, l.in, elem_size(l.dw_dtype));
    g.dz = src;
    set_tiles(g, f.prod.w, ws + f.dw_part);
    a.dw_blocks = (int32_t)f.prod.w.blocks();
  }
  int64_t bias_blocks = 0;
  if (l.dbias) {
    a.bias.part = f.strip_bias ? (const float*)(ws + f.bias_off) : nullptr;
    a.bias.dbias = l.dbias;
    a.bias.width = wide;
    a.bias.strips = (int32_t)f.strips;
    a.bias.accumulate = accumulate;
    a.bias.src = src;
    a.bias.tokens = (int32_t)l.tokens;
    bias_blocks = f.strip_bias ? div_up(wide, 64) : div_up(l.out, BD_COLS);
  }
  const int64_t blocks = (int64_t)a.dx_blocks + a.dw_blocks + bias_blocks;
  if (!a.dx_blocks && !a.dw_blocks)
    return launch("layer_bias", s, [&] {
      hipLaunchKernelGGL((k_bias<T>), dim3((unsigned)bias_blocks), dim3(512), 0, s, a.bias);
    });
  const dim3 grid((unsigned)blocks), block(512);
  auto direct = [&] {
    return launch("layer_bwd", s, [&] { hipLaunchKernelGGL((k_backward_direct<T>), grid, block, 0, s, a); });
  };
  auto products = [&](auto operand) {
    using TI = decltype(operand);
    return launch("layer_bwd", s, [&] {
      switch (f.prod.tile) {
        case TILE_256: hipLaunchKernelGGL((k_backward<TI, T, Form256>), grid, block, 0, s, a); break;
        case TILE_128: hipLaunchKernelGGL((k_backward<TI, T, Form128>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((k_backward<TI, T, Form64>), grid, block, 0, s, a); break;
      }
    });
  };
  if (f.direct) OCC_TRY(direct());
  else if (f.planes) OCC_TRY(products(uint16_t{}));
  else OCC_TRY(products(T{}));
  const unsigned jx = l.dX && a.dx.splits > 1 ? join_blocks(a.dx) : 0;
  const unsigned jw = l.dW && a.dw.splits > 1 ? join_blocks(a.dw) : 0;
  if (!jx && !jw) return OCC_OK;
  return launch("layer_join", s, [&] {
    hipLaunchKernelGGL((k_backward_join<T>), dim3(jx + jw), dim3(256), 0, s, a.dx, a.dw, (int)jx);
  });
}

template <class T>
occ_status_t zero_rows(void* p, int64_t rows, int64_t cols, int64_t ld, hipStream_t s) {
  return launch("zero_grad", s, [&] {
    hipLaunchKernelGGL((k_zero_rows<T>), dim3((unsigned)std::min<int64_t>(div_up(rows * cols, 256), 8192)), dim3(256),
                       0, s, (T*)p, rows, (int)cols, ld);
  });
}

template <bool GATED>
occ_status_t backward(const occ_linear_grad_t* lp, unsigned flags, void* ws, size_t ws_bytes, occ_stream_t stream) {
  OCC_TRY(check_bwd(lp, GATED));
  if (flags & ~(unsigned)OCC_GRAD_ACCUMULATE) return OCC_E_FLAGS;
  const occ_linear_grad_t& l = *lp;
  const bool accumulate = flags & OCC_GRAD_ACCUMULATE;
  const size_t es = elem_size(l.dtype), ws_es = elem_size(l.dw_dtype);
  const int64_t wide = GATED ? 2 * l.out : l.out;
  const bool act = GATED || l.act != OCC_ACT_NONE;
  if (!aligned(l.dY, es) || !aligned(l.X, es) || !aligned(l.W, es) || !aligned(l.Z, es) || !aligned(l.dX, es) ||
      !aligned(l.dW, ws_es) || !aligned(l.dbias, 4))
    return OCC_E_ALIGN;
  hipStream_t s = (hipStream_t)stream;
  BwdPlan f;
  if (l.tokens > 0) {
    if (!l.dY || (act && !l.Z) || (l.dX && !l.W) || (l.dW && !l.X)) return OCC_E_NULL;
    OCC_TRY(plan_bwd(l, GATED, f));
    OCC_TRY(check_ws(ws, ws_bytes, f.bytes));
  }
  Spans sp;
  sp.add(l.dY, l.tokens, l.out, l.lddy, es, false);
  if (act) sp.add(l.Z, l.tokens, wide, l.ldz, es, false);
  if (l.dW) sp.add(l.X, l.tokens, l.in, l.ldx, es, false);
  if (l.dX) sp.add(l.W, wide, l.in, l.ldw, es, false);
  sp.add(l.dX, l.tokens, l.in, l.lddx, es, true);
  sp.add(l.dW, wide, l.in, l.lddw, ws_es, true);
  sp.add(l.dbias, 1, wide, wide, 4, true);
  if (f.bytes) sp.add(ws, 1, (int64_t)f.bytes, (int64_t)f.bytes, 1, true);
  if (sp.clash()) return OCC_E_ALIAS;
  if (l.tokens == 0) {
    if (accumulate) return OCC_OK;
    if (l.dW) OCC_TRY(ws_es == 2 ? zero_rows<uint16_t>(l.dW, wide, l.in, l.lddw, s)
                                 : zero_rows<float>(l.dW, wide, l.in, l.lddw, s));
    return l.dbias ? zero_rows<float>(l.dbias, 1, wide, wide, s) : OCC_OK;
  }
  return l.dtype == OCC_BF16 ? run_bwd<uint16_t, GATED>(l, f, accumulate, (char*)ws, s)
                             : run_bwd<float, GATED>(l, f, accumulate, (char*)ws, s);
}

// ----------------------------------------------------------------------------
// AdamW
// ----------------------------------------------------------------------------
enum AdamKind { AK_F32_32, AK_BF16_32, AK_F32_8, AK_BF16_8, AK_FACTORS_32, AK_FACTORS_8, AK_NUM };

AdamKind kind_of(const occ_param_t& p) {
  if (!p.G) return p.state_bits == 32 ? AK_FACTORS_32 : AK_FACTORS_8;
  if (p.state_bits == 32) return p.g_dtype == OCC_BF16 ? AK_BF16_32 : AK_F32_32;
  return p.g_dtype == OCC_BF16 ? AK_BF16_8 : AK_F32_8;
}

// Factors with 32-bit moments are taken 256 columns a block where that makes
// at least this many blocks, all of them whole runs: 403M elements at rank 32
// 1.96 ms, 2.05 in blocks of 64 columns; but 0.4M at rank 78 38 us against 17,
// 39M at rank 128 275 against 229, and rows of 1817 2.15 ms against 1.95.
constexpr int64_t kNarrowBlocks = 4096;

// A launch holds fewer than 2^32 threads, 512 or 256 a block.
constexpr int64_t kMaxAdamBlocks = (((int64_t)1 << 32) - 1) / 512;

// narrow: factors in blocks of 64 columns
int64_t adam_blocks(const occ_param_t& p, bool narrow) {
  const int64_t per_row = div_up(p.cols, kRun);
  if (!p.G) return div_up(p.rows, ADF_ROWS) * (narrow && p.state_bits == 32 ? div_up(p.cols, 64) : per_row);
  return p.state_bits == 32 ? div_up(p.rows * p.cols, AD_BLOCK) : div_up(p.rows * per_row, AD8_BLOCK);
}

occ_status_t check_param(const occ_param_t& p, std::vector<Span>& spans) {
  if (p.rows < 1 || p.cols < 1 || p.rows >= kMaxTokens || p.cols >= kMaxTokens ||
      p.rows * p.cols >= ((int64_t)1 << 42) || adam_blocks(p, true) >= kMaxTokens)
    return OCC_E_SHAPE;
  if (p.state_bits != 32 && p.state_bits != 8) return OCC_E_VALUE;
  if (!std::isfinite(p.decay)) return OCC_E_VALUE;
  if (!p.W || !p.m || !p.v || (p.state_bits == 8 && (!p.m_scale || !p.v_scale))) return OCC_E_NULL;
  const size_t ss = p.state_bits == 32 ? 4 : 1;
  const int64_t per_row = div_up(p.cols, kRun);
  if (!aligned(p.W, 4) || !aligned(p.W16, 2) || !aligned(p.m, ss) || !aligned(p.v, ss)) return OCC_E_ALIGN;
  if (p.G) {
    if (p.g_dtype != OCC_F32 && p.g_dtype != OCC_BF16) return OCC_E_DTYPE;
    if (!ld_ok(p.cols, p.ldg)) return OCC_E_SHAPE;
    if (!aligned(p.G, elem_size(p.g_dtype))) return OCC_E_ALIGN;
    spans.push_back(span2d(p.G, p.rows, p.cols, p.ldg, elem_size(p.g_dtype), false));
  } else {
    if (!p.P || !p.Q) return OCC_E_NULL;
    if (p.rank < 1 || p.rank > OCC_MAX_RANK) return OCC_E_RANK;
    if (!aligned(p.P, 4) || !aligned(p.Q, 4)) return OCC_E_ALIGN;
    spans.push_back(span2d(p.P, p.rows, p.rank, p.rank, 4, false));
    spans.push_back(span2d(p.Q, p.cols, p.rank, p.rank, 4, false));
  }
  spans.push_back(span2d(p.W, p.rows, p.cols, p.cols, 4, true));
  if (p.W16) spans.push_back(span2d(p.W16, p.rows, p.cols, p.cols, 2, true));
  spans.push_back(span2d(p.m, p.rows, p.cols, p.cols, ss, true));
  spans.push_back(span2d(p.v, p.rows, p.cols, p.cols, ss, true));
  if (p.state_bits == 8) {
    if (!aligned(p.m_scale, 4) || !aligned(p.v_scale, 4)) return OCC_E_ALIGN;
    spans.push_back(span2d(p.m_scale, p.rows, per_row, per_row, 4, true));
    spans.push_back(span2d(p.v_scale, p.rows, per_row, per_row, 4, true));
  }
  return OCC_OK;
}

// Bytes read and written, factors aside.
double adam_bytes(const occ_param_t& p) {
  return (double)p.rows * (double)p.cols *
         (8.0 + (p.state_bits == 32 ? 16.0 : 4.0) + (p.W16 ? 2.0 : 0.0) + (p.G ? (double)elem_size(p.g_dtype) : 0.0));
}

// Whole rows on 64 bytes: the streams may bypass the caches, which they do
// where all tensors of a call are more than the memory-side cache holds from
// one step to the next (3.1M elements, 94 MB: 17.9 us through the caches, 19.1
// past them; 403M elements 2.30 against 2.06 ms).
bool streams(const occ_param_t& p) {
  const bool rows = p.state_bits == 8 || !p.G;   // else W and the moments are one run each
  if (!aligned(p.W, 64) || !aligned(p.W16, 64) || (rows && p.cols % 32)) return false;
  if (p.state_bits == 32 && (!aligned(p.m, 64) || !aligned(p.v, 64))) return false;
  return !p.G || (aligned(p.G, 64) && (p.ldg == p.cols || (size_t)p.ldg * elem_size(p.g_dtype) % 64 == 0));
}

template <bool NT>
void start_adam(AdamKind kind, bool narrow, const AdamArgs& a, unsigned blocks, hipStream_t s) {
  const dim3 grid(blocks), block(256), fblock(ADF_WAVES * 64);
  switch (kind) {
    case AK_F32_32: hipLaunchKernelGGL((k_adamw32<float, NT>), grid, block, 0, s, a); break;
    case AK_BF16_32: hipLaunchKernelGGL((k_adamw32<uint16_t, NT>), grid, block, 0, s, a); break;
    case AK_F32_8: hipLaunchKernelGGL((k_adamw8<float, NT>), grid, block, 0, s, a); break;
    case AK_BF16_8: hipLaunchKernelGGL((k_adamw8<uint16_t, NT>), grid, block, 0, s, a); break;
    case AK_FACTORS_32:
      if (narrow) hipLaunchKernelGGL((k_adamw_factors<32, NT, 1>), grid, fblock, 0, s, a);
      else hipLaunchKernelGGL((k_adamw_factors<32, NT, 4>), grid, fblock, 0, s, a);
      break;
    default: hipLaunchKernelGGL((k_adamw_factors<8, NT, 4>), grid, fblock, 0, s, a); break;
  }
}

occ_status_t launch_adam(AdamKind kind, bool nt, bool narrow, AdamArgs& a, int count, int64_t blocks, hipStream_t s) {
  for (int i = count; i < kAdamTensors; ++i) a.start[i] = INT32_MAX;
  return launch("adamw", s, [&] {
    if (nt) start_adam<true>(kind, narrow, a, (unsigned)blocks, s);
    else start_adam<false>(kind, narrow, a, (unsigned)blocks, s);
  });
}

occ_status_t adamw(const occ_param_t* params, int count, const occ_adamw_t* h, hipStream_t s) {
  if (count < 1) return OCC_E_SHAPE;
  if (!params || !h) return OCC_E_NULL;
  if (!std::isfinite(h->lr) || !(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0) ||
      !(h->eps >= 0.0 && std::isfinite(h->eps)) || h->step < 1)
    return OCC_E_VALUE;
  if (!aligned(h->grad_scale, 4) || !aligned(h->flags, 4)) return OCC_E_ALIGN;
  std::vector<Span> spans;
  spans.reserve((size_t)count * 8 + 2);
  for (int j = 0; j < count; ++j) OCC_TRY(check_param(params[j], spans));
  if (h->grad_scale) spans.push_back({(uintptr_t)h->grad_scale, (uintptr_t)h->grad_scale + 4, false});
  if (h->flags) spans.push_back({(uintptr_t)h->flags, (uintptr_t)h->flags + 4, false});
  if (overlaps(std::move(spans))) return OCC_E_ALIAS;
  double bytes = 0.0;
  int64_t wide_blocks = 0;   // of factors
  bool whole = true;
  for (int j = 0; j < count; ++j) {
    bytes += adam_bytes(params[j]);
    if (params[j].G) continue;
    wide_blocks += adam_blocks(params[j], false);
    whole = whole && params[j].cols % kRun == 0;
  }
  const bool far = bytes > kStreamBytes;
  const bool narrow = wide_blocks < kNarrowBlocks || !whole;
  AdamArgs a{};
  a.b1 = (float)h->beta1;
  a.c1 = (float)(1.0 - h->beta1);
  a.b2 = (float)h->beta2;
  a.c2 = (float)(1.0 - h->beta2);
  a.a = (float)(h->lr / (1.0 - std::pow(h->beta1, (double)h->step)));
  a.c = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, (double)h->step)));
  a.eps = (float)h->eps;
  a.grad_scale = h->grad_scale;
  a.flags = h->flags;
  // one launch for each form of gradient, moments and alignment among the tensors
  for (int form = 0; form < 2 * AK_NUM; ++form) {
    const AdamKind kind = (AdamKind)(form >> 1);
    const bool nt = form & 1;
    int64_t blocks = 0;
    int in = 0;   // tensors of this launch
    for (int j = 0; j < count; ++j) {
      const occ_param_t& p = params[j];
      if (kind_of(p) != kind || (far && streams(p)) != nt) continue;
      const int64_t nb = adam_blocks(p, narrow);
      // a tensor of more blocks than a launch has left is taken in parts
      for (int64_t done = 0, take; done < nb; done += take) {
        if (in == kAdamTensors || blocks == kMaxAdamBlocks) {
          OCC_TRY(launch_adam(kind, nt, narrow, a, in, blocks, s));
          in = 0;
          blocks = 0;
        }
        take = std::min(nb - done, kMaxAdamBlocks - blocks);
        a.start[in] = (int32_t)(blocks - done);
        AdamTensor& t = a.t[in++];
        t.W = p.W;
        t.W16 = (uint16_t*)p.W16;
        t.G = p.G;
        t.P = p.P;
        t.Q = p.Q;
        t.m = p.m;
        t.v = p.v;
        t.m_scale = p.m_scale;
        t.v_scale = p.v_scale;
        t.ldg = p.G ? p.ldg : p.rank;
        t.rows = (int32_t)p.rows;
        t.cols = (int32_t)p.cols;
        t.keep = (float)(1.0 - h->lr * (double)p.decay);
        t.key = (h->seed + (uint32_t)j * 0x6A09E667u) * 0xBB67AE85u;
        blocks += take;
      }
    }
    if (in) OCC_TRY(launch_adam(kind, nt, narrow, a, in, blocks, s));
  }
  return OCC_OK;
}

}  // namespace

extern "C" {

size_t occ_linear_fwd_workspace_bytes(const occ_linear_t* l) {
  FwdPlan f;
  return check_fwd(l, false) == OCC_OK && plan_fwd(*l, false, f) == OCC_OK ? f.bytes : 0;
}

size_t occ_gated_fwd_workspace_bytes(const occ_linear_t* l) {
  FwdPlan f;
  return check_fwd(l, true) == OCC_OK && plan_fwd(*l, true, f) == OCC_OK ? f.bytes : 0;
}

size_t occ_linear_bwd_workspace_bytes(const occ_linear_grad_t* l) {
  BwdPlan f;
  return check_bwd(l, false) == OCC_OK && plan_bwd(*l, false, f) == OCC_OK ? f.bytes : 0;
}

size_t occ_gated_bwd_workspace_bytes(const occ_linear_grad_t* l) {
  BwdPlan f;
  return check_bwd(l, true) == OCC_OK && plan_bwd(*l, true, f) == OCC_OK ? f.bytes : 0;
}

occ_status_t occ_linear_fwd(const occ_linear_t* l, void* ws, size_t ws_bytes, occ_stream_t stream) {
  return forward<false>(l, ws, ws_bytes, stream);
}

occ_status_t occ_gated_fwd(const occ_linear_t* l, void* ws, size_t ws_bytes, occ_stream_t stream) {
  return forward<true>(l, ws, ws_bytes, stream);
}

occ_status_t occ_linear_bwd(const occ_linear_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                            occ_stream_t stream) {
  return backward<false>(l, flags, ws, ws_bytes, stream);
}

occ_status_t occ_gated_bwd(const occ_linear_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                           occ_stream_t stream) {
  return backward<true>(l, flags, ws, ws_bytes, stream);
}

occ_status_t occ_adamw_step(const occ_param_t* params, int count, const occ_adamw_t* h, occ_stream_t stream) {
  try {
    return adamw(params, count, h, (hipStream_t)stream);
  } catch (...) {   // no memory for the list of spans
    return OCC_E_HIP;
  }
}

}  // extern "C"
