// C ABI of the experts' layers: argument checks and launches, on the host.  A
// part of stage_ops.hip.
#pragma once

#include "kernels_experts.hpp"
#include "plan_experts.hpp"

namespace {

Groups groups_of(const int32_t* offsets, uint32_t* flags, int64_t experts, int64_t rows) {
  return Groups{offsets, flags, (int32_t)experts, (int32_t)rows};
}

// The weights of every expert as one operand of whole 16-byte pieces (planes
// each in one run).
template <class T>
ExpertsCopyArgs copy_weights(const void* src, int64_t ld, int64_t wide, int64_t in, int64_t stride, int64_t experts,
                             char* dst, bool planes) {
  ExpertsCopyArgs a{};
  a.c = copy_operand<T>(src, ld, experts * wide, in, dst, planes);
  a.step = stride;
  a.per = experts == 1 || stride == wide * ld ? 0 : (int32_t)wide;
  return a;
}

template <class T, bool GATED>
occ_status_t run_experts_prep(const ExpertsPrepArgs& p, hipStream_t s) {
  const int blocks = p.dz_blocks + p.copy[0].c.blocks + p.copy[1].c.blocks + p.copy[2].c.blocks;
  if (!blocks) return OCC_OK;
  return launch("experts_prep", s, [&] {
    hipLaunchKernelGGL((k_experts_prep<T, GATED>), dim3((unsigned)blocks), dim3(256), 0, s, p);
  });
}

template <class T, bool GATED>
occ_status_t run_experts_fwd(const occ_experts_t& p, const ExpertsFwdPlan& f, char* ws, hipStream_t s) {
  const occ_linear_t& l = p.l;
  const int64_t wide = GATED ? 2 * l.out : l.out;
  const Groups of = groups_of(p.offsets, p.flags, p.experts, l.tokens);
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
  const double bytes = (double)sizeof(T) * ((double)l.tokens * (double)(l.in + l.out + (l.Z ? wide : 0)) +
                                            (double)(p.experts * wide) * (double)l.in);
  e.stream = bytes > kStreamBytes && rows_on_lines(l.Y, l.ldy, l.out, sizeof(T)) &&
             rows_on_lines(l.Z, l.ldz, l.out, sizeof(T));
  const dim3 grid((unsigned)f.blocks);
  const char* const name = GATED ? "experts_gated_fwd" : "experts_linear_fwd";
  if (f.few) {
    ExpertsFewArgs a{};
    a.g.X = l.X;
    a.g.W = l.W;
    a.g.ldx = l.ldx;
    a.g.ldw = l.ldw;
    a.g.in = (int32_t)l.in;
    a.g.fwd = e;
    a.of = of;
    a.w_step = p.stride_w * (int64_t)sizeof(T);
    a.wide = (int32_t)wide;
    a.across = (int32_t)few_across(f.few, l.out, GATED);
    return launch(GATED ? "experts_gated_few" : "experts_linear_few", s, [&] {
      const dim3 waves(DOT_WAVES * 64), block(SK_WAVES * 64);
      if (f.few == 1) hipLaunchKernelGGL((k_experts_dot<T, GATED>), grid, waves, 0, s, a);
      else if (f.few == 16) hipLaunchKernelGGL((k_experts_skinny<T, 1, GATED>), grid, block, 0, s, a);
      else if (f.few == 32) hipLaunchKernelGGL((k_experts_skinny<T, 2, GATED>), grid, block, 0, s, a);
      else if constexpr (GATED) hipLaunchKernelGGL((k_experts_skinny<T, 4, GATED>), grid, block, 0, s, a);
    });
  }
  ExpertsArgs a{};
  GemmArgs& g = a.g;
  g.A = l.X;
  g.lda = l.ldx;
  g.B = l.W;
  g.ldb = l.ldw;
  a.w_step = p.stride_w * (int64_t)sizeof(T);
  const size_t os = f.planes ? 2 : sizeof(T);
  const int64_t ldp = piece_ld(l.in, os);
  ExpertsPrepArgs prep{};
  if (f.copy_x) {
    prep.copy[0].c = copy_operand<T>(l.X, l.ldx, l.tokens, l.in, ws + f.x_off, f.planes);
    g.A = ws + f.x_off;
    g.lda = ldp;
    g.plane_a = prep.copy[0].c.plane * 2;
  }
  if (f.copy_w) {
    prep.copy[1] = copy_weights<T>(l.W, l.ldw, wide, l.in, p.stride_w, p.experts, ws + f.w_off, f.planes);
    g.B = ws + f.w_off;
    g.ldb = ldp;
    g.plane_b = prep.copy[1].c.plane * 2;
    a.w_step = wide * ldp * (int64_t)os;
  }
  OCC_TRY((run_experts_prep<T, GATED>(prep, s)));
  g.N = (int32_t)l.out;
  g.ka = g.kb = (int32_t)(f.direct ? l.in : ldp);
  g.fwd = e;
  const int side = f.direct ? 64 : kTiles[f.tile].side;
  g.tiles_n = (int32_t)(GATED ? div_up(l.out, side / 2) : div_up(l.out, side));
  g.splits = 1;
  g.seg_tiles = (int32_t)div_up(l.in, kRowBytes / (int64_t)os);
  g.tiles_k = g.k_per_split = g.seg_tiles * (f.planes ? kPairs : 1);
  a.of = of;
  a.wide = (int32_t)wide;
  constexpr int EP = GATED ? EP_GATED : EP_FWD;
  const dim3 block(512);
  if (f.direct)
    return launch(name, s, [&] { hipLaunchKernelGGL((k_experts_direct<T, EP>), grid, block, 0, s, a); });
  auto product = [&](auto operand) {
    using TI = decltype(operand);
    return launch(name, s, [&] {
      switch (f.tile) {
        case TILE_256: hipLaunchKernelGGL((k_experts_fwd<TI, T, Form256, EP>), grid, block, 0, s, a); break;
        case TILE_128: hipLaunchKernelGGL((k_experts_fwd<TI, T, Form128, EP>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((k_experts_fwd<TI, T, Form64, EP>), grid, block, 0, s, a); break;
      }
    });
  };
  return f.planes ? product(uint16_t{}) : product(T{});
}

template <bool GATED>
occ_status_t experts_forward_call(const occ_experts_t* pp, void* ws, size_t ws_bytes, occ_stream_t stream) {
  OCC_TRY(check_experts_fwd(pp, GATED));
  const occ_experts_t& p = *pp;
  const occ_linear_t& l = p.l;
  if (l.tokens == 0) return OCC_OK;
  if (!l.X || !l.W || !l.Y || !p.offsets) return OCC_E_NULL;
  const size_t es = elem_size(l.dtype);
  if (!aligned(l.X, es) || !aligned(l.W, es) || !aligned(l.Y, es) || !aligned(l.R, es) || !aligned(l.Z, es) ||
      !aligned(l.bias, 4) || !aligned(p.offsets, 4) || !aligned(p.flags, 4))
    return OCC_E_ALIGN;
  ExpertsFwdPlan f;
  OCC_TRY(plan_experts_fwd(p, GATED, f));
  OCC_TRY(check_ws(ws, ws_bytes, f.bytes));
  const int64_t wide = GATED ? 2 * l.out : l.out;
  Spans sp;
  sp.add(l.X, l.tokens, l.in, l.ldx, es, false);
  sp.add(l.W, 1, (p.experts - 1) * p.stride_w + (wide - 1) * l.ldw + l.in, 0, es, false);
  sp.add(l.bias, 1, p.experts * wide, 0, 4, false);
  sp.add(l.Y, l.tokens, l.out, l.ldy, es, true);
  sp.add(l.Z, l.tokens, wide, l.ldz, es, true);
  if (l.R && (l.R != l.Y || l.ldr != l.ldy)) sp.add(l.R, l.tokens, l.out, l.ldr, es, false);
  sp.add(p.offsets, 1, p.experts + 1, 0, 4, false);
  sp.add(p.flags, 1, 1, 0, 4, true);
  if (f.bytes) sp.add(ws, 1, (int64_t)f.bytes, 0, 1, true);
  if (sp.clash()) return OCC_E_ALIAS;
  hipStream_t s = (hipStream_t)stream;
  return l.dtype == OCC_BF16 ? run_experts_fwd<uint16_t, GATED>(p, f, (char*)ws, s)
                             : run_experts_fwd<float, GATED>(p, f, (char*)ws, s);
}

template <class T, bool GATED>
occ_status_t run_experts_bwd(const occ_experts_grad_t& p, const ExpertsBwdPlan& f, bool accumulate, char* ws,
                             hipStream_t s) {
  const occ_linear_grad_t& l = p.l;
  const int64_t wide = GATED ? 2 * l.out : l.out;
  const bool act = GATED || l.act != OCC_ACT_NONE;
  const Groups of = groups_of(p.offsets, p.flags, p.experts, l.tokens);
  const size_t os = f.planes ? 2 : sizeof(T);
  ExpertsPrepArgs prep{};
  prep.of = of;
  if (f.strips) {
    DzArgs& d = prep.dz;
    d.dY = l.dY;
    d.ldy = l.lddy;
    d.Z = act ? l.Z : nullptr;
    d.ldz = l.ldz;
    d.dZ = f.has_dz ? ws + f.dz_off : nullptr;
    d.ldd = f.ldd;
    d.bias_part = l.dbias ? (float*)(ws + f.bias_off) : nullptr;
    d.tokens = (int32_t)l.tokens;
    d.out = (int32_t)l.out;
    d.act = l.act;
    d.strip = (int32_t)f.strip;
    d.across = (int32_t)f.across;
    d.plane = f.planes && f.has_dz ? l.tokens * f.ldd : 0;
    prep.dz_blocks = (int32_t)(f.across * f.strips);
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
  if (f.copy_dy) prep.copy[0].c = copy_operand<T>(l.dY, l.lddy, l.tokens, l.out, ws + f.dz_off, f.planes);
  if (f.copy_w)
    prep.copy[1] = copy_weights<T>(l.W, l.ldw, wide, l.in, p.stride_w, p.experts, ws + f.w_off, f.planes);
  if (f.copy_x) prep.copy[2].c = copy_operand<T>(l.X, l.ldx, l.tokens, l.in, ws + f.x_off, f.planes);
  OCC_TRY((run_experts_prep<T, GATED>(prep, s)));

  const double bytes = (double)sizeof(T) * ((double)l.tokens * (double)(2 * l.in + wide) +
                                            2.0 * (double)(p.experts * wide) * (double)l.in);
  const bool stream = bytes > kStreamBytes;
  ExpertsBackwardArgs a{};
  a.of = of;
  a.strip = (int32_t)std::max<int64_t>(f.strip, 1);
  const int side = f.direct ? 64 : kTiles[f.tile].side;
  const int64_t ldp = piece_ld(l.in, os);
  const int64_t dz_plane = f.planes ? l.tokens * f.ldd * 2 : 0;
  if (l.dX) {
    GemmArgs& g = a.dx;
    g.A = dz;
    g.lda = ldd;
    g.B = f.copy_w ? ws + f.w_off : l.W;
    g.ldb = f.copy_w ? ldp : l.ldw;
    a.w_step = f.copy_w ? wide * ldp * (int64_t)os : p.stride_w * (int64_t)sizeof(T);
    g.plane_a = dz_plane;
    g.plane_b = p.experts * wide * ldp * 2;
    g.N = (int32_t)l.in;
    g.ka = (int32_t)(f.has_dz || f.copy_dy ? f.ldd : wide);
    g.kb = (int32_t)wide;
    g.C = l.dX;
    g.ldc = l.lddx;
    g.stream = stream && rows_on_lines(l.dX, l.lddx, l.in, sizeof(T));
    g.dz = src;
    g.tiles_n = (int32_t)div_up(l.in, side);
    g.splits = 1;
    g.seg_tiles = (int32_t)div_up(wide, kRowBytes / (int64_t)os);
    g.tiles_k = g.k_per_split = g.seg_tiles * (f.planes ? kPairs : 1);
    a.dx_blocks = (int32_t)f.dx_blocks;
  }
  if (l.dW) {
    GemmArgs& g = a.dw;
    g.A = dz;
    g.lda = ldd;
    g.B = f.copy_x ? ws + f.x_off : l.X;
    g.ldb = f.copy_x ? ldp : l.ldx;
    g.plane_a = dz_plane;
    g.plane_b = l.tokens * ldp * 2;
    g.M = (int32_t)wide;
    g.N = (int32_t)l.in;
    g.C = l.dW;
    g.ldc = l.lddw;
    g.c_f32 = l.dw_dtype == OCC_F32;
    g.accumulate = accumulate;
    g.stream = stream && rows_on_lines(l.dW, l.lddw, l.in, elem_size(l.dw_dtype)) &&
               (size_t)p.stride_dw * elem_size(l.dw_dtype) % 64 == 0;
    g.dz = src;
    g.tiles_m = (int32_t)div_up(wide, side);
    g.tiles_n = (int32_t)div_up(l.in, side);
    g.splits = 1;
    a.dw_step = p.stride_dw * (int64_t)elem_size(l.dw_dtype);
    a.dw_blocks = (int32_t)f.dw_blocks;
  }
  int64_t bias_blocks = 0;
  if (l.dbias) {
    a.bias.part = (const float*)(ws + f.bias_off);
    a.bias.dbias = l.dbias;
    a.bias.width = wide;
    a.bias.accumulate = accumulate;
    bias_blocks = p.experts * div_up(wide, 64);
  }
  const dim3 grid((unsigned)(f.dx_blocks + f.dw_blocks + bias_blocks)), block(512);
  if (!f.dx_blocks && !f.dw_blocks)
    return launch("experts_bias", s, [&] { hipLaunchKernelGGL(k_experts_bias, grid, block, 0, s, a); });
  if (f.direct)
    return launch("experts_bwd", s, [&] { hipLaunchKernelGGL((k_experts_bwd_direct<T>), grid, block, 0, s, a); });
  auto products = [&](auto operand) {
    using TI = decltype(operand);
    return launch("experts_bwd", s, [&] {
      switch (f.tile) {
        case TILE_256: hipLaunchKernelGGL((k_experts_bwd<TI, T, Form256>), grid, block, 0, s, a); break;
        case TILE_128: hipLaunchKernelGGL((k_experts_bwd<TI, T, Form128>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((k_experts_bwd<TI, T, Form64>), grid, block, 0, s, a); break;
      }
    });
  };
  return f.planes ? products(uint16_t{}) : products(T{});
}

template <bool GATED>
occ_status_t experts_backward_call(const occ_experts_grad_t* pp, unsigned flags, void* ws, size_t ws_bytes,
                                   occ_stream_t stream) {
  OCC_TRY(check_experts_bwd(pp, GATED));
  if (flags & ~(unsigned)OCC_GRAD_ACCUMULATE) return OCC_E_FLAGS;
  const occ_experts_grad_t& p = *pp;
  const occ_linear_grad_t& l = p.l;
  const bool accumulate = flags & OCC_GRAD_ACCUMULATE;
  const size_t es = elem_size(l.dtype), ws_es = elem_size(l.dw_dtype);
  const int64_t wide = GATED ? 2 * l.out : l.out;
  const bool act = GATED || l.act != OCC_ACT_NONE;
  if (!aligned(l.dY, es) || !aligned(l.X, es) || !aligned(l.W, es) || !aligned(l.Z, es) || !aligned(l.dX, es) ||
      !aligned(l.dW, ws_es) || !aligned(l.dbias, 4) || !aligned(p.offsets, 4) || !aligned(p.flags, 4))
    return OCC_E_ALIGN;
  ExpertsBwdPlan f;
  if (l.tokens > 0) {
    if (!p.offsets || !l.dY || (act && !l.Z) || (l.dX && !l.W) || (l.dW && !l.X)) return OCC_E_NULL;
    OCC_TRY(plan_experts_bwd(p, GATED, f));
    OCC_TRY(check_ws(ws, ws_bytes, f.bytes));
  }
  Spans sp;
  sp.add(l.dY, l.tokens, l.out, l.lddy, es, false);
  if (act) sp.add(l.Z, l.tokens, wide, l.ldz, es, false);
  if (l.dW) sp.add(l.X, l.tokens, l.in, l.ldx, es, false);
  if (l.dX) sp.add(l.W, 1, (p.experts - 1) * p.stride_w + (wide - 1) * l.ldw + l.in, 0, es, false);
  sp.add(l.dX, l.tokens, l.in, l.lddx, es, true);
  sp.add(l.dW, 1, (p.experts - 1) * p.stride_dw + (wide - 1) * l.lddw + l.in, 0, ws_es, true);
  sp.add(l.dbias, 1, p.experts * wide, 0, 4, true);
  if (l.tokens > 0) {
    sp.add(p.offsets, 1, p.experts + 1, 0, 4, false);
    sp.add(p.flags, 1, 1, 0, 4, true);
  }
  if (f.bytes) sp.add(ws, 1, (int64_t)f.bytes, 0, 1, true);
  if (sp.clash()) return OCC_E_ALIAS;
  hipStream_t s = (hipStream_t)stream;
  if (l.tokens == 0) {
    if (accumulate) return OCC_OK;
    // one launch where the experts' rows follow each other
    const bool whole = p.experts == 1 || p.stride_dw == wide * l.lddw;
    const int64_t calls = whole ? 1 : p.experts, rows = whole ? p.experts * wide : wide;
    for (int64_t e = 0; l.dW && e < calls; ++e) {
      char* const w = (char*)l.dW + e * p.stride_dw * (int64_t)ws_es;
      OCC_TRY(ws_es == 2 ? zero_rows<uint16_t>(w, rows, l.in, l.lddw, s) : zero_rows<float>(w, rows, l.in, l.lddw, s));
    }
    return l.dbias ? zero_rows<float>(l.dbias, 1, p.experts * wide, p.experts * wide, s) : OCC_OK;
  }
  return l.dtype == OCC_BF16 ? run_experts_bwd<uint16_t, GATED>(p, f, accumulate, (char*)ws, s)
                             : run_experts_bwd<float, GATED>(p, f, accumulate, (char*)ws, s);
}

}  // namespace

extern "C" {

size_t occ_experts_linear_fwd_workspace_bytes(const occ_experts_t* l) {
  ExpertsFwdPlan f;
  return check_experts_fwd(l, false) == OCC_OK && plan_experts_fwd(*l, false, f) == OCC_OK ? f.bytes : 0;
}

size_t occ_experts_gated_fwd_workspace_bytes(const occ_experts_t* l) {
  ExpertsFwdPlan f;
  return check_experts_fwd(l, true) == OCC_OK && plan_experts_fwd(*l, true, f) == OCC_OK ? f.bytes : 0;
}

size_t occ_experts_linear_bwd_workspace_bytes(const occ_experts_grad_t* l) {
  ExpertsBwdPlan f;
  return check_experts_bwd(l, false) == OCC_OK && plan_experts_bwd(*l, false, f) == OCC_OK ? f.bytes : 0;
}

size_t occ_experts_gated_bwd_workspace_bytes(const occ_experts_grad_t* l) {
  ExpertsBwdPlan f;
  return check_experts_bwd(l, true) == OCC_OK && plan_experts_bwd(*l, true, f) == OCC_OK ? f.bytes : 0;
}

occ_status_t occ_experts_linear_fwd(const occ_experts_t* l, void* ws, size_t ws_bytes, occ_stream_t stream) {
  return experts_forward_call<false>(l, ws, ws_bytes, stream);
}

occ_status_t occ_experts_gated_fwd(const occ_experts_t* l, void* ws, size_t ws_bytes, occ_stream_t stream) {
  return experts_forward_call<true>(l, ws, ws_bytes, stream);
}

occ_status_t occ_experts_linear_bwd(const occ_experts_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                                    occ_stream_t stream) {
  return experts_backward_call<false>(l, flags, ws, ws_bytes, stream);
}

occ_status_t occ_experts_gated_bwd(const occ_experts_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                                   occ_stream_t stream) {
  return experts_backward_call<true>(l, flags, ws, ws_bytes, stream);
}

}  // extern "C"
