// C ABI of the router and the exchange of rows: argument checks and launches,
// on the host.  A part of stage_ops.hip.
#pragma once

#include "kernels_route.hpp"
#include "plan_experts.hpp"

namespace {

// f(T{}) with a call's type
template <class F>
occ_status_t by_type(int dtype, F&& f) {
  return dtype == OCC_BF16 ? f(uint16_t{}) : f(float{});
}

occ_status_t check_route(const occ_route_t* r) {
  if (!r) return OCC_E_NULL;
  if (r->dtype != OCC_F32 && r->dtype != OCC_BF16) return OCC_E_DTYPE;
  if (r->renorm != 0 && r->renorm != 1) return OCC_E_VALUE;
  if (r->experts < 1 || r->experts > OCC_MAX_EXPERTS || r->k < 1 || r->k > OCC_MAX_CHOICES || r->k > r->experts ||
      r->tokens < 0 || r->tokens * r->k >= kMaxTokens || r->tokens >= kMaxTokens || !ld_ok(r->experts, r->ldl))
    return OCC_E_SHAPE;
  return OCC_OK;
}

// One block makes the whole plan of up to RT_CHUNK tokens, in one launch, where
// its LDS holds it.
size_t route_small_lds(const occ_route_t& r) {
  return 4 * ((size_t)r.experts * (RT_WORDS + 1) + (size_t)r.tokens * r.k);
}

bool route_small(const occ_route_t& r) { return r.tokens <= RT_CHUNK && route_small_lds(r) <= 65536; }

// Tokens of a block, and blocks (256 at most: each adds up the counts of all).
int64_t route_per(const occ_route_t& r) { return up(div_up(r.tokens, 256), RT_CHUNK); }

size_t route_bytes(const occ_route_t& r) {
  if (!r.tokens || route_small(r)) return 0;
  Carve c;
  c.take((size_t)div_up(r.tokens, route_per(r)) * up(r.experts, 4) * 4);
  return c.total();
}

// f(lanes that share a token, quads that each holds of it)
template <class F>
occ_status_t by_experts(const occ_route_t& r, F&& f) {
  using std::integral_constant;
  if (route_lanes(r.experts, r.k) == 64) return f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (r.experts > 128) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (r.experts > 64) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
}

// f(the way of choosing)
template <class T, class F>
occ_status_t by_choices(const occ_route_t& r, F&& f) {
  if (r.k > 16 || (r.k > RT_LIST && r.experts > 256)) return f(ChooseMany<T, 64>{});
  if (r.k > RT_LIST) return f(ChooseMany<T, 16>{});
  constexpr int V = sizeof(T) == 2 ? 32 : 16;   // fp32 keys take two registers
  if (r.experts <= 32) return f(ChooseFew<T, 4, 8>{});
  if (r.experts <= 64) return f(ChooseFew<T, 4, 16>{});
  if (r.experts <= 128) return f(ChooseFew<T, 128 / V, V>{});
  if (r.experts <= 256) return f(ChooseFew<T, 256 / V, V>{});
  if (r.experts <= 512) return f(ChooseFew<T, 512 / V, V>{});
  return f(ChooseFew<T, 32, 32>{});
}

template <class T>
occ_status_t run_route(const occ_route_t& r, char* ws, hipStream_t s) {
  RouteArgs a{};
  a.logits = r.logits;
  a.ldl = r.ldl;
  a.tokens = r.tokens;
  a.experts = (int32_t)r.experts;
  a.k = r.k;
  a.renorm = r.renorm;
  a.per = (int32_t)route_per(r);
  a.index = r.index;
  a.weights = r.weights;
  a.offsets = r.offsets;
  a.order = r.order;
  a.slots = r.slots;
  a.counts = (int32_t*)(ws + kWsHeader);
  if (route_small(r))
    return by_choices<T>(r, [&](auto c) {
      return launch("route", s, [&] {
        hipLaunchKernelGGL((k_route_small<decltype(c)>), dim3(1), dim3(1024), route_small_lds(r), s, a);
      });
    });
  const dim3 grid((unsigned)div_up(r.tokens, a.per));
  OCC_TRY(by_choices<T>(r, [&](auto c) {
    return launch("route_choose", s, [&] {
      hipLaunchKernelGGL((k_route_choose<decltype(c)>), grid, dim3(1024), 0, s, a);
    });
  }));
  return launch("route_place", s, [&] { hipLaunchKernelGGL(k_route_place, grid, dim3(1024), 0, s, a); });
}

template <class T>
occ_status_t run_route_bwd(const occ_route_t& r, const float* dweights, void* dlogits, int64_t ldd, hipStream_t s) {
  RouteGradArgs all{};
  all.logits = r.logits;
  all.dlogits = dlogits;
  all.index = r.index;
  all.weights = r.weights;
  all.dweights = dweights;
  all.ldl = r.ldl;
  all.ldd = ldd;
  all.experts = (int32_t)r.experts;
  all.k = r.k;
  all.renorm = r.renorm;
  const int64_t part = route_bwd_part(r.experts, r.k);
  return by_experts(r, [&](auto lanes, auto quads) {
    for (int64_t t = 0; t < r.tokens; t += part) {
      RouteGradArgs a = all;
      a.tokens = std::min(part, r.tokens - t);
      if (a.logits) a.logits = (const T*)a.logits + t * a.ldl;
      a.dlogits = (T*)a.dlogits + t * a.ldd;
      a.index += t * a.k;
      a.weights += t * a.k;
      a.dweights += t * a.k;
      OCC_TRY(launch("route_bwd", s, [&] {
        hipLaunchKernelGGL((k_route_bwd<T, lanes, quads>), dim3((unsigned)div_up(a.tokens, 256 / lanes)), dim3(256), 0,
                           s, a);
      }));
    }
    return OCC_OK;
  });
}

void add_plan(Spans& sp, const occ_route_t& r, bool written) {
  const int64_t n = r.tokens * r.k;
  sp.add(r.index, 1, n, n, 4, written);
  sp.add(r.weights, 1, n, n, 4, written);
  if (!written) return;
  sp.add(r.offsets, 1, r.experts + 1, 0, 4, true);
  sp.add(r.order, 1, n, n, 4, true);
  sp.add(r.slots, 1, n, n, 4, true);
}

occ_status_t check_exchange(const occ_exchange_t* x) {
  if (!x) return OCC_E_NULL;
  if (x->dtype != OCC_F32 && x->dtype != OCC_BF16) return OCC_E_DTYPE;
  if (x->experts < 1 || x->experts > OCC_MAX_EXPERTS || x->k < 1 || x->k > OCC_MAX_CHOICES || x->tokens < 0 ||
      x->tokens >= kMaxTokens || x->tokens * x->k >= kMaxTokens || x->rows < 0 || x->rows >= kMaxTokens ||
      x->width < 1 || x->width > kMaxWidth)
    return OCC_E_SHAPE;
  if (!aligned(x->offsets, 4) || !aligned(x->order, 4) || !aligned(x->slots, 4) || !aligned(x->flags, 4))
    return OCC_E_ALIGN;
  return OCC_OK;
}

ExchangeArgs exchange_args(const occ_exchange_t& x) {
  ExchangeArgs a{};
  a.offsets = x.offsets;
  a.order = x.order;
  a.slots = x.slots;
  a.flags = x.flags;
  a.tokens = x.tokens;
  a.rows = x.rows;
  a.experts = (int32_t)x.experts;
  a.k = x.k;
  a.width = (int32_t)x.width;
  a.parts = (int32_t)div_up(x.width, EX_PIECES * 1024 / (int64_t)elem_size(x.dtype));
  return a;
}

dim3 exchange_grid(int64_t units) { return dim3((unsigned)std::min(div_up(units, EX_WAVES), EX_BLOCKS)); }

}  // namespace

extern "C" {

size_t occ_route_fwd_workspace_bytes(const occ_route_t* r) { return check_route(r) == OCC_OK ? route_bytes(*r) : 0; }

occ_status_t occ_route_fwd(const occ_route_t* rp, void* ws, size_t ws_bytes, occ_stream_t stream) {
  OCC_TRY(check_route(rp));
  const occ_route_t& r = *rp;
  if (!r.offsets || (r.tokens && (!r.logits || !r.index || !r.weights || !r.order || !r.slots))) return OCC_E_NULL;
  if (!aligned(r.logits, elem_size(r.dtype)) || !aligned(r.index, 4) || !aligned(r.weights, 4) ||
      !aligned(r.offsets, 4) || !aligned(r.order, 4) || !aligned(r.slots, 4))
    return OCC_E_ALIGN;
  hipStream_t s = (hipStream_t)stream;
  if (!r.tokens) return zero_rows<float>(r.offsets, 1, r.experts + 1, r.experts + 1, s);   // no rows: all bits 0
  const size_t need = route_bytes(r);
  OCC_TRY(check_ws(ws, ws_bytes, need));
  Spans sp;
  sp.add(r.logits, r.tokens, r.experts, r.ldl, elem_size(r.dtype), false);
  add_plan(sp, r, true);
  if (need) sp.add(ws, 1, (int64_t)need, 0, 1, true);
  if (sp.clash()) return OCC_E_ALIAS;
  return by_type(r.dtype, [&](auto t) { return run_route<decltype(t)>(r, (char*)ws, s); });
}

occ_status_t occ_route_bwd(const occ_route_t* rp, const float* dweights, void* dlogits, int64_t ldd,
                           occ_stream_t stream) {
  OCC_TRY(check_route(rp));
  const occ_route_t& r = *rp;
  if (!ld_ok(r.experts, ldd)) return OCC_E_SHAPE;
  if (!r.tokens) return OCC_OK;
  if (!r.index || !r.weights || !dweights || !dlogits || (!r.renorm && !r.logits)) return OCC_E_NULL;
  const size_t es = elem_size(r.dtype);
  if (!aligned(r.logits, es) || !aligned(dlogits, es) || !aligned(r.index, 4) || !aligned(r.weights, 4) ||
      !aligned(dweights, 4))
    return OCC_E_ALIGN;
  Spans sp;
  // dlogits may take the logits' place: a token's are read before they are written
  if (!r.renorm && (r.logits != dlogits || r.ldl != ldd)) sp.add(r.logits, r.tokens, r.experts, r.ldl, es, false);
  add_plan(sp, r, false);
  sp.add(dweights, 1, r.tokens * r.k, 0, 4, false);
  sp.add(dlogits, r.tokens, r.experts, ldd, es, true);
  if (sp.clash()) return OCC_E_ALIAS;
  return by_type(r.dtype,
                 [&](auto t) { return run_route_bwd<decltype(t)>(r, dweights, dlogits, ldd, (hipStream_t)stream); });
}

occ_status_t occ_dispatch(const occ_exchange_t* xp, const void* X, int64_t ldx, void* Xs, int64_t ldxs,
                          occ_stream_t stream) {
  OCC_TRY(check_exchange(xp));
  const occ_exchange_t& x = *xp;
  if (!ld_ok(x.width, ldx) || !ld_ok(x.width, ldxs)) return OCC_E_SHAPE;
  if (!x.rows) return OCC_OK;
  if (!x.offsets || !x.order || !Xs || (x.tokens && !X)) return OCC_E_NULL;
  const size_t es = elem_size(x.dtype);
  if (!aligned(X, es) || !aligned(Xs, es)) return OCC_E_ALIGN;
  Spans sp;
  sp.add(X, x.tokens, x.width, ldx, es, false);
  sp.add(Xs, x.rows, x.width, ldxs, es, true);
  sp.add(x.offsets, 1, x.experts + 1, 0, 4, false);
  sp.add(x.order, 1, x.rows, 0, 4, false);
  sp.add(x.flags, 1, 1, 0, 4, true);
  if (sp.clash()) return OCC_E_ALIAS;
  ExchangeArgs a = exchange_args(x);
  a.in = X;
  a.ldi = ldx;
  a.out = Xs;
  a.ldo = ldxs;
  return by_type(x.dtype, [&](auto t) {
    return launch("dispatch", (hipStream_t)stream, [&] {
      hipLaunchKernelGGL((k_dispatch<decltype(t)>), exchange_grid(x.rows * a.parts), dim3(EX_WAVES * 64), 0,
                         (hipStream_t)stream, a);
    });
  });
}

occ_status_t occ_combine(const occ_exchange_t* xp, const float* weights, const void* Ys, int64_t ldys, const void* R,
                         int64_t ldr, void* Y, int64_t ldy, occ_stream_t stream) {
  OCC_TRY(check_exchange(xp));
  const occ_exchange_t& x = *xp;
  if (!ld_ok(x.width, ldys) || !ld_ok(x.width, ldy) || (R && !ld_ok(x.width, ldr))) return OCC_E_SHAPE;
  if (!x.tokens) return OCC_OK;
  if (!x.slots || !Y || (x.rows && !Ys)) return OCC_E_NULL;
  const size_t es = elem_size(x.dtype);
  if (!aligned(Ys, es) || !aligned(R, es) || !aligned(Y, es) || !aligned(weights, 4)) return OCC_E_ALIGN;
  Spans sp;
  sp.add(Ys, x.rows, x.width, ldys, es, false);
  if (R && (R != Y || ldr != ldy)) sp.add(R, x.tokens, x.width, ldr, es, false);
  sp.add(Y, x.tokens, x.width, ldy, es, true);
  sp.add(x.slots, 1, x.tokens * x.k, 0, 4, false);
  sp.add(weights, 1, x.tokens * x.k, 0, 4, false);
  sp.add(x.flags, 1, 1, 0, 4, true);
  if (sp.clash()) return OCC_E_ALIAS;
  ExchangeArgs a = exchange_args(x);
  a.in = Ys;
  a.ldi = ldys;
  a.other = R;
  a.ldt = ldr;
  a.out = Y;
  a.ldo = ldy;
  a.weights = weights;
  return by_type(x.dtype, [&](auto t) {
    return launch("combine", (hipStream_t)stream, [&] {
      hipLaunchKernelGGL((k_combine<decltype(t)>), exchange_grid(x.tokens * a.parts), dim3(EX_WAVES * 64), 0,
                         (hipStream_t)stream, a);
    });
  });
}

occ_status_t occ_combine_bwd(const occ_exchange_t* xp, const float* weights, const void* dY, int64_t lddy,
                             const void* Ys, int64_t ldys, void* dYs, int64_t lddys, float* dweights,
                             occ_stream_t stream) {
  OCC_TRY(check_exchange(xp));
  const occ_exchange_t& x = *xp;
  if (!dYs && !dweights) return OCC_E_NULL;
  if (!ld_ok(x.width, lddy) || (dweights && !ld_ok(x.width, ldys)) || (dYs && !ld_ok(x.width, lddys)))
    return OCC_E_SHAPE;
  if (!x.tokens) return OCC_OK;
  if (!x.slots || !dY || (x.rows && (!x.order || (dweights && !Ys)))) return OCC_E_NULL;
  const size_t es = elem_size(x.dtype);
  if (!aligned(dY, es) || !aligned(Ys, es) || !aligned(dYs, es) || !aligned(weights, 4) || !aligned(dweights, 4))
    return OCC_E_ALIGN;
  Spans sp;
  sp.add(dY, x.tokens, x.width, lddy, es, false);
  if (dweights) sp.add(Ys, x.rows, x.width, ldys, es, false);
  sp.add(dYs, x.rows, x.width, lddys, es, true);
  sp.add(dweights, 1, x.tokens * x.k, 0, 4, true);
  sp.add(weights, 1, x.tokens * x.k, 0, 4, false);
  sp.add(x.slots, 1, x.tokens * x.k, 0, 4, false);
  sp.add(x.order, 1, x.rows, 0, 4, false);
  sp.add(x.flags, 1, 1, 0, 4, true);
  if (sp.clash()) return OCC_E_ALIAS;
  ExchangeArgs a = exchange_args(x);
  a.in = dY;
  a.ldi = lddy;
  a.other = Ys;
  a.ldt = ldys;
  a.out = dYs;
  a.ldo = lddys;
  a.weights = weights;
  a.dweights = dweights;
  return by_type(x.dtype, [&](auto t) {
    return launch("combine_bwd", (hipStream_t)stream, [&] {
      hipLaunchKernelGGL((k_combine_bwd<decltype(t)>), exchange_grid(x.tokens * x.k), dim3(EX_WAVES * 64), 0,
                         (hipStream_t)stream, a);
    });
  });
}

}  // extern "C"
