// C ABI of the distillation loss: argument checks and launches, on the host.
// A part of stage_ops.hip.
#pragma once

#include "kernels_distill.hpp"

namespace {

constexpr int64_t kMaxVocab = (int64_t)1 << 24;

occ_status_t check_distill(const occ_distill_t* d) {
  if (!d) return OCC_E_NULL;
  if ((d->dtype != OCC_F32 && d->dtype != OCC_BF16) || (d->t_dtype != OCC_F32 && d->t_dtype != OCC_BF16))
    return OCC_E_DTYPE;
  // T^2 and 1 / T are factors, and neither may overflow or be lost
  if (!(d->temperature > 0.0f) || !std::isnormal(d->temperature * d->temperature) ||
      !(d->alpha >= 0.0f && d->alpha <= 1.0f))
    return OCC_E_VALUE;
  if (d->tokens < 0 || d->tokens >= kMaxTokens || d->vocab < 1 || d->vocab > kMaxVocab || d->k < 0 ||
      d->k > OCC_MAX_TEACHER || !ld_ok(d->vocab, d->lds) || (d->dS && !ld_ok(d->vocab, d->ldds)))
    return OCC_E_SHAPE;
  if (d->k && (!ld_ok(d->k, d->ldi) || !ld_ok(d->k, d->ldt))) return OCC_E_SHAPE;
  return OCC_OK;
}

// What both passes ask of their pointers.
occ_status_t distill_pointers(const occ_distill_t& d, Spans& sp) {
  if (!d.S || (d.k && (!d.index || !d.teacher))) return OCC_E_NULL;
  const size_t es = elem_size(d.dtype), ts = elem_size(d.t_dtype);
  if (!aligned(d.S, es) || !aligned(d.dS, es) || !aligned(d.teacher, ts) || !aligned(d.index, 4) ||
      !aligned(d.labels, 4) || !aligned(d.scale, 4) || !aligned(d.loss, 4) || !aligned(d.lse, 4) ||
      !aligned(d.flags, 4))
    return OCC_E_ALIGN;
  // dS may take the place of the logits
  if (d.S != d.dS || d.lds != d.ldds) sp.add(d.S, d.tokens, d.vocab, d.lds, es, false);
  sp.add(d.dS, d.tokens, d.vocab, d.ldds, es, true);
  if (d.k) {
    sp.add(d.index, d.tokens, d.k, d.ldi, 4, false);
    sp.add(d.teacher, d.tokens, d.k, d.ldt, ts, false);
  }
  sp.add(d.labels, 1, d.tokens, 0, 4, false);
  sp.add(d.scale, 1, d.tokens, 0, 4, false);
  sp.add(d.flags, 1, 1, 0, 4, true);
  return OCC_OK;
}

DistillArgs distill_args(const occ_distill_t& d) {
  DistillArgs a{};
  a.S = d.S;
  a.lds = d.lds;
  a.index = d.index;
  a.teacher = d.teacher;
  a.ldi = d.ldi;
  a.ldt = d.ldt;
  a.labels = d.labels;
  a.scale = d.scale;
  a.loss = d.loss;
  a.lse = d.lse;
  a.dS = d.dS;
  a.ldd = d.ldds;
  a.flags = d.flags;
  a.vocab = (int32_t)d.vocab;
  a.k = d.k;
  a.teacher_bf16 = d.t_dtype == OCC_BF16;
  a.temperature = d.temperature;
  a.alpha = d.alpha;
  const size_t es = elem_size(d.dtype);
  a.stream = d.dS && 2.0 * (double)d.tokens * (double)d.vocab * (double)es > kStreamBytes &&
             rows_on_lines(d.dS, d.ldds, d.vocab, es);
  return a;
}

// Launches hold fewer than 2^32 threads: the tokens are taken in parts.
template <class F>
occ_status_t by_tokens(const occ_distill_t& d, const DistillArgs& all, int threads, F&& f) {
  const int64_t most = (((int64_t)1 << 32) - 1) / threads, es = (int64_t)elem_size(d.dtype);
  for (int64_t t = 0; t < d.tokens; t += most) {
    DistillArgs a = all;
    a.S = (const char*)a.S + t * a.lds * es;
    if (a.dS) a.dS = (char*)a.dS + t * a.ldd * es;
    if (a.index) a.index += t * a.ldi;
    if (a.teacher) a.teacher = (const char*)a.teacher + t * a.ldt * (int64_t)elem_size(d.t_dtype);
    if (a.labels) a.labels += t;
    if (a.scale) a.scale += t;
    if (a.loss) a.loss += t;
    if (a.lse) a.lse += 2 * t;
    OCC_TRY(f(a, dim3((unsigned)std::min(most, d.tokens - t))));
  }
  return OCC_OK;
}

template <class T, int NW, int VPT>
occ_status_t start_distill(const occ_distill_t& d, const DistillArgs& all, hipStream_t s) {
  return by_tokens(d, all, NW * 64, [&](const DistillArgs& a, dim3 grid) {
    return launch("distill", s, [&] {
      if (a.stream) hipLaunchKernelGGL((k_distill<T, NW, VPT, true>), grid, dim3(NW * 64), 0, s, a);
      else hipLaunchKernelGGL((k_distill<T, NW, VPT, false>), grid, dim3(NW * 64), 0, s, a);
    });
  });
}

// Waves of a block: four, which leaves other blocks of a CU to load while one
// computes, or eight where four do not hold a row; sixteen, and the exponentials
// kept, up to a token a CU.  us with sixteen and with four or eight, 511 and 512
// tokens: bf16 8000 columns 11.5 and 8.0, 51200 29.3 and 24.2; fp32 8000 12.5 and
// 9.3, 51200 41.7 and 41.8; with sixteen, 256 tokens take half of these.
constexpr int64_t kDistillTokens = 256;

template <class T, int NW>
occ_status_t distill_steps(const occ_distill_t& d, const DistillArgs& a, int64_t whole, hipStream_t s) {
  if constexpr (NW != 8) {   // eight waves: more than sixteen steps of four
    if (whole <= 2) return start_distill<T, NW, 2>(d, a, s);
    if (whole <= 4) return start_distill<T, NW, 4>(d, a, s);
  }
  if constexpr (NW == 16) {
    if (whole <= 6) return start_distill<T, NW, 6>(d, a, s);
  }
  if (whole <= 8) return start_distill<T, NW, 8>(d, a, s);
  return start_distill<T, NW, 16>(d, a, s);
}

template <class T>
occ_status_t run_distill(const occ_distill_t& d, hipStream_t s) {
  const DistillArgs a = distill_args(d);
  const int64_t four = d.vocab / (256 * (16 / (int64_t)sizeof(T)));   // whole steps of four waves
  if (d.tokens > kDistillTokens || four <= 2) {
    if (four <= 16) return distill_steps<T, 4>(d, a, four, s);
    if (four / 2 <= 16) return distill_steps<T, 8>(d, a, four / 2, s);
  }
  if (four / 4 <= 16) return distill_steps<T, 16>(d, a, four / 4, s);
  return by_tokens(d, a, 1024, [&](const DistillArgs& b, dim3 grid) {
    return launch("distill", s, [&] { hipLaunchKernelGGL((k_distill_long<T>), grid, dim3(1024), 0, s, b); });
  });
}

template <class T>
occ_status_t run_distill_bwd(const occ_distill_t& d, hipStream_t s) {
  const DistillArgs all = distill_args(d);
  const bool wide = d.tokens <= kDistillTokens;
  return by_tokens(d, all, wide ? 1024 : 256, [&](const DistillArgs& a, dim3 grid) {
    return launch("distill_bwd", s, [&] {
      if (wide) hipLaunchKernelGGL((k_distill_bwd<T, 16, false>), grid, dim3(1024), 0, s, a);
      else if (a.stream) hipLaunchKernelGGL((k_distill_bwd<T, 4, true>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((k_distill_bwd<T, 4, false>), grid, dim3(256), 0, s, a);
    });
  });
}

}  // namespace

extern "C" {

occ_status_t occ_distill_fwd(const occ_distill_t* dp, occ_stream_t stream) {
  OCC_TRY(check_distill(dp));
  const occ_distill_t& d = *dp;
  if (!d.tokens) return OCC_OK;
  if (!d.loss) return OCC_E_NULL;
  Spans sp;
  OCC_TRY(distill_pointers(d, sp));
  sp.add(d.loss, 1, d.tokens, 0, 4, true);
  sp.add(d.lse, 1, 2 * d.tokens, 0, 4, true);
  if (sp.clash()) return OCC_E_ALIAS;
  hipStream_t s = (hipStream_t)stream;
  return by_type(d.dtype, [&](auto t) { return run_distill<decltype(t)>(d, s); });
}

occ_status_t occ_distill_bwd(const occ_distill_t* dp, occ_stream_t stream) {
  OCC_TRY(check_distill(dp));
  const occ_distill_t& d = *dp;
  if (!d.tokens) return OCC_OK;
  if (!d.dS || !d.lse) return OCC_E_NULL;
  Spans sp;
  OCC_TRY(distill_pointers(d, sp));
  sp.add(d.lse, 1, 2 * d.tokens, 0, 4, false);
  if (sp.clash()) return OCC_E_ALIAS;
  hipStream_t s = (hipStream_t)stream;
  return by_type(d.dtype, [&](auto t) { return run_distill_bwd<decltype(t)>(d, s); });
}

}  // extern "C"
