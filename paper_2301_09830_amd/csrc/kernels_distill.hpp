// Loss of a language model's logits against a teacher's top logits and the
// labels, with its gradient.  For a token with logits s, temperature T and
// weight alpha, with the teacher's k entries t at columns i:
//
//   p = softmax(t / T) over the entries, q = softmax(s / T), c = softmax(s)
//   loss = scale [alpha T^2 sum p (log p - log q_i) + (1 - alpha) (-log c_label)]
//   ds_j = scale [alpha T (q_j - p_j) + (1 - alpha) (c_j - [j = label])]
//
// Bound by memory: the loss with its gradient reads every logit once and
// writes it once, the row held in registers in between (8192 x 51200 bf16 314 us,
// 5.3 TB/s; fp32 1003 x 32003 without the gradient 28 us, 4.2 TB/s, the gradient from
// stored logarithms 45, 5.6 TB/s; 2048 x 200000 bf16, in two passes, 417).  Few
// tokens are bound by the instructions of a CU that has a row to itself (4 x 51200
// 9 us, 4 x 500 5.5).
#pragma once

#include "kernels_route.hpp"

namespace occ {

constexpr int DL_ENTRIES = 1024;   // of a teacher's list

struct DistillArgs {
  const void* S;          // tokens x vocab
  int64_t lds;
  const int32_t* index;   // tokens x k
  const void* teacher;    // tokens x k
  int64_t ldi, ldt;
  const int32_t* labels;  // may be null
  const float* scale;     // may be null
  float* loss;
  float* lse;             // tokens x 2: at the temperature, at 1; may be null
  void* dS;               // may be null
  int64_t ldd;
  uint32_t* flags;
  int32_t vocab, k, teacher_bf16;
  float temperature, alpha;
  int32_t stream;         // dS bypasses the caches
};

// One token's entries, in LDS; the label's is behind the teacher's.  Entries of
// one column are taken together in the gradient: the first of them (column)
// has what all of them take off it (off).
template <int N>
struct DistillToken {
  int32_t index[N + 1], column[N + 1];   // -1: masked
  float p[N + 1], s[N + 1], off[N + 1];
};

// Sum (or maximum) over a block of NW waves, in every thread.
template <int NW, class F>
__device__ __forceinline__ float block_reduce(float x, float* lds, F&& f) {
  x = __uint_as_float(over_lanes<64>(__float_as_uint(x), [&](uint32_t a, uint32_t b) {
    return __float_as_uint(f(__uint_as_float(a), __uint_as_float(b)));
  }));
  if constexpr (NW == 1) return x;
  __syncthreads();   // the last use of lds has ended
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  x = lds[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) x = f(x, lds[w]);
  return x;
}

// NaN wins.
__device__ __forceinline__ float max_nan(float a, float b) { return a != a || a > b ? a : b; }

template <int NW>
__device__ __forceinline__ float block_max(float x, float* lds) {
  return block_reduce<NW>(x, lds, [](float a, float b) { return max_nan(a, b); });
}

template <int NW>
__device__ __forceinline__ float block_sum(float x, float* lds) {
  return block_reduce<NW>(x, lds, [](float a, float b) { return a + b; });
}

// A token's part in the loss, the same in all threads.
struct DistillRow {
  float scale;
  bool soft, hard;    // has entries; has a label
  float entropy;      // sum of p log p
};

// Reads the entries and their logits, makes p.  Returns with the block in step.
template <class T, int NW>
__device__ __forceinline__ DistillRow distill_entries(const DistillArgs& g, int64_t token, DistillToken<DL_ENTRIES>& e,
                                                      float* lds) {
  constexpr int NT = NW * 64;
  DistillRow r;
  r.scale = g.scale ? g.scale[token] : 1.0f;
  const int label = g.labels && g.alpha != 1.0f ? g.labels[token] : -1;
  r.hard = r.scale != 0.0f && label >= 0 && label < g.vocab;
  r.soft = false;
  r.entropy = 0.0f;
  bool bad = label >= g.vocab;
  const int k = g.alpha != 0.0f ? g.k : 0;
  auto raise = [&] {
    if (__ballot(bad) && (threadIdx.x & 63) == 0 && g.flags) atomicOr(g.flags, kBadRows);
  };
  if (r.scale == 0.0f) {   // no part in the loss; its columns are checked all the same
    if (!g.flags) return r;
    for (int j = threadIdx.x; j < k; j += NT) bad |= g.index[token * g.ldi + j] >= g.vocab;
    raise();
    return r;
  }
  const T* const row = (const T*)g.S + token * g.lds;
  const float inv = 1.0f / g.temperature;
  for (int j = threadIdx.x; j < k; j += NT) {
    const int i = g.index[token * g.ldi + j];
    const bool in = i >= 0 && i < g.vocab;
    bad |= i >= g.vocab;
    float t = g.teacher_bf16 ? ld_elem<uint16_t>((const uint16_t*)g.teacher + token * g.ldt + j)
                             : ((const float*)g.teacher)[token * g.ldt + j];
    t = in ? t : -INFINITY;   // what stands at a masked entry is not looked at
    const bool live = t != -INFINITY;
    e.index[j] = live ? i : -1;
    e.p[j] = t;
    e.s[j] = live ? ld_elem<T>(row + i) : 0.0f;
  }
  if (threadIdx.x == 0) {
    e.index[g.k] = r.hard ? label : -1;
    e.s[g.k] = r.hard ? ld_elem<T>(row + label) : 0.0f;
  }
  raise();
  __syncthreads();
  // the teacher's softmax by one wave, while the row is on its way to the others;
  // the maximum is subtracted before the division by T, as in the row's
  if (threadIdx.x < 64) {
    float top = -INFINITY, sum = 0.0f, plog = 0.0f;
    for (int j = threadIdx.x; j < k; j += 64) top = max_nan(top, e.p[j]);
    top = block_max<1>(top, lds);
    if (top != -INFINITY) {
      for (int j = threadIdx.x; j < k; j += 64) sum += exp_f((e.p[j] - top) * inv);
      sum = block_sum<1>(sum, lds);
      const float log_sum = logf(sum), part = 1.0f / sum;
      for (int j = threadIdx.x; j < k; j += 64) {
        const float d = (e.p[j] - top) * inv, p = exp_f(d) * part;
        plog += p > 0.0f || p != p ? p * (d - log_sum) : 0.0f;
        e.p[j] = p;
      }
      plog = block_sum<1>(plog, lds);
    }
    if (threadIdx.x == 0) {
      lds[0] = top;
      lds[1] = plog;
    }
  }
  __syncthreads();
  r.soft = lds[0] != -INFINITY;
  r.entropy = lds[1];
  if (g.dS) {
    const float soft = r.scale * g.alpha * g.temperature, hard = r.scale * (1.0f - g.alpha);
    for (int j = threadIdx.x; j <= g.k; j += NT) {
      const int at = j == g.k || r.soft ? e.index[j] : -1;
      float off = 0.0f;
      bool first = at >= 0;
      if (first && r.soft) {
        // every entry with every other, k^2 pairs of reads: 8192 x 51200 takes 344 us at
        // k 128, 408 at 256, 613 at 512, 1565 at 1024; without branches, so that the
        // reads are in flight together
#pragma unroll 8
        for (int i = 0; i < k; ++i) {
          const bool same = e.index[i] == at;
          const float p = e.p[i];
          first &= !same | (i >= j);
          off += same ? p : 0.0f;
        }
      }
      off *= soft;
      if (r.hard && e.index[g.k] == at) off += hard;
      e.column[j] = first ? at : -1;
      e.off[j] = off;
    }
    __syncthreads();
  }
  return r;
}

// The loss from a row's statistics: m its maximum, z and z1 the sums of
// exp((s - m) / T) and exp(s - m).
template <int NW>
__device__ __forceinline__ void distill_loss(const DistillArgs& g, int64_t token, const DistillRow& r,
                                             const DistillToken<DL_ENTRIES>& e, float m, float z, float z1,
                                             float* lds) {
  if (threadIdx.x >= 64) return;   // one wave
  const float inv = 1.0f / g.temperature, log_z = logf(z), log_1 = logf(z1);
  float cross = 0.0f;   // -sum p log q
  if (r.soft) {
    for (int j = threadIdx.x; j < g.k; j += 64) {
      const float p = e.p[j];
      if (p > 0.0f || p != p) cross += p * (log_z - (e.s[j] - m) * inv);
    }
    cross = block_sum<1>(cross, lds);
  }
  if (threadIdx.x) return;
  float loss = 0.0f;
  if (r.soft) loss = g.alpha * g.temperature * g.temperature * (r.entropy + cross);
  if (r.hard) loss += (1.0f - g.alpha) * (log_1 - (e.s[g.k] - m));
  g.loss[token] = r.scale * loss;
  if (g.lse) {
    g.lse[2 * token] = r.soft ? m * inv + log_z : 0.0f;
    g.lse[2 * token + 1] = r.hard ? m + log_1 : 0.0f;
  }
}

constexpr float kLog2e = 1.4426950408889634f;

// Exponentials of a row: e^((s - m) / T), or e^(s - m) for the labels alone or
// at T = 1, and both where a token has entries and a label at another
// temperature (`two`).  m is the row's maximum, subtracted before anything is
// multiplied, so that rows of the type's lowest values stay exact.
struct DistillExp {
  float m, ka, kb;
  bool two;
  __device__ __forceinline__ DistillExp(const DistillArgs& g, const DistillRow& r, float top) {
    m = top;
    ka = r.soft ? kLog2e / g.temperature : kLog2e;
    kb = kLog2e;
    two = r.soft && r.hard && g.temperature != 1.0f;
  }
  __device__ __forceinline__ float a(float s) const { return __builtin_amdgcn_exp2f((s - m) * ka); }
  __device__ __forceinline__ float b(float s) const { return __builtin_amdgcn_exp2f((s - m) * kb); }
};

// The same over their sums, from stored logarithms of these: e^(s / T - lse).
// The logarithm is subtracted before anything is rounded but it and 1 / T, so an
// exponent is off by a few 2^-24 of |lse| + |s| / T.  That is too much for rows
// whose logarithm is beyond kFarLse (6e-4 of the softmax there; all of it for a
// row of the type's lowest values): they are summed anew, and use the maximum
// (2048 x 51200 bf16 102 us, 72 from the logarithms).
constexpr float kFarLse = 1024.0f;

struct DistillLse {
  float ia, oa, ob, ka;
  bool two;
  __device__ __forceinline__ DistillLse(const DistillArgs& g, const DistillRow& r, float soft, float hard) {
    ia = r.soft ? 1.0f / g.temperature : 1.0f;
    oa = r.soft ? soft : hard;
    ob = hard;
    ka = kLog2e;
    two = r.soft && r.hard && g.temperature != 1.0f;
  }
  __device__ __forceinline__ void from_maximum(const DistillExp& x) {
    ia = 1.0f;
    oa = ob = x.m;
    ka = x.ka;
  }
  __device__ __forceinline__ float a(float s) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(s, ia, -oa) * ka); }
  __device__ __forceinline__ float b(float s) const { return __builtin_amdgcn_exp2f((s - ob) * kLog2e); }
};

// Factors of the exponentials in the gradient.
struct DistillGrad {
  float fa, fb;
  __device__ __forceinline__ DistillGrad(const DistillArgs& g, const DistillRow& r, bool two, float z, float z1) {
    const float soft = r.soft ? r.scale * g.alpha * g.temperature / z : 0.0f;
    const float hard = r.hard ? r.scale * (1.0f - g.alpha) / z1 : 0.0f;
    fa = two ? soft : soft + hard;
    fb = two ? hard : 0.0f;
  }
};

template <class T, class X>
__device__ __forceinline__ f32x4_t grad_piece(f32x4_t v, const X& x, const DistillGrad& d) {
  constexpr int CH = 16 / sizeof(T);
  float e[CH];
  widen<T>(v, e);
  if (x.two) {
#pragma unroll
    for (int i = 0; i < CH; ++i) e[i] = __builtin_fmaf(d.fb, x.b(e[i]), d.fa * x.a(e[i]));
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) e[i] = d.fa * x.a(e[i]);
  }
  return narrow<T>(e);
}

template <class T, bool NT>
__device__ __forceinline__ void st_row_piece(T* p, f32x4_t v, int left) {
  constexpr int CH = 16 / sizeof(T);
  if constexpr (NT) {
    if (left >= CH) return __builtin_nontemporal_store(v, (f32x4_t*)p);
  }
  st_piece<T>(p, v, left);
}

// The columns of the entries, over what the rest of the row stored there: each
// by the wave that stored it, whose stores to one place stay in order.
template <class T, int NW, class X>
__device__ __forceinline__ void store_entries(const DistillArgs& g, int64_t token, const DistillToken<DL_ENTRIES>& e,
                                              const X& x, const DistillGrad& d) {
  constexpr int CH = 16 / sizeof(T);
  wave_step();
  const int wave = wave_id();
  for (int j = threadIdx.x & 63; j <= g.k; j += 64) {
    const int at = e.column[j];
    if (at < 0 || (int)((uint32_t)at / (64 * CH) % NW) != wave) continue;
    const float s = e.s[j];
    float v = d.fa * x.a(s);
    if (x.two) v = __builtin_fmaf(d.fb, x.b(s), v);
    st_elem((T*)g.dS + token * g.ldd + at, v - e.off[j]);
  }
}

template <class T, int NW>
__device__ __forceinline__ void zero_row(const DistillArgs& g, int64_t token) {
  constexpr int CH = 16 / sizeof(T);
  T* const row = (T*)g.dS + token * g.ldd;
  for (int c = threadIdx.x * CH; c < g.vocab; c += NW * 64 * CH) st_piece<T>(row + c, f32x4_t{}, g.vocab - c);
}

// A token that has no part in the loss: its logits are not read.
template <class T, int NW>
__device__ __forceinline__ void ignored_token(const DistillArgs& g, int64_t token) {
  if (threadIdx.x == 0) {
    if (g.loss) g.loss[token] = 0.0f;
    if (g.lse) g.lse[2 * token] = g.lse[2 * token + 1] = 0.0f;
  }
  if (g.dS) zero_row<T, NW>(g, token);
}

// A token a block, its row in the registers of NW waves: one pass over memory.
// A step is a piece of 16 bytes a thread; of a row's steps at most VPT are
// whole, and one more may be partial.  A piece is widened anew in each pass
// over the registers (`fresh`): kept from one to the next, bf16 rows would take
// twice the registers that they are loaded into.  The array has nine
// pieces or more: the compiler makes one vector of up to 32 registers, which a
// conditional load of a piece copies as a whole, and spills it.
__device__ __forceinline__ f32x4_t fresh(f32x4_t& v) {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" : "+v"(v));
  return v;
}

template <class T>
__device__ __forceinline__ float piece_max(f32x4_t v, float m) {
  constexpr int CH = 16 / sizeof(T);
  float f[CH];
  widen<T>(v, f);
#pragma unroll
  for (int i = 0; i < CH; ++i) m = fmaxf(m, f[i]);
  return m;
}

// keep, if not null, receives the exponentials (unless there are two of each).
template <class T>
__device__ __forceinline__ void piece_sums(f32x4_t v, const DistillExp& x, float& z, float& z1, float* keep = nullptr) {
  constexpr int CH = 16 / sizeof(T);
  float f[CH];
  widen<T>(v, f);
  if (x.two) {
#pragma unroll
    for (int i = 0; i < CH; ++i) z1 += x.b(f[i]);
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const float a = x.a(f[i]);
    if (keep) keep[i] = a;
    z += a;
  }
}

template <class T, int NW, int VPT, bool NT>
__global__ __launch_bounds__(NW * 64, 4) void k_distill(DistillArgs g) {
  constexpr int CH = 16 / sizeof(T), STEP = NW * 64 * CH;
  __shared__ DistillToken<DL_ENTRIES> e;
  __shared__ float lds[NW];
  const int64_t token = blockIdx.x;
  const T* const row = (const T*)g.S + token * g.lds;
  const int c0 = threadIdx.x * CH, whole = g.vocab / STEP, c1 = c0 + whole * STEP;
  f32x4_t v[VPT < 9 ? 9 : VPT], last;
  // on its way while the entries are read; of few tokens without a look at the scale
  if (NW == 16 || !g.scale || g.scale[token] != 0.0f) {
#pragma unroll
    for (int p = 0; p < VPT; ++p)
      if (p < whole) v[p] = ld_piece<T>(row + c0 + p * STEP, CH);
    last = row_piece<T>(row, c1, g.vocab);
  }
  const DistillRow r = distill_entries<T, NW>(g, token, e, lds);
  if (!r.soft && !r.hard) return ignored_token<T, NW>(g, token);
  float m = piece_max<T>(fresh(last), -INFINITY);
#pragma unroll
  for (int p = 0; p < VPT; ++p)
    if (p < whole) m = piece_max<T>(fresh(v[p]), m);
  m = block_reduce<NW>(m, lds, [](float a, float b) { return fmaxf(a, b); });
  const DistillExp x(g, r, m);
  // sixteen waves take few tokens, a CU each, and are bound by instructions: the
  // exponentials stay in registers
  constexpr bool KEEP = NW == 16 && VPT * CH <= 48;   // of 128 registers
  float z = 0.0f, z1 = 0.0f, kept[KEEP ? (VPT + 1) * CH : 1];
#pragma unroll
  for (int p = 0; p < VPT; ++p)
    if (p < whole) piece_sums<T>(fresh(v[p]), x, z, z1, KEEP ? kept + p * CH : nullptr);
  piece_sums<T>(fresh(last), x, z, z1, KEEP ? kept + VPT * CH : nullptr);
  z = block_sum<NW>(z, lds);
  z1 = x.two ? block_sum<NW>(z1, lds) : z;
  distill_loss<NW>(g, token, r, e, m, z, z1, lds);
  if (!g.dS) return;
  const DistillGrad d(g, r, x.two, z, z1);
  T* const out = (T*)g.dS + token * g.ldd;
  if (KEEP && !x.two) {
    auto scaled = [&](const float* a) {
      float f[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) f[i] = d.fa * a[i];
      return narrow<T>(f);
    };
#pragma unroll
    for (int p = 0; p < VPT; ++p)
      if (p < whole) st_row_piece<T, NT>(out + c0 + p * STEP, scaled(kept + p * CH), CH);
    if (c1 < g.vocab) st_row_piece<T, NT>(out + c1, scaled(kept + VPT * CH), g.vocab - c1);
    return store_entries<T, NW>(g, token, e, x, d);
  }
#pragma unroll
  for (int p = 0; p < VPT; ++p)
    if (p < whole) st_row_piece<T, NT>(out + c0 + p * STEP, grad_piece<T>(fresh(v[p]), x, d), CH);
  if (c1 < g.vocab) st_row_piece<T, NT>(out + c1, grad_piece<T>(fresh(last), x, d), g.vocab - c1);
  store_entries<T, NW>(g, token, e, x, d);
}

// A row's maximum, and the sums of its exponentials, kept together in one pass
// of U pieces at a time.  unit: an exponential's factors (its m is not used).
struct DistillSums {
  float m, z, z1;
};

template <class T, int NW, int U>
__device__ __forceinline__ DistillSums row_sums(const T* row, int vocab, const DistillExp& unit, float* lds) {
  constexpr int CH = 16 / sizeof(T), STEP = NW * 64 * CH;
  float m = -INFINITY, z = 0.0f, z1 = 0.0f;
  for (int c0 = threadIdx.x * CH; c0 < vocab; c0 += U * STEP) {
    f32x4_t v[U];
    float f[U][CH], top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = row_piece<T>(row, c0 + u * STEP, vocab);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      widen<T>(v[u], f[u]);
#pragma unroll
      for (int i = 0; i < CH; ++i) top = fmaxf(top, f[u][i]);
    }
    const float by = top == -INFINITY ? 0.0f : top;   // only -inf (or NaN) so far
    z *= __builtin_amdgcn_exp2f(unit.ka * (m - by));
    if (unit.two) z1 *= __builtin_amdgcn_exp2f(unit.kb * (m - by));
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        z += __builtin_amdgcn_exp2f(unit.ka * (f[u][i] - by));
        if (unit.two) z1 += __builtin_amdgcn_exp2f(unit.kb * (f[u][i] - by));
      }
    m = top;
  }
  DistillSums r;
  r.m = block_reduce<NW>(m, lds, [](float a, float b) { return fmaxf(a, b); });
  const float own = m == -INFINITY && z == 0.0f ? 0.0f : m - r.m;   // a thread without a column has nothing to add
  r.z = block_sum<NW>(z * __builtin_amdgcn_exp2f(unit.ka * own), lds);
  r.z1 = unit.two ? block_sum<NW>(z1 * __builtin_amdgcn_exp2f(unit.kb * own), lds) : r.z;
  if (r.m == -INFINITY) r.z = r.z1 = NAN;
  return r;
}

// Rows that the registers of a block do not hold: the maximum and the sums in
// one pass, then the gradient from a second one, which finds the row in the
// memory-side cache.
template <class T>
__global__ __launch_bounds__(1024) void k_distill_long(DistillArgs g) {
  constexpr int NW = 16, CH = 16 / sizeof(T), STEP = NW * 64 * CH, U = 4;
  __shared__ DistillToken<DL_ENTRIES> e;
  __shared__ float lds[NW];
  const int64_t token = blockIdx.x;
  const DistillRow r = distill_entries<T, NW>(g, token, e, lds);
  if (!r.soft && !r.hard) return ignored_token<T, NW>(g, token);
  const T* const row = (const T*)g.S + token * g.lds;
  const DistillSums sums = row_sums<T, NW, U>(row, g.vocab, DistillExp(g, r, 0.0f), lds);
  distill_loss<NW>(g, token, r, e, sums.m, sums.z, sums.z1, lds);
  if (!g.dS) return;
  const DistillExp x(g, r, sums.m);
  const DistillGrad d(g, r, x.two, sums.z, sums.z1);
  T* const out = (T*)g.dS + token * g.ldd;
  for (int c0 = threadIdx.x * CH; c0 < g.vocab; c0 += U * STEP) {
    f32x4_t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = row_piece<T>(row, c0 + u * STEP, g.vocab);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * STEP;
      if (c < g.vocab) st_piece<T>(out + c, grad_piece<T>(v[u], x, d), g.vocab - c);
    }
  }
  store_entries<T, NW>(g, token, e, x, d);
}

// The gradient from the stored logarithms of the sums.
template <class T, int NW, bool NT>
__global__ __launch_bounds__(NW * 64) void k_distill_bwd(DistillArgs g) {
  constexpr int CH = 16 / sizeof(T), STEP = NW * 64 * CH, U = 4;
  __shared__ DistillToken<DL_ENTRIES> e;
  __shared__ float lds[NW];
  const int64_t token = blockIdx.x;
  const float soft = g.lse[2 * token], hard = g.lse[2 * token + 1];
  const DistillRow r = distill_entries<T, NW>(g, token, e, lds);
  if (!r.soft && !r.hard) return zero_row<T, NW>(g, token);
  DistillLse x(g, r, soft, hard);
  const T* const row = (const T*)g.S + token * g.lds;
  float z = 1.0f, z1 = 1.0f;
  if ((r.soft && !(fabsf(soft) <= kFarLse)) || (r.hard && !(fabsf(hard) <= kFarLse))) {
    const DistillExp unit(g, r, 0.0f);
    const DistillSums sums = row_sums<T, NW, 1>(row, g.vocab, unit, lds);   // all read before a column is written
    x.from_maximum(DistillExp(g, r, sums.m));
    z = sums.z;
    z1 = sums.z1;
  }
  const DistillGrad d(g, r, x.two, z, z1);
  T* const out = (T*)g.dS + token * g.ldd;
  for (int c0 = threadIdx.x * CH; c0 < g.vocab; c0 += U * STEP) {
    f32x4_t v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = row_piece<T>(row, c0 + u * STEP, g.vocab);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * STEP;
      if (c < g.vocab) st_row_piece<T, NT>(out + c, grad_piece<T>(v[u], x, d), g.vocab - c);
    }
  }
  store_entries<T, NW>(g, token, e, x, d);
}

}  // namespace occ
