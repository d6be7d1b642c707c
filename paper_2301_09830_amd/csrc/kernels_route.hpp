// The router of a layer of experts, and the exchange of rows between the
// tokens' order and the experts'.
#pragma once

#include "kernels_experts.hpp"

namespace occ {

template <class T>
__device__ __forceinline__ void st_piece(T* p, f32x4_t v, int left) {
  constexpr int CH = 16 / sizeof(T);
  if (left >= CH) {
    if constexpr (sizeof(T) == 4) *(f4u_t*)p = f4u_t{v[0], v[1], v[2], v[3]};
    else *(u4h_t*)p = __builtin_bit_cast(u4h_t, v);
    return;
  }
  T e[CH];
  __builtin_memcpy(e, &v, 16);
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (i < left) p[i] = e[i];
}

// A piece of a row, -inf behind its end.
template <class T>
__device__ __forceinline__ f32x4_t row_piece(const T* row, int c, int vocab) {
  constexpr int CH = 16 / sizeof(T);
  if (c + CH <= vocab) return ld_piece<T>(row + c, CH);
  const uint32_t low = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  f32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(low);
  if (c >= vocab) return v;
  T e[CH];
  __builtin_memcpy(e, &v, 16);
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (c + i < vocab) e[i] = row[c + i];
  __builtin_memcpy(&v, e, 16);
  return v;
}

// The elements of a piece as fp32, and back.
template <class T>
__device__ __forceinline__ void widen(f32x4_t v, float* e) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e[2 * i] = bf16_lo(__float_as_uint(v[i]));
      e[2 * i + 1] = bf16_hi(__float_as_uint(v[i]));
    }
  }
}

template <class T>
__device__ __forceinline__ f32x4_t narrow(const float* e) {
  if constexpr (sizeof(T) == 4) return f32x4_t{e[0], e[1], e[2], e[3]};
  f32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(bf16_pack2(e[2 * i], e[2 * i + 1]));
  return v;
}

// ----------------------------------------------------------------------------
// choice of the experts
// ----------------------------------------------------------------------------
struct RouteArgs {
  const void* logits;   // tokens x experts
  int64_t ldl;
  int64_t tokens;
  int32_t experts, k, renorm;
  int32_t per;          // tokens of a block
  int32_t* index;       // tokens x k
  float* weights;
  int32_t* offsets;     // experts + 1
  int32_t* order;       // tokens * k: entries (token * k + j) by expert, in order
  int32_t* slots;       // tokens x k: an entry's place in it
  int32_t* counts;      // workspace, blocks x experts
};

// Order of the logits as unsigned integers: -0 as 0; 0 for -inf and NaN, which
// are never chosen.
__device__ __forceinline__ uint32_t rank_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  if (!(x > -INFINITY)) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r); }

// A reduction over the L lanes (16 or 64) that share a token, in every one.
template <int CTRL>
__device__ __forceinline__ uint32_t row_turn(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}

template <int L, class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t x, F&& f) {
  x = f(x, row_turn<0x128>(x));   // 8, 4, 2 and 1 lanes round a row of 16
  x = f(x, row_turn<0x124>(x));
  x = f(x, row_turn<0x122>(x));
  x = f(x, row_turn<0x121>(x));
  if constexpr (L == 64) {
    x = f(x, (uint32_t)__shfl_xor((int)x, 16));
    x = f(x, (uint32_t)__shfl_xor((int)x, 32));
  }
  return x;
}

template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  return over_lanes<L>(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

template <int L>
__device__ __forceinline__ uint32_t lanes_min(uint32_t x) {
  return over_lanes<L>(x, [](uint32_t a, uint32_t b) { return min(a, b); });
}

template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
  return __uint_as_float(over_lanes<L>(__float_as_uint(x), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

// exp(x) with the hardware's exp2: x log2(e) rounded, |x| 2^-24 relative
__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(1.4426950408889634f * x); }

// A token's logits, of which each of L lanes holds Q quads: columns 4 (q L +
// lane) .. + 3.  Those behind the last expert are -inf.
template <class T, int L, int Q>
__device__ __forceinline__ void load_logits(const void* p, int64_t ld, int64_t token, int experts, int lane, float* x) {
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int c = (q * L + lane) * 4, left = experts - c;
    f32x4_t v = {};
    if (left > 0) v = ld_quad<T>((const T*)p + token * ld + c, left);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * q + i] = i < left ? v[i] : -INFINITY;
  }
}

// Choices of a token: index -1 and weight 0 where there is none.  The lower
// index comes first among equals, so a logit and its column are one key: in
// bf16 they fit one word; in fp32 they take 42 bits of a double's fraction,
// whose maximum and minimum are one instruction too.
template <class T> struct RouteKey;

// What is never chosen has the rank of -inf, the lowest.
constexpr uint32_t kLowestRank = 0x007fffffu;

__device__ __forceinline__ uint32_t rank_or_lowest(float x) {
  const uint32_t u = __float_as_uint(fmaxf(x + 0.0f, -INFINITY));   // -0 is 0, NaN -inf
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

template <> struct RouteKey<uint16_t> {
  using type = uint32_t;
  static __device__ __forceinline__ type make(float x, int column) {
    return (rank_or_lowest(x) & 0xffff0000u) | (0xffffu - column);
  }
  static __device__ __forceinline__ bool some(type k) { return k > kLowestRank; }
  static __device__ __forceinline__ int column(type k) { return (int)(0xffffu - (k & 0xffffu)); }
  // the low bits of a negative value's rank are ones
  static __device__ __forceinline__ float value(type k) { return value_of(k & 0x80000000u ? k & 0xffff0000u : k | 0xffffu); }
  static __device__ __forceinline__ type larger(type a, type b) { return max(a, b); }
  static __device__ __forceinline__ type smaller(type a, type b) { return min(a, b); }
  template <class F>
  static __device__ __forceinline__ type moved(type k, F&& f) { return f(k); }
};

template <> struct RouteKey<float> {
  using type = double;
  static __device__ __forceinline__ uint64_t bits(type k) { return __builtin_bit_cast(uint64_t, k); }
  static __device__ __forceinline__ type make(float x, int column) {   // 1.0 and up: no denormal, infinity or NaN
    const uint32_t r = rank_or_lowest(x);
    return __builtin_bit_cast(double, (uint64_t)(0x3ff00000u | r >> 22) << 32 | (r << 10 | (uint32_t)(1023 - column)));
  }
  static __device__ __forceinline__ uint32_t rank(type k) { return (uint32_t)(bits(k) >> 10); }
  static __device__ __forceinline__ bool some(type k) { return rank(k) > kLowestRank; }
  static __device__ __forceinline__ int column(type k) { return 1023 - (int)(bits(k) & 1023); }
  static __device__ __forceinline__ float value(type k) { return value_of(rank(k)); }
  static __device__ __forceinline__ type larger(type a, type b) { return __builtin_fmax(a, b); }
  static __device__ __forceinline__ type smaller(type a, type b) { return __builtin_fmin(a, b); }
  template <class F>
  static __device__ __forceinline__ type moved(type k, F&& f) {
    const uint64_t u = bits(k);
    return __builtin_bit_cast(double, (uint64_t)f((uint32_t)(u >> 32)) << 32 | f((uint32_t)u));
  }
};

// Value of a lane of the other half of 2 D lanes (D up to 8: of lane ^ D, or of
// the mirrored one), for lists that are the same in all D lanes of a half.
template <int D>
__device__ __forceinline__ uint32_t other_half(uint32_t x) {
  if constexpr (D == 1) return row_turn<0xb1>(x);
  else if constexpr (D == 2) return row_turn<0x4e>(x);
  else if constexpr (D == 4) return row_turn<0x141>(x);
  else if constexpr (D == 8) return row_turn<0x140>(x);
  else return (uint32_t)__shfl_xor((int)x, D);
}

constexpr int RT_LIST = 8;   // keys of a list

template <class K>
__device__ __forceinline__ void in_order(typename K::type& a, typename K::type& b) {
  const auto x = a;
  a = K::larger(x, b);
  b = K::smaller(x, b);
}

// Falling order, by Batcher's network for eight (19 exchanges).
template <class K>
__device__ __forceinline__ void sort_list(typename K::type* k) {
  constexpr int at[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                             {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
  for (int i = 0; i < 19; ++i) in_order<K>(k[at[i][0]], k[at[i][1]]);
}

// The eight largest of two sorted lists: of a falling and a rising one the
// larger at each place, which rise and fall once and are sorted in three steps.
template <class K>
__device__ __forceinline__ void merge_list(typename K::type* k, const typename K::type* o) {
#pragma unroll
  for (int i = 0; i < RT_LIST; ++i) k[i] = K::larger(k[i], o[RT_LIST - 1 - i]);
#pragma unroll
  for (int d = RT_LIST / 2; d; d >>= 1)
#pragma unroll
    for (int i = 0; i < RT_LIST; ++i)
      if (!(i & d)) in_order<K>(k[i], k[i + d]);
}

template <class K, int D>
__device__ __forceinline__ void merge_lanes(typename K::type* k) {
  typename K::type o[RT_LIST];
#pragma unroll
  for (int i = 0; i < RT_LIST; ++i) o[i] = K::moved(k[i], [](uint32_t x) { return other_half<D>(x); });
  merge_list<K>(k, o);
}

template <int L>
__device__ __forceinline__ float sum_halves(float x) {
  auto add = [&](uint32_t y) { x += __uint_as_float(y); };
  add(other_half<1>(__float_as_uint(x)));
  add(other_half<2>(__float_as_uint(x)));
  if constexpr (L > 4) add(other_half<4>(__float_as_uint(x)));
  if constexpr (L > 8) add(other_half<8>(__float_as_uint(x)));
  if constexpr (L > 16) add(other_half<16>(__float_as_uint(x)));
  return x;
}

// Up to RT_LIST choices, of L lanes (4 to 32) that hold V (8 to 32) logits
// each: every lane sorts its keys by eights and keeps the largest, then the
// lanes' lists are merged.  Lane l ends with the choices l, l + L, ...: PER of
// them.  Bound by the exchanges, two instructions each: 128 logits are 20 a
// token of 16 in a wave (four lanes; 17 in one lane, which leaves three of four
// waves out; a pick a round, 112).  65536 x 128 bf16, k 8: 10 us, 36 a pick a round.
template <int L> constexpr int route_per() { return L < RT_LIST ? RT_LIST / L : 1; }

template <class T, int L, int V>
__device__ __forceinline__ void choose(const RouteArgs& g, int64_t token, int lane, int* index, float* weight) {
  using K = RouteKey<T>;
  constexpr int CH = 16 / sizeof(T), PER = route_per<L>();
  const T* const row = (const T*)g.logits + token * g.ldl;
  float x[V];
#pragma unroll
  for (int v = 0; v < V; v += CH) {
    widen<T>(row_piece<T>(row, (v / CH * L + lane) * CH, g.experts), x + v);
  }
  typename K::type best[RT_LIST];
  uint32_t largest = 0;   // magnitude: above infinity's, a NaN
#pragma unroll
  for (int v = 0; v < V; v += RT_LIST) {
    typename K::type k[RT_LIST];
#pragma unroll
    for (int i = 0; i < RT_LIST; ++i) {
      const int u = v + i;
      largest = max(largest, __float_as_uint(x[u]) & 0x7fffffffu);
      k[i] = K::make(x[u], (u / CH * L + lane) * CH + u % CH);
    }
    sort_list<K>(k);
    if (v) {
      merge_list<K>(best, k);
    } else {
#pragma unroll
      for (int i = 0; i < RT_LIST; ++i) best[i] = k[i];
    }
  }
  merge_lanes<K, 1>(best);
  merge_lanes<K, 2>(best);
  if constexpr (L > 4) merge_lanes<K, 4>(best);
  if constexpr (L > 8) merge_lanes<K, 8>(best);
  if constexpr (L > 16) merge_lanes<K, 16>(best);
  const float first = K::value(best[0]);
  float e[PER], part = 0.0f;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    auto mine = best[p * L];
#pragma unroll
    for (int i = 1; i < L && i < RT_LIST; ++i) mine = lane == i ? best[p * L + i] : mine;
    const int j = p * L + lane;
    const bool some = j < g.k && j < RT_LIST && K::some(mine);
    index[p] = some ? K::column(mine) : -1;
    e[p] = some ? exp_f(K::value(mine) - first) : 0.0f;
    part += e[p];
  }
  if (!g.renorm) {
    part = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) part += exp_f(x[v] - first);
  }
  const float sum = sum_halves<L>(largest > 0x7f800000u ? NAN : part);
#pragma unroll
  for (int p = 0; p < PER; ++p) weight[p] = index[p] >= 0 ? e[p] / sum : 0.0f;
}

// More than RT_LIST choices: lane j of the L that share a token ends with the
// j-th.  One pick a round: the largest of the lanes' largest.
template <class T, int L>
__device__ __forceinline__ void choose_many(const RouteArgs& g, int64_t token, int lane, int& index, float& weight) {
  constexpr int Q = 4, V = 4 * Q;
  constexpr bool PACK = sizeof(T) == 2;
  float x[V];
  uint32_t r[V];
  load_logits<T, L, Q>(g.logits, g.ldl, token, g.experts, lane, x);
  auto column = [&](int v) { return (uint32_t)(((v >> 2) * L + lane) * 4 + (v & 3)); };
  bool nan = false;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    nan |= x[v] != x[v];
    r[v] = rank_of(x[v]);
    if (PACK && r[v]) r[v] = (r[v] & 0xffff0000u) | (0xffffu - column(v));
  }
  index = -1;
  uint32_t mine = 0, top = 0;
  for (int j = 0; j < g.k; ++j) {
    uint32_t best = 0, at = 0;
    if constexpr (PACK) {
#pragma unroll
      for (int v = 0; v < V; ++v) best = max(best, r[v]);
      best = lanes_max<L>(best);
      at = 0xffffu - (best & 0xffffu);
#pragma unroll
      for (int v = 0; v < V; ++v) r[v] = r[v] == best ? 0 : r[v];
      best &= 0xffff0000u;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        at = r[v] > best ? column(v) : at;
        best = max(best, r[v]);
      }
      const uint32_t most = lanes_max<L>(best);
      at = lanes_min<L>(best == most ? at : 0xffffffffu);
      best = most;
#pragma unroll
      for (int v = 0; v < V; ++v) r[v] = column(v) == at ? 0 : r[v];
    }
    if (!j) top = best;
    if (lane == j && best) {
      mine = best;
      index = (int)at;
    }
  }
  // bf16: the low bits of a negative value's rank are ones
  auto value = [](uint32_t u) { return value_of(PACK && !(u & 0x80000000u) ? u | 0xffffu : u); };
  const float first = value(top);
  const float e = index >= 0 ? exp_f(value(mine) - first) : 0.0f;
  float part = e;
  if (!g.renorm) {
    part = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) part += x[v] > -INFINITY ? exp_f(x[v] - first) : 0.0f;
  }
  const float sum = lanes_sum<L>(nan ? NAN : part);
  weight = index >= 0 ? e / sum : 0.0f;
}

// The lanes of a token, and each one's choices: f(choice, index, weight).
template <class T, int L, int V>
struct ChooseFew {
  static constexpr int lanes = L;
  template <class F>
  static __device__ __forceinline__ void run(const RouteArgs& g, int64_t token, int lane, F&& f) {
    int index[route_per<L>()];
    float weight[route_per<L>()];
    choose<T, L, V>(g, token, lane, index, weight);
#pragma unroll
    for (int p = 0; p < route_per<L>(); ++p)
      if (p * L + lane < g.k) f(p * L + lane, index[p], weight[p]);
  }
};

template <class T, int L>
struct ChooseMany {
  static constexpr int lanes = L;
  template <class F>
  static __device__ __forceinline__ void run(const RouteArgs& g, int64_t token, int lane, F&& f) {
    int index;
    float weight;
    choose_many<T, L>(g, token, lane, index, weight);
    if (lane < g.k) f(lane, index, weight);
  }
};

// ----------------------------------------------------------------------------
// places of the entries: a stable sort by expert without a race
// ----------------------------------------------------------------------------
// Of a chunk of tokens every expert has a bit mask of those that chose it, so
// an entry's rank among its expert's is a count of bits, whatever the order in
// which the bits were set.
constexpr int RT_CHUNK = 256, RT_WORDS = RT_CHUNK / 32;
constexpr int RT_EXPERTS = 1024;

// Exclusive prefix of n values in LDS, in place, by one wave; returns the sum.
__device__ __forceinline__ int prefix_lds(int* v, int n) {
  int carry = 0;
  const int lane = threadIdx.x & 63;
  for (int i = 0; i < n; i += 64) {
    const int x = i + lane < n ? v[i + lane] : 0;
    const int sum = wave_scan(x);
    if (i + lane < n) v[i + lane] = carry + sum - x;
    carry += __builtin_amdgcn_readlane(sum, 63);
  }
  return carry;
}

__device__ __forceinline__ int mask_count(const uint32_t* m) {
  int n = 0;
#pragma unroll
  for (int w = 0; w < RT_WORDS; ++w) n += __popc(m[w]);
  return n;
}

__device__ __forceinline__ int mask_rank(const uint32_t* m, int bit) {
  int n = 0;
#pragma unroll
  for (int w = 0; w < RT_WORDS; ++w) {
    const int b = bit - 32 * w;
    n += __popc(b >= 32 ? m[w] : b > 0 ? m[w] & ((1u << b) - 1) : 0u);
  }
  return n;
}

// Up to RT_CHUNK tokens: all of it in one block and one launch.
template <class C>
__global__ __launch_bounds__(1024) void k_route_small(RouteArgs g) {
  constexpr int L = C::lanes;
  extern __shared__ uint32_t route_lds[];
  uint32_t* const mask = route_lds;                      // experts x RT_WORDS
  int* const base = (int*)(mask + g.experts * RT_WORDS);   // experts
  int* const picks = base + g.experts;                   // tokens x k
  for (int i = threadIdx.x; i < g.experts * RT_WORDS; i += 1024) mask[i] = 0;
  __syncthreads();
  const int lane = threadIdx.x % L;
  for (int t = threadIdx.x / L; t < g.tokens; t += 1024 / L) {
    C::run(g, t, lane, [&](int j, int index, float weight) {
      const int i = t * g.k + j;
      g.index[i] = index;
      g.weights[i] = weight;
      picks[i] = index;
      if (index >= 0) atomicOr(&mask[index * RT_WORDS + t / 32], 1u << (t & 31));
    });
  }
  __syncthreads();
  for (int e = threadIdx.x; e < g.experts; e += 1024) base[e] = mask_count(mask + e * RT_WORDS);
  __syncthreads();
  if (threadIdx.x < 64) {
    const int all = prefix_lds(base, g.experts);
    if (threadIdx.x == 0) g.offsets[g.experts] = all;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < g.experts; e += 1024) g.offsets[e] = base[e];
  const int n = (int)g.tokens * g.k;
  for (int i = threadIdx.x; i < n; i += 1024) {
    const int e = picks[i];
    int slot = -1;
    if (e >= 0) {
      slot = base[e] + mask_rank(mask + e * RT_WORDS, i / g.k);
      g.order[slot] = i;
    }
    g.slots[i] = slot;
  }
}

// More tokens, first launch: the choices, and how many of a block's tokens
// chose each expert (rows of whole 16 bytes).
__device__ __forceinline__ int count_row(const RouteArgs& g) { return (g.experts + 3) & ~3; }

template <class C>
__global__ __launch_bounds__(1024) void k_route_choose(RouteArgs g) {
  constexpr int L = C::lanes;
  __shared__ int count[RT_EXPERTS];
  const int row = count_row(g);
  for (int e = threadIdx.x; e < row; e += 1024) count[e] = 0;
  __syncthreads();
  const int lane = threadIdx.x % L;
  const int64_t t0 = (int64_t)blockIdx.x * g.per, t1 = min(t0 + g.per, g.tokens);
  for (int64_t t = t0 + threadIdx.x / L; t < t1; t += 1024 / L)
    C::run(g, t, lane, [&](int j, int index, float weight) {
      g.index[t * g.k + j] = index;
      g.weights[t * g.k + j] = weight;
      if (index >= 0) atomicAdd(&count[index], 1);
    });
  __syncthreads();
  for (int e = threadIdx.x; e < row; e += 1024) g.counts[(int64_t)blockIdx.x * row + e] = count[e];
}

// Second launch: every block adds up the counts before its own.  Bound by the
// latency of its few steps (8.5 us for 65536 tokens, k 8; 18.5 with 256 threads),
// so all loads of a step are in flight together: four experts a thread, the
// blocks' rows dealt to groups of threads.  Some 1.6 us of it are conflicts of
// LDS banks: the same word of random experts' masks lies in an eighth of them.
__global__ __launch_bounds__(1024) void k_route_place(RouteArgs g) {
  __shared__ uint32_t mask[RT_EXPERTS * RT_WORDS];
  __shared__ int total[RT_EXPERTS], prior[RT_EXPERTS];
  const int blocks = gridDim.x, me = blockIdx.x, row = count_row(g);
  for (int e = threadIdx.x; e < row; e += 1024) total[e] = prior[e] = 0;
  __syncthreads();
  const int quads = row / 4, groups = 1024 / quads, group = threadIdx.x / quads;
  if (group < groups) {
    const int q = threadIdx.x - group * quads;
    i32x4_t all = {}, before = {};
#pragma unroll 8
    for (int b = group; b < blocks; b += groups) {
      const i32x4_t n = *(const i32x4_t*)(g.counts + (int64_t)b * row + 4 * q);
      all += n;
      if (b < me) before += n;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      atomicAdd(&total[4 * q + i], all[i]);
      atomicAdd(&prior[4 * q + i], before[i]);
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int all = prefix_lds(total, g.experts);
    if (me == 0 && threadIdx.x == 0) g.offsets[g.experts] = all;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < g.experts; e += 1024) {
    if (me == 0) g.offsets[e] = total[e];
    prior[e] += total[e];
  }
  const int64_t t0 = (int64_t)me * g.per, t1 = min(t0 + g.per, g.tokens);
  for (int64_t c = t0; c < t1; c += RT_CHUNK) {
    const int n = (int)min((int64_t)RT_CHUNK, t1 - c) * g.k;
    const int64_t i0 = c * g.k;
    for (int i = threadIdx.x; i < g.experts * RT_WORDS; i += 1024) mask[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024) {
      const int e = g.index[i0 + i], t = i / g.k;
      if (e >= 0) atomicOr(&mask[e * RT_WORDS + t / 32], 1u << (t & 31));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024) {
      const int e = g.index[i0 + i];
      int slot = -1;
      if (e >= 0) {
        slot = prior[e] + mask_rank(mask + e * RT_WORDS, i / g.k);
        g.order[slot] = (int)(i0 + i);
      }
      g.slots[i0 + i] = slot;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < g.experts; e += 1024) prior[e] += mask_count(mask + e * RT_WORDS);
    __syncthreads();
  }
}

// ----------------------------------------------------------------------------
// gradient of the logits
// ----------------------------------------------------------------------------
// Bound by memory and its few dependent steps (65536 x 128 bf16, k 8, softmax
// over all experts: 39.8 MB in 11 to 13 us; renormalised, without the logits,
// 23.1 MB in 5.9 where they lie in the caches).  With s = sum of w dw over the
// choices: renormalised weights give the chosen logits w (dw - s); weights of the
// softmax over all experts give -p s at every expert and w dw more at the chosen
// ones.
struct RouteGradArgs {
  const void* logits;
  void* dlogits;
  const int32_t* index;
  const float* weights;
  const float* dweights;
  int64_t ldl, ldd, tokens;
  int32_t experts, k, renorm;
};

// The compiler keeps memory accesses on their side of this.
__device__ __forceinline__ void wave_step() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <class T, int L, int Q>
__global__ __launch_bounds__(256) void k_route_bwd(RouteGradArgs g) {
  constexpr int V = 4 * Q;
  const int lane = threadIdx.x % L;
  const int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const bool in = t < g.tokens;   // the lanes of a token go together
  int index = -1;
  float w = 0.0f, up = 0.0f;
  if (in && lane < g.k) {
    index = g.index[t * g.k + lane];
    if (index >= 0) {   // what stands at a choice that is none is not looked at
      w = g.weights[t * g.k + lane];
      up = w * g.dweights[t * g.k + lane];
    }
  }
  const float s = lanes_sum<L>(up);
  const float d = g.renorm ? up - w * s : up;
  float x[V];
  if (!g.renorm) {
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = -INFINITY;
    if (in) load_logits<T, L, Q>(g.logits, g.ldl, t, g.experts, lane, x);
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) top = max(top, rank_of(x[v]));
    top = lanes_max<L>(top);
    const float first = top ? value_of(top) : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = x[v] == -INFINITY ? 0.0f : exp_f(x[v] - first);
      sum += x[v];
    }
    sum = lanes_sum<L>(sum);
    const float f = top ? -s / sum : sum;   // no expert to choose: zeros (NaN where a logit is)
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = x[v] * f;
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = 0.0f;
  }
  // the chosen ones through LDS, a row of the token's own; its lanes are of one
  // wave, whose LDS instructions stay in order
  __shared__ __attribute__((aligned(16))) float chosen[256 / L][4 * L * Q];
  float* const mine = chosen[threadIdx.x / L];
#pragma unroll
  for (int q = 0; q < Q; ++q) *(f32x4_t*)(mine + (q * L + lane) * 4) = f32x4_t{};
  wave_step();
  // every choice leaves its lane at its expert: one that finds another's there
  // shares the expert with it, and such are added up in order
  const bool some = index >= 0 && index < g.experts;
  if (some) mine[index] = (float)lane;
  wave_step();
  const bool shared = some && mine[index] != (float)lane;
  wave_step();
  if (__ballot(shared)) {
    if (some) mine[index] = 0.0f;
    for (int j = 0; j < g.k; ++j) {
      wave_step();
      if (some && lane == j) mine[index] += d;
    }
  } else if (some) {
    mine[index] = d;
  }
  wave_step();
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const f32x4_t c = *(const f32x4_t*)(mine + (q * L + lane) * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * q + i] += c[i];
  }
  if (!in) return;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int c = (q * L + lane) * 4, left = g.experts - c;
    if (left > 0) st_quad((T*)g.dlogits + t * g.ldd + c, f32x4_t{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]}, left);
  }
}

// ----------------------------------------------------------------------------
// exchange of rows
// ----------------------------------------------------------------------------
// Bound by memory: 32768 rows of 4096 bf16 dispatched in 82 us, combined in 80 (110
// with a residual), the gradient of that in 121, 4.9 to 5.6 TB/s.  A wave moves
// EX_PIECES KiB of one row, so that a row of a place, or of a token, is uniform and
// a call of few rows still spreads over the chip.
struct ExchangeArgs {
  const void* in;       // dispatch: X; combine: Ys; combine_bwd: dY
  const void* other;    // combine: R; combine_bwd: Ys (either may be null)
  void* out;            // combine_bwd: dYs (may be null)
  int64_t ldi, ldt, ldo;
  const int32_t* offsets;   // dispatch: rows behind offsets[experts] are left alone
  const int32_t* order;
  const int32_t* slots;
  const float* weights;     // may be null
  float* dweights;          // combine_bwd, may be null
  uint32_t* flags;
  int64_t tokens, rows;
  int32_t experts, k, width;
  int32_t parts;            // waves of a row
};

constexpr int EX_WAVES = 4, EX_PIECES = 2;
constexpr int64_t EX_BLOCKS = 1 << 20;   // of a launch; more units are taken in turns

// Unit `unit` of `total`: its row, and the part of it.
__device__ __forceinline__ int64_t row_of_unit(int64_t unit, int64_t total, int parts, int& part) {
  const int64_t row = total >> 32 ? unit / parts : (int64_t)((uint32_t)unit / (uint32_t)parts);
  part = (int)(unit - row * parts);
  return row;
}

__device__ __forceinline__ void raise_rows(uint32_t* flags) {
  if (flags && (threadIdx.x & 63) == 0) atomicOr(flags, kBadRows);
}

template <class T>
__global__ __launch_bounds__(EX_WAVES * 64) void k_dispatch(ExchangeArgs g) {
  constexpr int CH = 16 / sizeof(T);
  const int64_t last = g.offsets[g.experts], rows = min(max(last, (int64_t)0), g.rows), total = rows * g.parts;
  if (last != rows && blockIdx.x == 0 && wave_id() == 0) raise_rows(g.flags);
  for (int64_t unit = (int64_t)blockIdx.x * EX_WAVES + wave_id(); unit < total; unit += (int64_t)gridDim.x * EX_WAVES) {
    int part;
    const int64_t s = row_of_unit(unit, total, g.parts, part);
    const int c0 = part * (EX_PIECES * 64 * CH) + (threadIdx.x & 63) * CH;
    const int entry = g.order[s];
    if (entry < 0 || entry >= g.tokens * g.k) {
      raise_rows(g.flags);
      continue;
    }
    const T* const x = (const T*)g.in + (int64_t)(entry / g.k) * g.ldi;
    T* const o = (T*)g.out + s * g.ldo;
    f32x4_t v[EX_PIECES];
#pragma unroll
    for (int p = 0; p < EX_PIECES; ++p) {
      const int c = c0 + p * 64 * CH;
      if (c < g.width) v[p] = ld_piece<T>(x + c, g.width - c);
    }
#pragma unroll
    for (int p = 0; p < EX_PIECES; ++p) {
      const int c = c0 + p * 64 * CH;
      if (c < g.width) st_piece<T>(o + c, v[p], g.width - c);
    }
  }
}

// Y of a token: its experts' rows times their weights, in order, and R.
template <class T>
__device__ __forceinline__ void combine_part(const ExchangeArgs& g, int64_t t, int part) {
  constexpr int CH = 16 / sizeof(T), U = 4;
  const int c0 = part * (EX_PIECES * 64 * CH) + (threadIdx.x & 63) * CH;
  float sum[EX_PIECES][CH] = {};
  f32x4_t r[EX_PIECES] = {};
  if (g.other) {
#pragma unroll
    for (int p = 0; p < EX_PIECES; ++p) {
      const int c = c0 + p * 64 * CH;
      if (c < g.width) r[p] = ld_piece<T>((const T*)g.other + t * g.ldt + c, g.width - c);
    }
  }
  for (int j0 = 0; j0 < g.k; j0 += U) {   // U rows' loads are in flight together
    f32x4_t v[U][EX_PIECES] = {};
    float w[U];
    bool have[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      have[u] = false;
      if (j0 + u >= g.k) continue;
      const int64_t s = g.slots[t * g.k + j0 + u];
      if (s < -1 || s >= g.rows) raise_rows(g.flags);
      if (s < 0 || s >= g.rows) continue;
      have[u] = true;
      w[u] = g.weights ? g.weights[t * g.k + j0 + u] : 1.0f;
#pragma unroll
      for (int p = 0; p < EX_PIECES; ++p) {
        const int c = c0 + p * 64 * CH;
        if (c < g.width) v[u][p] = ld_piece<T>((const T*)g.in + s * g.ldi + c, g.width - c);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!have[u]) continue;
#pragma unroll
      for (int p = 0; p < EX_PIECES; ++p) {
        float e[CH];
        widen<T>(v[u][p], e);
#pragma unroll
        for (int i = 0; i < CH; ++i) sum[p][i] = __builtin_fmaf(w[u], e[i], sum[p][i]);
      }
    }
  }
#pragma unroll
  for (int p = 0; p < EX_PIECES; ++p) {
    const int c = c0 + p * 64 * CH;
    if (c >= g.width) continue;
    if (g.other) {
      float e[CH];
      widen<T>(r[p], e);
#pragma unroll
      for (int i = 0; i < CH; ++i) sum[p][i] += e[i];
    }
    st_piece<T>((T*)g.out + t * g.ldo + c, narrow<T>(sum[p]), g.width - c);
  }
}

template <class T>
__global__ __launch_bounds__(EX_WAVES * 64) void k_combine(ExchangeArgs g) {
  const int64_t total = g.tokens * g.parts;
  for (int64_t unit = (int64_t)blockIdx.x * EX_WAVES + wave_id(); unit < total; unit += (int64_t)gridDim.x * EX_WAVES) {
    int part;
    const int64_t t = row_of_unit(unit, total, g.parts, part);
    combine_part<T>(g, t, part);
  }
}
// A wave takes one entry: dYs of its row and the gradient of its weight.  An
// entry's place has to name the entry, so that no row is written twice.
template <class T>
__device__ __forceinline__ void combine_entry(const ExchangeArgs& g, int64_t entry) {
  constexpr int CH = 16 / sizeof(T), U = 4;
  const int lane = threadIdx.x & 63;
  const int64_t s = g.slots[entry];
  const bool in = s >= 0 && s < g.rows, have = in && g.order[s] == entry;
  if (s < -1 || s >= g.rows || in != have) raise_rows(g.flags);
  if (!have) {
    if (g.dweights && lane == 0) g.dweights[entry] = 0.0f;
    return;
  }
  const T* const dy = (const T*)g.in + entry / g.k * g.ldi;
  const T* const y = (const T*)g.other + s * g.ldt;
  T* const o = (T*)g.out + s * g.ldo;
  const float w = g.weights ? g.weights[entry] : 1.0f;
  float dot = 0.0f;
  for (int c0 = lane * CH; c0 < g.width; c0 += U * 64 * CH) {
    f32x4_t a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 64 * CH;
      if (c >= g.width) continue;
      a[u] = ld_piece<T>(dy + c, g.width - c);
      if (g.dweights) b[u] = ld_piece<T>(y + c, g.width - c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 64 * CH;
      if (c >= g.width) continue;
      float e[CH], f[CH];
      widen<T>(a[u], e);
      if (g.dweights) {
        widen<T>(b[u], f);
#pragma unroll
        for (int i = 0; i < CH; ++i) dot = __builtin_fmaf(e[i], f[i], dot);
      }
      if (g.out) {
#pragma unroll
        for (int i = 0; i < CH; ++i) e[i] *= w;
        st_piece<T>(o + c, narrow<T>(e), g.width - c);
      }
    }
  }
  if (!g.dweights) return;
  dot = wave_sum(dot);
  if (lane == 0) g.dweights[entry] = dot;
}

template <class T>
__global__ __launch_bounds__(EX_WAVES * 64) void k_combine_bwd(ExchangeArgs g) {
  const int64_t total = g.tokens * g.k;
  for (int64_t entry = (int64_t)blockIdx.x * EX_WAVES + wave_id(); entry < total; entry += (int64_t)gridDim.x * EX_WAVES)
    combine_entry<T>(g, entry);
}

}  // namespace occ
