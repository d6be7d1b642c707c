// Layers whose weights belong to experts: the rows of X lie in runs, one run
// for each expert, that `offsets` bounds on the device, and every run has a
// weight matrix of its own.  The products are those of the layers, tile by
// tile (gemm_tile); what is added here is which expert and which of its tiles
// a block has.  The host does not know the runs' lengths: it launches as many
// blocks as any lengths may need, and a block that finds no tile ends.
//
// Bound as the layers' products are: 16384 rows of 8 experts, gated 4096 x 8192 bf16
// 1901 us (1157 TFLOP/s of the rows that there are), backward 4096 x 4096 2101 with dZ;
// 32768 rows of 128 experts, 2048 x 1024, backward 541: dW has four K tiles an
// expert, beside which the first loads and the results take most of a block's time.
//
// A block finds its tile from the offsets themselves: a wave counts the tiles
// of 64 experts at a time and adds them up across its lanes, so that no launch
// and no table stands before the products.
#pragma once

#include "kernels_layer.hpp"

namespace occ {

struct Groups {
  const int32_t* offsets;   // experts + 1
  uint32_t* flags;          // raised where an offset falls or leaves 0 .. rows; may be null
  int32_t experts, rows;
};

constexpr uint32_t kBadRows = 4;   // OCC_F_BAD_ROWS

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // from 1, 2, 4, 8 lanes below in a row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // the last of a row, to the next
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // the last of the lower half, to the upper
  return x;
}

// Rows lo .. hi - 1 of expert e0 + lane (none behind the last expert).  An
// offset out of 0 .. rows is taken as the nearer end, one that falls as the
// largest before it; `reached` is that largest one so far.
__device__ __forceinline__ void expert_rows(const Groups& g, int e0, int& reached, int& lo, int& hi) {
  const int lane = threadIdx.x & 63;
  auto at = [&](int e) { return min(max(g.offsets[min(e, g.experts)], 0), g.rows); };
  lo = at(e0 + lane);
  hi = at(e0 + lane + 1);
  if (__ballot(lo > hi || lo < reached)) {
    int top = max(lo, reached);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int other = __shfl_up(top, s);
      if (lane >= s) top = max(top, other);
    }
    lo = top;
    hi = max(top, hi);
  }
  reached = __builtin_amdgcn_readlane(hi, 63);
}

// An expert's run of rows, and which unit of it a block has: units are tiles,
// strips or runs of rows, counted through the experts in order.
struct Expert {
  int e, start, count;
  int in, before;   // the unit in this expert; units of the experts before it
};

// The expert that unit order(total) belongs to; false: there is no such unit.
template <class U, class O>
__device__ __forceinline__ bool find_unit(const Groups& g, U&& units, O&& order, Expert& x) {
  int reached = 0, lo, hi;
  expert_rows(g, 0, reached, lo, hi);
  int sum = wave_scan(units(hi - lo));
  int total = __builtin_amdgcn_readlane(sum, 63);
  int r = reached;
  for (int e0 = 64; e0 < g.experts; e0 += 64) {
    int l, h;
    expert_rows(g, e0, r, l, h);
    total += __builtin_amdgcn_readlane(wave_scan(units(h - l)), 63);
  }
  const int t = order(total);
  if (t < 0 || t >= total) return false;
  int e0 = 0, before = 0;
  uint64_t past;
  while (!(past = __ballot(before + sum > t))) {
    before += __builtin_amdgcn_readlane(sum, 63);
    e0 += 64;
    if (e0 >= g.experts) return false;   // only if the offsets have changed since they were counted
    expert_rows(g, e0, reached, lo, hi);
    sum = wave_scan(units(hi - lo));
  }
  const int l = __builtin_ctzll(past);
  x.e = e0 + l;
  x.start = __builtin_amdgcn_readlane(lo, l);
  x.count = __builtin_amdgcn_readlane(hi, l) - x.start;
  x.before = before + __builtin_amdgcn_readlane(sum, l) - units(x.count);
  x.in = t - x.before;
  return true;
}

// The run of expert e, and the units before it.
template <class U>
__device__ __forceinline__ Expert expert_at(const Groups& g, int e, U&& units) {
  int reached = 0, lo, hi, before = 0, e0 = 0;
  expert_rows(g, 0, reached, lo, hi);
  int sum = wave_scan(units(hi - lo));
  for (; e0 + 64 <= e; sum = wave_scan(units(hi - lo))) {
    before += __builtin_amdgcn_readlane(sum, 63);
    e0 += 64;
    expert_rows(g, e0, reached, lo, hi);
  }
  const int l = e - e0;
  Expert x;
  x.e = e;
  x.start = __builtin_amdgcn_readlane(lo, l);
  x.count = __builtin_amdgcn_readlane(hi, l) - x.start;
  x.before = before + __builtin_amdgcn_readlane(sum, l) - units(x.count);
  x.in = 0;
  return x;
}

// Raises the flag for offsets that are not in order; one wave of a launch.
__device__ __forceinline__ void check_offsets(const Groups& g) {
  if (!g.flags || threadIdx.x >= 64) return;
  bool bad = false;
  for (int e = threadIdx.x; e <= g.experts; e += 64) {
    const int o = g.offsets[e];
    bad |= o < 0 || o > g.rows || (e && g.offsets[e - 1] > o);
  }
  if (__ballot(bad) && threadIdx.x == 0) atomicOr(g.flags, kBadRows);
}

// ----------------------------------------------------------------------------
// forward
// ----------------------------------------------------------------------------
template <class T>
__device__ __forceinline__ void* at_row(const void* p, int64_t row, int64_t ld) {
  return p ? (char*)p + row * ld * (int64_t)sizeof(T) : nullptr;
}

// The epilogue's matrices from row `row` on, and the expert's bias.
template <class T>
__device__ __forceinline__ void shift_epilogue(FwdEpi& f, int64_t row, int64_t bias) {
  f.Y = at_row<T>(f.Y, row, f.ldy);
  f.Z = at_row<T>(f.Z, row, f.ldz);
  f.R = at_row<T>(f.R, row, f.ldr);
  if (f.bias) f.bias += bias;
}

struct ExpertsArgs {
  GemmArgs g;       // of the first expert, from row 0 on
  Groups of;
  int64_t w_step;   // bytes from one expert's weights to the next
  int32_t wide;     // values of an expert's bias
};

// The last tile along the rows: where 128 of its 256 rows have nothing it is
// made by the form with half of them, which half of all experts' last tiles
// can be (32768 rows of 128 experts, 2048 x 1024, both gradients: 555 -> 541 us).
template <class T, class TE, class F, bool AKS, bool BKS, int EP>
__device__ __forceinline__ void ragged_tile(const GemmArgs& g, int tm, int tn, lds_char* lds) {
  if constexpr (F::BM == 256) {
    if (g.M - tm * F::BM <= F::BM / 2)
      return gemm_tile<T, TE, Form128x256, AKS, BKS, EP>(g, 2 * tm, tn, 0, lds);
  }
  gemm_tile<T, TE, F, AKS, BKS, EP>(g, tm, tn, 0, lds);
}

// Tiles are counted expert by expert, and each XCD takes a contiguous run of
// them, so that the tiles of an expert share its weights in one or two L2s.
template <class T, class TE, class F, int EP>
__device__ __forceinline__ void experts_forward(const ExpertsArgs& a, lds_char* lds) {
  const int b = blockIdx.x;
  if (b == 0) check_offsets(a.of);
  Expert x;
  if (!find_unit(
          a.of, [&](int rows) { return (rows + F::BM - 1) / F::BM * a.g.tiles_n; },
          [&](int total) { return b < total ? xcd_order(b, total) : -1; }, x))
    return;
  GemmArgs g = a.g;
  g.A = at_row<T>(g.A, x.start, g.lda);
  g.B = (const char*)g.B + x.e * a.w_step;
  g.M = x.count;
  shift_epilogue<TE>(g.fwd, x.start, (int64_t)x.e * a.wide);
  int tm, tn;
  band_tile(x.in, (x.count + F::BM - 1) / F::BM, g.tiles_n, tm, tn);
  ragged_tile<T, TE, F, false, false, EP>(g, tm, tn, lds);
}

template <class T, class TE, class F, int EP>
__global__ __launch_bounds__(F::NW * 64, 2) void k_experts_fwd(ExpertsArgs a) {
  __shared__ __attribute__((aligned(1024))) char sm[F::LDS];
  experts_forward<T, TE, F, EP>(a, (lds_char*)sm);
}

template <class T, int EP>
__global__ __launch_bounds__(512, 4) void k_experts_direct(ExpertsArgs a) {
  __shared__ __attribute__((aligned(1024))) char sm[FormDirect::LDS];
  experts_forward<T, T, FormDirect, EP>(a, (lds_char*)sm);
}

// Few rows an expert: its weights are streamed, once for every 4 rows (along
// K) or every 16 NT (through the matrix instructions).  16 gated rows over 64
// experts, 2048 x 1024 bf16: 17 us, 5.4 TB/s of weights.
struct ExpertsFewArgs {
  SkinnyArgs g;
  Groups of;
  int64_t w_step;
  int32_t wide, across;   // across: blocks along the columns
};

// Rows `in` of ROWS each of an expert, for a block of columns; runs of rows of
// the same columns follow each other, so that they find the weights in a cache.
template <class T, int ROWS>
__device__ __forceinline__ bool few_rows(const ExpertsFewArgs& a, SkinnyArgs& g, int& block) {
  if (blockIdx.x == 0) check_offsets(a.of);
  auto runs = [](int rows) { return (rows + ROWS - 1) / ROWS; };
  Expert x;
  if (!find_unit(
          a.of, [&](int rows) { return runs(rows) * a.across; }, [&](int) { return (int)blockIdx.x; }, x))
    return false;
  const int n = runs(x.count);
  block = x.in / n;
  const int first = (x.in - block * n) * ROWS;
  g = a.g;
  g.tokens = min(ROWS, x.count - first);
  g.X = at_row<T>(g.X, x.start + first, g.ldx);
  g.W = (const char*)g.W + x.e * a.w_step;
  shift_epilogue<T>(g.fwd, x.start + first, (int64_t)x.e * a.wide);
  return true;
}

template <class T, bool GATED>
__global__ __launch_bounds__(DOT_WAVES * 64) void k_experts_dot(ExpertsFewArgs a) {
  SkinnyArgs g;
  int block;
  if (!few_rows<T, 4>(a, g, block)) return;
  if (g.tokens == 1) dot_block<T, 1, GATED>(g, block);
  else if (g.tokens == 2) dot_block<T, 2, GATED>(g, block);
  else dot_block<T, 4, GATED>(g, block);
}

template <class T, int NT, bool GATED>
__global__ __launch_bounds__(SK_WAVES * 64) void k_experts_skinny(ExpertsFewArgs a) {
  SkinnyArgs g;
  int block;
  if (few_rows<T, 16 * NT>(a, g, block)) skinny_block<T, NT, GATED>(g, block);
}

// ----------------------------------------------------------------------------
// before the products of the backward pass, and aligned operands
// ----------------------------------------------------------------------------
// dZ and strips of the bias gradient as in a layer; a strip ends where its
// expert's rows do, so that bias_block can add an expert's strips.  As there, dZ
// is rounded to the layer's type, which the matrix instructions take: bf16
// gradients are off by 0.0024 of their norm (0.0017 with dZ in fp32, their own
// rounding alone), and the two differ by 0.0026.  dZ in two bf16 planes would
// take that away for twice the matrix instructions, the bound of the products.
struct ExpertsCopyArgs {
  CopyArgs c;
  int64_t step;   // elements from one expert's matrix to the next
  int32_t per;    // rows of an expert's matrix; 0: one matrix
};

struct ExpertsPrepArgs {
  DzArgs dz;
  Groups of;
  ExpertsCopyArgs copy[3];
  int32_t dz_blocks;
};

template <class T>
__device__ __forceinline__ void copy_experts(const ExpertsCopyArgs& a, int block) {
  if (!a.per) return copy_block<T>(a.c, block);
  constexpr int CH = 16 / sizeof(T);
  const CopyArgs& g = a.c;
  const int64_t total = g.rows * g.pieces;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < total; i += (int64_t)g.blocks * 256) {
    const int64_t r = i / g.pieces, e = r / a.per;
    const T* const row = (const T*)g.src + e * a.step + (r - e * a.per) * g.ld;
    if (sizeof(T) == 4 && g.plane) {
      const int c = (int)(i - r * g.pieces) * 8;
      uint16_t* const q = (uint16_t*)g.dst + i * 8;
      st_planes(q, g.plane, ld_quad<float>((const float*)row + c, g.cols - c), 4);
      st_planes(q + 4, g.plane, ld_quad<float>((const float*)row + c + 4, g.cols - c - 4), 4);
      continue;
    }
    const int c = (int)(i - r * g.pieces) * CH;
    *(f32x4_t*)((T*)g.dst + i * CH) = ld_piece<T>(row + c, g.cols - c);
  }
}

template <class T, bool GATED>
__global__ __launch_bounds__(256) void k_experts_prep(ExpertsPrepArgs g) {
  int b = blockIdx.x;
  if (b < g.dz_blocks) {
    const int t = b / g.dz.across, strip = g.dz.strip;
    Expert x;
    if (!find_unit(
            g.of, [&](int rows) { return (rows + strip - 1) / strip; }, [&](int) { return t; }, x))
      return;
    const int64_t r0 = x.start + (int64_t)x.in * strip;
    return dz_rows<T, GATED>(g.dz, b - t * g.dz.across, t, r0, min(r0 + strip, (int64_t)x.start + x.count));
  }
  b -= g.dz_blocks;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (b < g.copy[i].c.blocks) return copy_experts<T>(g.copy[i], b);
    b -= g.copy[i].c.blocks;
  }
}

// ----------------------------------------------------------------------------
// the products of the backward pass
// ----------------------------------------------------------------------------
struct ExpertsBackwardArgs {
  GemmArgs dx, dw;
  BiasArgs bias;
  Groups of;
  int64_t w_step, dw_step;    // bytes from one expert's W (dW) to the next
  int32_t dx_blocks, dw_blocks;   // dx_blocks: whole eights, so that dW's blocks keep their XCDs
  int32_t strip;              // rows of a strip of the bias gradient
};

__device__ __forceinline__ void shift_dz(DzSource& d, int64_t row, int es) {
  d.dY = (const char*)d.dY + row * d.ldy * es;
  if (d.Z) d.Z = (const char*)d.Z + row * d.ldz * es;
}

// A tile of zeros, for an expert without rows.
template <class TE, class F>
__device__ __forceinline__ void zero_tile(const GemmArgs& g, int tm, int tn) {
  constexpr int QPR = F::BN / 4;
  for (int i = threadIdx.x; i < F::BM * QPR; i += F::NW * 64) {
    const int m = tm * F::BM + i / QPR, n = tn * F::BN + i % QPR * 4, left = g.N - n;
    if (m >= g.M || left <= 0) continue;
    const int64_t at = (int64_t)m * g.ldc + n;
    if (sizeof(TE) == 4 || g.c_f32) st_quad((float*)g.C + at, f32x4_t{}, left);
    else st_quad((uint16_t*)g.C + at, f32x4_t{}, left);
  }
}

// dW of an expert is a product over its rows.  Experts' lengths differ, so the
// tiles of every expert are dealt to all XCDs, a contiguous run to each.  A tile
// is one block's, whatever the rows: few tiles over many rows leave CUs idle
// (16384 rows of one expert, 64 x 64 bf16: 75 us, the plain layer, whose rows are
// split, 13; 32768 x 2048 x 1024, half of the rows with one of 128 experts: 730
// us, 483 with all alike).
template <class T, class TE, class F>
__device__ __forceinline__ void experts_dw(const ExpertsBackwardArgs& a, int b, lds_char* lds) {
  const int tiles = a.dw.tiles_m * a.dw.tiles_n;
  int e, in;
  if (tiles >= 8) {
    const int per = (tiles + 7) >> 3, i = b >> 3;
    e = i / per;
    in = (b & 7) * per + i - e * per;
    if (in >= tiles) return;
  } else {
    e = b / tiles;
    in = b - e * tiles;
  }
  if (e >= a.of.experts) return;
  const Expert x = expert_at(a.of, e, [](int) { return 0; });
  if (!x.count && a.dw.accumulate) return;
  GemmArgs g = a.dw;
  g.A = at_row<T>(g.A, x.start, g.lda);
  g.B = at_row<T>(g.B, x.start, g.ldb);
  shift_dz(g.dz, x.start, sizeof(TE));
  g.C = (char*)g.C + e * a.dw_step;
  g.ka = g.kb = x.count;
  constexpr int BK = kRowBytes / sizeof(T);
  g.tiles_k = (x.count + BK - 1) / BK;
  if constexpr (sizeof(T) != sizeof(TE)) {
    g.seg_tiles = max(g.tiles_k, 1);
    g.tiles_k *= kPairs;
  }
  g.k_per_split = g.tiles_k;
  int tm, tn;
  band_tile(in, g.tiles_m, g.tiles_n, tm, tn);
  if (!x.count) return zero_tile<TE, F>(g, tm, tn);
  ragged_tile<T, TE, F, true, true, EP_STORE>(g, tm, tn, lds);
}

template <class T, class TE, class F>
__device__ __forceinline__ void experts_dx(const ExpertsBackwardArgs& a, int b, lds_char* lds) {
  Expert x;
  if (!find_unit(
          a.of, [&](int rows) { return (rows + F::BM - 1) / F::BM * a.dx.tiles_n; },
          [&](int total) { return b < total ? xcd_order(b, total) : -1; }, x))
    return;
  GemmArgs g = a.dx;
  g.A = at_row<T>(g.A, x.start, g.lda);
  g.B = (const char*)g.B + x.e * a.w_step;
  shift_dz(g.dz, x.start, sizeof(TE));
  g.C = at_row<TE>(g.C, x.start, g.ldc);
  g.M = x.count;
  int tm, tn;
  band_tile(x.in, (x.count + F::BM - 1) / F::BM, g.tiles_n, tm, tn);
  ragged_tile<T, TE, F, false, true, EP_STORE>(g, tm, tn, lds);
}

// 64 columns of an expert's bias gradient: the sum of its strips.
__device__ __forceinline__ void experts_bias(const ExpertsBackwardArgs& a, int b, float* lds) {
  const int across = (int)((a.bias.width + 63) / 64), e = b / across;
  if (e >= a.of.experts) return;
  const int strip = a.strip;
  auto strips = [&](int rows) { return (rows + strip - 1) / strip; };
  const Expert x = expert_at(a.of, e, strips);
  BiasArgs g = a.bias;
  g.part += x.before * g.width;
  g.dbias += e * g.width;
  g.strips = strips(x.count);
  bias_block(g, b - e * across, lds);
}

template <class T, class TE, class F>
__device__ __forceinline__ void experts_backward(const ExpertsBackwardArgs& a, char* sm) {
  lds_char* const lds = (lds_char*)sm;
  static_assert(F::NW == 8, "the bias blocks run on eight waves");
  int b = blockIdx.x;
  if (b == 0) check_offsets(a.of);
  if (b < a.dx_blocks) return experts_dx<T, TE, F>(a, b, lds);
  b -= a.dx_blocks;
  if (b < a.dw_blocks) return experts_dw<T, TE, F>(a, b, lds);
  experts_bias(a, b - a.dw_blocks, (float*)sm);
}

template <class T, class TE, class F>
__global__ __launch_bounds__(F::NW * 64, 2) void k_experts_bwd(ExpertsBackwardArgs a) {
  __shared__ __attribute__((aligned(1024))) char sm[F::LDS];
  experts_backward<T, TE, F>(a, sm);
}

template <class T>
__global__ __launch_bounds__(512, 4) void k_experts_bwd_direct(ExpertsBackwardArgs a) {
  __shared__ __attribute__((aligned(1024))) char sm[FormDirect::LDS];
  experts_backward<T, T, FormDirect>(a, sm);
}

// dbias alone
__global__ __launch_bounds__(512) void k_experts_bias(ExpertsBackwardArgs a) {
  __shared__ __attribute__((aligned(16))) float sm[512];
  if (blockIdx.x == 0) check_offsets(a.of);
  experts_bias(a, blockIdx.x, sm);
}

}  // namespace occ
