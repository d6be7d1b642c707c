// Matrix products of the linear and gated layers: C (M x N) = A B^T over a
// contraction of K, with bias, activation, gate and residual in the epilogue
// of the forward pass.  One kernel serves the three products of a layer:
//
//   forward        Z  = X W^T      both operands with K contiguous
//   input gradient dX = dZ W       W with K strided (its rows are K)
//   weight gradient dW = dZ^T X    both operands with K strided
//
// Both layouts are brought into LDS as they lie in memory, 16 bytes a lane
// with buffer_load_dwordx4 ... lds; an operand with K strided is turned while
// it is read from LDS (ds_read_b64_tr_b16, or single words for fp32).  Pieces
// of 16 bytes are exchanged within a row (on the global side of the DMA, so
// that LDS is written in order) such that the lanes of a read meet no bank
// twice.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device.hpp"

namespace occ {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4 };

// ----------------------------------------------------------------------------
// activations and their derivatives
// ----------------------------------------------------------------------------
// 1 / (1 + e^-x) with the hardware's exp2 and reciprocal (1 ulp each): 0 where
// e^-x is infinite.
__device__ __forceinline__ float sigmoid_f(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.442695040888963f * x));
}

// The normal distribution function at z and the density's exponential
// e = exp(-z^2/2): erfc(x) = e (a1 t + .. + a5 t^5), t = 1 / (1 + p x) for
// x = |z| / sqrt 2 (Abramowitz and Stegun 7.1.26: error below 1.5e-7).
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float x = fabsf(z) * 0.70710678118654752f;
  e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
  float p = 1.061405429f;
  p = __builtin_fmaf(p, t, -1.453152027f);
  p = __builtin_fmaf(p, t, 1.421413741f);
  p = __builtin_fmaf(p, t, -0.284496736f);
  p = __builtin_fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * p * t * e;   // the distribution at -|z|
  return z < 0.0f ? tail : 1.0f - tail;
}

constexpr float kGeluC = 0.79788456080286536f;   // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

__device__ __forceinline__ f32x4_t act_quad(int act, f32x4_t z) {
  f32x4_t y = z;
  float e;
  switch (act) {   // the same for all lanes
    case ACT_RELU:
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = z[i] > 0.0f || z[i] != z[i] ? z[i] : 0.0f;
      break;
    case ACT_GELU:
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = z[i] * normal_cdf(z[i], e);
      break;
    case ACT_GELU_TANH:   // (1 + tanh q) / 2 = sigmoid(2 q)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        y[i] = z[i] * sigmoid_f(z[i] * __builtin_fmaf(2.0f * kGeluC * kGeluA, z[i] * z[i], 2.0f * kGeluC));
      break;
    case ACT_SILU:
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = z[i] * sigmoid_f(z[i]);
      break;
    default: break;
  }
  return y;
}

// act(z) and act'(z)
__device__ __forceinline__ void act_grad_f(int act, float z, float& a, float& da) {
  float e;
  switch (act) {
    case ACT_RELU:
      a = z > 0.0f || z != z ? z : 0.0f;
      da = z > 0.0f ? 1.0f : 0.0f;
      return;
    case ACT_GELU: {
      const float c = normal_cdf(z, e);
      a = z * c;
      da = __builtin_fmaf(z * 0.3989422804014327f, e, c);
      return;
    }
    case ACT_GELU_TANH: {
      const float zz = fminf(z * z, 1e30f);   // finite: it meets a factor that is 0 there
      const float s = sigmoid_f(2.0f * kGeluC * z * __builtin_fmaf(kGeluA, zz, 1.0f));
      a = z * s;
      // z s (1 - s) 2 q'(z) + s
      da = __builtin_fmaf(a * (1.0f - s), 2.0f * kGeluC * __builtin_fmaf(3.0f * kGeluA, zz, 1.0f), s);
      return;
    }
    case ACT_SILU: {
      const float s = sigmoid_f(z);
      a = z * s;
      da = __builtin_fmaf(a, 1.0f - s, s);
      return;
    }
    default: a = z; da = 1.0f;
  }
}

// ----------------------------------------------------------------------------
// element access at any alignment
// ----------------------------------------------------------------------------
template <class T> __device__ __forceinline__ float ld_elem(const T* p);
template <> __device__ __forceinline__ float ld_elem<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float ld_elem<uint16_t>(const uint16_t* p) {
  return __uint_as_float((uint32_t)*p << 16);
}
__device__ __forceinline__ void st_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_elem(uint16_t* p, float v) { *p = bf16_rne(v); }

// Four consecutive elements, the first `left` of them inside the row.  NT:
// nontemporal, for streams whose rows all start on 64 bytes.
template <class T, bool NT = false>
__device__ __forceinline__ f32x4_t ld_quad(const T* p, int left) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) {
      if constexpr (NT) return __builtin_nontemporal_load((const f32x4_t*)p);
      const f4u_t v = *(const f4u_t*)p;
      return f32x4_t{v[0], v[1], v[2], v[3]};
    } else {
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
      u32x2_t v;
      if constexpr (NT) {
        v = __builtin_nontemporal_load((const u32x2_t*)p);
      } else {
        const u2h_t u = *(const u2h_t*)p;
        v = u32x2_t{u[0], u[1]};
      }
      return f32x4_t{bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1])};
    }
  }
  f32x4_t r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < left) r[i] = ld_elem<T>(p + i);
  return r;
}

template <class T, bool NT = false>
__device__ __forceinline__ void st_quad(T* p, f32x4_t v, int left) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) {
      if constexpr (NT) __builtin_nontemporal_store(v, (f32x4_t*)p);
      else *(f4u_t*)p = f4u_t{v[0], v[1], v[2], v[3]};
    } else {
      typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
      const u32x2_t u = {bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3])};
      if constexpr (NT) __builtin_nontemporal_store(u, (u32x2_t*)p);
      else *(u2h_t*)p = u2h_t{u[0], u[1]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < left) st_elem(p + i, v[i]);
}

// ----------------------------------------------------------------------------
// the epilogue of the forward pass, shared by all forms of the product
// ----------------------------------------------------------------------------
struct FwdEpi {
  void* Y;
  int64_t ldy;
  void* Z;          // may be null
  int64_t ldz;
  const void* R;    // may be null
  int64_t ldr;
  const float* bias;   // may be null
  int32_t act;
  int32_t out;         // columns of Y; gated: W, bias and Z hold the gate's rows, then the others'
};

// bias[n .. n + 3], zeros without one
__device__ __forceinline__ f32x4_t bias_quad(const FwdEpi& e, int n, int left) {
  return e.bias ? ld_quad<float>(e.bias + n, left) : f32x4_t{};
}

// Columns n .. n + 3 of token m: z (and u, the other projection, when gated)
// are sums of products in fp32, the bias added.
template <class T, bool GATED>
__device__ __forceinline__ void fwd_epilogue(const FwdEpi& e, int64_t m, int n, f32x4_t z, f32x4_t u) {
  const int left = e.out - n;
  if (left <= 0) return;
  if (e.Z) {
    st_quad((T*)e.Z + m * e.ldz + n, z, left);
    if constexpr (GATED) st_quad((T*)e.Z + m * e.ldz + e.out + n, u, left);
  }
  f32x4_t y = act_quad(e.act, z);
  if constexpr (GATED) y *= u;
  if (e.R) y += ld_quad<T>((const T*)e.R + m * e.ldr + n, left);
  st_quad((T*)e.Y + m * e.ldy + n, y, left);
}

// ----------------------------------------------------------------------------
// tiled product
// ----------------------------------------------------------------------------
struct GemmArgs {
  const void* A;      // K contiguous: M x K; K strided: K x M
  const void* B;      // K contiguous: N x K; K strided: K x N
  int64_t lda, ldb;   // elements
  int32_t M, N;       // N: columns of the result (gated: of one projection)
  int32_t ka, kb;     // K of each operand; K contiguous: whole 16-byte pieces, zeros behind K's end
  int32_t tiles_m, tiles_n;
  int32_t splits, tiles_k, k_per_split;   // K in tiles of 128 bytes of elements
  float* part;        // splits > 1: partial sums, splits x M x width
  void* C;            // EP_STORE: the result
  int64_t ldc;
  int32_t c_f32, accumulate;
  FwdEpi fwd;
};

enum { EP_STORE = 0, EP_FWD = 1, EP_GATED = 2 };

constexpr int kRowBytes = 128;   // of a row of K in a tile: 64 bf16 or 32 fp32

// Offsets at or above this are out of range of the buffer descriptors below;
// such a lane of a DMA writes zeros.
constexpr uint32_t kOut = 0x80000000u;

__device__ __forceinline__ i32x4_t make_rsrc(uintptr_t p) {
  return i32x4_t{(int32_t)(uint32_t)p, (int32_t)(uint32_t)((uint64_t)p >> 32) & 0xffff,
                 (int32_t)kOut, 0x00020000};
}

// 64 lanes x 16 bytes from memory to LDS at `lds` + 16 * lane.  Written as
// assembly so that the compiler does not wait for it before LDS reads of
// other stages; the kernels below wait themselves.  No register is written.
__device__ __forceinline__ void dma16(i32x4_t rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(voff), "s"(rsrc));
}

// One operand: rows R of the block's tile, in the layout KS (K strided) or
// not, of elements of ES bytes, moved by NW waves.
template <int R, bool KS, int ES, int NW>
struct Operand {
  static constexpr int BK = kRowBytes / ES;          // K of a tile
  static constexpr int CH = 16 / ES;                 // elements of a piece
  static constexpr int BYTES = R * kRowBytes;
  static constexpr int NI = BYTES / 1024 / NW;       // DMA instructions of a wave
  static constexpr int KROW = R * ES;                // bytes of a row, K strided
  uint32_t voff[NI];
  int kk[KS ? NI : 1];   // first K of the lane's piece
  uintptr_t base;
  int64_t step;

  // Exchange of 16-byte pieces within row k of a K-strided tile.  A read
  // takes rows k + {0..3} (bf16: of two groups 8 rows apart; fp32: rows 4
  // apart) and a run of 32 (64) bytes of each.
  static __device__ __forceinline__ int turn(int k) {
    return ES == 2 ? ((k & 3) | ((k >> 1) & 4)) << 1 : ((k >> 2) & 3) << 2;
  }

  // row_of(r): row of the operand held in row r of the tile, inside the array;
  // the 32 rows (K strided: 8 or fewer) that a wave moves are addressed from
  // the first of them, in 31 bits.
  template <class F>
  __device__ __forceinline__ void init(const void* p, int64_t ld, int rows, int row0, int wave, int lane,
                                       int64_t k0, F&& row_of) {
    if constexpr (!KS) {
      const int ch = (lane & 7) ^ (lane >> 3);
      kk[0] = ch * CH;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int r = (wave * NI + j) * 8 + (lane >> 3);
        voff[j] = (uint32_t)(row_of(r) - row_of(wave * NI * 8)) * (uint32_t)(ld * ES) + ch * 16;
      }
      base = (uintptr_t)p + ((uintptr_t)row_of(wave * NI * 8) * ld + k0) * ES;
      step = kRowBytes;
    } else {
      constexpr int PER = 1024 / KROW;       // rows of K an instruction covers
      constexpr int LPR = 64 / PER;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int k = (wave * NI + j) * PER + lane / LPR;
        const int c = ((lane % LPR) ^ turn(k)) * CH;
        kk[j] = k;
        voff[j] = row0 + c < rows ? (uint32_t)(k - wave * NI * PER) * (uint32_t)(ld * ES) + c * ES : kOut;
      }
      base = (uintptr_t)p + ((uintptr_t)(k0 + wave * NI * PER) * ld + row0) * ES;
      step = (int64_t)BK * ld * ES;
    }
  }

  // `left`: K from this tile's start to its end; what lies past it is zero.
  __device__ __forceinline__ void load(uint32_t lds, int wave, int left) {
    const i32x4_t rs = make_rsrc(base);
#pragma unroll
    for (int j = 0; j < NI; ++j)
      dma16(rs, kk[KS ? j : 0] < left ? voff[j] : kOut, lds + (wave * NI + j) * 1024);
    base += step;
  }
};

// One fragment: 16 rows of an operand over a whole K tile, for the lane's row
// lane % 16.  v[0..1] hold K (bf16) 32 s + 8 (lane / 16) + 0..7 of half s, or
// (fp32) 16 s + 4 (lane / 16) + 0..3.
template <int ES> struct Frag { f32x4_t v[2]; };

template <int R, bool KS, int ES>
struct Reader {
  uint32_t at[KS ? R / 16 : 2];

  // first: the wave's first row in the tile (K strided: a multiple of R rows)
  __device__ __forceinline__ void init(int first, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (!KS) {
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = (first + i) * kRowBytes + (((4 * s + g) ^ (i & 7)) << 4);
    } else if constexpr (ES == 2) {
      const int r = i >> 2, f = r | ((g & 1) << 2);
#pragma unroll
      for (int a = 0; a < R / 16; ++a) at[a] = ((((first >> 4) + a) ^ f) << 5) + (i & 3) * 8;
    } else {
#pragma unroll
      for (int a = 0; a < R / 16; ++a) at[a] = ((((first >> 4) + a) ^ g) << 6) + i * 4;
    }
  }

  template <int KROW>
  __device__ __forceinline__ void add_row(int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (KS) {
      const int k = ES == 2 ? 8 * g + (i >> 2) : 4 * g;
#pragma unroll
      for (int a = 0; a < R / 16; ++a) at[a] += k * KROW;
    }
  }

  template <int KROW>
  __device__ __forceinline__ Frag<ES> read(const lds_char* tile, int a) const {
    Frag<ES> f;
    if constexpr (!KS) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
        f.v[s] = *(const __attribute__((address_space(3))) f32x4_t*)(tile + at[s] + a * 16 * kRowBytes);
    } else if constexpr (ES == 2) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        typedef __attribute__((address_space(3))) s16x4_t lds_s4;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + at[a] + 32 * s * KROW));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + at[a] + (32 * s + 4) * KROW));
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        f.v[s] = __builtin_bit_cast(f32x4_t, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          f.v[s][j] = *(const __attribute__((address_space(3))) float*)(tile + at[a] + (16 * s + j) * KROW);
    }
    return f;
  }
};

template <int ES>
__device__ __forceinline__ f32x4_t mfma_tile(const Frag<ES>& b, const Frag<ES>& a, f32x4_t c) {
  if constexpr (ES == 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b.v[s]),
                                                  __builtin_bit_cast(bf16x8_t, a.v[s]), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b.v[s][j], a.v[s][j], c, 0, 0, 0);
  }
  return c;
}

// Tile (tm, tn) of a block.  Workgroups are dealt to the XCDs round-robin;
// xcd_tile() gives each XCD a contiguous run of tiles, and the run walks
// bands of kBand tile rows column by column, so that the tiles of one XCD at
// one time form a near-square and share rows of A and B in its L2.
constexpr int kBand = 8;

__device__ __forceinline__ void band_tile(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int per = kBand * tiles_n;
  const int band = t / per, in = t - band * per;
  const int h = min(kBand, tiles_m - band * kBand);
  tn = in / h;
  tm = band * kBand + in - tn * h;
}

// Passes that the results of a tile take through the LDS of its two stages.
template <int BM, int BN, int STAGE>
constexpr int PR_PASSES = BM * BN * 4 / (2 * STAGE) > 0 ? BM * BN * 4 / (2 * STAGE) : 1;

// Four results of a gradient: stored, or added to what is there.
template <class T>
__device__ __forceinline__ void store_result(const GemmArgs& g, int64_t m, int n, f32x4_t v, int left) {
  if (sizeof(T) == 4 || g.c_f32) {
    float* const p = (float*)g.C + m * g.ldc + n;
    if (g.accumulate) v += ld_quad<float>(p, left);
    st_quad(p, v, left);
  } else {
    uint16_t* const p = (uint16_t*)g.C + m * g.ldc + n;
    if (g.accumulate) v += ld_quad<uint16_t>(p, left);
    st_quad(p, v, left);
  }
}

// WM x WN waves, each 16 FA x 16 FB results.  PP: the waves form two groups
// (one wave of each on every SIMD) that alternate between matrix
// instructions and LDS reads; see the loop.
template <class T, int WM, int WN, int FA, int FB, bool AKS, bool BKS, int EP, bool PP>
__global__ __launch_bounds__(WM * WN * 64, PP ? 2 : 2) void k_gemm(GemmArgs g) {
  constexpr int ES = sizeof(T), NW = WM * WN;
  constexpr int BM = WM * FA * 16, BN = WN * FB * 16;
  using OA = Operand<BM, AKS, ES, NW>;
  using OB = Operand<BN, BKS, ES, NW>;
  constexpr int STAGE = OA::BYTES + OB::BYTES;
  constexpr int BK = OA::BK;
  __shared__ __attribute__((aligned(1024))) char sm[2 * STAGE];
  lds_char* const lds = (lds_char*)sm;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  const int t = xcd_tile();
  const int per_split = g.tiles_m * g.tiles_n;
  const int split = t / per_split;
  band_tile(t - split * per_split, g.tiles_m, g.tiles_n, tm, tn);
  const int kt0 = split * g.k_per_split;
  const int nk = min(g.k_per_split, g.tiles_k - kt0);
  const int m0 = tm * BM;
  constexpr int BNC = EP == EP_GATED ? BN / 2 : BN;   // columns of the result
  const int n0 = tn * BNC;

  OA oa;
  OB ob;
  oa.init(g.A, g.lda, g.M, m0, wave, lane, (int64_t)kt0 * BK, [&](int r) { return min(m0 + r, g.M - 1); });
  ob.init(g.B, g.ldb, g.N, n0, wave, lane, (int64_t)kt0 * BK, [&](int r) {
    if constexpr (EP == EP_GATED) {
      // each wave's columns: half of them the gate's, then the same of the other projection
      constexpr int TN = FB * 16;
      const int c = min(n0 + r / TN * (TN / 2) + r % (TN / 2), g.N - 1);
      return (r % TN) >= TN / 2 ? c + g.N : c;
    } else {
      return min(n0 + r, g.N - 1);
    }
  });
  Reader<FA * 16, AKS, ES> ra;
  Reader<FB * 16, BKS, ES> rb;
  ra.init(wm * FA * 16, lane);
  rb.init(wn * FB * 16, lane);
  ra.template add_row<OA::KROW>(lane);
  rb.template add_row<OB::KROW>(lane);

  f32x4_t acc[FA][FB];
#pragma unroll
  for (int a = 0; a < FA; ++a)
#pragma unroll
    for (int b = 0; b < FB; ++b) acc[a][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

  int left_a = g.ka - kt0 * BK, left_b = g.kb - kt0 * BK;   // of K, at the next tile to load
  auto load_a = [&](int stage) { oa.load(lds0 + stage * STAGE, wave, left_a); left_a -= BK; };
  auto load_b = [&](int stage) { ob.load(lds0 + stage * STAGE + OA::BYTES, wave, left_b); left_b -= BK; };

  constexpr int HA = FA / 2, HB = FB / 2;
  Frag<ES> a0[HA], a1[HA], b0[HB], b1[HB];
  // fragments i0 .. i1 - 1 of a half
  auto read_a = [&](Frag<ES>* f, int stage, int half, int i0, int i1) {
    const lds_char* p = lds + stage * STAGE;
#pragma unroll
    for (int i = 0; i < HA; ++i)
      if (i >= i0 && i < i1) f[i] = ra.template read<OA::KROW>(p, half * HA + i);
  };
  auto read_b = [&](Frag<ES>* f, int stage, int half) {
    const lds_char* p = lds + stage * STAGE + OA::BYTES;
#pragma unroll
    for (int i = 0; i < HB; ++i) f[i] = rb.template read<OB::KROW>(p, half * HB + i);
  };
  auto multiply = [&](const Frag<ES>* a, const Frag<ES>* b, int ha, int hb) {
#pragma unroll
    for (int i = 0; i < HA; ++i)
#pragma unroll
      for (int j = 0; j < HB; ++j)
        acc[ha * HA + i][hb * HB + j] = mfma_tile<ES>(b[j], a[i], acc[ha * HA + i][hb * HB + j]);
  };
  auto before = [&]() {   // of a run of matrix instructions
    if constexpr (PP) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
    }
  };
  auto after = [&]() {
    if constexpr (PP) {
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_barrier" ::: "memory");
    }
  };

  load_a(0);
  load_b(0);
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  if (nk > 1) {
    load_b(1);
    load_a(1);
  }
  read_a(a0, 0, 0, 0, HA);
  if constexpr (PP) {
    if (wave >= NW / 2) asm volatile("s_barrier" ::: "memory");
  }
  // The quarters of the wave's results, in an order that needs one new half
  // operand each; the reads are spread so that each run of matrix
  // instructions covers the same number of them.  Loads of tile t + 1 end
  // before its first read (the wait before the second quarter, and a barrier
  // after it); the stage of tile t is loaded again only after every wave's
  // last read of it: B from the third quarter on, A from the fourth.
  constexpr int Q1 = HA / 4, Q2 = HA / 2;
  for (int kt = 0; kt < nk; ++kt) {
    const int st = kt & 1;
    read_b(b0, st, 0);
    read_a(a1, st, 1, 0, Q1);
    before();
    multiply(a0, b0, 0, 0);
    after();
    read_b(b1, st, 1);
    read_a(a1, st, 1, Q1, Q2);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (!PP) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    before();
    multiply(a0, b1, 0, 1);
    after();
    read_a(a1, st, 1, Q2, HA);
    if (kt + 1 < nk) read_a(a0, st ^ 1, 0, 0, Q1);
    if (kt + 2 < nk) load_b(st);
    if constexpr (!PP) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    before();
    multiply(a1, b1, 1, 1);
    after();
    if (kt + 1 < nk) read_a(a0, st ^ 1, 0, Q1, HA);
    if (kt + 2 < nk) load_a(st);
    before();
    multiply(a1, b0, 1, 0);
    after();
  }
  if constexpr (PP) {
    if (wave < NW / 2) asm volatile("s_barrier" ::: "memory");
  }

  // The results go through LDS, so that the epilogue runs along whole rows of
  // the tile: a wave's stores then cover 512 (256) consecutive bytes instead
  // of 32 in each of 16 rows, which lie in one memory channel when the row
  // length is a power of two (8192 x 16384 results: 229 us at K = 64 that way).
  // Pieces of 16 bytes are exchanged within a row by the row's number: a
  // lane holds 4 columns of row lane % 16 of each 16 x 16 block.
  constexpr int NP = PR_PASSES<BM, BN, STAGE>;
  constexpr int WR = FA / NP * 16, PR = WM * WR;   // rows of a wave and of a pass
  constexpr int QPR = BNC / 4, RPI = 64 / QPR;     // quads of a row; rows at a time
  const int li = lane & 15, lg = lane >> 4;
  const int q = lane % QPR, n = n0 + q * 4, left = g.N - n;
  const bool split_k = g.splits > 1;
  f32x4_t bz = {}, bu = {};
  if (EP != EP_STORE && !split_k && left > 0) {
    bz = bias_quad(g.fwd, n, left);
    if constexpr (EP == EP_GATED) bu = bias_quad(g.fwd, g.N + n, left);
  }
  const int64_t width = EP == EP_GATED ? 2 * (int64_t)g.N : g.N;
  typedef __attribute__((address_space(3))) f32x4_t lds_f4;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    // (the stores of the pass before need not have ended)
    if (p) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int a = 0; a < FA / NP; ++a)
#pragma unroll
      for (int b = 0; b < FB; ++b) {
        const int c = EP == EP_GATED ? (b >= FB / 2 ? QPR : 0) + (wn * (FB / 2) + b % (FB / 2)) * 4 + lg
                                     : (wn * FB + b) * 4 + lg;
        *(lds_f4*)(lds + (wm * WR + a * 16 + li) * BN * 4 + ((c ^ li) << 4)) = acc[p * (FA / NP) + a][b];
      }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll 4
    for (int r = 0; r < PR / NW / RPI; ++r) {
      const int row = wave * (PR / NW) + r * RPI + lane / QPR;
      const int64_t m = m0 + row / WR * (FA * 16) + p * WR + row % WR;
      if (m >= g.M || left <= 0) continue;
      f32x4_t z = *(const lds_f4*)(lds + row * BN * 4 + ((q ^ (row & 15)) << 4)), u = {};
      if constexpr (EP == EP_GATED) u = *(const lds_f4*)(lds + row * BN * 4 + (((QPR + q) ^ (row & 15)) << 4));
      if (split_k) {
        float* const dst = g.part + ((int64_t)split * g.M + m) * width + n;
        st_quad(dst, z, left);
        if constexpr (EP == EP_GATED) st_quad(dst + g.N, u, left);
      } else if constexpr (EP == EP_STORE) {
        store_result<T>(g, m, n, z, left);
      } else {
        fwd_epilogue<T, EP == EP_GATED>(g.fwd, m, n, z + bz, u + bu);
      }
    }
  }
}

// Sum of the partial products of a split K, in split order, and the epilogue.
template <class T, int EP>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs g) {
  const int quads = (g.N + 3) / 4;
  const int width = EP == EP_GATED ? 2 * g.N : g.N;
  const int64_t total = (int64_t)g.M * quads, stride = (int64_t)g.M * width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / quads;
    const int n = (int)(i - m * quads) * 4, left = g.N - n;
    const float* p = g.part + m * width + n;
    f32x4_t z = {}, u = {};
    for (int s = 0; s < g.splits; ++s, p += stride) {
      z += ld_quad<float>(p, left);
      if constexpr (EP == EP_GATED) u += ld_quad<float>(p + g.N, left);
    }
    if constexpr (EP == EP_STORE) {
      store_result<T>(g, m, n, z, left);
    } else {
      z += bias_quad(g.fwd, n, left);
      if constexpr (EP == EP_GATED) u += bias_quad(g.fwd, g.N + n, left);
      fwd_epilogue<T, EP == EP_GATED>(g.fwd, m, n, z, u);
    }
  }
}

}  // namespace occ
