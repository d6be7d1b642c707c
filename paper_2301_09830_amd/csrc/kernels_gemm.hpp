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
// twice (no conflict cycles counted in the products).
//
// Bound by the matrix units and what keeps them fed: bf16 8192^3 runs forward
// at 1510 TFLOP/s, both gradients at 1330 (K strided takes twice the LDS reads
// for the same instructions), with the units busy 60 to 67 % of the time; 8192 x
// 4096 x 16384 with GELU and Z stored 806 to 949 us on different boards, 1160 to
// 1360 TFLOP/s; fp32 4096^3, on bf16 planes, 215.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device.hpp"
#include "layer_tiles.hpp"

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
// e = exp(-z^2/2): at -|z| it is e (a1 t + .. + a8 t^8), t = 1 / (1 + p |z|).
// The polynomial is the least largest relative error's (8.4e-8, 1.1e-7 with the
// coefficients in fp32) against e^(x^2) erfc(x) / 2, x = |z| / sqrt 2 up to 9.5,
// fitted by reweighted least squares.  So the relative error stays that of a few
// roundings over the whole range, z^2 2^-24 where the exponential's argument is
// large (z in [-5, -4] 3e-7 in norm; a polynomial of 5 terms good to 1.5e-7 of 1
// has 6e-4 there).
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.30405593f, fabsf(z), 1.0f));
  float p = 0.036853954f;
  p = __builtin_fmaf(p, t, -0.15518664f);
  p = __builtin_fmaf(p, t, 0.19185275f);
  p = __builtin_fmaf(p, t, -0.042862806f);
  p = __builtin_fmaf(p, t, 0.12342219f);
  p = __builtin_fmaf(p, t, 0.10247556f);
  p = __builtin_fmaf(p, t, 0.122187726f);
  p = __builtin_fmaf(p, t, 0.12125731f);
  const float tail = p * t * e;   // the distribution at -|z|
  return z < 0.0f ? tail : 1.0f - tail;
}

constexpr float kGeluC = 0.79788456080286536f;   // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

// y = act(z) of N quads: one branch for all of them
template <int N>
__device__ __forceinline__ void act_quads(int act, const f32x4_t* z, f32x4_t* y) {
  auto each = [&](auto&& f) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[k][i] = f(z[k][i]);
  };
  switch (act) {   // the same for all lanes
    case ACT_RELU: each([](float v) { return v > 0.0f || v != v ? v : 0.0f; }); break;
    case ACT_GELU:
      each([](float v) {
        float e;
        return v * normal_cdf(v, e);
      });
      break;
    case ACT_GELU_TANH:   // (1 + tanh q) / 2 = sigmoid(2 q)
      each([](float v) {
        return v * sigmoid_f(v * __builtin_fmaf(2.0f * kGeluC * kGeluA, v * v, 2.0f * kGeluC));
      });
      break;
    case ACT_SILU: each([](float v) { return v * sigmoid_f(v); }); break;
    default: each([](float v) { return v; });
  }
}

__device__ __forceinline__ f32x4_t act_quad(int act, f32x4_t z) {
  f32x4_t y;
  act_quads<1>(act, &z, &y);
  return y;
}

// act(z) and act'(z)
__device__ __forceinline__ void act_grad_quad(int act, f32x4_t z, f32x4_t& a, f32x4_t& da) {
  float e;
  switch (act) {
    case ACT_RELU:
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = z[i] > 0.0f || z[i] != z[i] ? z[i] : 0.0f;
        da[i] = z[i] > 0.0f ? 1.0f : z[i] != z[i] ? z[i] : 0.0f;
      }
      break;
    case ACT_GELU:
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float c = normal_cdf(z[i], e);
        a[i] = z[i] * c;
        da[i] = __builtin_fmaf(z[i] * 0.3989422804014327f, e, c);
      }
      break;
    case ACT_GELU_TANH:
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float zz = fminf(z[i] * z[i], 1e30f);   // finite: it meets a factor that is 0 there
        const float s = sigmoid_f(z[i] * __builtin_fmaf(2.0f * kGeluC * kGeluA, zz, 2.0f * kGeluC));
        a[i] = z[i] * s;
        // z s (1 - s) 2 q'(z) + s
        da[i] = __builtin_fmaf(a[i] * (1.0f - s), __builtin_fmaf(6.0f * kGeluC * kGeluA, zz, 2.0f * kGeluC), s);
      }
      break;
    case ACT_SILU:
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float s = sigmoid_f(z[i]);
        a[i] = z[i] * s;
        da[i] = __builtin_fmaf(a[i], 1.0f - s, s);
      }
      break;
    default:
      a = z;
      da = f32x4_t{1.0f, 1.0f, 1.0f, 1.0f};
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

// 16 bytes of a row, at any alignment; `left` elements of it are inside.
template <class T>
__device__ __forceinline__ f32x4_t ld_piece(const T* p, int left) {
  constexpr int CH = 16 / sizeof(T);
  if (left >= CH) {
    if constexpr (sizeof(T) == 4) {
      const f4u_t v = *(const f4u_t*)p;
      return f32x4_t{v[0], v[1], v[2], v[3]};
    } else {
      const u4h_t v = *(const u4h_t*)p;
      return f32x4_t{__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3])};
    }
  }
  T e[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) e[i] = i < left ? p[i] : (T)0;
  f32x4_t r;
  __builtin_memcpy(&r, e, 16);
  return r;
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
  int32_t stream;      // Y and Z bypass the caches (rows on 64 bytes)
  int32_t out;         // columns of Y; gated: W, bias and Z hold the gate's rows, then the others'
};

// bias[n .. n + 3], zeros without one
__device__ __forceinline__ f32x4_t bias_quad(const FwdEpi& e, int n, int left) {
  return e.bias ? ld_quad<float>(e.bias + n, left) : f32x4_t{};
}

// R[m][n .. n + 3], zeros without one
template <class T>
__device__ __forceinline__ f32x4_t residual_quad(const FwdEpi& e, int64_t m, int n, int left) {
  return e.R ? ld_quad<T>((const T*)e.R + m * e.ldr + n, left) : f32x4_t{};
}

// Columns n .. n + 3 of token m: z (and u, the other projection, when gated)
// are sums of products in fp32, the bias added; r is the residual.
template <class T, bool GATED>
__device__ __forceinline__ void fwd_epilogue(const FwdEpi& e, int64_t m, int n, f32x4_t z, f32x4_t u, f32x4_t r) {
  const int left = e.out - n;
  if (left <= 0) return;
  T* const zp = (T*)e.Z + m * e.ldz + n;
  T* const yp = (T*)e.Y + m * e.ldy + n;
  f32x4_t y = act_quad(e.act, z);
  if constexpr (GATED) y *= u;
  y += r;
  if (e.stream) {
    if (e.Z) {
      st_quad<T, true>(zp, z, left);
      if constexpr (GATED) st_quad<T, true>(zp + e.out, u, left);
    }
    st_quad<T, true>(yp, y, left);
  } else {
    if (e.Z) {
      st_quad(zp, z, left);
      if constexpr (GATED) st_quad(zp + e.out, u, left);
    }
    st_quad(yp, y, left);
  }
}

// ----------------------------------------------------------------------------
// tiled product
// ----------------------------------------------------------------------------
// dZ of a layer, made from dY and Z where it is loaded.  Z null: dZ = dY.
struct DzSource {
  const void* dY;
  const void* Z;
  int64_t ldy, ldz;
  int32_t out, act, gated;
};

struct GemmArgs {
  const void* A;      // K contiguous: M x K; K strided: K x M
  const void* B;      // K contiguous: N x K; K strided: K x N
  int64_t lda, ldb;   // elements
  int32_t M, N;       // N: columns of the result (gated: of one projection)
  int32_t ka, kb;     // K of each operand; K contiguous: whole 16-byte pieces, zeros behind K's end
  int32_t tiles_m, tiles_n;
  int32_t splits, tiles_k, k_per_split;   // K in tiles of 128 bytes of elements
  float* part;        // splits > 1: partial sums, splits x M x part_width(N)
  void* C;            // EP_STORE: the result
  int64_t ldc;
  int32_t c_f32, accumulate, stream;
  int64_t plane_a, plane_b;   // fp32 as three bf16 planes: bytes from one to the next
  int32_t seg_tiles;          // K tiles of one pair of planes
  FwdEpi fwd;
  DzSource dz;                // direct form: dz.Z, if given, in place of A
};

// fp32 operands on the bf16 matrix units: x = h + m + l, each the bf16 nearest
// to what the ones before leave, holds x to 2^-27 of itself, and six of the
// nine products of two such sums hold the product to 2^-25 (those left out are
// m l, l m and l l), less than its rounding to fp32.  The product runs over K
// once for each pair, the small ones first.

// plane of pair p: A takes l h m m h h, B takes h l m h m h
__device__ __forceinline__ int plane_of_a(int p) { return (0x052 >> (2 * p)) & 3; }
__device__ __forceinline__ int plane_of_b(int p) { return (0x118 >> (2 * p)) & 3; }

// An infinity ends as NaN; a finite value that bf16 would round to infinity
// keeps the largest bf16 as its first part.
__device__ __forceinline__ void split3(float x, uint16_t* p) {
  p[0] = bf16_rne(x);
  if ((p[0] & 0x7fff) == 0x7f80) p[0] -= 1;
  const float r = x - __uint_as_float((uint32_t)p[0] << 16);
  p[1] = bf16_rne(r);
  p[2] = bf16_rne(r - __uint_as_float((uint32_t)p[1] << 16));
}

enum { EP_STORE = 0, EP_FWD = 1, EP_GATED = 2 };

// Columns of a partial sum's row: whole quads, the gate's and then the others'.
template <int EP>
__device__ __forceinline__ int64_t part_width(const GemmArgs& g) {
  return (int64_t)((g.N + 3) & ~3) * (EP == EP_GATED ? 2 : 1);
}

// Offsets at or above this are out of range of the buffer descriptors below;
// such a lane of a DMA writes zeros.
constexpr uint32_t kOut = 0x80000000u;

__device__ __forceinline__ i32x4_t make_rsrc(uintptr_t p) {
  return i32x4_t{(int32_t)(uint32_t)p, (int32_t)(uint32_t)((uint64_t)p >> 32) & 0xffff,
                 (int32_t)kOut, 0x00020000};
}

// 64 lanes x 16 bytes from memory to LDS at `lds` + 16 * lane.  Written as
// assembly so that the compiler does not wait for it before LDS reads of
// other stages; the kernels below wait themselves.  No register is written but
// m0, which is reserved: it cannot be named as clobbered, and the compiler sets
// it before each use of its own (these kernels have none).
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
  uintptr_t base, start;   // of the present tile, and of K = 0
  int64_t step;

  // Exchange of 16-byte pieces within row k of a K-strided tile.  A read
  // takes rows k + {0..3} (bf16: of two groups 8 rows apart; fp32: rows 4
  // apart) and a run of 32 (64) bytes of each.
  static __device__ __forceinline__ int turn(int k) {
    if (ES == 4) return ((k >> 2) & 3) << 2;
    // rows of 128 bytes: odd and even rows lie in different halves of the banks
    return (KROW == 128 ? (k & 3) ^ ((k >> 3) & 1) : (k & 3) | ((k >> 1) & 4)) << 1;
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
      start = (uintptr_t)p + (uintptr_t)row_of(wave * NI * 8) * ld * ES;
      base = start + k0 * ES;
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
      start = (uintptr_t)p + ((uintptr_t)(wave * NI * PER) * ld + row0) * ES;
      base = start + (uintptr_t)k0 * ld * ES;
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

  // first: the wave's first row in the tile (K strided: a multiple of R rows);
  // KROW: bytes of a row of the tile, K strided
  template <int KROW>
  __device__ __forceinline__ void init(int first, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (!KS) {
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = (first + i) * kRowBytes + (((4 * s + g) ^ (i & 7)) << 4);
    } else if constexpr (ES == 2) {
      const int k = 8 * g + (i >> 2), f = Operand<KROW / ES, true, ES, 1>::turn(k) >> 1;
#pragma unroll
      for (int a = 0; a < R / 16; ++a) at[a] = k * KROW + ((((first >> 4) + a) ^ f) << 5) + (i & 3) * 8;
    } else {
#pragma unroll
      for (int a = 0; a < R / 16; ++a) at[a] = 4 * g * KROW + ((((first >> 4) + a) ^ g) << 6) + i * 4;
    }
  }

  // half s of K, of rows 16 a .. 16 a + 15
  template <int KROW>
  __device__ __forceinline__ f32x4_t read_half(const lds_char* tile, int a, int s) const {
    if constexpr (!KS) {
      return *(const __attribute__((address_space(3))) f32x4_t*)(tile + at[s] + a * 16 * kRowBytes);
    } else if constexpr (ES == 2) {
      typedef __attribute__((address_space(3))) s16x4_t lds_s4;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + at[a] + 32 * s * KROW));
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + at[a] + (32 * s + 4) * KROW));
      typedef short s16x8_t __attribute__((ext_vector_type(8)));
      return __builtin_bit_cast(f32x4_t, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f32x4_t v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *(const __attribute__((address_space(3))) float*)(tile + at[a] + (16 * s + j) * KROW);
      return v;
    }
  }

  template <int KROW>
  __device__ __forceinline__ Frag<ES> read(const lds_char* tile, int a) const {
    Frag<ES> f;
#pragma unroll
    for (int s = 0; s < 2; ++s) f.v[s] = read_half<KROW>(tile, a, s);
    return f;
  }
};

template <int ES>
__device__ __forceinline__ f32x4_t mfma_half(f32x4_t b, f32x4_t a, f32x4_t c) {
  if constexpr (ES == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b), __builtin_bit_cast(bf16x8_t, a), c,
                                                   0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j], a[j], c, 0, 0, 0);
    return c;
  }
}

template <int ES>
__device__ __forceinline__ f32x4_t mfma_tile(const Frag<ES>& b, const Frag<ES>& a, f32x4_t c) {
#pragma unroll
  for (int s = 0; s < 2; ++s) c = mfma_half<ES>(b.v[s], a.v[s], c);
  return c;
}

// Tile (tm, tn) of a block.  Workgroups are dealt to the XCDs round-robin;
// xcd_order gives each XCD a contiguous run of the n tiles, and the run walks
// bands of kBand tile rows column by column, so that the tiles of one XCD at
// one time form a near-square and share rows of A and B in its L2.
constexpr int kBand = 8;

__device__ __forceinline__ int xcd_order(int b, int n) {
  const int n8 = n & ~7;
  return b < n8 ? (b & 7) * (n8 >> 3) + (b >> 3) : b;
}

__device__ __forceinline__ void band_tile(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int per = kBand * tiles_n;
  const int band = t / per, in = t - band * per;
  const int h = min(kBand, tiles_m - band * kBand);
  tn = in / h;
  tm = band * kBand + in - tn * h;
}

// Passes that the results of a tile take through the LDS of its stages.
template <int BM, int BN, int BYTES>
constexpr int PR_PASSES = (BM * BN * 4 + BYTES - 1) / BYTES;

// Four results of a gradient: stored, or added to what is there.
template <class TC>
__device__ __forceinline__ void store_as(const GemmArgs& g, int64_t m, int n, f32x4_t v, int left) {
  TC* const p = (TC*)g.C + m * g.ldc + n;
  if (g.accumulate) v += ld_quad<TC>(p, left);
  if (g.stream) st_quad<TC, true>(p, v, left);
  else st_quad(p, v, left);
}

template <class T>
__device__ __forceinline__ void store_result(const GemmArgs& g, int64_t m, int n, f32x4_t v, int left) {
  if (sizeof(T) == 4 || g.c_f32) store_as<float>(g, m, n, v, left);
  else store_as<uint16_t>(g, m, n, v, left);
}

// Rows m, m + RPI, .. (EDGE: those below M) of a lane whose four columns lie
// inside the result.
template <class TC, int RUN, int RPI, bool EDGE>
__device__ __forceinline__ void store_rows(const GemmArgs& g, int64_t m, int n, f32x4_t* v) {
  TC* const p = (TC*)g.C + m * g.ldc + n;
  const int64_t step = RPI * g.ldc;
  auto in = [&](int r) { return !EDGE || m + r * RPI < g.M; };
  if (g.accumulate) {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
      if (in(r)) v[r] += ld_quad<TC>(p + r * step, 4);
  }
  if (g.stream) {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
      if (in(r)) st_quad<TC, true>(p + r * step, v[r], 4);
  } else {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
      if (in(r)) st_quad(p + r * step, v[r], 4);
  }
}

template <class T, bool GATED, int RUN, int RPI, bool EDGE>
__device__ __forceinline__ void fwd_rows(const FwdEpi& e, int64_t M, int64_t m, int n, const f32x4_t* z,
                                         const f32x4_t* u) {
  f32x4_t res[RUN] = {}, y[RUN];
  auto in = [&](int r) { return !EDGE || m + r * RPI < M; };
  if (e.R) {
    const T* const p = (const T*)e.R + m * e.ldr + n;
#pragma unroll
    for (int r = 0; r < RUN; ++r)
      if (in(r)) res[r] = ld_quad<T>(p + r * RPI * e.ldr, 4);
#pragma unroll
    for (int r = 0; r < RUN; ++r) asm volatile("" : "+v"(res[r]));
  }
  if (e.Z) {
    T* const p = (T*)e.Z + m * e.ldz + n;
    const int64_t step = RPI * e.ldz;
    if (e.stream) {
#pragma unroll
      for (int r = 0; r < RUN; ++r)
        if (in(r)) {
          st_quad<T, true>(p + r * step, z[r], 4);
          if constexpr (GATED) st_quad<T, true>(p + r * step + e.out, u[r], 4);
        }
    } else {
#pragma unroll
      for (int r = 0; r < RUN; ++r)
        if (in(r)) {
          st_quad(p + r * step, z[r], 4);
          if constexpr (GATED) st_quad(p + r * step + e.out, u[r], 4);
        }
    }
  }
  act_quads<RUN>(e.act, z, y);
#pragma unroll
  for (int r = 0; r < RUN; ++r) {
    if constexpr (GATED) y[r] *= u[r];
    y[r] += res[r];
  }
  T* const p = (T*)e.Y + m * e.ldy + n;
  const int64_t step = RPI * e.ldy;
  if (e.stream) {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
      if (in(r)) st_quad<T, true>(p + r * step, y[r], 4);
  } else {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
      if (in(r)) st_quad(p + r * step, y[r], 4);
  }
}

// One operand of the direct form: 64 rows, a piece of 16 bytes for each of 512
// threads, through registers to the places of a tile that the DMA above fills.
// Rows may lie at any alignment.  A source of dZ is turned into it on the way,
// rounded to the layer's type as it would be if it were stored.
template <class T, bool KS>
struct DirectOperand {
  static constexpr int CH = 16 / sizeof(T), KROW = 64 * sizeof(T);
  struct Raw {
    f32x4_t p[3];   // of the matrix or dY; of Z: gate, other projection
  };
  const T* base;
  int64_t ld;
  DzSource dz;
  int at, kk, rows, k_end;   // at: the lane's row; K strided: first of its columns

  template <class F>
  __device__ __forceinline__ void init(const void* p, int64_t ld_, const DzSource& d, int rows_, int k_end_, int row0,
                                       int wave, int lane, F&& row_of) {
    base = (const T*)p;
    ld = ld_;
    dz = d;
    rows = rows_;
    k_end = k_end_;
    if constexpr (KS) {
      constexpr int LPR = KROW / 16;
      const int k = wave * (64 / LPR) + lane / LPR;
      kk = k;
      at = row0 + ((lane % LPR) ^ Operand<64, true, sizeof(T), 8>::turn(k)) * CH;
    } else {
      kk = ((lane & 7) ^ (lane >> 3)) * CH;
      at = row_of(wave * 8 + (lane >> 3));
    }
  }

  __device__ __forceinline__ void place(int k0, int64_t& row, int& col, int& left) const {
    row = KS ? k0 + kk : at;
    col = KS ? at : k0 + kk;
    left = KS ? (row < k_end ? rows - col : 0) : k_end - col;
  }

  __device__ __forceinline__ Raw fetch(int k0) const {
    int64_t row;
    int col, left;
    place(k0, row, col, left);
    Raw r = {};
    if (!dz.Z) {
      r.p[0] = ld_piece<T>(base + row * ld + col, left);
      return r;
    }
    const T* const y = (const T*)dz.dY + row * dz.ldy;
    const T* const z = (const T*)dz.Z + row * dz.ldz;
    if (!dz.gated || col + CH <= dz.out) {
      r.p[0] = ld_piece<T>(y + col, left);
      r.p[1] = ld_piece<T>(z + col, left);
      if (dz.gated) r.p[2] = ld_piece<T>(z + dz.out + col, left);
    } else if (col >= dz.out) {
      r.p[0] = ld_piece<T>(y + col - dz.out, left);
      r.p[1] = ld_piece<T>(z + col - dz.out, left);
    } else {   // columns of both projections
      T e[3][CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const bool other = col + i >= dz.out;
        const int c = col + i - (other ? dz.out : 0);
        e[0][i] = i < left ? y[c] : (T)0;
        e[1][i] = i < left ? z[c] : (T)0;
        e[2][i] = i < left && !other ? z[dz.out + c] : (T)0;
      }
      __builtin_memcpy(r.p, e, 48);
    }
    return r;
  }

  // four elements from the i-th of a piece
  static __device__ __forceinline__ f32x4_t quad(f32x4_t p, int i) {
    if constexpr (sizeof(T) == 4) return p;
    const uint32_t lo = __float_as_uint(p[2 * i]), hi = __float_as_uint(p[2 * i + 1]);
    return f32x4_t{bf16_lo(lo), bf16_hi(lo), bf16_lo(hi), bf16_hi(hi)};
  }

  __device__ __forceinline__ f32x4_t finish(const Raw& r, int k0) const {
    if (!dz.Z) return r.p[0];
    int64_t row;
    int col, left;
    place(k0, row, col, left);
    f32x4_t o;
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) {
      const f32x4_t dy = quad(r.p[0], i), z = quad(r.p[1], i);
      f32x4_t a, da, d;
      act_grad_quad(dz.act, z, a, da);
      d = dy * da;
      if (dz.gated) {
        const f32x4_t u = quad(r.p[2], i);
#pragma unroll
        for (int k = 0; k < 4; ++k) d[k] = col + 4 * i + k >= dz.out ? dy[k] * a[k] : dy[k] * u[k] * da[k];
      }
      if constexpr (sizeof(T) == 4) {
        o = d;
      } else {
        o[2 * i] = __uint_as_float(bf16_pack2(d[0], d[1]));
        o[2 * i + 1] = __uint_as_float(bf16_pack2(d[2], d[3]));
      }
    }
    return o;
  }
};

// A form of the product: WM x WN waves, each 16 FA x 16 FB results, S stages
// of K tiles in LDS.
// S == 2 (256 x 256): the waves form two groups, one wave of each on every
// SIMD, that alternate between matrix instructions and LDS reads.
// S == 4 (128 x 128 and 64 x 64): tiles are loaded three ahead, one barrier a
// tile; two waves a SIMD, since one alone stands still while its loads are
// issued (4096^3 bf16 at 128 x 128: 203 us on four waves, 151 on eight).
// DIRECT: operands come through registers, two stages.
template <int WM_, int WN_, int FA_, int FB_, int S_, bool DIRECT_ = false>
struct Form {
  static constexpr bool DIRECT = DIRECT_;
  static constexpr int WM = WM_, WN = WN_, FA = FA_, FB = FB_, S = S_;
  static constexpr int NW = WM * WN, BM = WM * FA * 16, BN = WN * FB * 16;
  static constexpr int LDS = S * (BM + BN) * kRowBytes;
};
using Form256 = Form<2, 4, 8, 4, 2>;
using Form128 = Form<2, 4, 4, 2, 4>;
using Form64 = Form<4, 2, 1, 2, 4>;
using FormDirect = Form<4, 2, 1, 2, 2, true>;

// Block `block` of a product: all of its tile's K, or one part of it.  T: type
// of the operands, TE: of the layer (fp32 on bf16 planes: T bf16, TE fp32).
template <class T, class TE, class F, bool AKS, bool BKS, int EP>
__device__ __forceinline__ void gemm_block(const GemmArgs& g, int block, lds_char* lds) {
  constexpr int ES = sizeof(T), S = F::S, NW = F::NW, WM = F::WM, WN = F::WN, FA = F::FA, FB = F::FB;
  constexpr int BM = F::BM, BN = F::BN;
  constexpr bool PP = S == 2 && !F::DIRECT, SEG = sizeof(T) != sizeof(TE);
  using OA = Operand<BM, AKS, ES, NW>;
  using OB = Operand<BN, BKS, ES, NW>;
  constexpr int STAGE = OA::BYTES + OB::BYTES;
  constexpr int BK = OA::BK;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  const int per_split = g.tiles_m * g.tiles_n;
  const int t = xcd_order(block, per_split * g.splits);
  const int split = t / per_split;
  band_tile(t - split * per_split, g.tiles_m, g.tiles_n, tm, tn);
  const int kt0 = split * g.k_per_split;
  const int nk = min(g.k_per_split, g.tiles_k - kt0);
  const int m0 = tm * BM;
  constexpr int BNC = EP == EP_GATED ? BN / 2 : BN;   // columns of the result
  const int n0 = tn * BNC;

  // planes: the pair that the first tile belongs to, and the tile in it
  int pair_a = SEG ? kt0 / g.seg_tiles : 0, pair_b = pair_a;
  int in_a = SEG ? kt0 - pair_a * g.seg_tiles : kt0, in_b = in_a;
  const char* const A = (const char*)g.A;
  const char* const B = (const char*)g.B;
  auto row_of_a = [&](int r) { return min(m0 + r, g.M - 1); };
  auto row_of_b = [&](int r) {
    if constexpr (EP == EP_GATED) {
      // each wave's columns: half of them the gate's, then the same of the other projection
      constexpr int TN = FB * 16;
      const int c = min(n0 + r / TN * (TN / 2) + r % (TN / 2), g.N - 1);
      return (r % TN) >= TN / 2 ? c + g.N : c;
    } else {
      return min(n0 + r, g.N - 1);
    }
  };
  OA oa;
  OB ob;
  if constexpr (!F::DIRECT) {
    oa.init(SEG ? A + plane_of_a(pair_a) * g.plane_a : A, g.lda, g.M, m0, wave, lane, (int64_t)in_a * BK, row_of_a);
    ob.init(SEG ? B + plane_of_b(pair_b) * g.plane_b : B, g.ldb, g.N, n0, wave, lane, (int64_t)in_b * BK, row_of_b);
  }
  if constexpr (SEG) {   // plane 0
    oa.start -= plane_of_a(pair_a) * g.plane_a;
    ob.start -= plane_of_b(pair_b) * g.plane_b;
  }
  Reader<FA * 16, AKS, ES> ra;
  Reader<FB * 16, BKS, ES> rb;
  ra.template init<OA::KROW>(wm * FA * 16, lane);
  rb.template init<OB::KROW>(wn * FB * 16, lane);

  f32x4_t acc[FA][FB];
#pragma unroll
  for (int a = 0; a < FA; ++a)
#pragma unroll
    for (int b = 0; b < FB; ++b) acc[a][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

  int left_a = g.ka - in_a * BK, left_b = g.kb - in_b * BK;   // of K, at the next tile to load
  auto load_a = [&](int stage) {
    oa.load(lds0 + stage * STAGE, wave, left_a);
    left_a -= BK;
    if (SEG && ++in_a == g.seg_tiles) {
      in_a = 0;
      oa.base = oa.start + plane_of_a(++pair_a) * g.plane_a;
      left_a = g.ka;
    }
  };
  auto load_b = [&](int stage) {
    ob.load(lds0 + stage * STAGE + OA::BYTES, wave, left_b);
    left_b -= BK;
    if (SEG && ++in_b == g.seg_tiles) {
      in_b = 0;
      ob.base = ob.start + plane_of_b(++pair_b) * g.plane_b;
      left_b = g.kb;
    }
  };

  if constexpr (F::DIRECT) {
    // Three tiles' loads are in flight, in registers; a stage is written again
    // behind the barrier that follows every wave's last read of it.
    constexpr int D = 3;
    DirectOperand<T, AKS> da;
    DirectOperand<T, BKS> db;
    da.init(g.A, g.lda, g.dz, g.M, g.ka, m0, wave, lane, row_of_a);
    db.init(g.B, g.ldb, DzSource{}, g.N, g.kb, n0, wave, lane, row_of_b);
    typename DirectOperand<T, AKS>::Raw xa[D];
    typename DirectOperand<T, BKS>::Raw xb[D];
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (d < nk) {
        xa[d] = da.fetch((kt0 + d) * BK);
        xb[d] = db.fetch((kt0 + d) * BK);
      }
    typedef __attribute__((address_space(3))) f32x4_t lds_piece;
    for (int k3 = 0; k3 < nk; k3 += D) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const int kt = k3 + d;
        if (kt >= nk) continue;
        lds_char* const p = lds + (kt & 1) * STAGE;
        *(lds_piece*)(p + threadIdx.x * 16) = da.finish(xa[d], (kt0 + kt) * BK);
        *(lds_piece*)(p + OA::BYTES + threadIdx.x * 16) = db.finish(xb[d], (kt0 + kt) * BK);
        if (kt + D < nk) {
          xa[d] = da.fetch((kt0 + kt + D) * BK);
          xb[d] = db.fetch((kt0 + kt + D) * BK);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4_t fa[FA], fb[FB];
#pragma unroll
          for (int i = 0; i < FA; ++i) fa[i] = ra.template read_half<OA::KROW>(p, i, h);
#pragma unroll
          for (int i = 0; i < FB; ++i) fb[i] = rb.template read_half<OB::KROW>(p + OA::BYTES, i, h);
#pragma unroll
          for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[i][j] = mfma_half<ES>(fb[j], fa[i], acc[i][j]);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // every wave's reads have ended
  } else if constexpr (PP) {
    constexpr int HA = FA / 2, HB = FB / 2, Q1 = HA / 4, Q2 = HA / 2;
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
    // a run of matrix instructions, while the other group reads
    auto multiply = [&](const Frag<ES>* a, const Frag<ES>* b, int ha, int hb) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < HA; ++i)
#pragma unroll
        for (int j = 0; j < HB; ++j)
          acc[ha * HA + i][hb * HB + j] = mfma_tile<ES>(b[j], a[i], acc[ha * HA + i][hb * HB + j]);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_barrier" ::: "memory");
    };
    load_a(0);
    load_b(0);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    if (nk > 1) {
      load_b(1);
      load_a(1);
    }
    read_a(a0, 0, 0, 0, HA);
    if (wave >= NW / 2) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    // The quarters of the wave's results, in an order that needs one new half
    // operand each; the reads are spread so that each run of matrix
    // instructions covers the same number of them.  Loads of tile t + 1 end
    // before its first read (the wait before the second quarter, and a barrier
    // after it); the stage of tile t is loaded again only after every wave's
    // last read of it: B from the third quarter on, A from the fourth.
    for (int kt = 0; kt < nk; ++kt) {
      const int st = kt & 1;
      read_b(b0, st, 0);
      read_a(a1, st, 1, 0, Q1);
      multiply(a0, b0, 0, 0);
      read_b(b1, st, 1);
      read_a(a1, st, 1, Q1, Q2);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      multiply(a0, b1, 0, 1);
      read_a(a1, st, 1, Q2, HA);
      if (kt + 1 < nk) read_a(a0, st ^ 1, 0, 0, Q1);
      if (kt + 2 < nk) load_b(st);
      multiply(a1, b1, 1, 1);
      if (kt + 1 < nk) read_a(a0, st ^ 1, 0, Q1, HA);
      if (kt + 2 < nk) load_a(st);
      multiply(a1, b0, 1, 0);
    }
    if (wave < NW / 2) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  } else {
    constexpr int NI = OA::NI + OB::NI;   // loads of a tile, in flight together
    struct Half {
      f32x4_t a[FA], b[FB];
    } h0, h1;
    auto read = [&](Half& h, int stage, int s) {
      const lds_char* p = lds + stage * STAGE;
#pragma unroll
      for (int i = 0; i < FA; ++i) h.a[i] = ra.template read_half<OA::KROW>(p, i, s);
#pragma unroll
      for (int i = 0; i < FB; ++i) h.b[i] = rb.template read_half<OB::KROW>(p + OA::BYTES, i, s);
    };
    auto multiply = [&](const Half& h) {
#pragma unroll
      for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = mfma_half<ES>(h.b[j], h.a[i], acc[i][j]);
    };
#pragma unroll
    for (int j = 0; j < S - 1; ++j)
      if (j < nk) {
        load_a(j);
        load_b(j);
      }
    if (nk >= S - 1) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"((S - 2) * NI) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    read(h0, 0, 0);
    // In the middle of tile t every wave waits for its loads of tile t + 1
    // (those of the S - 3 tiles behind may be on their way) and for its own
    // reads; after the barrier tile t + 1 is whole and the stage of tile t - 1
    // is free.
    int st = 0, fill = S - 1;
    for (int kt = 0; kt < nk; ++kt) {
      read(h1, st, 1);
      multiply(h0);
      if (kt + 1 < nk) {
        if (kt + S - 2 < nk)
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((S - 3) * NI) : "memory");
        else
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (kt + S - 1 < nk) {
          load_a(fill);
          load_b(fill);
        }
        fill = fill == S - 1 ? 0 : fill + 1;
        st = st == S - 1 ? 0 : st + 1;
        read(h0, st, 0);
      }
      multiply(h1);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // every wave's reads have ended
  }

  // The results go through LDS, so that the epilogue runs along whole rows of
  // the tile: a wave's stores then cover 512 (256) consecutive bytes instead
  // of 32 in each of 16 rows, which lie in one memory channel when the row
  // length is a power of two (8192 x 16384 results: 229 us at K = 64 that way).
  // Pieces of 16 bytes are exchanged within a row by the row's number: a
  // lane holds 4 columns of row lane % 16 of each 16 x 16 block.
  constexpr int NP = PR_PASSES<BM, BN, S * STAGE>;
  constexpr int WR = FA / NP * 16, PR = WM * WR;   // rows of a wave and of a pass
  constexpr int QPR = BNC / 4, RPI = 64 / QPR;     // quads of a row; rows at a time
  const int li = lane & 15, lg = lane >> 4;
  const int q = lane % QPR, n = n0 + q * 4, left = g.N - n;
  const bool split_k = g.splits > 1;
  typedef __attribute__((address_space(3))) f32x4_t lds_f4;
  // Runs of rows without a test per element (tested per element, this part was
  // bound by its instructions: 8192 x 4096 x 16384 bf16 865 us, 814 this way).  The loads
  // of a run (the residual's) end before its stores begin, and the bias is in
  // before all of them: memory operations are counted in order, so a load that
  // is waited for behind stores waits for them too.
  f32x4_t bz = {}, bu = {};
  if (EP != EP_STORE && !split_k && left > 0) {
    bz = bias_quad(g.fwd, n, left);
    if constexpr (EP == EP_GATED) bu = bias_quad(g.fwd, g.N + n, left);
  }
  asm volatile("" : "+v"(bz), "+v"(bu));
  constexpr int STEPS = PR / NW / RPI, RUN = STEPS < 4 ? STEPS : 4;
  static_assert(PR / NW <= WR && WR % (PR / NW) == 0, "a wave's rows follow each other in the result");
  const int row0 = wave * (PR / NW) + lane / QPR;
  const bool whole = m0 + BM <= g.M && n0 + BNC <= g.N;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
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
    const int64_t mrow = m0 + row0 / WR * (FA * 16) + p * WR + row0 % WR;
#pragma unroll 1
    for (int r0 = 0; r0 < STEPS; r0 += RUN) {
      f32x4_t z[RUN], u[RUN] = {};
#pragma unroll
      for (int r = 0; r < RUN; ++r) {
        const int row = row0 + (r0 + r) * RPI;
        z[r] = *(const lds_f4*)(lds + row * BN * 4 + ((q ^ (row & 15)) << 4)) + bz;
        if constexpr (EP == EP_GATED) u[r] = *(const lds_f4*)(lds + row * BN * 4 + (((QPR + q) ^ (row & 15)) << 4)) + bu;
      }
      const int64_t m = mrow + r0 * RPI;
      if (split_k) {
        const int64_t w = part_width<EP>(g);
        float* const dst = g.part + ((int64_t)split * g.M + m) * w + n;
#pragma unroll
        for (int r = 0; r < RUN; ++r) {
          if (!whole && (m + r * RPI >= g.M || left <= 0)) continue;
          *(f32x4_t*)(dst + r * RPI * w) = z[r];
          if constexpr (EP == EP_GATED) *(f32x4_t*)(dst + r * RPI * w + w / 2) = u[r];
        }
      } else if (whole) {
        if constexpr (EP == EP_STORE) {
          if (sizeof(TE) == 4 || g.c_f32) store_rows<float, RUN, RPI, false>(g, m, n, z);
          else store_rows<uint16_t, RUN, RPI, false>(g, m, n, z);
        } else {
          fwd_rows<TE, EP == EP_GATED, RUN, RPI, false>(g.fwd, g.M, m, n, z, u);
        }
      } else if (left >= 4) {
        if constexpr (EP == EP_STORE) {
          if (sizeof(TE) == 4 || g.c_f32) store_rows<float, RUN, RPI, true>(g, m, n, z);
          else store_rows<uint16_t, RUN, RPI, true>(g, m, n, z);
        } else {
          fwd_rows<TE, EP == EP_GATED, RUN, RPI, true>(g.fwd, g.M, m, n, z, u);
        }
      } else if (left > 0) {   // the lanes of the last one to three columns
#pragma unroll 1
        for (int r = 0; r < RUN; ++r) {
          const int64_t mr = m + r * RPI;
          if (mr >= g.M) continue;
          if constexpr (EP == EP_STORE) store_result<TE>(g, mr, n, z[r], left);
          else fwd_epilogue<TE, EP == EP_GATED>(g.fwd, mr, n, z[r], u[r], residual_quad<TE>(g.fwd, mr, n, left));
        }
      }
    }
  }
}

template <class T, class TE, class F, int EP>
__global__ __launch_bounds__(F::NW * 64, 2) void k_gemm(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) char sm[F::LDS];
  gemm_block<T, TE, F, false, false, EP>(g, blockIdx.x, (lds_char*)sm);
}

template <class T, int EP>
__global__ __launch_bounds__(512, 4) void k_gemm_direct(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) char sm[FormDirect::LDS];
  gemm_block<T, T, FormDirect, false, false, EP>(g, blockIdx.x, (lds_char*)sm);
}

// Sum of the partial products of a split K, in split order, and the epilogue.
// Bound by memory (86 MB in 14.5 us, 6.0 TB/s).
template <class T, int EP>
__device__ __forceinline__ void join_block(const GemmArgs& g, int block, int blocks) {
  const int quads = (g.N + 3) / 4;
  const int64_t width = part_width<EP>(g), total = (int64_t)g.M * quads, stride = g.M * width;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < total; i += (int64_t)blocks * 256) {
    const int64_t m = total >> 32 ? i / quads : (int64_t)((uint32_t)i / (uint32_t)quads);
    const int n = (int)(i - m * quads) * 4, left = g.N - n;
    const float* p = g.part + m * width + n;
    f32x4_t z = {}, u = {};
    // four parts at a time, so that their loads are in flight together
    for (int s = 0; s < g.splits; s += 4, p += 4 * stride) {
      f32x4_t a[4], b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* const q = p + min(j, g.splits - 1 - s) * stride;
        a[j] = *(const f32x4_t*)q;
        if constexpr (EP == EP_GATED) b[j] = *(const f32x4_t*)(q + width / 2);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (s + j < g.splits) {
          z += a[j];
          if constexpr (EP == EP_GATED) u += b[j];
        }
    }
    if constexpr (EP == EP_STORE) {
      store_result<T>(g, m, n, z, left);
    } else {
      z += bias_quad(g.fwd, n, left);
      if constexpr (EP == EP_GATED) u += bias_quad(g.fwd, g.N + n, left);
      fwd_epilogue<T, EP == EP_GATED>(g.fwd, m, n, z, u, residual_quad<T>(g.fwd, m, n, left));
    }
  }
}

template <class T, int EP>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs g) {
  join_block<T, EP>(g, blockIdx.x, gridDim.x);
}

}  // namespace occ
