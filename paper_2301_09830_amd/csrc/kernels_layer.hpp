// The linear and gated layers beside their tiled products: products of few
// tokens, the gradient at the pre-activation with the bias gradient, and
// copies of operands that no 16-byte access fits.
#pragma once

#include "kernels_gemm.hpp"

namespace occ {

// ----------------------------------------------------------------------------
// few tokens: the weights are streamed once
// ----------------------------------------------------------------------------
struct SkinnyArgs {
  const void* X;   // tokens x in
  const void* W;   // out (gated: 2 out) x in
  int64_t ldx, ldw;
  int32_t tokens, in;
  FwdEpi fwd;
};

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

// A block makes 16 columns of Y (gated: the 16 rows of both projections) for
// up to 16 NT tokens: its SK_WAVES waves take K in turns of one tile of 128
// bytes a row, with weights and tokens loaded straight into the registers of
// the matrix instructions, and add their sums in wave order.
constexpr int SK_WAVES = 8;

template <class T, int NT, bool GATED>
__global__ __launch_bounds__(SK_WAVES * 64) void k_skinny(SkinnyArgs g) {
  constexpr int ES = sizeof(T), CH = 16 / ES, BK = kRowBytes / ES, NW = GATED ? 2 : 1;
  __shared__ f32x4_t sums[SK_WAVES][NW * NT][64];
  const int wave = wave_id(), lane = threadIdx.x & 63;
  const int i = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const int row = min(n0 + i, g.fwd.out - 1);
  const T* w[NW];
  w[0] = (const T*)g.W + (int64_t)row * g.ldw + q * CH;
  if constexpr (GATED) w[1] = w[0] + (int64_t)g.fwd.out * g.ldw;
  const T* x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) x[t] = (const T*)g.X + (int64_t)min(16 * t + i, g.tokens - 1) * g.ldx + q * CH;
  f32x4_t acc[NW][NT] = {};
  // pieces q and q + 4 of each row's tile
  auto load = [&](const T* p, int64_t k, int left) {
    Frag<ES> f;
#pragma unroll
    for (int s = 0; s < 2; ++s) f.v[s] = ld_piece<T>(p + k + s * 4 * CH, left - s * 4 * CH);
    return f;
  };
  struct Step {
    Frag<ES> w[NW], x[NT];
  };
  auto step = [&](const Step& f) {
#pragma unroll
    for (int a = 0; a < NW; ++a)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[a][t] = mfma_tile<ES>(f.w[a], f.x[t], acc[a][t]);
  };
  // Two runs of U tiles are in flight: one is multiplied while the next loads.
  constexpr int U = NT == 1 ? 4 : 2;
  const int full = g.in / BK;
  const int runs = full > wave ? ((full - wave - 1) / SK_WAVES + 1) / U : 0;   // whole runs of this wave
  Step one[U], two[U];
  auto fetch = [&](Step* f, int run) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = (int64_t)(wave + (run * U + u) * SK_WAVES) * BK;
#pragma unroll
      for (int a = 0; a < NW; ++a) f[u].w[a] = load(w[a], k, BK);
#pragma unroll
      for (int t = 0; t < NT; ++t) f[u].x[t] = load(x[t], k, BK);
    }
  };
  auto multiply = [&](const Step* f) {
#pragma unroll
    for (int u = 0; u < U; ++u) step(f[u]);
  };
  if (runs) fetch(one, 0);
  for (int r = 0; r < runs; r += 2) {
    if (r + 1 < runs) fetch(two, r + 1);
    multiply(one);
    if (r + 1 >= runs) break;
    if (r + 2 < runs) fetch(one, r + 2);
    multiply(two);
  }
  for (int kt = wave + runs * U * SK_WAVES; (int64_t)kt * BK < g.in; kt += SK_WAVES) {
    const int64_t k = (int64_t)kt * BK;
    const int left = (int)min((int64_t)BK, g.in - k) - q * CH;
    Step f;
#pragma unroll
    for (int a = 0; a < NW; ++a) f.w[a] = load(w[a], k, left);
#pragma unroll
    for (int t = 0; t < NT; ++t) f.x[t] = load(x[t], k, left);
    step(f);
  }
#pragma unroll
  for (int a = 0; a < NW; ++a)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][a * NT + t][lane] = acc[a][t];
  __syncthreads();
  // one wave a block of 16 tokens
  for (int t = wave; t < NT; t += SK_WAVES) {
    const int m = 16 * t + i;
    f32x4_t z = {}, u = {};
#pragma unroll
    for (int v = 0; v < SK_WAVES; ++v) {
      z += sums[v][t][lane];
      if constexpr (GATED) u += sums[v][NT + t][lane];
    }
    const int n = n0 + q * 4, left = g.fwd.out - n;
    if (m < g.tokens && left > 0) {
      z += bias_quad(g.fwd, n, left);
      if constexpr (GATED) u += bias_quad(g.fwd, g.fwd.out + n, left);
      fwd_epilogue<T, GATED>(g.fwd, m, n, z, u);
    }
  }
}

// ----------------------------------------------------------------------------
// gradient at the pre-activation, and the bias gradient
// ----------------------------------------------------------------------------
// dZ = dY act'(Z); gated, with Z = [G U]: dG = dY U act'(G), dU = dY act(G).
// dZ is rounded to the layer's type, the type its products take.  Bias sums
// are taken from the values before that rounding, in fp32 over a strip of
// rows, and the strips are added by k_dz_bias in strip order.
struct DzArgs {
  const void* dY;
  const void* Z;     // null: dZ = dY, and only the bias sums are made
  void* dZ;          // null: only the bias sums are made
  float* bias_part;  // strips x width, or null
  int64_t ldy, ldz, ldd;
  int32_t tokens, out, act, strip;   // strip: rows of a block
};

constexpr int DZ_LANES = 32;   // threads along a row, 4 columns each
constexpr int DZ_ROWS = 8;     // rows at a time

template <class T, bool GATED>
__global__ __launch_bounds__(256) void k_dz(DzArgs g) {
  const int cx = threadIdx.x & (DZ_LANES - 1), ry = threadIdx.x / DZ_LANES;
  const int n = (blockIdx.x * DZ_LANES + cx) * 4, left = g.out - n;
  const int64_t r0 = (int64_t)blockIdx.y * g.strip;
  const int64_t r1 = min(r0 + g.strip, (int64_t)g.tokens);
  f32x4_t s0 = {}, s1 = {};
  if (left > 0) {
    for (int64_t m = r0 + ry; m < r1; m += DZ_ROWS) {
      const f32x4_t dy = ld_quad<T>((const T*)g.dY + m * g.ldy + n, left);
      f32x4_t d0 = dy, d1 = {};
      if (g.Z) {
        const T* const zr = (const T*)g.Z + m * g.ldz + n;
        const f32x4_t z = ld_quad<T>(zr, left);
        f32x4_t u = {};
        if constexpr (GATED) u = ld_quad<T>(zr + g.out, left);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float a, da;
          act_grad_f(g.act, z[i], a, da);
          if constexpr (GATED) {
            d0[i] = dy[i] * u[i] * da;
            d1[i] = dy[i] * a;
          } else {
            d0[i] = dy[i] * da;
          }
        }
      }
      if (g.dZ) {
        T* const o = (T*)g.dZ + m * g.ldd + n;
        st_quad(o, d0, left);
        if constexpr (GATED) st_quad(o + g.out, d1, left);
        // rows end in whole 16-byte pieces, zeros behind the last column
        if (left <= 4)
          for (int64_t c = GATED ? 2 * (int64_t)g.out : g.out; c < g.ldd; ++c) ((T*)g.dZ)[m * g.ldd + c] = (T)0;
      }
      s0 += d0;
      if constexpr (GATED) s1 += d1;
    }
  }
  if (!g.bias_part) return;
  __shared__ f32x4_t part[GATED ? 2 : 1][DZ_ROWS][DZ_LANES];
  part[0][ry][cx] = s0;
  if constexpr (GATED) part[1][ry][cx] = s1;
  __syncthreads();
  if (ry < (GATED ? 2 : 1) && left > 0) {
    f32x4_t s = {};
#pragma unroll
    for (int r = 0; r < DZ_ROWS; ++r) s += part[ry][r][cx];
    const int64_t width = GATED ? 2 * (int64_t)g.out : g.out;
    st_quad(g.bias_part + blockIdx.y * width + ry * (int64_t)g.out + n, s, left);
  }
}

__global__ __launch_bounds__(256) void k_dz_bias(const float* part, int strips, int64_t width, float* dbias,
                                                 int accumulate) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= width) return;
  float s = accumulate ? dbias[n] : 0.0f;
  for (int i = 0; i < strips; ++i) s += part[i * width + n];
  dbias[n] = s;
}

// Copy of an operand with rows on 16 bytes, whole pieces and zeros behind
// their ends.
template <class T>
__global__ __launch_bounds__(256) void k_align_rows(const T* src, int64_t lds, T* dst, int64_t rows, int cols,
                                                    int pieces) {
  constexpr int CH = 16 / sizeof(T);
  const int64_t total = rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / pieces;
    const int c = (int)(i - r * pieces) * CH;
    *(f32x4_t*)(dst + i * CH) = ld_piece<T>(src + r * lds + c, cols - c);
  }
}

// Zeros where no token contributes to a gradient.
template <class T>
__global__ __launch_bounds__(256) void k_zero_rows(T* p, int64_t rows, int cols, int64_t ld) {
  const int64_t total = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256)
    p[i / cols * ld + i % cols] = (T)0;
}

}  // namespace occ
