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

// One column of one token.
template <class T, bool GATED>
__device__ __forceinline__ void fwd_epilogue_one(const FwdEpi& e, int64_t m, int n, float z, float u) {
  if (e.bias) {
    z += e.bias[n];
    if constexpr (GATED) u += e.bias[e.out + n];
  }
  if (e.Z) {
    st_elem((T*)e.Z + m * e.ldz + n, z);
    if constexpr (GATED) st_elem((T*)e.Z + m * e.ldz + e.out + n, u);
  }
  float y = act_quad(e.act, f32x4_t{z, z, z, z})[0];
  if constexpr (GATED) y *= u;
  if (e.R) y += ld_elem<T>((const T*)e.R + m * e.ldr + n);
  st_elem((T*)e.Y + m * e.ldy + n, y);
}

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s);
  return x;
}

// Up to NT tokens, NT <= 4: a wave takes two rows of W (gated: a gate's row
// and the other projection's) along K, 1024 bytes of a row an instruction, so
// that the stream runs through the memory channels in order; sums stay in the
// lanes until the end.  Bound by memory: one token, 4096 x 4096 bf16 5.5 us, 6.1
// TB/s; four tokens, gated 4096 x 8192 23.8 us, 5.7 TB/s.
constexpr int DOT_WAVES = 4;

template <class T, int NT, bool GATED>
__global__ __launch_bounds__(DOT_WAVES * 64) void k_dot(SkinnyArgs g) {
  constexpr int CH = 16 / sizeof(T), BK = 64 * CH;
  const int lane = threadIdx.x & 63;
  const int id = blockIdx.x * DOT_WAVES + wave_id();
  const int n0 = GATED ? id : 2 * id;
  if (n0 >= g.fwd.out) return;
  const bool both = GATED || n0 + 1 < g.fwd.out;
  const T* const w0 = (const T*)g.W + (int64_t)n0 * g.ldw;
  const T* const w1 = GATED ? w0 + (int64_t)g.fwd.out * g.ldw : both ? w0 + g.ldw : w0;
  float z[2][NT] = {};
  auto load = [&](const T* p, int64_t k) { return ld_piece<T>(p + k, (int)min((int64_t)CH, g.in - k)); };
  auto widen = [&](f32x4_t v, float* e) {
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
  };
  constexpr int U = NT <= 2 ? 4 : 2;
  auto add = [&](f32x4_t a, f32x4_t b, const f32x4_t* x) {
    float ea[CH], eb[CH], ex[CH];
    widen(a, ea);
    widen(b, eb);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      widen(x[t], ex);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        z[0][t] = __builtin_fmaf(ea[i], ex[i], z[0][t]);
        z[1][t] = __builtin_fmaf(eb[i], ex[i], z[1][t]);
      }
    }
  };
  const T* x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) x[t] = (const T*)g.X + (int64_t)min(t, g.tokens - 1) * g.ldx;
  int64_t k = lane * CH;
  for (; k + (U - 1) * BK + CH <= g.in; k += U * BK) {
    f32x4_t a[U], b[U], xv[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      a[u] = ld_piece<T>(w0 + k + u * BK, CH);
      b[u] = ld_piece<T>(w1 + k + u * BK, CH);
#pragma unroll
      for (int t = 0; t < NT; ++t) xv[u][t] = ld_piece<T>(x[t] + k + u * BK, CH);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) add(a[u], b[u], xv[u]);
  }
  for (; k < g.in; k += BK) {
    f32x4_t xv[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xv[t] = load(x[t], k);
    add(load(w0, k), load(w1, k), xv);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float s0 = wave_sum(z[0][t]), s1 = wave_sum(z[1][t]);
    if (t >= g.tokens) continue;
    if constexpr (GATED) {
      if (lane == t) fwd_epilogue_one<T, true>(g.fwd, t, n0, s0, s1);
    } else {
      const int c = lane - 2 * t;
      if (c == 0 || (c == 1 && both)) fwd_epilogue_one<T, false>(g.fwd, t, n0 + c, c ? s1 : s0, 0.0f);
    }
  }
}

// A block makes 16 columns of Y (gated: the 16 rows of both projections) for
// up to 16 NT tokens: its SK_WAVES waves take K in turns of one tile of 128
// bytes a row, with weights and tokens loaded straight into the registers of
// the matrix instructions, and add their sums in wave order.  8 tokens, 4096 x
// 4096 bf16 8.6 us: bound by the latency of the loads that a CU keeps in flight.
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
      fwd_epilogue<T, GATED>(g.fwd, m, n, z, u, residual_quad<T>(g.fwd, m, n, left));
    }
  }
}

// ----------------------------------------------------------------------------
// before the products: the gradient at the pre-activation, aligned operands
// ----------------------------------------------------------------------------
// dZ = dY act'(Z); gated, with Z = [G U]: dG = dY U act'(G), dU = dY act(G).
// dZ is rounded to the layer's type, the type its products take: in bf16 the
// gradients are then off by 0.0024 of their norm, against 0.0017 with dZ in fp32
// (their own rounding at the store).  dZ as two bf16 planes would have that too,
// for twice the matrix instructions, the bound of these products.  Bias sums
// are taken from the values before that rounding, in fp32 over a strip of
// rows; bias_block adds the strips.  Bound by memory (gated 8192 x 8192 bf16: 671
// MB in 116 us, 5.8 TB/s).
struct DzArgs {
  const void* dY;
  const void* Z;     // null: dZ = dY, and only the bias sums are made
  void* dZ;          // null: only the bias sums are made
  float* bias_part;  // strips x width, or null
  int64_t ldy, ldz, ldd;
  int32_t tokens, out, act, strip;   // strip: rows of a block
  int32_t across;                    // blocks along a row
  int64_t plane;                     // fp32: dZ as three bf16 planes this far apart (elements); else 0
};

// Four elements as three bf16 planes, the first `left` of them inside the row.
__device__ __forceinline__ void st_planes(uint16_t* p, int64_t plane, f32x4_t v, int left) {
  uint16_t e[4][kPlanes];
#pragma unroll
  for (int i = 0; i < 4; ++i) split3(v[i], e[i]);
#pragma unroll
  for (int k = 0; k < kPlanes; ++k) {
    uint16_t* const q = p + k * plane;
    if (left >= 4) {
      *(u2h_t*)q = u2h_t{e[0][k] | (uint32_t)e[1][k] << 16, e[2][k] | (uint32_t)e[3][k] << 16};
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < left) q[i] = e[i][k];
    }
  }
}

template <class T, bool GATED>
__device__ __forceinline__ void dz_block(const DzArgs& g, int block) {
  __shared__ f32x4_t part[GATED ? 2 : 1][DZ_ROWS][DZ_LANES];
  const int cx = threadIdx.x & (DZ_LANES - 1), ry = threadIdx.x / DZ_LANES;
  const int by = block / g.across, bx = block - by * g.across;
  const int n = (bx * DZ_LANES + cx) * 4, left = g.out - n;
  const int64_t r0 = (int64_t)by * g.strip;
  const int64_t r1 = min(r0 + g.strip, (int64_t)g.tokens);
  f32x4_t s0 = {}, s1 = {};
  if (left > 0) {
    for (int64_t m = r0 + ry; m < r1; m += DZ_ROWS) {
      const f32x4_t dy = ld_quad<T>((const T*)g.dY + m * g.ldy + n, left);
      f32x4_t d0 = dy, d1 = {};
      if (g.Z) {
        const T* const zr = (const T*)g.Z + m * g.ldz + n;
        const f32x4_t z = ld_quad<T>(zr, left);
        f32x4_t u = {}, a, da;
        if constexpr (GATED) u = ld_quad<T>(zr + g.out, left);
        act_grad_quad(g.act, z, a, da);
        if constexpr (GATED) {
          d0 = dy * u * da;
          d1 = dy * a;
        } else {
          d0 = dy * da;
        }
      }
      if (sizeof(T) == 4 && g.plane) {
        uint16_t* const o = (uint16_t*)g.dZ + m * g.ldd + n;
        st_planes(o, g.plane, d0, left);
        if constexpr (GATED) st_planes(o + g.out, g.plane, d1, left);
        if (left <= 4)
          for (int k = 0; k < kPlanes; ++k)
            for (int64_t c = GATED ? 2 * (int64_t)g.out : g.out; c < g.ldd; ++c)
              ((uint16_t*)g.dZ)[k * g.plane + m * g.ldd + c] = 0;
      } else if (g.dZ) {
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
  part[0][ry][cx] = s0;
  if constexpr (GATED) part[1][ry][cx] = s1;
  __syncthreads();
  if (ry < (GATED ? 2 : 1) && left > 0) {
    f32x4_t s = {};
#pragma unroll
    for (int r = 0; r < DZ_ROWS; ++r) s += part[ry][r][cx];
    const int64_t width = GATED ? 2 * (int64_t)g.out : g.out;
    st_quad(g.bias_part + by * width + ry * (int64_t)g.out + n, s, left);
  }
}

// Copy of an operand with rows on 16 bytes, whole pieces and zeros behind
// their ends.
struct CopyArgs {
  const void* src;
  void* dst;
  int64_t ld, rows;
  int32_t cols, pieces, blocks;
  int64_t plane;   // fp32: as three bf16 planes this far apart (elements); else 0
};

template <class T>
__device__ __forceinline__ void copy_block(const CopyArgs& g, int block) {
  constexpr int CH = 16 / sizeof(T);
  const int64_t total = g.rows * g.pieces;
  for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < total; i += (int64_t)g.blocks * 256) {
    const int64_t r = i / g.pieces;
    if (sizeof(T) == 4 && g.plane) {
      const int c = (int)(i - r * g.pieces) * 8;
      const float* const p = (const float*)g.src + r * g.ld + c;
      uint16_t* const q = (uint16_t*)g.dst + i * 8;
      st_planes(q, g.plane, ld_quad<float>(p, g.cols - c), 4);
      st_planes(q + 4, g.plane, ld_quad<float>(p + 4, g.cols - c - 4), 4);
      continue;
    }
    const int c = (int)(i - r * g.pieces) * CH;
    *(f32x4_t*)((T*)g.dst + i * CH) = ld_piece<T>((const T*)g.src + r * g.ld + c, g.cols - c);
  }
}

// All of it in one launch: dz_blocks blocks make dZ, the rest copy.
struct PrepArgs {
  DzArgs dz;
  CopyArgs copy[3];   // of dY, W and X
  int32_t dz_blocks;
};

template <class T, bool GATED>
__global__ __launch_bounds__(256) void k_prep(PrepArgs g) {
  int b = blockIdx.x;
  if (b < g.dz_blocks) return dz_block<T, GATED>(g.dz, b);
  b -= g.dz_blocks;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (b < g.copy[i].blocks) return copy_block<T>(g.copy[i], b);
    b -= g.copy[i].blocks;
  }
}

// ----------------------------------------------------------------------------
// the products of the backward pass
// ----------------------------------------------------------------------------
struct BiasArgs {
  const float* part;   // strips x width
  float* dbias;
  int64_t width;
  int32_t strips, accumulate;
  DzSource src;        // of the direct form, which has no parts
  int32_t tokens;
};

// 64 columns a block of 512 threads: 8 threads a column add every 8th strip,
// and their sums are added in order.
__device__ __forceinline__ void bias_block(const BiasArgs& g, int block, float* lds) {
  constexpr int G = 8;
  const int c = threadIdx.x & 63, r = threadIdx.x >> 6;
  const int64_t n = (int64_t)block * 64 + c;
  float s = 0.0f;
  if (n < g.width) {
    const float* p = g.part + n;
    int i = r;
    for (; i + 3 * G < g.strips; i += 4 * G) {
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = p[(i + u * G) * g.width];
#pragma unroll
      for (int u = 0; u < 4; ++u) s += v[u];
    }
    for (; i < g.strips; i += G) s += p[i * g.width];
  }
  lds[threadIdx.x] = s;
  __syncthreads();
  if (r || n >= g.width) return;
#pragma unroll
  for (int u = 1; u < G; ++u) s += lds[u * 64 + c];
  g.dbias[n] = g.accumulate ? g.dbias[n] + s : s;
}

// Straight from dY and Z: 16 columns of dY a block of 512 threads, four of
// them and every 128th row a thread, both projections together (64 columns and
// every 32nd row: the backward pass of 991 x 1076 x 390 bf16 24 us, a chain of
// loads; 14 this way).
constexpr int BD_COLS = 16, BD_ROWS = 128;
constexpr int BD_LDS = 2 * BD_ROWS * BD_COLS * 4;

template <class T>
__device__ __forceinline__ void bias_direct(const BiasArgs& g, int block, float* lds) {
  constexpr int U = 4;   // rows whose loads are in flight together
  const DzSource& d = g.src;
  const int c = threadIdx.x % (BD_COLS / 4), r = threadIdx.x / (BD_COLS / 4);
  const int n = block * BD_COLS + c * 4, left = d.out - n;
  f32x4_t s0 = {}, s1 = {};
  if (left > 0) {
    for (int64_t m = r; m < g.tokens; m += U * BD_ROWS) {
      f32x4_t dy[U], z[U], u[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t row = min(m + i * BD_ROWS, (int64_t)g.tokens - 1);
        dy[i] = ld_quad<T>((const T*)d.dY + row * d.ldy + n, left);
        const T* const zr = (const T*)d.Z + row * d.ldz + n;
        if (d.Z) z[i] = ld_quad<T>(zr, left);
        if (d.gated) u[i] = ld_quad<T>(zr + d.out, left);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (m + i * BD_ROWS >= g.tokens) continue;
        f32x4_t a, da;
        if (d.Z) act_grad_quad(d.act, z[i], a, da);
        s0 += d.gated ? dy[i] * u[i] * da : d.Z ? dy[i] * da : dy[i];
        if (d.gated) s1 += dy[i] * a;
      }
    }
  }
  f32x4_t* const part = (f32x4_t*)lds;
  part[threadIdx.x] = s0;
  if (d.gated) part[512 + threadIdx.x] = s1;
  __syncthreads();
  // 16 threads a column, 8 rows each, then their sums in order
  constexpr int G = 16, PER = BD_ROWS / G;
  const int col = threadIdx.x % BD_COLS, k = threadIdx.x / BD_COLS % G, half = threadIdx.x / (BD_COLS * G);
  float s = 0.0f;
  const float* const p = lds + (half * BD_ROWS + k * PER) * BD_COLS + col;
  if (half == 0 || d.gated) {
#pragma unroll
    for (int i = 0; i < PER; ++i) s += p[i * BD_COLS];
  }
  __syncthreads();
  lds[threadIdx.x] = s;
  __syncthreads();
  if (k || (half && !d.gated) || block * BD_COLS + col >= d.out) return;
#pragma unroll
  for (int i = 1; i < G; ++i) s += lds[threadIdx.x + i * BD_COLS];
  const int64_t at = (int64_t)half * d.out + block * BD_COLS + col;
  g.dbias[at] = g.accumulate ? g.dbias[at] + s : s;
}

template <class T>
__device__ __forceinline__ void bias_any(const BiasArgs& g, int block, float* lds) {
  if (g.part) bias_block(g, block, lds);
  else bias_direct<T>(g, block, lds);
}

// The bias gradient, dX = dZ W and dW = dZ^T X in one launch: where one of the
// products alone leaves CUs idle, or ends in a part of a round, the other's
// blocks fill them.
struct BackwardArgs {
  GemmArgs dx, dw;
  BiasArgs bias;
  int32_t dx_blocks, dw_blocks;
};

template <class T, class TE, class F>
__global__ __launch_bounds__(F::NW * 64, 2) void k_backward(BackwardArgs g) {
  __shared__ __attribute__((aligned(1024))) char sm[F::LDS];
  int b = blockIdx.x;
  if (b < g.dx_blocks) return gemm_block<T, TE, F, false, true, EP_STORE>(g.dx, b, (lds_char*)sm);
  b -= g.dx_blocks;
  if (b < g.dw_blocks) return gemm_block<T, TE, F, true, true, EP_STORE>(g.dw, b, (lds_char*)sm);
  static_assert(F::NW == 8, "the bias blocks run on eight waves");
  bias_any<TE>(g.bias, b - g.dw_blocks, (float*)sm);
}

// The same from dY and Z themselves, with no launch before it.
template <class T>
__global__ __launch_bounds__(512, 4) void k_backward_direct(BackwardArgs g) {
  __shared__ __attribute__((aligned(1024))) char sm[FormDirect::LDS];
  int b = blockIdx.x;
  if (b < g.dx_blocks) return gemm_block<T, T, FormDirect, false, true, EP_STORE>(g.dx, b, (lds_char*)sm);
  b -= g.dx_blocks;
  if (b < g.dw_blocks) return gemm_block<T, T, FormDirect, true, true, EP_STORE>(g.dw, b, (lds_char*)sm);
  bias_direct<T>(g.bias, b - g.dw_blocks, (float*)sm);
}

// Joins the parts of both products.
template <class T>
__global__ __launch_bounds__(256) void k_backward_join(GemmArgs dx, GemmArgs dw, int dx_blocks) {
  const int b = blockIdx.x;
  if (b < dx_blocks) return join_block<T, EP_STORE>(dx, b, dx_blocks);
  join_block<T, EP_STORE>(dw, b - dx_blocks, gridDim.x - dx_blocks);
}

// dbias alone
template <class T>
__global__ __launch_bounds__(512) void k_bias(BiasArgs g) {
  __shared__ __attribute__((aligned(16))) float sm[BD_LDS / 4];
  bias_any<T>(g, blockIdx.x, sm);
}

// Zeros where no token contributes to a gradient.
template <class T>
__global__ __launch_bounds__(256) void k_zero_rows(T* p, int64_t rows, int cols, int64_t ld) {
  const int64_t total = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256)
    p[i / cols * ld + i % cols] = (T)0;
}

}  // namespace occ
