// AdamW over many tensors in one launch, with moments in 32 bits or in 8, on
// gradients as they are stored (fp32, bf16) or as the compressor's factors.
//
// Per element, in fp32 and in this order (no contraction, so that every form
// of the kernel rounds alike):
//   g = grad_scale G
//   m = b1 m + (1 - b1) g
//   v = b2 v + (1 - b2) (g g)
//   W = keep W - a (m / (sqrt(v) c + eps))
// keep = 1 - lr decay, a = lr / (1 - b1^t), c = 1 / sqrt(1 - b2^t).
//
// 8-bit moments: m and sqrt(v) as OCP e4m3 codes times an fp32 scale for each
// run of 256 columns of a row, scale = (largest magnitude) / 448.  The square
// root halves the range that v spans in a run, and is what the update divides
// by.  Codes are rounded up with the probability of the part cut off (16
// random bits from a counter hash of seed, tensor and element): an average
// whose step is below half a code's distance would never move under rounding
// to nearest.  A positive sqrt(v) keeps a positive code, so that no update
// divides a stored m by zero.  The step itself uses the moments before they
// are rounded.
#pragma once

#include "kernels_gemm.hpp"

namespace occ {

constexpr int kRun = 256;   // columns that share a scale

struct AdamTensor {
  float* W;
  uint16_t* W16;        // bf16 copy of W, or null
  const void* G;        // gradient rows x cols (ldg), or null: P Q^T
  const float* P;       // rows x rank
  const float* Q;       // cols x rank
  void* m;              // fp32, or e4m3 codes
  void* v;
  float* m_scale;       // 8-bit moments: rows x ceil(cols / 256)
  float* v_scale;
  int64_t ldg;
  int32_t rows, cols, rank;
  int32_t block0;       // first block of this tensor in the launch
  float keep;
  uint32_t key;         // of the tensor's random bits
};

constexpr int kAdamTensors = 30;   // of one launch: their descriptors are kernel arguments

struct AdamArgs {
  AdamTensor t[kAdamTensors];
  int32_t count;
  float b1, c1, b2, c2;   // c1 = 1 - b1, c2 = 1 - b2
  float a, c, eps;
  const float* grad_scale;   // device scalar, or null
  const uint32_t* flags;     // device word, or null: FLAG 1 set = leave everything as it is
};

__device__ __forceinline__ int adam_tensor(const AdamArgs& g, int b) {
  int lo = 0, hi = g.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (g.t[mid].block0 <= b) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One step of four elements: w, m and v are updated, root = sqrt(v).
__device__ __forceinline__ void adam_quad(const AdamArgs& g, float keep, float scale, f32x4_t grad, f32x4_t& w,
                                          f32x4_t& m, f32x4_t& v, f32x4_t& root) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float gr = grad[i] * scale;
    m[i] = m[i] * g.b1 + gr * g.c1;
    v[i] = v[i] * g.b2 + (gr * gr) * g.c2;
    root[i] = __builtin_sqrtf(v[i]);
    w[i] = w[i] * keep - (m[i] / (root[i] * g.c + g.eps)) * g.a;
  }
}

// 32 random bits for element `index` of the tensor with this key: 16 for m
// (low), 16 for v.  Two rounds of an odd multiplier and a shifted exclusive or.
__device__ __forceinline__ uint32_t adam_bits(uint64_t index, uint32_t key) {
  uint32_t x = (uint32_t)index * 0x9E3779B1u + key + (uint32_t)(index >> 32) * 0xBB67AE85u;
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// Magnitude code of |y| <= 448 in e4m3, rounded up with probability (part cut
// off): the 16 bits of `rnd` are added below the 3 bits kept.  Below the
// smallest normal, 2^-6, the codes have the distance of the binade [2^-6,
// 2^-5), and adding 2^-6 puts y there.
__device__ __forceinline__ uint32_t e4m3_code(float y, uint32_t rnd) {
  const float a = fabsf(y);
  const bool small = a < 0.015625f;
  const uint32_t bits = __float_as_uint(small ? a + 0.015625f : a) + (rnd << 4);
  const uint32_t code = min((bits >> 20) - (small ? 968u : 960u), 126u);
  return y != y ? 127u : code;
}

__device__ __forceinline__ f32x4_t e4m3_decode(uint32_t w) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return f32x4_t{lo[0], lo[1], hi[0], hi[1]};
}

typedef uint32_t u32_any_t __attribute__((aligned(1)));

// Four codes at any alignment, the first `left` of them inside the row.
__device__ __forceinline__ uint32_t ld_codes(const uint8_t* p, int left) {
  if (left >= 4) return *(const u32_any_t*)p;
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < left) w |= (uint32_t)p[i] << (8 * i);
  return w;
}

__device__ __forceinline__ void st_codes(uint8_t* p, uint32_t w, int left) {
  if (left >= 4) {
    *(u32_any_t*)p = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < left) p[i] = (uint8_t)(w >> (8 * i));
}

__device__ __forceinline__ float quad_top(f32x4_t x) {
  return fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
}

// Scales of a run from its largest magnitude.  The floor keeps 448 / top
// finite; a run of zeros has it as its scale.
__device__ __forceinline__ float run_top(float x) { return fmaxf(x, 7.888609052210118e-31f); }   // 2^-100

__device__ __forceinline__ void encode_quad(f32x4_t m, f32x4_t root, float inv_m, float inv_v, uint64_t index,
                                            uint32_t key, uint32_t& cm, uint32_t& cv) {
  cm = cv = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = adam_bits(index + i, key);
    const float y = m[i] * inv_m;
    cm |= (e4m3_code(y, r & 0xffffu) | (__float_as_uint(y) >> 31 << 7)) << (8 * i);
    uint32_t c = e4m3_code(root[i] * inv_v, r >> 16);
    if (root[i] > 0.0f && c == 0) c = 1;
    cv |= c << (8 * i);
  }
}

// ----------------------------------------------------------------------------
// stored gradients, 32-bit moments: runs over the elements in order
// ----------------------------------------------------------------------------
constexpr int AD_QUADS = 4;                      // quads of a thread
constexpr int AD_BLOCK = 256 * 4 * AD_QUADS;     // elements of a block

template <class TG>
__device__ __forceinline__ f32x4_t ld_grad(const AdamTensor& t, int64_t e, int left) {
  const TG* const G = (const TG*)t.G;
  if (t.ldg == t.cols) return ld_quad<TG>(G + e, left);
  f32x4_t r = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i >= left) break;
    const int64_t row = (e + i) / t.cols;
    r[i] = ld_elem<TG>(G + row * t.ldg + (e + i - row * t.cols));
  }
  return r;
}

template <class TG>
__global__ __launch_bounds__(256) void k_adamw32(AdamArgs g) {
  if (g.flags && (*g.flags & 1u)) return;
  const AdamTensor& t = g.t[adam_tensor(g, blockIdx.x)];
  const float scale = g.grad_scale ? *g.grad_scale : 1.0f;
  const int64_t total = (int64_t)t.rows * t.cols;
  const int64_t e0 = (int64_t)((int)blockIdx.x - t.block0) * AD_BLOCK + threadIdx.x * 4;
  float* const M = (float*)t.m;
  float* const V = (float*)t.v;
  f32x4_t gr[AD_QUADS], w[AD_QUADS], m[AD_QUADS], v[AD_QUADS], root;
#pragma unroll
  for (int q = 0; q < AD_QUADS; ++q) {
    const int64_t e = e0 + q * 1024;
    const int left = (int)max((int64_t)0, min((int64_t)4, total - e));
    gr[q] = ld_grad<TG>(t, e, left);
    w[q] = ld_quad<float>(t.W + e, left);
    m[q] = ld_quad<float>(M + e, left);
    v[q] = ld_quad<float>(V + e, left);
  }
#pragma unroll
  for (int q = 0; q < AD_QUADS; ++q) {
    const int64_t e = e0 + q * 1024;
    const int left = (int)max((int64_t)0, min((int64_t)4, total - e));
    adam_quad(g, t.keep, scale, gr[q], w[q], m[q], v[q], root);
    st_quad(t.W + e, w[q], left);
    st_quad(M + e, m[q], left);
    st_quad(V + e, v[q], left);
    if (t.W16) st_quad(t.W16 + e, w[q], left);
  }
}

// ----------------------------------------------------------------------------
// stored gradients, 8-bit moments: a wave takes runs of 256 columns
// ----------------------------------------------------------------------------
constexpr int AD8_RUNS = 4;                    // runs of a wave
constexpr int AD8_BLOCK = 4 * AD8_RUNS;        // runs of a block

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 32; s; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}

template <class TG>
__global__ __launch_bounds__(256) void k_adamw8(AdamArgs g) {
  if (g.flags && (*g.flags & 1u)) return;
  const AdamTensor& t = g.t[adam_tensor(g, blockIdx.x)];
  const float scale = g.grad_scale ? *g.grad_scale : 1.0f;
  const int lane = threadIdx.x & 63;
  const int per_row = (t.cols + kRun - 1) / kRun;
  const int64_t runs = (int64_t)t.rows * per_row;
  const int64_t r0 = (int64_t)((int)blockIdx.x - t.block0) * AD8_BLOCK + wave_id() * AD8_RUNS;
  uint8_t* const M = (uint8_t*)t.m;
  uint8_t* const V = (uint8_t*)t.v;
  f32x4_t gr[AD8_RUNS], w[AD8_RUNS];
  uint32_t cm[AD8_RUNS], cv[AD8_RUNS];
  float sm[AD8_RUNS], sv[AD8_RUNS];
  int64_t at[AD8_RUNS];
  int lf[AD8_RUNS];
#pragma unroll
  for (int q = 0; q < AD8_RUNS; ++q) {
    const int64_t run = r0 + q;
    if (run < runs) {
      const int64_t row = run / per_row;
      const int c = (int)(run - row * per_row) * kRun + lane * 4;
      lf[q] = t.cols - c;
      at[q] = row * t.cols + c;
      gr[q] = ld_quad<TG>((const TG*)t.G + row * t.ldg + c, lf[q]);
      w[q] = ld_quad<float>(t.W + at[q], lf[q]);
      cm[q] = ld_codes(M + at[q], lf[q]);
      cv[q] = ld_codes(V + at[q], lf[q]);
      sm[q] = t.m_scale[run];
      sv[q] = t.v_scale[run];
    }
  }
#pragma unroll
  for (int q = 0; q < AD8_RUNS; ++q) {
    const int64_t run = r0 + q;
    if (run >= runs) break;
    f32x4_t m = e4m3_decode(cm[q]) * sm[q], root = e4m3_decode(cv[q]) * sv[q];
    f32x4_t v = root * root;
    adam_quad(g, t.keep, scale, gr[q], w[q], m, v, root);
    // lanes behind the row's end hold zeros and do not count
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i >= lf[q]) m[i] = root[i] = 0.0f;
    const float tm = run_top(wave_max(quad_top(m))), tv = run_top(wave_max(quad_top(root)));
    const float im = (1.0f / tm) * 448.0f, iv = (1.0f / tv) * 448.0f;
    encode_quad(m, root, im, iv, (uint64_t)at[q], t.key, cm[q], cv[q]);
    st_quad(t.W + at[q], w[q], lf[q]);
    if (t.W16) st_quad(t.W16 + at[q], w[q], lf[q]);
    st_codes(M + at[q], cm[q], lf[q]);
    st_codes(V + at[q], cv[q], lf[q]);
    if (lane == 0) {
      t.m_scale[run] = tm * (1.0f / 448.0f);
      t.v_scale[run] = tv * (1.0f / 448.0f);
    }
  }
}

// ----------------------------------------------------------------------------
// gradients as factors: G = P Q^T is made in registers and never stored
// ----------------------------------------------------------------------------
// A wave takes 16 rows x 256 columns (one run of each row), a block 64 rows.
// The products are fp32 on v_mfma_f32_16x16x4_f32 with Q as the first
// operand: a lane then holds four consecutive columns of row lane % 16 of
// each 16 x 16 block.  The order of the rank within the products is that of
// the 16-byte pieces both operands are loaded in.
constexpr int ADF_ROWS = 64;

template <int BITS>
__global__ __launch_bounds__(256) void k_adamw_factors(AdamArgs g) {
  if (g.flags && (*g.flags & 1u)) return;
  const AdamTensor& t = g.t[adam_tensor(g, blockIdx.x)];
  const float scale = g.grad_scale ? *g.grad_scale : 1.0f;
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  const int per_row = (t.cols + kRun - 1) / kRun;
  const int b = (int)blockIdx.x - t.block0;
  const int rb = b / per_row, run = b - rb * per_row;
  const int row = rb * ADF_ROWS + wave_id() * 16 + i;
  const bool mine = row < t.rows;
  const int c0 = run * kRun;
  const int nf = min(16, (t.cols - c0 + 15) / 16);
  f32x4_t acc[16];
#pragma unroll
  for (int f = 0; f < 16; ++f) acc[f] = f32x4_t{};
  const float* const p = t.P + (int64_t)min(row, t.rows - 1) * t.rank + 4 * q;
  const float* const qp = t.Q + 4 * q;
  for (int k = 0; k < t.rank; k += 16) {
    const int left = t.rank - k - 4 * q;
    const f32x4_t pv = ld_quad<float>(p + k, left);
#pragma unroll
    for (int f = 0; f < 16; ++f) {
      if (f >= nf) continue;
      const f32x4_t qv = ld_quad<float>(qp + (int64_t)min(c0 + 16 * f + i, t.cols - 1) * t.rank + k, left);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(qv[j], pv[j], acc[f], 0, 0, 0);
    }
  }
  const int64_t e0 = (int64_t)row * t.cols + c0 + 4 * q;
  const int left0 = mine ? t.cols - c0 - 4 * q : 0;
  if constexpr (BITS == 32) {
    float* const M = (float*)t.m;
    float* const V = (float*)t.v;
#pragma unroll
    for (int f = 0; f < 16; ++f) {
      if (f >= nf) continue;
      const int64_t e = e0 + 16 * f;
      const int left = left0 - 16 * f;
      f32x4_t w = ld_quad<float>(t.W + e, left), m = ld_quad<float>(M + e, left), v = ld_quad<float>(V + e, left);
      f32x4_t root;
      adam_quad(g, t.keep, scale, acc[f], w, m, v, root);
      st_quad(t.W + e, w, left);
      st_quad(M + e, m, left);
      st_quad(V + e, v, left);
      if (t.W16) st_quad(t.W16 + e, w, left);
    }
  } else {
    uint8_t* const M = (uint8_t*)t.m;
    uint8_t* const V = (uint8_t*)t.v;
    const int64_t sr = (int64_t)min(row, t.rows - 1) * per_row + run;
    const float sm = t.m_scale[sr], sv = t.v_scale[sr];
    float tm = 0.0f, tv = 0.0f;
    f32x4_t roots[16];
#pragma unroll
    for (int f = 0; f < 16; ++f) {
      if (f >= nf) continue;
      const int64_t e = e0 + 16 * f;
      const int left = left0 - 16 * f;
      f32x4_t w = ld_quad<float>(t.W + e, left);
      f32x4_t m = e4m3_decode(ld_codes(M + e, left)) * sm, root = e4m3_decode(ld_codes(V + e, left)) * sv;
      f32x4_t v = root * root;
      adam_quad(g, t.keep, scale, acc[f], w, m, v, root);
      st_quad(t.W + e, w, left);
      if (t.W16) st_quad(t.W16 + e, w, left);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k >= left) m[k] = root[k] = 0.0f;
      tm = fmaxf(tm, quad_top(m));
      tv = fmaxf(tv, quad_top(root));
      acc[f] = m;
      roots[f] = root;
    }
    // a row's run lies in the lanes i, i + 16, i + 32 and i + 48
    tm = fmaxf(tm, __shfl_xor(tm, 16));
    tv = fmaxf(tv, __shfl_xor(tv, 16));
    tm = run_top(fmaxf(tm, __shfl_xor(tm, 32)));
    tv = run_top(fmaxf(tv, __shfl_xor(tv, 32)));
    const float im = (1.0f / tm) * 448.0f, iv = (1.0f / tv) * 448.0f;
#pragma unroll
    for (int f = 0; f < 16; ++f) {
      if (f >= nf) continue;
      const int64_t e = e0 + 16 * f;
      const int left = left0 - 16 * f;
      uint32_t cm, cv;
      encode_quad(acc[f], roots[f], im, iv, (uint64_t)e, t.key, cm, cv);
      st_codes(M + e, cm, left);
      st_codes(V + e, cv, left);
    }
    if (q == 0 && mine) {
      t.m_scale[sr] = tm * (1.0f / 448.0f);
      t.v_scale[sr] = tv * (1.0f / 448.0f);
    }
  }
}

}  // namespace occ
