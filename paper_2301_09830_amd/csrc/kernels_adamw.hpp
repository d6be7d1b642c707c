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
  int64_t ldg;          // of G; of factors: their rank
  int32_t rows, cols;
  float keep;
  uint32_t key;         // of the tensor's random bits
};

// Tensors of one launch.  Their descriptors are kernel arguments, 4 KB of them.
constexpr int kAdamTensors = 40;

struct AdamArgs {
  AdamTensor t[kAdamTensors];
  int32_t start[kAdamTensors];   // first block of each tensor (negative: earlier launches took some); behind the last one INT_MAX
  float b1, c1, b2, c2;   // c1 = 1 - b1, c2 = 1 - b2
  float a, c, eps;
  const float* grad_scale;   // device scalar, or null
  const uint32_t* flags;     // device word, or null: FLAG 1 set = leave everything as it is
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// The tensor of a block: which eight, then which of them, so that it waits
// for the arguments' memory twice (a step of 70 tensors, 3.1M elements, 20.9 us;
// by halves, 30 tensors a launch, 28.5).
__device__ __forceinline__ int adam_tensor(const AdamArgs& g, int b) {
  int n = 0;
#pragma unroll
  for (int i = 8; i < kAdamTensors; i += 8) n += g.start[i] <= b ? 8 : 0;
  const int32_t* const p = g.start + n;
#pragma unroll
  for (int i = 1; i < 8; ++i) n += p[i] <= b ? 1 : 0;
  return n;
}

// sqrt(x) to nearest, by the known test of a root against its neighbours with a
// fused residual: the hardware's result (1 ulp) gives way to a neighbour by the
// sign of x minus the product of the two values a midpoint lies between.
// 0, infinity and NaN pass the comparisons unchanged.  Below 2^-100, where the
// residual loses bits, the result may be 1 ulp off.
__device__ __forceinline__ float sqrt_rn(float x) {
  const float s = __builtin_amdgcn_sqrtf(x);
  const float lo = __uint_as_float(__float_as_uint(s) - 1u), hi = __uint_as_float(__float_as_uint(s) + 1u);
  float r = __builtin_fmaf(-lo, s, x) <= 0.0f ? lo : s;
  return __builtin_fmaf(-hi, s, x) > 0.0f ? hi : r;
}

// One step of four elements: w, m and v are updated, root = sqrt(v).
__device__ __forceinline__ void adam_quad(const AdamArgs& g, float keep, float scale, f32x4_t grad, f32x4_t& w,
                                          f32x4_t& m, f32x4_t& v, f32x4_t& root) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float gr = grad[i] * scale;
    m[i] = m[i] * g.b1 + gr * g.c1;
    v[i] = v[i] * g.b2 + (gr * gr) * g.c2;
    root[i] = sqrt_rn(v[i]);
    // the reciprocal's last bit is 2^-23 of the step, not of W
    w[i] = w[i] * keep - (m[i] * __builtin_amdgcn_rcpf(root[i] * g.c + g.eps)) * g.a;
  }
}

// 32 random bits for an element, 16 for m (low) and 16 for v: two rounds of an
// odd multiplier and a shifted exclusive or on x = index * 0x9E3779B1 + key +
// (index >> 32) * 0xBB67AE85 (mod 2^32).
__device__ __forceinline__ uint32_t adam_bits(uint32_t x) {
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
  const uint32_t start = (uint32_t)index * 0x9E3779B1u + key;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = adam_bits(start + i * 0x9E3779B1u + (uint32_t)((index + i) >> 32) * 0xBB67AE85u);
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
// Bound by memory.  One quad a thread and many short blocks, all of it
// nontemporal where every buffer starts on 64 bytes: 403M elements (30 bytes
// each with the bf16 copy) 2.06 ms, 5.8 TB/s; four quads a thread 2.17 ms,
// with ordinary loads and stores 2.30 ms.
constexpr int AD_BLOCK = 256 * 4;   // elements of a block

// A gradient whose rows lie apart is found element by element; the divisions
// hide behind the streams (268M elements, fp32: 1254 us with rows 32 elements
// apart, 1220 in one run; off 64 bytes 1371 and 1389).
template <class TG, bool NT>
__device__ __forceinline__ f32x4_t ld_grad(const AdamTensor& t, int64_t e, int left) {
  const TG* const G = (const TG*)t.G;
  if (t.ldg == t.cols) return ld_quad<TG, NT>(G + e, left);
  f32x4_t r = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i >= left) break;
    const int64_t row = (e + i) / t.cols;
    r[i] = ld_elem<TG>(G + row * t.ldg + (e + i - row * t.cols));
  }
  return r;
}

template <class TG, bool NT>
__global__ __launch_bounds__(256) void k_adamw32(AdamArgs g) {
  if (g.flags && (*g.flags & 1u)) return;
  const int index = adam_tensor(g, blockIdx.x);
  const AdamTensor& t = g.t[index];
  const float scale = g.grad_scale ? *g.grad_scale : 1.0f;
  const int64_t total = (int64_t)t.rows * t.cols;
  const int64_t e = (int64_t)((int)blockIdx.x - g.start[index]) * AD_BLOCK + threadIdx.x * 4;
  if (e >= total) return;
  const int left = (int)min((int64_t)4, total - e);
  float* const M = (float*)t.m + e;
  float* const V = (float*)t.v + e;
  f32x4_t w = ld_quad<float, NT>(t.W + e, left), m = ld_quad<float, NT>(M, left), v = ld_quad<float, NT>(V, left);
  f32x4_t root;
  adam_quad(g, t.keep, scale, ld_grad<TG, NT>(t, e, left), w, m, v, root);
  st_quad<float, NT>(t.W + e, w, left);
  st_quad<float, NT>(M, m, left);
  st_quad<float, NT>(V, v, left);
  if (t.W16) st_quad<uint16_t, NT>(t.W16 + e, w, left);
}

// ----------------------------------------------------------------------------
// stored gradients, 8-bit moments: a wave takes runs of 256 columns
// ----------------------------------------------------------------------------
// Two runs a wave (403M elements on bf16 gradients, 16 bytes each, 1.14 ms =
// 5.7 TB/s; four runs are as fast, but 10 % slower for 12.6M elements).  Bound
// by memory, closely followed by the instructions of the two encodings.
constexpr int AD8_RUNS = 2;                    // runs of a wave
constexpr int AD8_BLOCK = 4 * AD8_RUNS;        // runs of a block

// Largest value of the wave, in every lane.  Within 16 lanes by DPP: the
// neighbour, the other pair, the mirrored 8, the mirrored 16.
template <int CTRL>
__device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false)));
}

__device__ __forceinline__ float row_max(float x) {   // of 16 lanes
  x = dpp_max<0xB1>(x);    // quad_perm 1 0 3 2
  x = dpp_max<0x4E>(x);    // quad_perm 2 3 0 1
  x = dpp_max<0x141>(x);   // row_half_mirror
  return dpp_max<0x140>(x);   // row_mirror
}

__device__ __forceinline__ float wave_max(float x) {
  x = row_max(x);
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// One run of a row; FULL: all its 256 columns are there.
template <class TG, bool NT, bool FULL>
struct Adam8Run {
  f32x4_t grad, w;
  uint32_t cm, cv;
  float sm, sv;
  int64_t at, run;
  int left;

  __device__ __forceinline__ void load(const AdamTensor& t, int64_t row, int c0, int64_t r, int lane) {
    const int c = c0 + lane * 4;
    run = r;
    left = FULL ? 4 : t.cols - c;
    at = row * t.cols + c;
    grad = ld_quad<TG, NT>((const TG*)t.G + row * t.ldg + c, left);
    w = ld_quad<float, NT>(t.W + at, left);
    cm = ld_codes((const uint8_t*)t.m + at, left);
    cv = ld_codes((const uint8_t*)t.v + at, left);
    sm = t.m_scale[r];
    sv = t.v_scale[r];
  }

  __device__ __forceinline__ void step(const AdamArgs& g, const AdamTensor& t, float scale, int lane) {
    f32x4_t m = e4m3_decode(cm) * sm, root = e4m3_decode(cv) * sv;
    f32x4_t v = root * root;
    adam_quad(g, t.keep, scale, grad, w, m, v, root);
    // lanes behind the row's end hold zeros and do not count
    if constexpr (!FULL) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= left) m[i] = root[i] = 0.0f;
    }
    st_quad<float, NT>(t.W + at, w, left);
    if (t.W16) st_quad<uint16_t, NT>(t.W16 + at, w, left);
    const float tm = run_top(wave_max(quad_top(m))), tv = run_top(wave_max(quad_top(root)));
    const float im = (1.0f / tm) * 448.0f, iv = (1.0f / tv) * 448.0f;
    encode_quad(m, root, im, iv, (uint64_t)at, t.key, cm, cv);
    st_codes((uint8_t*)t.m + at, cm, left);
    st_codes((uint8_t*)t.v + at, cv, left);
    if (lane == 0) {
      t.m_scale[run] = tm * (1.0f / 448.0f);
      t.v_scale[run] = tv * (1.0f / 448.0f);
    }
  }
};

template <class TG, bool NT>
__global__ __launch_bounds__(256) void k_adamw8(AdamArgs g) {
  if (g.flags && (*g.flags & 1u)) return;
  const int index = adam_tensor(g, blockIdx.x);
  const AdamTensor& t = g.t[index];
  const float scale = g.grad_scale ? *g.grad_scale : 1.0f;
  const int lane = threadIdx.x & 63;
  const int per_row = (t.cols + kRun - 1) / kRun;
  const int64_t runs = (int64_t)t.rows * per_row;
  const int64_t r0 = (int64_t)((int)blockIdx.x - g.start[index]) * AD8_BLOCK + wave_id() * AD8_RUNS;
  if (r0 >= runs) return;
  int64_t row = runs >> 31 ? r0 / per_row : (int64_t)((uint32_t)r0 / (uint32_t)per_row);
  int b = (int)(r0 - row * per_row);
  if (t.cols % kRun == 0 && r0 + AD8_RUNS <= runs) {
    Adam8Run<TG, NT, true> f[AD8_RUNS];
#pragma unroll
    for (int q = 0; q < AD8_RUNS; ++q) {
      f[q].load(t, row, b * kRun, r0 + q, lane);
      if (++b == per_row) b = 0, ++row;
    }
#pragma unroll
    for (int q = 0; q < AD8_RUNS; ++q) f[q].step(g, t, scale, lane);
    return;
  }
#pragma unroll 1
  for (int q = 0; q < AD8_RUNS && r0 + q < runs; ++q) {
    Adam8Run<TG, NT, false> f;
    f.load(t, row, b * kRun, r0 + q, lane);
    f.step(g, t, scale, lane);
    if (++b == per_row) b = 0, ++row;
  }
}

// ----------------------------------------------------------------------------
// gradients as factors: G = P Q^T is made in registers and never stored
// ----------------------------------------------------------------------------
// A block takes 128 rows x 256 columns (one run of each row), a wave 16 of the
// rows.  The products are fp32 on v_mfma_f32_16x16x4_f32; Q, which all waves
// share, passes through LDS 32 ranks at a time, P goes straight to registers.
// A lane's results are four columns of row lane % 16 of each 16 x 16 block;
// 64 columns at a time they are turned through LDS, so that W and the moments
// are read and written in runs of 256 bytes of a row (16 runs of 64 bytes at a
// power of two apart meet in one memory channel: 2.8 ms for the 403M elements
// of eight layers of width 2048 at rank 32, 1.99 ms this way, 5.3 TB/s).  The first
// columns' W and moments are asked for before the products, each next 64
// columns' while the present ones are worked on.
// With fp32 moments, which have no runs, a block may take 64 columns (NJ = 1):
// twice the waves a SIMD, and four times the blocks where there are few.
constexpr int ADF_WAVES = 8;
constexpr int ADF_ROWS = 16 * ADF_WAVES;
constexpr int ADF_RANKS = 32;

template <int BITS>
struct AdamPiece {   // 4 rows x 4 columns of a lane, 4 rows apart
  f32x4_t w[4], m[BITS == 32 ? 4 : 1], v[BITS == 32 ? 4 : 1];
  uint32_t cm[4], cv[4];
};

// Rows 128 rb .. and columns 64 NJ run .. of a tensor.  FULL: all of them are there.
template <int BITS, bool NT, bool FULL, int NJ>
__device__ __forceinline__ void adamw_factors(const AdamArgs& g, const AdamTensor& t, int rb, int run, int per_row,
                                              f32x4_t* qs, f32x4_t (*turn)[16 * 16]) {
  constexpr int COLS = 64 * NJ;
  static_assert(BITS == 32 || COLS == kRun, "scales of whole runs");
  const float scale = g.grad_scale ? *g.grad_scale : 1.0f;
  const int rank = (int)t.ldg;
  const int wave = wave_id(), lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  const int row0 = rb * ADF_ROWS + wave * 16;
  const int c0 = run * COLS;
  const int cols_left = FULL ? COLS : t.cols - c0;
  auto left_of = [&](int row, int j) { return FULL ? 4 : row < t.rows ? cols_left - 64 * j - 4 * i : 0; };

  // rows row0 + 4 k + q, columns c0 + 64 j + 4 i of piece j
  AdamPiece<BITS> now, next;
  auto load = [&](AdamPiece<BITS>& p, int j) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = row0 + 4 * k + q;
      const int64_t e = (int64_t)row * t.cols + c0 + 64 * j + 4 * i;
      const int left = left_of(row, j);
      p.w[k] = ld_quad<float, NT>(t.W + e, left);
      if constexpr (BITS == 32) {
        p.m[k] = ld_quad<float, NT>((const float*)t.m + e, left);
        p.v[k] = ld_quad<float, NT>((const float*)t.v + e, left);
      } else {
        p.cm[k] = ld_codes((const uint8_t*)t.m + e, left);
        p.cv[k] = ld_codes((const uint8_t*)t.v + e, left);
      }
    }
  };
  load(now, 0);
  float sm[4], sv[4];   // scales of the four rows
  if constexpr (BITS == 8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t sr = (int64_t)min(row0 + 4 * k + q, t.rows - 1) * per_row + run;
      sm[k] = t.m_scale[sr];
      sv[k] = t.v_scale[sr];
    }
  }

  f32x4_t acc[4 * NJ];
#pragma unroll
  for (int f = 0; f < 4 * NJ; ++f) acc[f] = f32x4_t{};
  const float* const prow = t.P + (int64_t)min(row0 + i, t.rows - 1) * rank;
  // thread: pieces of 4 ranks of rows threadIdx / 8 + 64 u of the run's Q
  constexpr int QN = COLS * ADF_RANKS / 4 / (ADF_WAVES * 64);
  const int qr = threadIdx.x >> 3, qc = threadIdx.x & 7;
  f32x4_t qn[QN];
  auto load_q = [&](int k) {
#pragma unroll
    for (int u = 0; u < QN; ++u)
      qn[u] = ld_quad<float>(t.Q + (int64_t)min(c0 + qr + u * (ADF_WAVES * 8), t.cols - 1) * rank + k + 4 * qc,
                             rank - k - 4 * qc);
  };
  load_q(0);
  for (int k = 0; k < rank; k += ADF_RANKS) {
    f32x4_t pv[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) pv[s] = ld_quad<float>(prow + k + 16 * s + 4 * q, rank - k - 16 * s - 4 * q);
    if (k) __syncthreads();
#pragma unroll
    for (int u = 0; u < QN; ++u) {
      const int r = qr + u * (ADF_WAVES * 8);
      qs[r * 8 + (qc ^ (r & 7))] = qn[u];
    }
    __syncthreads();
    if (k + ADF_RANKS < rank) load_q(k + ADF_RANKS);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (k + 16 * s >= rank) continue;
#pragma unroll
      for (int f = 0; f < 4 * NJ; ++f) {
        const f32x4_t qv = qs[(16 * f + i) * 8 + ((4 * s + q) ^ (i & 7))];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(qv[j], pv[s][j], acc[f], 0, 0, 0);
      }
    }
  }

  float tm[4] = {}, tv[4] = {};
  f32x4_t ms[BITS == 8 ? NJ : 1][4], roots[BITS == 8 ? NJ : 1][4];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (64 * j >= cols_left) continue;
    if (j < NJ - 1 && 64 * (j + 1) < cols_left) load(next, j + 1);
#pragma unroll
    for (int f = 0; f < 4; ++f) turn[wave][i * 16 + ((4 * f + q) ^ i)] = acc[4 * j + f];
    __builtin_amdgcn_wave_barrier();
    f32x4_t gr[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) gr[k] = turn[wave][(4 * k + q) * 16 + (i ^ (4 * k + q))];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = row0 + 4 * k + q;
      const int64_t e = (int64_t)row * t.cols + c0 + 64 * j + 4 * i;
      const int left = left_of(row, j);
      f32x4_t m, v, root;
      if constexpr (BITS == 32) {
        m = now.m[k];
        v = now.v[k];
      } else {
        m = e4m3_decode(now.cm[k]) * sm[k];
        root = e4m3_decode(now.cv[k]) * sv[k];
        v = root * root;
      }
      adam_quad(g, t.keep, scale, gr[k], now.w[k], m, v, root);
      st_quad<float, NT>(t.W + e, now.w[k], left);
      if (t.W16) st_quad<uint16_t, NT>(t.W16 + e, now.w[k], left);
      if constexpr (BITS == 32) {
        st_quad<float, NT>((float*)t.m + e, m, left);
        st_quad<float, NT>((float*)t.v + e, v, left);
      } else {
        if constexpr (!FULL) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (c >= left) m[c] = root[c] = 0.0f;
        }
        tm[k] = fmaxf(tm[k], quad_top(m));
        tv[k] = fmaxf(tv[k], quad_top(root));
        ms[j][k] = m;
        roots[j][k] = root;
      }
    }
    if constexpr (NJ > 1) now = next;
  }
  if constexpr (BITS == 8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      tm[k] = run_top(row_max(tm[k]));   // a row's run lies in 16 lanes
      tv[k] = run_top(row_max(tv[k]));
      const float im = (1.0f / tm[k]) * 448.0f, iv = (1.0f / tv[k]) * 448.0f;
      const int row = row0 + 4 * k + q;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (64 * j >= cols_left) continue;
        const int64_t e = (int64_t)row * t.cols + c0 + 64 * j + 4 * i;
        const int left = left_of(row, j);
        uint32_t cm, cv;
        encode_quad(ms[j][k], roots[j][k], im, iv, (uint64_t)e, t.key, cm, cv);
        st_codes((uint8_t*)t.m + e, cm, left);
        st_codes((uint8_t*)t.v + e, cv, left);
      }
      if (i == 0 && (FULL || row < t.rows)) {
        const int64_t sr = (int64_t)row * per_row + run;
        t.m_scale[sr] = tm[k] * (1.0f / 448.0f);
        t.v_scale[sr] = tv[k] * (1.0f / 448.0f);
      }
    }
  }
}

template <int BITS, bool NT, int NJ>
__global__ __launch_bounds__(ADF_WAVES * 64) void k_adamw_factors(AdamArgs g) {
  if (g.flags && (*g.flags & 1u)) return;
  constexpr int COLS = 64 * NJ;
  __shared__ f32x4_t qs[COLS * ADF_RANKS / 4];
  __shared__ f32x4_t turn[ADF_WAVES][16 * 16];
  const int index = adam_tensor(g, blockIdx.x);
  const AdamTensor& t = g.t[index];
  const int per_row = (t.cols + COLS - 1) / COLS;
  const int b = (int)blockIdx.x - g.start[index];
  const int rb = b / per_row, run = b - rb * per_row;
  if ((rb + 1) * ADF_ROWS <= t.rows && (run + 1) * COLS <= t.cols)
    adamw_factors<BITS, NT, true, NJ>(g, t, rb, run, per_row, qs, turn);
  else
    adamw_factors<BITS, NT, false, NJ>(g, t, rb, run, per_row, qs, turn);
}

}  // namespace occ
