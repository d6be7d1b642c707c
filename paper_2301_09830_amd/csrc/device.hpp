// Device helpers shared by all kernels of liboptcc: wave index, bf16, vector
// accesses at any alignment, XCD-aware block order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace occ {

// Index of this thread's wave in its block, as a wave-uniform (SGPR) value so
// that addresses derived from it qualify for scalar loads.
__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// bf16 bit pattern of an fp32 value, rounded to nearest even (NaN stays NaN).
__device__ __forceinline__ uint16_t bf16_rne(float v) {
  return __builtin_bit_cast(uint16_t, (__bf16)v);
}

__device__ __forceinline__ uint32_t bf16_pack2(float lo, float hi) {
  return (uint32_t)bf16_rne(lo) | ((uint32_t)bf16_rne(hi) << 16);
}

// Vector accesses at element alignment.  The hardware takes 16-byte global
// loads and stores at any address that is a multiple of the element size, so
// rows that start at any element use the same instructions as aligned ones
// (measured on a 1 GiB stream: loads at 4-byte alignment 5.1 TB/s, as aligned;
// at 2-byte alignment 4.9 TB/s).  `AL` only states that the address is known
// to be naturally aligned.
typedef float f4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef float f2u_t __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u4h_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u2h_t __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u1h_t __attribute__((aligned(2)));

template <bool AL>
__device__ __forceinline__ float4 ld_f4(const float* p) {
  if constexpr (AL) {
    return *(const float4*)p;
  } else {
    const f4u_t v = *(const f4u_t*)p;
    return make_float4(v[0], v[1], v[2], v[3]);
  }
}

// eight / four bf16 elements
template <bool AL>
__device__ __forceinline__ uint4 ld_h8(const uint16_t* p) {
  if constexpr (AL) {
    return *(const uint4*)p;
  } else {
    const u4h_t v = *(const u4h_t*)p;
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
}

template <bool AL>
__device__ __forceinline__ uint2 ld_h4(const uint16_t* p) {
  if constexpr (AL) {
    return *(const uint2*)p;
  } else {
    const u2h_t v = *(const u2h_t*)p;
    return make_uint2(v[0], v[1]);
  }
}

// One value, stored nontemporally or plainly.
template <bool NT, class T>
__device__ __forceinline__ void st_as(T v, T* p) {
  if constexpr (NT) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// Four consecutive elements of an output row.  NT (every output row on
// 64-byte boundaries): nontemporal, since the dirty lines of these streaming
// outputs would otherwise be written back during the next pass.  Other rows:
// plain stores at element alignment, whose partly written lines meet in the
// L2 (16-byte stores along rows 16 bytes off the 64-byte grid: 6.3 TB/s
// plain, 3.1 TB/s nontemporal; on the grid 6.9 and 5.6-5.8).
template <bool NT>
__device__ __forceinline__ void store_f4(float* o, float a, float b, float c, float e) {
  typedef float nt4 __attribute__((ext_vector_type(4)));
  if constexpr (NT) __builtin_nontemporal_store(nt4{a, b, c, e}, (nt4*)o);
  else *(f4u_t*)o = f4u_t{a, b, c, e};
}

// Tile index of a block of a kernel whose neighbouring tiles share an operand
// slice (the Q columns of a left-product split, the P_hat rows of a
// right-product split or reconstruction row block).  Workgroups are dealt to
// the 8 XCDs round-robin (workgroup b to XCD b % 8), each XCD with its own L2;
// renumbering so that XCD x takes the contiguous tile range
// [x G8 / 8, (x + 1) G8 / 8) (G8 = the grid rounded down to a multiple of 8;
// the last G - G8 blocks keep their index) keeps the tiles that run on one
// XCD on few slices.  A bijection of [0, G): results do not change.
__device__ __forceinline__ int xcd_tile() {
  const int g8 = (int)gridDim.x & ~7, b = (int)blockIdx.x;
  return b < g8 ? (b & 7) * (g8 >> 3) + (b >> 3) : b;
}

}  // namespace occ
