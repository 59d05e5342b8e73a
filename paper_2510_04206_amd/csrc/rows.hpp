// Rows of bf16 or fp32 elements that may start at any element: 8 elements of a lane at a time,
// sums over a wave, and the host's refusals.
#pragma once
#include <stdio.h>

#include "../../include/agrl.h"
#include "common.hpp"

namespace agrl {
namespace {

inline int fail(int code, const char* fn, const char* what) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s: %s", fn, what);
  set_last_error(buf);
  return code;
}

// Whether the heads of an output [T, n_head, d], rows `ld` and heads `hs` elements apart, are apart: each
// row's heads within the next row's distance, or each head's rows within the next head's.
inline bool heads_apart(int64_t T, int64_t n_head, int64_t d, int64_t ld, int64_t hs) {
  if (T <= 1 && n_head <= 1) return true;
  if (ld < 0 || hs < 0) return false;
  if (T <= 1) return hs >= d;
  if (n_head <= 1) return ld >= d;
  return (hs >= d && ld >= (__int128)(n_head - 1) * hs + d) ||
         (ld >= d && hs >= (__int128)(T - 1) * ld + d);
}

// rows may start at any element: 16-byte accesses of the element's alignment
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int CH = 8;   // elements per chunk

template <typename T>
struct Chunk;
template <>
struct Chunk<uint16_t> {   // bf16 bits
  u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *(const u32x4_a2*)p; }
  __device__ __forceinline__ void load_some(const uint16_t* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < CH - 1; ++k)
      if (k < n) w[k >> 1] |= (uint32_t)p[k] << (16 * (k & 1));
    v = u32x4{w[0], w[1], w[2], w[3]};
  }
  __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int k) const {
    return __uint_as_float(k & 1 ? v[k >> 1] & 0xffff0000u : v[k >> 1] << 16);
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&f)[CH]) {
    u32x4 o;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      o[k] = __builtin_bit_cast(
          uint32_t, __builtin_convertvector(f32x2{f[2 * k], f[2 * k + 1]}, bf16x2));
    *(u32x4_a2*)p = o;
  }
  static __device__ __forceinline__ void store_some(uint16_t* p, const float (&f)[CH], int n) {
#pragma unroll
    for (int k = 0; k < CH - 1; ++k)
      if (k < n) p[k] = f32_to_bf16_bits(f[k]);
  }
};
template <>
struct Chunk<float> {
  u32x4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *(const u32x4_a4*)p;
    hi = *(const u32x4_a4*)(p + 4);
  }
  __device__ __forceinline__ void load_some(const float* p, int n) {
    zero();
#pragma unroll
    for (int k = 0; k < CH - 1; ++k)
      if (k < n) {
        if (k < 4)
          lo[k] = __float_as_uint(p[k]);
        else
          hi[k - 4] = __float_as_uint(p[k]);
      }
  }
  __device__ __forceinline__ void zero() { lo = hi = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int k) const {
    return __uint_as_float(k < 4 ? lo[k & 3] : hi[k & 3]);
  }
  static __device__ __forceinline__ void store(float* p, const float (&f)[CH]) {
    typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
    *(f32x4_a4*)p = f32x4{f[0], f[1], f[2], f[3]};
    *(f32x4_a4*)(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
  }
  static __device__ __forceinline__ void store_some(float* p, const float (&f)[CH], int n) {
#pragma unroll
    for (int k = 0; k < CH - 1; ++k)
      if (k < n) p[k] = f[k];
  }
};

// Sum over a wave, the same in every lane: two exchanges within quads, two within 16 lanes
// (the VALU's own lane permutations), then the four 16-lane sums as scalars.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(
                 __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0xb1>(v);    // quad_perm 1,0,3,2
  v = dpp_add<0x4e>(v);    // quad_perm 2,3,0,1
  v = dpp_add<0x141>(v);   // mirror within 8 lanes
  v = dpp_add<0x140>(v);   // mirror within 16 lanes
  const int b = __float_as_int(v);
  return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) +
          __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(b, 32)) +
          __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}

}  // namespace
}  // namespace agrl
