// Rotation of the query and key heads of packed tokens by their positions (gfx950).
//
//   y = R x: for each pair (p, q) of a head's first `rot` elements, with the angle
//   t = position * base^(-2 i / rot),   y_p = x_p cos t - x_q sin t,  y_q = x_p sin t + x_q cos t
//   pair i: (i, i + rot / 2), or (2 i, 2 i + 1) interleaved.  The gradient is the rotation by -t.
//
// Memory bounds it: each head is read and written once.  A lane keeps its place in a head (8
// elements of each half, or of four pairs) over all tokens and heads it meets, so its frequencies are
// formed once, and a token's angles once for the heads that it takes of it (a workgroup has 256 lanes, 32 heads of
// 128, and goes through the rest).  The angle is counted in turns in 64
// bits (position 2^20: what 32 bits would leave of it is off by 0.06 radians) and its fraction
// is rounded to 32, where sine and cosine are taken.
//
// Measured (MI355X; a copy of 2 GiB moves 4.9 TB/s): 65536 tokens, 48 of 56 heads of 128 bf16, 351 us, 4.6 TB/s (a first dozen 371); 150
// tokens, 12 heads of 64 fp32, 3.5 us on the GPU, 7.7 from Python.
#include <math.h>

#include "rows.hpp"

namespace agrl {
namespace {

struct RotateArgs {
  int64_t T;
  int32_t heads, d, rot, units, hgroup, tgroup;   // hgroup x tgroup heads and tokens at a time
  const void* x;
  int64_t ld_x, hs_x;
  const int32_t* position;
  double log2_base;
  float sign;
  void* y;
  int64_t ld_y, hs_y;
  int32_t copy;         // y is not x: elements past rot are copied
};

// VEC = 8: units of 8 elements (half pairing: 8 of each half), then chunks past rot.
// VEC = 1: one pair, or one element past rot.
template <typename X, int VEC, bool INTER>
__global__ void __launch_bounds__(512) rotate_kernel(RotateArgs a) {
  constexpr int PAIRS = VEC == 1 ? 1 : INTER ? VEC / 2 : VEC;
  const int per = a.hgroup * a.units;              // lanes of a token
  const int tsub = threadIdx.x / per, in = threadIdx.x - tsub * per;
  const int hsub = in / a.units, u = in - hsub * a.units;
  if (tsub >= a.tgroup) return;
  const int rotating = a.rot / 2 / PAIRS;          // units that rotate
  const bool rotates = u < rotating;
  if (!rotates && !a.copy) return;
  // elements: first of the unit, and of its partner
  const int e0 = rotates ? (INTER ? u * 2 * PAIRS : u * PAIRS) : a.rot + (u - rotating) * VEC;
  const int e1 = INTER ? e0 + 1 : e0 + a.rot / 2;
  double turns[PAIRS];
#pragma unroll
  for (int k = 0; k < PAIRS; ++k)
    turns[k] = exp2(a.log2_base * (-2.0 * (u * PAIRS + k) / a.rot)) * 0.15915494309189535;
  for (int64_t t = (int64_t)blockIdx.x * a.tgroup + tsub; t < a.T; t += (int64_t)gridDim.x * a.tgroup) {
    float co[PAIRS], si[PAIRS];
    if (rotates) {
      const double pos = a.position ? (double)a.position[t] : (double)t;
#pragma unroll
      for (int k = 0; k < PAIRS; ++k) {
        const double f = pos * turns[k];
        sincospif(2.0f * (float)(f - rint(f)), &si[k], &co[k]);
        si[k] *= a.sign;
      }
    }
    for (int h = hsub; h < a.heads; h += a.hgroup) {
      const X* x = (const X*)a.x + t * a.ld_x + h * a.hs_x;
      X* y = (X*)a.y + t * a.ld_y + h * a.hs_y;
      if constexpr (VEC == 1) {
        auto get = [](X v) { return sizeof(X) == 2 ? bf16_bits_to_f32((uint16_t)v) : (float)v; };
        if (!rotates) {
          y[e0] = x[e0];
          continue;
        }
        const float p = get(x[e0]), q = get(x[e1]);
        const float yp = fmaf(p, co[0], -(q * si[0])), yq = fmaf(p, si[0], q * co[0]);
        if constexpr (sizeof(X) == 2) {
          y[e0] = f32_to_bf16_bits(yp);
          y[e1] = f32_to_bf16_bits(yq);
        } else {
          y[e0] = yp;
          y[e1] = yq;
        }
      } else {
        Chunk<X> p, q;
        float f[CH], g[CH];
        p.load(x + e0);
        if (!rotates) {
#pragma unroll
          for (int k = 0; k < CH; ++k) f[k] = p.get(k);
          Chunk<X>::store(y + e0, f);
        } else if constexpr (INTER) {
#pragma unroll
          for (int k = 0; k < PAIRS; ++k) {
            const float v = p.get(2 * k), w = p.get(2 * k + 1);
            f[2 * k] = fmaf(v, co[k], -(w * si[k]));
            f[2 * k + 1] = fmaf(v, si[k], w * co[k]);
          }
          Chunk<X>::store(y + e0, f);
        } else {
          q.load(x + e1);
#pragma unroll
          for (int k = 0; k < CH; ++k) {
            const float v = p.get(k), w = q.get(k);
            f[k] = fmaf(v, co[k], -(w * si[k]));
            g[k] = fmaf(v, si[k], w * co[k]);
          }
          Chunk<X>::store(y + e0, f);
          Chunk<X>::store(y + e1, g);
        }
      }
    }
  }
}

}  // namespace
}  // namespace agrl

extern "C" int agrl_rotate_heads(int64_t T, int32_t n_head, int32_t d, int32_t rot, int32_t dtype,
                                 const void* x, int64_t ld_x, int64_t head_x, const int32_t* position,
                                 double base, int32_t interleaved, int32_t inverse, void* y,
                                 int64_t ld_y, int64_t head_y, void* stream) {
  using namespace agrl;
  const char* fn = "agrl_rotate_heads";
  if (dtype != AGRL_BF16 && dtype != AGRL_F32)
    return fail(AGRL_E_DTYPE, fn, "dtype must be AGRL_BF16 or AGRL_F32");
  if (T < 0 || T > ((int64_t)1 << 40) || n_head < 0 || n_head > (1 << 20) || d <= 0)
    return fail(AGRL_E_SHAPE, fn, "bad T, n_head or d");
  if (rot < 0 || rot > d || rot % 2) return fail(AGRL_E_SHAPE, fn, "rot must be even, at most d");
  if (d > 512) return fail(AGRL_E_UNSUPPORTED, fn, "d is larger than 512");
  if (ld_x < 0 || head_x < 0) return fail(AGRL_E_SHAPE, fn, "a stride of x is negative");
  if (!heads_apart(T, n_head, d, ld_y, head_y))
    return fail(AGRL_E_SHAPE, fn, "the heads of y overlap");
  if (!(base > 0.0) || !isfinite(base)) return fail(AGRL_E_FLAGS, fn, "base must be finite and > 0");
  if ((interleaved != 0 && interleaved != 1) || (inverse != 0 && inverse != 1))
    return fail(AGRL_E_FLAGS, fn, "interleaved and inverse must be 0 or 1");
  if (T == 0 || n_head == 0) return AGRL_OK;
  if (!x || !y) return fail(AGRL_E_NULL, fn, "x or y is NULL");
  const bool same = x == y;
  if (same && ((T > 1 && ld_x != ld_y) || (n_head > 1 && head_x != head_y)))
    return fail(AGRL_E_SHAPE, fn, "y is x with other strides");
  if (same && rot == 0) return AGRL_OK;
  // whole groups of 8 elements, or element by element
  const bool vec = d % 8 == 0 && rot % (interleaved ? 8 : 16) == 0;
  RotateArgs a = {T, n_head, d, rot, 0, 0, 0, x, ld_x, head_x, position, log2(base),
                  inverse ? -1.0f : 1.0f, y, ld_y, head_y, !same};
  const int pairs = vec ? (interleaved ? 4 : 8) : 1;
  a.units = rot / 2 / pairs + (d - rot) / (vec ? 8 : 1);
  const int threads = a.units <= 256 ? 256 : 512, fit = threads / a.units;
  a.hgroup = n_head < fit ? n_head : fit;
  a.tgroup = fit / a.hgroup;
  const int64_t need = cdiv(T, (int64_t)a.tgroup), most = (int64_t)device_cu_count() * 8;
  const dim3 grid((unsigned)(need < most ? need : most)), block(threads);
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto z) {
    using X = decltype(z);
    if (vec && interleaved)
      hipLaunchKernelGGL((rotate_kernel<X, 8, true>), grid, block, 0, s, a);
    else if (vec)
      hipLaunchKernelGGL((rotate_kernel<X, 8, false>), grid, block, 0, s, a);
    else if (interleaved)
      hipLaunchKernelGGL((rotate_kernel<X, 1, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((rotate_kernel<X, 1, false>), grid, block, 0, s, a);
  };
  if (dtype == AGRL_BF16)
    go(uint16_t{});
  else
    go(float{});
  return hip_status(hipGetLastError());
}
