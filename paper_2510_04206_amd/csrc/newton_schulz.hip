// Newton-Schulz orthogonalisation of matrices and the optimiser step around it (gfx950).
//
//   X = G / (|G|_F + eps);  `steps` times: A = X X^T, B = b A + c A A, X = a X + B X
//
// on the side with fewer rows (r = min(m, n) rows of k = max(m, n); G^T for m > n).
#include <math.h>
#include <stdio.h>

#include "../../include/agrl.h"
#include "common.hpp"
#include "gemm.hpp"

namespace agrl {
namespace {

int fail(int code, const char* fn, const char* what) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s: %s", fn, what);
  set_last_error(buf);
  return code;
}

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// What the matrix cores multiply is fp16 (11 bits), scaled by S so that entries far below the
// largest keep their bits: |X|, |A|, |B| stay below about 4 for coefficients that keep the
// singular values bounded, and fp16 reaches 65504 = 16 S.
//
// The iterate X is held in two fp16 numbers, hi + lo (22 bits and the scale's range, the state
// that the term a X carries on), whose hi is the operand.  For a bf16 result the products take
// hi alone: the rounding of the operands to 11 bits leaves 2e-4 to 1.6e-3 relative in the result
// (the more, the flatter the singular values), which the result's own rounding (1.7e-3) covers.
// For an fp32 result every operand is hi + lo and a product is three (hi hi + hi lo + lo hi),
// which is as exact as fp32 products.
constexpr float S = 4096.0f;

struct HiLo {
  _Float16 hi, lo;
};
__device__ __forceinline__ HiLo split(float v) {
  const _Float16 h = (_Float16)v;
  return HiLo{h, (_Float16)(v - (float)h)};
}

// One stack of matrices in the workspace: plane p (0 hi, 1 lo), matrix z.
struct Planes {
  _Float16* at;
  int64_t plane, matrix;   // elements
  __host__ __device__ _Float16* get(int p, int64_t z) const { return at + p * plane + z * matrix; }
};

enum { GRAM, SQUARE, UPDATE };   // A = X X^T; B = bA + cAA + shift I; X = aX + BX

// What the last product writes: O, or the weight it updates.
struct Result {
  void* out;
  int64_t ld, matrix;
  int32_t f32, rows, cols, tall;   // rows x cols of the result; tall: X is its transpose
  int32_t step;                    // 1: out = keep * out - rate * O
  float keep, rate;
};

struct Args {
  Planes P, Q;        // P: rows of the tile (UPDATE: X, read transposed); Q: columns
  int64_t ldp, ldq;
  int32_t K, tiles_m, tiles_n;
  Planes C;           // A, B or the next X
  int64_t ldc;
  float alpha, beta, shift;   // UPDATE: beta X + P Q; SQUARE: beta A + alpha P Q + shift I
  int32_t last;
  Result res;
};

// A tile of BM x BN by WM x WN waves, each BI x BJ blocks of 16 x 16; NST stages of 64 k in LDS
template <int WM_, int WN_, int BI_, int BJ_, int NST_>
struct Tile {
  static constexpr int WM = WM_, WN = WN_, BI = BI_, BJ = BJ_, NST = NST_;
  static constexpr int BM = WM * BI * 16, BN = WN * BJ * 16, WAVES = WM * WN;
  static constexpr int SK = 64, ROW = 2 * SK;
  static constexpr int P_BYTES = BM * ROW, STAGE = (BM + BN) * ROW;
  static constexpr int CP = BM / 8 / WAVES, CQ = BN / 8 / WAVES;   // 1 KiB copies per wave
};

template <int MODE, bool SPLIT, class T>
__global__ void __launch_bounds__(64 * T::WAVES) ns_product_kernel(Args a) {
  constexpr int BM = T::BM, BN = T::BN, BI = T::BI, BJ = T::BJ, ROW = T::ROW, NST = T::NST;
  constexpr int CP = T::CP, CQ = T::CQ;
  constexpr bool TR = MODE == UPDATE;
  constexpr int TROW = BM * 2;                   // bytes of a k-row of a transposed stage
  constexpr int LPR = TROW / 16;                 // lanes of a copy per k-row
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NST * T::STAGE];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int64_t z = blockIdx.y;
  int tm, tn;
  if constexpr (TR) {
    tm = blockIdx.x % a.tiles_m;
    tn = blockIdx.x / a.tiles_m;
  } else {
    // lower triangle, row by row: tile t is (tm, tn <= tm)
    const int t = blockIdx.x;
    tm = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
    while (tm * (tm + 1) / 2 > t) --tm;
    tn = t - tm * (tm + 1) / 2;
  }
  const int m0 = tm * BM, n0 = tn * BN;

  uint32_t offp[CP], offq[CQ];
  // row-major: 8 rows of 128 bytes per copy, chunk c of row r at c ^ ((r >> 1) & 7)
#pragma unroll
  for (int q = 0; q < CQ; ++q) {
    const int row = (wave * CQ + q) * 8 + (lane >> 3);
    offq[q] = (uint32_t)(row * (a.ldq * 2)) + (((lane & 7) ^ row_swizzle(row)) << 4);
  }
#pragma unroll
  for (int q = 0; q < CP; ++q) {
    if constexpr (TR) {
      // k-rows of BM entries: 64-byte window w of k-row k at w ^ swz(k), its 32-byte halves
      // swapped when bit 3 of k is set (see the reads below)
      const int kr = (wave * CP + q) * (64 / LPR) + lane / LPR, p = lane % LPR;
      const int w = (p >> 2) ^ (BM >= 128 ? kr & 3 : (kr >> 1) & 1);
      const int col = w * 32 + ((((p >> 1) & 1) ^ ((kr >> 3) & 1)) << 4) + (p & 1) * 8;
      offp[q] = (uint32_t)(kr * (a.ldp * 2) + col * 2);
    } else {
      const int row = (wave * CP + q) * 8 + (lane >> 3);
      offp[q] = (uint32_t)(row * (a.ldp * 2)) + (((lane & 7) ^ row_swizzle(row)) << 4);
    }
  }
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)smem);
  const int nk = a.K / T::SK, total = SPLIT ? 3 * nk : nk;
  const int64_t p_first = TR ? (int64_t)m0 : m0 * a.ldp, p_step = TR ? T::SK * a.ldp : T::SK;
  auto copy_stage = [&](int s) {
    const int buf = s % NST;
    int kk = min(s, total - 1), pp = 0, pq = 0;
    if constexpr (SPLIT) {
      const int seg = kk / nk;       // hi lo, lo hi, then hi hi: the small terms first
      kk -= seg * nk;
      pp = seg == 1, pq = seg == 0;
    }
    const _Float16* p = a.P.get(pp, z) + p_first + kk * p_step;
    const _Float16* q = a.Q.get(pq, z) + n0 * a.ldq + kk * T::SK;
    const uint32_t lp = lds0 + buf * T::STAGE + wave * CP * 1024;
    const uint32_t lq = lds0 + buf * T::STAGE + T::P_BYTES + wave * CQ * 1024;
    static_for<CP>([&](auto c) { bf16k::copy16<c.value * 1024>(p, offp[c.value], lp); });
    static_for<CQ>([&](auto c) { bf16k::copy16<c.value * 1024>(q, offq[c.value], lq); });
  };

  f32x4 acc[BI][BJ];
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int fr = lane & 15, g = lane >> 4;
  int rp[2], rq[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    const int chk = ((kk * 4 + g) ^ row_swizzle(fr)) << 4;
    rp[kk] = (wm * BI * 16 + fr) * ROW + chk;
    rq[kk] = T::P_BYTES + (wn * BJ * 16 + fr) * ROW + chk;
  }
  // transposing reads: in 16-lane group g, lane s supplies k-row 8 g + (s >> 2) (+ 4 in the
  // second read) and rows 4 (s & 3) .. + 3 of the block; it receives row s of those k-rows
  const int q4 = (lane >> 2) & 3;
  const int tswz = BM >= 128 ? q4 : q4 >> 1;     // (the same for k-row + 4, + 8, + 32)
  const int tp = (8 * g + q4) * TROW + 8 * (lane & 3);

#pragma unroll
  for (int s = 0; s < NST - 1; ++s) copy_stage(s);
  for (int s = 0; s < total; ++s) {
    // this wave's copies of stage s have landed, then every wave's; and every wave has read
    // the buffer that the next copies refill (stages past the last copy it again)
    bf16k::wait_vmcnt<(NST - 2) * (CP + CQ)>();
    lds_barrier();
    copy_stage(s + NST - 1);
    const uint8_t* st = smem + (s % NST) * T::STAGE;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      f16x8 fp[BI], fq[BJ];
#pragma unroll
      for (int i = 0; i < BI; ++i) {
        if constexpr (TR) {
          const int b = wm * BI + i;             // block of 16 rows: window b / 2, half b & 1
          const uint8_t* at = st + tp + kk * 32 * TROW + (((b >> 1) ^ tswz) << 6) +
                              (((b & 1) ^ (g & 1)) << 5);
          bf16x8 v;
          v.lo = bf16k::read_tr(at);
          v.hi = bf16k::read_tr(at + 4 * TROW);
          fp[i] = __builtin_bit_cast(f16x8, v);
        } else {
          fp[i] = *(const f16x8*)(st + rp[kk] + i * 16 * ROW);
        }
      }
#pragma unroll
      for (int j = 0; j < BJ; ++j) fq[j] = *(const f16x8*)(st + rq[kk] + j * 16 * ROW);
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int j = 0; j < BJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[i], fq[j], acc[i][j], 0, 0, 0);
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");

  // block (i, j) of a lane: column c = 16 j + (lane & 15), rows r .. r + 3, r = 16 i + 4 g
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j) {
      const int64_t r = m0 + (wm * BI + i) * 16 + 4 * g, c = n0 + (wn * BJ + j) * 16 + fr;
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q] * (1.0f / S);
      if constexpr (MODE == SQUARE) {
        const f16x4 h = *(const f16x4*)(a.P.get(0, z) + c * a.ldp + r);
        f16x4 l = {0, 0, 0, 0};
        if constexpr (SPLIT) l = *(const f16x4*)(a.P.get(1, z) + c * a.ldp + r);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[q] = fmaf(a.alpha, v[q], a.beta * ((float)h[q] + (float)l[q]));
          if (r + q == c) v[q] += a.shift * S;
        }
      }
      if constexpr (MODE == UPDATE) {
        const f16x4 h = *(const f16x4*)(a.P.get(0, z) + c * a.ldp + r);
        const f16x4 l = *(const f16x4*)(a.P.get(1, z) + c * a.ldp + r);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = fmaf(a.beta, (float)h[q] + (float)l[q], v[q]);
        if (a.last) {
          const Result& o = a.res;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int64_t row = o.tall ? r + q : c, col = o.tall ? c : r + q;
            if (row < o.rows && col < o.cols) {
              const int64_t at = z * o.matrix + row * o.ld + col;
              float w = v[q] * (1.0f / S);
              if (o.f32) {
                float* p = (float*)o.out + at;
                *p = o.step ? fmaf(o.keep, *p, -o.rate * w) : w;
              } else {
                uint16_t* p = (uint16_t*)o.out + at;
                if (o.step) w = fmaf(o.keep, bf16_bits_to_f32(*p), -o.rate * w);
                *p = f32_to_bf16_bits(w);
              }
            }
          }
          continue;
        }
      }
      f16x4 h, l;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const HiLo s = split(v[q]);
        h[q] = s.hi, l[q] = s.lo;
      }
      constexpr bool LO = SPLIT || MODE == UPDATE;
      *(f16x4*)(a.C.get(0, z) + c * a.ldc + r) = h;
      if constexpr (LO) *(f16x4*)(a.C.get(1, z) + c * a.ldc + r) = l;
      if constexpr (MODE != UPDATE) {
        if (tm != tn) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            a.C.get(0, z)[(r + q) * a.ldc + c] = h[q];
            if constexpr (LO) a.C.get(1, z)[(r + q) * a.ldc + c] = l[q];
          }
        }
      }
    }
}

// ---------------------------------------------------------------------------
// Before the products: u = G, or the momentum's update M <- mu M + g and u = g + mu M (or M);
// the sum of u^2 in 64 bits, one partial sum per workgroup; then X = u / (|u| + eps) in hi + lo.
struct Source {
  const void* g;
  int64_t ld, matrix;
  int32_t f32, rows, cols;
  float* m;              // momentum [rows, cols] contiguous per matrix, or nullptr
  float mu;
  int32_t nesterov;
};
constexpr int NORM_GROUPS = 256;   // workgroups of a matrix's sum of squares, at most
constexpr int PRE = 256;

__device__ __forceinline__ float grad_at(const Source& s, int64_t z, int64_t i, int64_t j) {
  const int64_t at = z * s.matrix + i * s.ld + j;
  return s.f32 ? ((const float*)s.g)[at] : bf16_bits_to_f32(((const uint16_t*)s.g)[at]);
}

__global__ void __launch_bounds__(PRE) ns_norm_kernel(Source s, double* part) {
  const int64_t z = blockIdx.y, n = (int64_t)s.rows * s.cols;
  double sum = 0.0;
  for (int64_t e = (int64_t)blockIdx.x * PRE + threadIdx.x; e < n; e += (int64_t)gridDim.x * PRE) {
    const int64_t i = e / s.cols, j = e - i * s.cols;
    float u = grad_at(s, z, i, j);
    if (s.m) {
      float* m = s.m + z * n + e;
      const float v = fmaf(s.mu, *m, u);
      *m = v;
      u = s.nesterov ? fmaf(s.mu, v, u) : v;
    }
    sum += (double)u * (double)u;
  }
  __shared__ double red[PRE];
  red[threadIdx.x] = sum;
  __syncthreads();
#pragma unroll
  for (int o = PRE / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[z * gridDim.x + blockIdx.x] = red[0];
}

// X [r_pad, k_pad], 64 x 64 tiles (transposed through LDS where the matrix is tall)
__global__ void __launch_bounds__(PRE)
    ns_start_kernel(Source s, const double* part, int n_part, float eps, int tall, Planes X,
                    int64_t ldx) {
  __shared__ double red[PRE];
  __shared__ float tile[64][65];
  const int64_t z = blockIdx.z;
  const int t = threadIdx.x;
  red[t] = t < n_part ? part[z * n_part + t] : 0.0;
  __syncthreads();
#pragma unroll
  for (int o = PRE / 2; o > 0; o >>= 1) {
    if (t < o) red[t] += red[t + o];
    __syncthreads();
  }
  const float inv = (float)((double)S / (sqrt(red[0]) + (double)eps));
  const int64_t i0 = (int64_t)(tall ? blockIdx.x : blockIdx.y) * 64;   // in the matrix
  const int64_t j0 = (int64_t)(tall ? blockIdx.y : blockIdx.x) * 64;
  const int tx = t & 63, ty = t >> 6;
  for (int y = ty; y < 64; y += 4) {
    const int64_t i = i0 + y, j = j0 + tx;
    float u = 0.0f;
    if (i < s.rows && j < s.cols) {
      u = grad_at(s, z, i, j);
      if (s.m) {
        const float v = s.m[z * s.rows * s.cols + i * s.cols + j];
        u = s.nesterov ? fmaf(s.mu, v, u) : v;
      }
    }
    tile[y][tx] = u * inv;
  }
  __syncthreads();
  const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;   // in X
  for (int y = ty; y < 64; y += 4) {
    const HiLo v = split(tall ? tile[tx][y] : tile[y][tx]);
    const int64_t at = (r0 + y) * ldx + c0 + tx;
    X.get(0, z)[at] = v.hi;
    X.get(1, z)[at] = v.lo;
  }
}

// ---------------------------------------------------------------------------
constexpr int64_t MAX_SIDE = (int64_t)1 << 20, MAX_SHORT = (int64_t)1 << 16, MAX_BATCH = 65535;

// Sizes and the workspace of a stack of matrices
struct Plan {
  int64_t batch;
  int32_t r, k, tall, tile;
  int64_t r_pad, k_pad;
  int32_t split, n_part;
  int64_t x_plane, a_plane;                 // elements
  size_t part, x[2], a, b, total;           // bytes
};

bool make_plan(int64_t batch, int64_t m, int64_t n, int32_t out_dtype, Plan* p) {
  if (batch <= 0 || batch > MAX_BATCH || m <= 0 || n <= 0 || m > MAX_SIDE || n > MAX_SIDE)
    return false;
  const int64_t r = m < n ? m : n, k = m < n ? n : m;
  if (r > MAX_SHORT) return false;
  p->batch = batch, p->r = (int32_t)r, p->k = (int32_t)k, p->tall = m > n;
  auto tiles = [&](int64_t t) { return batch * cdiv(r, t) * cdiv(k, t); };
  p->tile = tiles(256) >= 192 ? 256 : tiles(128) >= 128 ? 128 : 64;
  p->r_pad = cdiv(r, (int64_t)p->tile) * p->tile;
  p->k_pad = cdiv(k, (int64_t)p->tile) * p->tile;
  p->split = out_dtype == AGRL_F32;
  const int64_t per = cdiv(m * n, (int64_t)PRE * 8);
  p->n_part = (int32_t)(per < NORM_GROUPS ? per : NORM_GROUPS);
  p->x_plane = batch * p->r_pad * p->k_pad;
  p->a_plane = batch * p->r_pad * p->r_pad;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p->part = take((size_t)batch * p->n_part * sizeof(double));
  for (int i = 0; i < 2; ++i) p->x[i] = take((size_t)p->x_plane * 4);
  const size_t a_bytes = (size_t)p->a_plane * (p->split ? 4 : 2);
  p->a = take(a_bytes);
  p->b = take(a_bytes);
  p->total = at;
  return true;
}

template <int MODE, class T>
void launch(const Plan& p, Args a, hipStream_t s) {
  a.tiles_m = (int32_t)((MODE == UPDATE ? p.k_pad : p.r_pad) / T::BM);
  a.tiles_n = (int32_t)(p.r_pad / T::BN);
  const int64_t tiles = MODE == UPDATE ? (int64_t)a.tiles_m * a.tiles_n
                                       : (int64_t)a.tiles_n * (a.tiles_n + 1) / 2;
  const dim3 grid((unsigned)tiles, (unsigned)p.batch), block(64 * T::WAVES);
  if (p.split)
    hipLaunchKernelGGL((ns_product_kernel<MODE, true, T>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((ns_product_kernel<MODE, false, T>), grid, block, 0, s, a);
}

struct Steps {
  int32_t n;
  float a, b, c, eps;
};

template <class T>
void run(const Plan& p, const Steps& o, const Source& src, const Result& res, uint8_t* ws,
         hipStream_t s) {
  double* part = (double*)(ws + p.part);
  hipLaunchKernelGGL(ns_norm_kernel, dim3(p.n_part, (unsigned)p.batch), dim3(PRE), 0, s, src, part);
  Planes X[2], A, B;
  for (int i = 0; i < 2; ++i)
    X[i] = Planes{(_Float16*)(ws + p.x[i]), p.x_plane, p.r_pad * p.k_pad};
  A = Planes{(_Float16*)(ws + p.a), p.a_plane, p.r_pad * p.r_pad};
  B = Planes{(_Float16*)(ws + p.b), p.a_plane, p.r_pad * p.r_pad};
  hipLaunchKernelGGL(ns_start_kernel,
                     dim3((unsigned)(p.k_pad / 64), (unsigned)(p.r_pad / 64), (unsigned)p.batch),
                     dim3(PRE), 0, s, src, part, p.n_part, o.eps, p.tall, X[0], p.k_pad);
  for (int i = 0; i < o.n; ++i) {
    Args a = {};
    a.P = a.Q = X[i & 1], a.ldp = a.ldq = p.k_pad, a.K = (int32_t)p.k_pad;
    a.C = A, a.ldc = p.r_pad;
    launch<GRAM, T>(p, a, s);
    const float sigma = p.split || i < o.n - 2 ? 0.0f : -(o.b + o.c) * (i == o.n - 1 ? 1.0f : 0.5f);
    a.P = a.Q = A, a.ldp = a.ldq = p.r_pad, a.K = (int32_t)p.r_pad;
    a.C = B, a.alpha = o.c, a.beta = o.b, a.shift = sigma;
    launch<SQUARE, T>(p, a, s);
    a.P = X[i & 1], a.ldp = p.k_pad, a.Q = B;
    a.C = X[(i + 1) & 1], a.ldc = p.k_pad, a.beta = o.a - sigma;
    a.last = i == o.n - 1, a.res = res;
    launch<UPDATE, T>(p, a, s);
  }
}

using Tile64 = Tile<2, 2, 2, 2, 4>;
using Tile128 = Tile<2, 2, 4, 4, 2>;
using Tile256 = Tile<2, 4, 8, 4, 2>;

int start(const char* fn, const Plan& p, const agrl_ns_options* opt, const Source& src,
          const Result& res, void* ws, size_t ws_bytes, hipStream_t s) {
  Steps o = {5, 3.4445f, -4.7750f, 2.0315f, 1e-7f};
  if (opt) {
    if (opt->steps < 0 || opt->steps > 100) return fail(AGRL_E_FLAGS, fn, "steps must be in [0, 100]");
    if (!isfinite(opt->a) || !isfinite(opt->b) || !isfinite(opt->c))
      return fail(AGRL_E_FLAGS, fn, "coefficients must be finite");
    if (!(opt->eps >= 0.0f) || !isfinite(opt->eps))
      return fail(AGRL_E_FLAGS, fn, "eps must be finite and >= 0");
    if (opt->steps) o.n = opt->steps;
    if (opt->a != 0.0f || opt->b != 0.0f || opt->c != 0.0f) o.a = opt->a, o.b = opt->b, o.c = opt->c;
    if (opt->eps != 0.0f) o.eps = opt->eps;
  }
  if (!ws || ws_bytes < p.total) return fail(AGRL_E_WORKSPACE, fn, "workspace missing or too small");
  if ((uintptr_t)ws % 256 != 0) return fail(AGRL_E_UNSUPPORTED, fn, "workspace must be 256-byte aligned");
  if (p.tile == 256)
    run<Tile256>(p, o, src, res, (uint8_t*)ws, s);
  else if (p.tile == 128)
    run<Tile128>(p, o, src, res, (uint8_t*)ws, s);
  else
    run<Tile64>(p, o, src, res, (uint8_t*)ws, s);
  return hip_status(hipGetLastError());
}

int check(const char* fn, int64_t batch, int64_t m, int64_t n, int32_t in_dtype, int64_t ld_in,
          int64_t stride_in, int32_t out_dtype, int64_t ld_out, int64_t stride_out, Plan* p) {
  if ((in_dtype != AGRL_BF16 && in_dtype != AGRL_F32) ||
      (out_dtype != AGRL_BF16 && out_dtype != AGRL_F32))
    return fail(AGRL_E_DTYPE, fn, "dtype must be AGRL_BF16 or AGRL_F32");
  if (batch < 0 || m < 0 || n < 0) return fail(AGRL_E_SHAPE, fn, "negative size");
  if (ld_in < n || ld_out < n) return fail(AGRL_E_SHAPE, fn, "a row stride is smaller than n");
  if (batch > 1 && (stride_in < 0 || stride_out < m * ld_out))
    return fail(AGRL_E_SHAPE, fn, "a matrix stride is too small");
  if (batch == 0 || m == 0 || n == 0) return AGRL_OK;
  if (!make_plan(batch, m, n, out_dtype, p)) return fail(AGRL_E_SHAPE, fn, "sizes too large");
  return AGRL_OK;
}

}  // namespace
}  // namespace agrl

extern "C" size_t agrl_orthogonalize_workspace_size(int64_t batch, int64_t m, int64_t n,
                                                    int32_t out_dtype) {
  agrl::Plan p;
  if (out_dtype != AGRL_BF16 && out_dtype != AGRL_F32) return 0;
  return agrl::make_plan(batch, m, n, out_dtype, &p) ? p.total : 0;
}

extern "C" int agrl_orthogonalize(int64_t batch, int64_t m, int64_t n, int32_t dtype,
                                  const void* G, int64_t ld_g, int64_t stride_g,
                                  int32_t out_dtype, const agrl_ns_options* ns, void* workspace,
                                  size_t ws_bytes, void* O, int64_t ld_o, int64_t stride_o,
                                  void* stream) {
  using namespace agrl;
  const char* fn = "agrl_orthogonalize";
  Plan p;
  int rc = check(fn, batch, m, n, dtype, ld_g, stride_g, out_dtype, ld_o, stride_o, &p);
  if (rc) return rc;
  if (batch == 0 || m == 0 || n == 0) return AGRL_OK;
  if (!G || !O) return fail(AGRL_E_NULL, fn, "G or O is NULL");
  const Source src = {G, ld_g, stride_g, dtype == AGRL_F32, (int32_t)m, (int32_t)n, nullptr, 0.0f, 0};
  const Result res = {O, ld_o, stride_o, out_dtype == AGRL_F32, (int32_t)m, (int32_t)n, p.tall,
                      0, 0.0f, 0.0f};
  return start(fn, p, ns, src, res, workspace, ws_bytes, (hipStream_t)stream);
}

extern "C" int agrl_muon_step(int64_t batch, int64_t m, int64_t n, int32_t grad_dtype,
                              const void* grad, int64_t ld_grad, int64_t stride_grad,
                              int32_t param_dtype, void* param, int64_t ld_param,
                              int64_t stride_param, float* momentum, float lr, float mu,
                              int32_t nesterov, float weight_decay, float scale,
                              const agrl_ns_options* ns, void* workspace, size_t ws_bytes,
                              void* stream) {
  using namespace agrl;
  const char* fn = "agrl_muon_step";
  Plan p;
  int rc = check(fn, batch, m, n, grad_dtype, ld_grad, stride_grad, param_dtype, ld_param,
                 stride_param, &p);
  if (rc) return rc;
  if (!isfinite(lr) || !isfinite(mu) || !isfinite(weight_decay) || !isfinite(scale) || scale < 0.0f)
    return fail(AGRL_E_FLAGS, fn, "lr, mu, weight_decay and scale must be finite, scale >= 0");
  if (nesterov != 0 && nesterov != 1) return fail(AGRL_E_FLAGS, fn, "nesterov must be 0 or 1");
  if (batch == 0 || m == 0 || n == 0) return AGRL_OK;
  if (!grad || !param || !momentum) return fail(AGRL_E_NULL, fn, "grad, param or momentum is NULL");
  if (scale == 0.0f) scale = m > n ? sqrtf((float)m / (float)n) : 1.0f;
  const Source src = {grad, ld_grad, stride_grad, grad_dtype == AGRL_F32, (int32_t)m, (int32_t)n,
                      momentum, mu, nesterov};
  const Result res = {param, ld_param, stride_param, param_dtype == AGRL_F32, (int32_t)m, (int32_t)n,
                      p.tall, 1, (float)(1.0 - (double)lr * weight_decay), lr * scale};
  return start(fn, p, ns, src, res, workspace, ws_bytes, (hipStream_t)stream);
}
