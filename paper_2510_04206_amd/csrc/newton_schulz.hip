// Newton-Schulz orthogonalisation of matrices and the optimiser step around it (gfx950).
//
//   X = G / (|G|_F + eps);  `steps` times: A = X X^T, B = b A + c A A, X = a X + B X
//
// on the side with fewer rows (r = min(m, n) rows of k = max(m, n); G^T for m > n).
//
// Matrix cores bound it.  A and A A are symmetric, so half of their tiles are formed and written
// twice: 3 r^2 k + r^3 operations a step instead of 4 r^2 k + 2 r^3.  One workgroup per tile,
// persistent, the K extent in stages of 128 bytes a row that the LDS copies keep in flight; which
// tile and how many stages is chosen per product by the time it is expected to take (choose_tiles).
// B X reads X transposed out of LDS, so X lies in memory once, and every product writes its result
// as the next one's operand.  A step is three launches; two before the first make |G| and X.
//
// Measured (MI355X, five steps): 5120 x 5120 fp32 -> bf16 2.5 ms, 1.07 PFLOP/s of the operations
// above (a 16384^3 library product in fp16 reaches 1.41), 8192 x 8192 8.6 ms, 1.28; 14336 x 3584 with
// momentum and a bf16 weight 3.0 ms, 1.00, with an fp32 weight 8.3 ms, 1.08 PFLOP/s of fp16 products;
// 8 x 1024 x 1024 fp32 -> fp32 0.75 ms, 0.69 of the same; 128 x 512 114 us and 256 x 256 fp32 124 us,
// of which 17 launches' own 4 us each are 60 and 55%.
// What is left: the last round of tiles is not full (B X of 5120 x 5120: 400 tiles of 256 x 256 for
// 256 units: matrix cores busy 0.47 of its time, 0.55 in 14336 x 3584's), at a tile's end all compute
// units move 512 KiB at once (20 of 140 us a tile there), and a 256 x 256 stage of 64 takes 1.4 us
// where the matrix cores alone would take 1.0 at the clock that the power limit leaves (1.9 to 2.1
// GHz).  In two parts, 8 x 1024 x 1024, they are busy 0.2 (A A) to 0.4 (B X) of the time; a wave waits a
// third of its cycles for memory or a barrier and another third to issue, without bank conflicts and
// with LDS 0.13 busy at most: which of the three dependent products of a block, the 64 additions
// beside each 48 and the last round's 32 tiles of 288 weighs most has not been measured.
#include <math.h>
#include <stdio.h>

#include "../../include/agrl.h"
#include "common.hpp"
#include "gemm.hpp"
#include "ns_plan.hpp"

namespace agrl {
namespace {

using namespace ns;

int fail(int code, const char* fn, const char* what) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s: %s", fn, what);
  set_last_error(buf);
  return code;
}

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// What the matrix cores multiply is fp16 (11 bits), scaled by S so that entries far below the
// largest keep their bits: |X|, |A|, |B| stay below about 4 for the default coefficients, and fp16
// reaches 65504 = 16 S.
//
// The iterate X is held in two fp16 numbers, hi + lo (22 bits and the scale's range, the state
// that the term a X carries on), whose hi is the operand.  For a bf16 result the products take
// hi alone.  Of the result's norm, the rounding of the operands to 11 bits leaves 2e-4 to 2e-3 where
// it averages over many unequal entries, as in gradients (the more, the flatter the singular
// values), as much as the result's own rounding (1.7e-3).  Where entries repeat it adds up: over
// 1 to 256 equal blocks of one value 5e-3 at the median, 2.6e-2 at most (emulated); the recursion of a
// singular value, with every rounding 2^-11 and of the worst sign, gives 6.2e-2 to first order.
// For an fp32 result every operand is hi + lo and a product is three (hi hi + hi lo + lo hi): 0.2 to
// 1.4 times what fp32 products are off by on noise, at most 9e-6 on the blocks, where those reach
// 1e-3.  Matrices of few rows take that way too: there the roundings average over few entries (33 x
// 65: 2.0e-3) and the time is latency.
constexpr float S = 4096.0f;

struct HiLo {
  _Float16 hi, lo;
};
// (v as it was rounded to fp32: merged into the conversion, a product or sum that forms v would be
// rounded once to hi and, for lo, twice, and the two would differ by a unit of hi now and then)
__device__ __forceinline__ HiLo split(float v) {
  asm("" : "+v"(v));
  const _Float16 h = (_Float16)v;
  return HiLo{h, (_Float16)(v - (float)h)};
}

// One stack of matrices in the workspace.  What is multiplied lies in memory as the matrix
// cores' stages take it, 128 bytes of a row at a time:
//   one part    64 columns of hi; lo, where it is kept (X), in a plane of its own
//   two parts   32 columns of hi, then the same 32 of lo
struct Planes {
  _Float16* at;
  int64_t matrix, lo;      // elements between matrices; from a hi to its lo's plane (one part)
  int64_t ld;              // columns (padded)
};
template <bool SPLIT>
__device__ __forceinline__ int64_t place(int64_t ld, int64_t row, int64_t col) {
  return SPLIT ? row * 2 * ld + ((col >> 5) << 6) + (col & 31) : row * ld + col;
}
template <bool SPLIT>
__device__ __forceinline__ int64_t lo_at(const Planes& p) {
  return SPLIT ? 32 : p.lo;
}

// A = X X^T; B = b A + c A A + shift I; X = beta X + B X, and the last of these
enum { GRAM, SQUARE, UPDATE, RESULT };

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
  int32_t K;
  // The stack's products are numbered in units of unit_m x unit_n (matrix by matrix, `units` each,
  // units_m down and units_n across); a launch takes `count` of them from `first` on, by tiles
  // that divide a unit.
  int32_t unit_m, unit_n, units_m, units_n, units, first, count;
  int32_t sub_m_log, sub_n_log, halves_log;      // tiles of a unit down and across; units of a square
  Planes C;           // A, B or the next X
  float alpha, beta, shift;   // UPDATE: beta X + P Q; SQUARE: beta A + alpha P Q + shift I
  int32_t keep_lo;            // UPDATE of one part: lo is read again
  Result res;         // RESULT: in place of C
};

// A tile of BM x BN by WM x WN waves, each BI x BJ blocks of 16 x 16; NST stages in LDS, each 128
// bytes of every row: 64 k, or 32 k in two parts.
template <int WM_, int WN_, int BI_, int BJ_, int NST_, int PER_CU_, bool EARLY_ = false>
struct Tile {
  static constexpr bool EARLY = EARLY_;          // the epilogue's inputs are read ahead of the products
  static constexpr int WM = WM_, WN = WN_, BI = BI_, BJ = BJ_, NST = NST_;
  static constexpr int PER_CU = PER_CU_;         // workgroups of a compute unit
  // waves of a SIMD: with two, a lane has 256 registers, which hold a tile of 128 x 128 without a
  // move between the two register files
  static constexpr int EU_WAVES = BI_ * BJ_ <= 4 || PER_CU_ > 1 ? 2 : 1;
  static constexpr int BM = WM * BI * 16, BN = WN * BJ * 16, WAVES = WM * WN;
  // a register set of fragments holds a stage, or, for the largest tile, half of one
  static constexpr bool HALVES = BI_ * BJ_ > 32;
  static constexpr int P_BYTES = BM * 128, STAGE = (BM + BN) * 128;
  static constexpr int CP = BM / 8 / WAVES, CQ = BN / 8 / WAVES;   // 1 KiB copies of a wave
};

// Tile t of the lower triangle (rows of tiles 0 .. n - 1, columns up to the row's own), in
// groups of 8 rows, column by column inside a group: tiles that follow each other share panels.
__device__ __forceinline__ void triangle_tile(int t, int n, int& tm, int& tn) {
  int g = 0;
  while (8 * (g + 1) < n && 32 * (g + 1) * (g + 1) + 4 * (g + 1) <= t) ++g;
  t -= 32 * g * g + 4 * g;
  const int h = min(8, n - 8 * g);
  if (t < 8 * g * h) {
    tm = 8 * g + t % h;
    tn = t / h;
  } else {
    t -= 8 * g * h;
    int c = 0;
    while (t >= h - c) t -= h - c, ++c;
    tm = 8 * g + c + t;
    tn = 8 * g + c;
  }
}

// Part 0 (hi) or 1 (lo) of four entries, two to a register.
__device__ __forceinline__ u32x2 packed(const f32x4& v, int part) {
  f16x4 f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const HiLo s = split(v[q]);
    f[q] = part ? s.lo : s.hi;
  }
  return __builtin_bit_cast(u32x2, f);
}

// Four lanes with rows 0..3 of a column each -> lane k with row k of the four columns.
template <int CTRL>
__device__ __forceinline__ uint32_t quad(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ u32x2 quad_transpose(u32x2 v, int lane) {
  const u32x2 o = {quad<0xb1>(v[0]), quad<0xb1>(v[1])};       // the other lane of the pair
  const uint32_t sel = lane & 1 ? 0x03020706u : 0x05040100u;  // (other's, own) odd or (own, other's) even
  const u32x2 w = {__builtin_amdgcn_perm(o[0], v[0], sel), __builtin_amdgcn_perm(o[1], v[1], sel)};
  const u32x2 t = {quad<0x4e>(w[0]), quad<0x4e>(w[1])};       // the other pair
  return lane & 2 ? u32x2{t[1], w[1]} : u32x2{w[0], t[0]};
}

// The same for 32-bit entries.
__device__ __forceinline__ f32x4 quad_transpose(const f32x4& v, int lane) {
  uint32_t w[4], o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = quad<0xb1>(__float_as_uint(v[q]));
#pragma unroll
  for (int h = 0; h < 2; ++h) {      // even lanes: entry 2 h of the pair's columns, odd: 2 h + 1
    w[2 * h] = lane & 1 ? o[2 * h + 1] : __float_as_uint(v[2 * h]);
    w[2 * h + 1] = lane & 1 ? __float_as_uint(v[2 * h + 1]) : o[2 * h];
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = quad<0x4e>(w[q]);
  const uint32_t x0 = lane & 2 ? o[2] : w[0], x1 = lane & 2 ? o[3] : w[1];
  const uint32_t x2 = lane & 2 ? w[2] : o[0], x3 = lane & 2 ? w[3] : o[1];
  return f32x4{__uint_as_float(x0), __uint_as_float(x1), __uint_as_float(x2), __uint_as_float(x3)};
}

// The last product's entries: rows r .. r + 3 (16 apart by block i) of column c (by block j) of
// X, which are four neighbours in a row of the result (behind a transpose of lane quads where X
// is the result's transpose).  A step reads its old values ahead of its stores, eight blocks' at a
// time; a one-part product's result is bf16.
// FULL: the whole tile lies in the result (no bounds, so no branches between the loads).
template <bool SPLIT, bool FULL, int BI, int BJ>
__device__ __forceinline__ void write_result(const Result& o, const f32x4 (&val)[BI][BJ], int z,
                                             int r0, int c0, int lane) {
  typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
  typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
  typedef std::conditional_t<SPLIT, f32x4, u32x2> Old;       // fp32, or four bf16
  constexpr int N = !FULL || BI * BJ < 8 ? BJ : 8;           // blocks at once
  const bool f32 = SPLIT && o.f32;
  float* const out32 = (float*)o.out + (int64_t)z * o.matrix;
  uint16_t* const out16 = (uint16_t*)o.out + (int64_t)z * o.matrix;
  // (r, c) and the steps of i and j in the result's rows and columns
  const int row0 = o.tall ? r0 + (lane & 3) : c0, col0 = o.tall ? c0 - (lane & 3) : r0;
  static_for<BI * BJ / N>([&](auto part_c) {
    constexpr int first = decltype(part_c)::value * N;
    auto each = [&](auto&& f) {
      static_for<N>([&](auto b_c) {
        constexpr int i = 16 * ((first + decltype(b_c)::value) / BJ);
        constexpr int j = 16 * ((first + decltype(b_c)::value) % BJ);
        const int row = row0 + (o.tall ? i : j), col = col0 + (o.tall ? j : i);
        const int there = FULL ? 4 : row < o.rows ? min(o.cols - col, 4) : 0;
        f(b_c, there, (int64_t)row * o.ld + col);
      });
    };
    Old old[N];
    if (o.step)
      each([&](auto b_c, int there, int64_t to) {
        Old& v = old[decltype(b_c)::value];
        u32x2 u = {0, 0};
        if (there >= 4) {
          if constexpr (SPLIT)
            if (f32) v = *(const f32x4_a4*)(out32 + to);
          if (!f32) u = *(const u32x2_a2*)(out16 + to);
        } else if constexpr (!FULL) {
#pragma unroll
          for (int q = 0; q < 3; ++q)
            if (q < there) {
              if constexpr (SPLIT)
                if (f32) v[q] = out32[to + q];
              if (!f32) u[q >> 1] |= (uint32_t)out16[to + q] << (16 * (q & 1));
            }
        }
        if constexpr (!SPLIT)
          v = u;
        else if (!f32)
          v[0] = __uint_as_float(u[0]), v[1] = __uint_as_float(u[1]);
      });
    f32x4 w[N];
#pragma unroll
    for (int b = 0; b < N; ++b) w[b] = val[(first + b) / BJ][(first + b) % BJ];
    if (o.tall)
#pragma unroll
      for (int b = 0; b < N; ++b) w[b] = quad_transpose(w[b], lane);
#pragma unroll
    for (int b = 0; b < N; ++b) {
      w[b] *= 1.0f / S;
      if (o.step) {
        f32x4 was;
        u32x2 u = {0, 0};
        if constexpr (SPLIT) {
          was = old[b];
          u = u32x2{__float_as_uint(old[b][0]), __float_as_uint(old[b][1])};
        } else {
          u = old[b];
        }
        if (!f32)
          was = f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u),
                      __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xffff0000u)};
#pragma unroll
        for (int q = 0; q < 4; ++q) w[b][q] = fmaf(o.keep, was[q], -o.rate * w[b][q]);
      }
    }
    each([&](auto b_c, int there, int64_t to) {
      const f32x4 v = w[decltype(b_c)::value];
      uint16_t h[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) h[q] = f32_to_bf16_bits(v[q]);
      if (there >= 4) {
        if (f32)
          *(f32x4_a4*)(out32 + to) = v;
        else
          *(u32x2_a2*)(out16 + to) =
              u32x2{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16};
      } else if constexpr (!FULL) {
#pragma unroll
        for (int q = 0; q < 3; ++q)
          if (q < there) {
            if (f32)
              out32[to + q] = v[q];
            else
              out16[to + q] = h[q];
          }
      }
    });
  });
}

// Fragment reads before slot q of a stage: spread over the first 7/8 of the slots, so that the
// last ones have come back when the stage ends.
constexpr int reads_before(int q, int reads, int slots) {
  return q * reads * 8 / (slots * 7) < reads ? q * reads * 8 / (slots * 7) : reads;
}

// C = P Q^T, a persistent grid over the tiles of a stack.  The loop keeps a stage's fragments in
// registers and, between its matrix instructions, reads the next stage's from LDS and starts the
// copies of the stage NST ahead, so one barrier a stage orders everything: behind it every wave
// has its fragments of this stage (whose buffer the new copies refill), and the next stage has
// landed.  Stages run on from a workgroup's tile to its next one (an even number of them per
// tile: the two register sets alternate), so a tile's first stages arrive under the last
// products and the epilogue of the tile before.
// (items item, item + stride, ... below end; smem: NST stages)
template <int MODE, bool SPLIT, class T>
__device__ __forceinline__ void product(const Args& a, int item, const int end, const int stride,
                                        uint8_t* const smem) {
  constexpr int BM = T::BM, BN = T::BN, BI = T::BI, BJ = T::BJ, NST = T::NST;
  constexpr int CP = T::CP, CQ = T::CQ, COPIES = CP + CQ;
  constexpr bool TR = MODE == UPDATE || MODE == RESULT;
  constexpr bool SMALL = BI * BJ <= 4;
  constexpr int KROWS = SPLIT ? 32 : 64;         // k of a stage
  constexpr int TROW = BM * 128 / KROWS;         // bytes of a k-row of a transposed stage
  constexpr int LPR = TROW / 16;                 // lanes of a copy per k-row
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int sub_log = a.sub_m_log + a.sub_n_log;
  struct At {
    int z, m0, n0;
    bool below;       // a tile below the diagonal squares of its symmetric product
  };
  auto tile_at = [&](int item) {
    const int unit = a.first + (item >> sub_log), sub = item & ((1 << sub_log) - 1);
    const int mat = unit < a.units ? 0 : unit / a.units, t = unit - mat * a.units;
    int um, un;
    if constexpr (TR) {
      grouped_tile(t, a.units_m, a.units_n, 8, um, un);
    } else {
      triangle_tile(t >> a.halves_log, a.units_m, um, un);
      un = (un << a.halves_log) + (t & ((1 << a.halves_log) - 1));
    }
    At at;
    at.z = __builtin_amdgcn_readfirstlane(mat);
    at.m0 = __builtin_amdgcn_readfirstlane(um * a.unit_m + (sub & ((1 << a.sub_m_log) - 1)) * BM);
    at.n0 = __builtin_amdgcn_readfirstlane(un * a.unit_n + (sub >> a.sub_m_log) * BN);
    at.below = __builtin_amdgcn_readfirstlane(un < um << a.halves_log);
    return at;
  };

  uint32_t offp[CP], offq[CQ];
  const uint32_t pitch_p = (uint32_t)(place<SPLIT>(a.P.ld, 1, 0) * 2);
  const uint32_t pitch_q = (uint32_t)(place<SPLIT>(a.Q.ld, 1, 0) * 2);
  // row-major: 8 rows of 128 bytes per copy, chunk c of row r at c ^ ((r >> 1) & 7)
#pragma unroll
  for (int q = 0; q < CQ; ++q) {
    const int row = (wave * CQ + q) * 8 + (lane >> 3);
    offq[q] = row * pitch_q + (((lane & 7) ^ row_swizzle(row)) << 4);
  }
#pragma unroll
  for (int q = 0; q < CP; ++q) {
    if constexpr (TR) {
      // k-rows of the tile's rows, 64-byte window w of k-row k at w ^ swz(k), its 32-byte halves
      // swapped when bit 3 of k is set: the 8 k-rows that half a wave reads (see below) then lie
      // in 8 distinct parts of the 256 bytes that LDS serves at once
      const int kr = (wave * CP + q) * (64 / LPR) + lane / LPR, p = lane % LPR;
      const int w = (p >> 2) ^ (TROW >= 256 ? kr & 3 : (kr >> 1) & 1);
      const int half = ((p >> 1) & 1) ^ ((kr >> 3) & 1);
      offp[q] = kr * pitch_p + w * 64 + half * 32 + (p & 1) * 16;
    } else {
      const int row = (wave * CP + q) * 8 + (lane >> 3);
      offp[q] = row * pitch_p + (((lane & 7) ^ row_swizzle(row)) << 4);
    }
  }
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)smem);
  const int total = a.K / KROWS;
  const int64_t p_step = TR ? (int64_t)KROWS * pitch_p : 128;
  // the next stage to copy: its operands, the stages left of its tile (0: none), that tile's item
  const uint8_t *p_at, *q_at;
  int left, copying = item;
  auto aim = [&](int it) {
    const At at = tile_at(it);
    p_at = (const uint8_t*)(a.P.at + at.z * a.P.matrix +
                            place<SPLIT>(a.P.ld, TR ? 0 : at.m0, TR ? at.m0 : 0));
    q_at = (const uint8_t*)(a.Q.at + at.z * a.Q.matrix + place<SPLIT>(a.Q.ld, at.n0, 0));
    left = total;
  };
  auto copy = [&](uint32_t buf, auto c_c) {
    constexpr int c = decltype(c_c)::value;
    if constexpr (c < CQ)
      bf16k::copy16<T::P_BYTES + c * 1024>(q_at, offq[c], buf + wave * CQ * 1024);
    else
      bf16k::copy16<(c - CQ) * 1024>(p_at, offp[c - CQ], buf + wave * CP * 1024);
  };
  // Behind the last tile's last stage a small tile copies nothing more (its launches are latency,
  // and of few stages); the others copy that stage again and read it for nothing, which keeps
  // branches out of their stages.
  auto advance = [&]() {
    if (--left > 0) {
      p_at += p_step;
      q_at += 128;
    } else if (copying + stride < end) {
      copying += stride;
      aim(copying);
    } else {
      left = SMALL ? 0 : 1;
    }
  };
  aim(item);

  // Two parts: a stage's three terms are summed by themselves and then added (rounded to
  // nearest) to the running sum: the matrix cores' own additions onto a large sum would lose
  // more than the operands do.
  f32x4 acc[BI][BJ], terms[SPLIT ? 3 : 1];
  const int fr = lane & 15, g = lane >> 4;
  int rp[2], rq[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    const int chk = ((kk * 4 + g) ^ row_swizzle(fr)) << 4;
    rp[kk] = (wm * BI * 16 + fr) * 128 + chk;
    rq[kk] = T::P_BYTES + (wn * BJ * 16 + fr) * 128 + chk;
  }
  // transposing reads: in 16-lane group g, lane s supplies k-row 8 g + (s >> 2) (+ 4 in the
  // second read) and rows 4 (s & 3) .. + 3 of the block; it receives row s of those k-rows
  const int q4 = (lane >> 2) & 3;
  const int tswz = ((TROW >= 256 ? q4 : q4 >> 1) << 6) | ((g & 1) << 5);
  int ta[TR ? BI : 1][TR && SPLIT ? 2 : 1];
  if constexpr (TR) {
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int part = 0; part < (SPLIT ? 2 : 1); ++part) {
        const int b = wm * BI + i;             // block of 16 rows: window b / 2, half b & 1
        const int win = SPLIT ? (b >> 1) * 2 + part : b >> 1;
        ta[i][part] = (8 * g + q4) * TROW + 8 * (lane & 3) + ((win << 6 | (b & 1) << 5) ^ tswz);
      }
  }

  // slice kk: the stage's k half, or its part
  constexpr int KK = T::HALVES ? 1 : 2;
  f16x8 fp[2][BI][KK], fq[2][BJ][KK];
  auto read_p = [&](const uint8_t* st, int i, int kk) {
    if constexpr (TR) {
      const uint8_t* at = st + ta[i][SPLIT ? kk : 0] + (SPLIT ? 0 : kk * 32 * TROW);
      bf16x8 v;
      v.lo = bf16k::read_tr(at);
      v.hi = bf16k::read_tr(at + 4 * TROW);
      return __builtin_bit_cast(f16x8, v);
    } else {
      return *(const f16x8*)(st + rp[kk] + i * 16 * 128);
    }
  };
  auto read_q = [&](const uint8_t* st, int j, int kk) {
    return *(const f16x8*)(st + rq[kk] + j * 16 * 128);
  };

  // half h of block b's sum (pinned where it stands: gathered behind the stage, the additions
  // would not hide under it)
  auto add = [&](auto b_c, auto h_c) {
    constexpr int b = decltype(b_c)::value, h = decltype(h_c)::value;
    f32x4& to = acc[b / BJ][b % BJ];
#pragma unroll
    for (int q = 2 * h; q < 2 * h + 2; ++q) {
      float v = to[q] + terms[b % 3][q];
      asm volatile("" : "+v"(v));
      to[q] = v;
    }
  };
  constexpr int READS = 2 * (BI + BJ), TERMS = SPLIT ? 3 : 2, SLOTS = BI * BJ * TERMS;
  int buf = 0;
  auto stage_with = [&](auto par_c, auto copies_c) {
    constexpr int P = decltype(par_c)::value;
    constexpr bool COPY = decltype(copies_c)::value;
    // the next stage has landed (vmcnt counts in order, and what else the wave has in flight is
    // younger or makes the wait longer, never shorter); once nothing is copied any more, all have
    bf16k::wait_vmcnt<COPY ? (NST - 2) * COPIES : 0>();
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
    const int next = buf + 1 == NST ? 0 : buf + 1;
    const uint8_t* st = smem + next * T::STAGE;
    const uint32_t into = lds0 + buf * T::STAGE;
    static_for<SLOTS>([&](auto q_c) {
      constexpr int q = decltype(q_c)::value;
      constexpr int term = q % TERMS, i = q / TERMS / BJ, j = q / TERMS % BJ;
      // two parts: hi lo, lo hi, hi hi; one part: the stage's two k halves
      constexpr int kp = SPLIT ? term == 1 : term, kq = SPLIT ? term == 0 : term;
      if constexpr (SPLIT) {
        // (a block's sum is added two blocks later: the matrix pipe has it by then)
        constexpr int b = q / TERMS;
        const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
        terms[b % 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
            fp[P][i][kp], fq[P][j][kq], term ? terms[b % 3] : zero, 0, 0, 0);
        if constexpr (term < 2 && b > 1)
          add(std::integral_constant<int, b - 2>{}, std::integral_constant<int, term>{});
      } else {
        acc[i][j] =
            __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[P][i][kp], fq[P][j][kq], acc[i][j], 0, 0, 0);
      }
      constexpr int r0 = reads_before(q, READS, SLOTS), r1 = reads_before(q + 1, READS, SLOTS);
      static_for<r1 - r0>([&](auto n_c) {
        constexpr int n = r0 + decltype(n_c)::value, kk = n / (BI + BJ), x = n % (BI + BJ);
        if constexpr (x < BJ)
          fq[P ^ 1][x][kk] = read_q(st, x, kk);
        else
          fp[P ^ 1][x - BJ][kk] = read_p(st, x - BJ, kk);
      });
      constexpr int c0 = q * COPIES / SLOTS, c1 = (q + 1) * COPIES / SLOTS;
      if constexpr (COPY)
        static_for<c1 - c0>([&](auto n_c) {
          copy(into, std::integral_constant<int, c0 + decltype(n_c)::value>{});
        });
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (SPLIT)
      static_for<2>([&](auto b) {
        constexpr int last = BI * BJ - 2 + decltype(b)::value;
        add(std::integral_constant<int, last>{}, std::integral_constant<int, 0>{});
        add(std::integral_constant<int, last>{}, std::integral_constant<int, 1>{});
      });
    if constexpr (COPY) advance();
    buf = next;
  };
  // The largest tile: set h holds the stage's k half h, and the next half is read under a half's
  // products.  The barrier stands between the halves.  The copies are spread over the second half:
  // all at its start, they took LDS from the reads (8192 x 8192: 427 us for A, so 400).  Its sums
  // fill the accumulation registers to the last, so the products are written with both sides tied
  // (left to the allocator, half of the sums moved to and fro between the register files); what
  // reads the sums behind the loop waits in pin().
  auto half_stage = [&](auto half_c) {
    constexpr int H = decltype(half_c)::value, PER = BI + BJ, N = BI * BJ;
    static_assert(!T::HALVES || 4 * COPIES == N, "a copy at every fourth product of half a stage");
    const int next = buf ^ 1;
    if constexpr (H == 1) {
      bf16k::wait_vmcnt<0>();
      lds_barrier();
      __builtin_amdgcn_sched_barrier(0);
    }
    const uint8_t* st = smem + (H == 1 ? next : buf) * T::STAGE;
    const uint32_t into = lds0 + buf * T::STAGE;
    static_for<N>([&](auto q_c) {
      constexpr int q = decltype(q_c)::value, i = q / BJ, j = q % BJ;
      asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0"
                   : "+a"(acc[i][j])
                   : "v"(fp[H][i][0]), "v"(fq[H][j][0]));
      constexpr int r0 = reads_before(q, PER, N), r1 = reads_before(q + 1, PER, N);
      static_for<r1 - r0>([&](auto n_c) {
        constexpr int x = r0 + decltype(n_c)::value;
        if constexpr (x < BJ)
          fq[H ^ 1][x][0] = read_q(st, x, H ^ 1);
        else
          fp[H ^ 1][x - BJ][0] = read_p(st, x - BJ, H ^ 1);
      });
      if constexpr (H == 1 && q % 4 == 3) copy(into, std::integral_constant<int, q / 4>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (H == 1) {
      advance();
      buf = next;
    }
  };
  auto stage = [&](auto par_c) {
    if constexpr (T::HALVES) {
      half_stage(std::integral_constant<int, 0>{});
      half_stage(std::integral_constant<int, 1>{});
    } else if (!SMALL || left > 0)
      stage_with(par_c, std::true_type{});
    else if constexpr (SMALL)
      stage_with(par_c, std::false_type{});
  };
  for (int s = 0; s < NST && left > 0; ++s) {
    static_for<COPIES>([&](auto c) { copy(lds0 + s * T::STAGE, c); });
    advance();
  }
  if (left > 0)
    bf16k::wait_vmcnt<(NST - 1) * COPIES>();
  else
    bf16k::wait_vmcnt<0>();
  lds_barrier();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
    for (int j = 0; j < BJ; ++j) fq[0][j][kk] = read_q(smem, j, kk);
#pragma unroll
    for (int i = 0; i < BI; ++i) fp[0][i][kk] = read_p(smem, i, kk);
  }
  for (; item < end; item += stride) {
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int j = 0; j < BJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // (the wide tile's sums live in the accumulation registers on both sides of the loop:
    // otherwise the allocator moves them to and fro inside it)
    auto pin = [&]() {
      // (a product written in assembly: no reader of its sum may follow within 18 cycles)
      if constexpr (T::HALVES) asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
      if constexpr (T::EU_WAVES == 1 && !SPLIT)
#pragma unroll
        for (int i = 0; i < BI; ++i)
#pragma unroll
          for (int j = 0; j < BJ; ++j) asm volatile("" : "+a"(acc[i][j]));
    };
    pin();
    const At at = tile_at(item);
    // block (i, j) of a lane: column c = 16 j + (lane & 15), rows r .. r + 3, r = 16 i + 4 g
    const int r0 = at.m0 + wm * BI * 16 + 4 * g, c0 = at.n0 + wn * BJ * 16 + fr;
    // What the epilogue adds to: a small tile reads it ahead of its products (a launch of few of
    // them is latency), a larger one half a tile at a time behind them, and the largest goes
    // through its epilogue by quarters, the next one's read ahead of the stores.
    constexpr bool OLD = MODE == SQUARE || MODE == UPDATE || (MODE == RESULT && SPLIT);
    constexpr bool LO = SPLIT || TR, OLD_LO = OLD && LO;
    constexpr int VAL_J = T::HALVES ? 1 : BJ;
    constexpr int OLD_J = T::EARLY ? BJ : T::HALVES ? VAL_J : BJ / 2, SETS = T::HALVES ? 2 : 1;
    f16x4 oh[SETS][OLD ? BI : 1][OLD_J], ol[SETS][OLD_LO ? BI : 1][OLD_J];
    auto read_old = [&](auto j_c) {
      constexpr int j0 = decltype(j_c)::value, set = j0 / OLD_J % SETS;
      const _Float16* const old = a.P.at + at.z * a.P.matrix;
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int j = 0; j < OLD_J; ++j) {
          const _Float16* p = old + place<SPLIT>(a.P.ld, c0 + 16 * (j0 + j), r0 + 16 * i);
          oh[set][i][j] = *(const f16x4*)p;
          if constexpr (OLD_LO) ol[set][i][j] = *(const f16x4*)(p + lo_at<SPLIT>(a.P));
        }
    };
    if constexpr (OLD && T::EARLY) read_old(std::integral_constant<int, 0>{});
    if constexpr (T::HALVES) asm volatile("s_nop 7" ::: "memory");
    for (int s = 0; s < total; s += 2) {
      stage(std::integral_constant<int, 0>{});
      stage(std::integral_constant<int, 1>{});
    }
    pin();
    if constexpr (OLD && T::HALVES) read_old(std::integral_constant<int, 0>{});
    static_for<BJ / VAL_J>([&](auto part_c) {
      constexpr int v0 = decltype(part_c)::value * VAL_J;
      const int cv = c0 + 16 * v0;
      f32x4 val[BI][VAL_J];
      if constexpr (OLD) {
        static_for<VAL_J / OLD_J>([&](auto half) {
          constexpr int h0 = decltype(half)::value * OLD_J, j0 = v0 + h0, set = j0 / OLD_J % SETS;
          if constexpr (!T::EARLY && !T::HALVES) read_old(std::integral_constant<int, j0>{});
#pragma unroll
          for (int i = 0; i < BI; ++i)
#pragma unroll
            for (int j = 0; j < OLD_J; ++j)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const float o = (float)oh[set][i][j][q] +
                                (OLD_LO ? (float)ol[set][OLD_LO ? i : 0][j][q] : 0.0f);
                float v = acc[i][j0 + j][q] * (1.0f / S);
                v = MODE == SQUARE ? fmaf(a.alpha, v, a.beta * o) : fmaf(a.beta, o, v);
                if (MODE == SQUARE && r0 + 16 * i + q == c0 + 16 * (j0 + j)) v += a.shift * S;
                val[i][h0 + j][q] = v;
              }
        });
        if constexpr (T::HALVES && v0 + VAL_J < BJ)
          read_old(std::integral_constant<int, v0 + VAL_J>{});
      } else {
#pragma unroll
        for (int i = 0; i < BI; ++i)
#pragma unroll
          for (int j = 0; j < VAL_J; ++j) val[i][j] = acc[i][v0 + j] * (1.0f / S);
      }
      if constexpr (MODE == RESULT) {
        const int end_m = a.res.tall ? a.res.rows : a.res.cols;
        const int end_n = a.res.tall ? a.res.cols : a.res.rows;
        if (at.m0 + BM <= end_m && at.n0 + BN <= end_n)
          write_result<SPLIT, true>(a.res, val, at.z, r0, cv, lane);
        else if (at.m0 < end_m && at.n0 < end_n)
          write_result<SPLIT, false>(a.res, val, at.z, r0, cv, lane);
      } else {
        _Float16* const out = a.C.at + at.z * a.C.matrix;
#pragma unroll
        for (int j = 0; j < VAL_J; ++j)
#pragma unroll
          for (int i = 0; i < BI; i += 2)
#pragma unroll
            for (int part = 0; part < (LO ? 2 : 1); ++part) {
              if (MODE == UPDATE && !SPLIT && part && !a.keep_lo) continue;
              const u32x2 x = packed(val[i][j], part), y = packed(val[i + 1][j], part);
              // blocks i and i + 1: after the swap a lane holds 8 consecutive rows of one of them,
              // and a store covers 64 consecutive bytes of 16 columns
              _Float16* p = out + part * lo_at<SPLIT>(a.C) +
                            place<SPLIT>(a.C.ld, cv + 16 * j,
                                         r0 - 4 * g + 16 * (i + (g & 1)) + 8 * (g >> 1));
              const auto s0 = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
              const auto s1 = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
              *(u32x4*)p = u32x4{s0[0], s1[0], s0[1], s1[1]};
            }
        if constexpr (!TR) {
          if (at.below) {                            // (a diagonal square is written whole)
#pragma unroll
            for (int i = 0; i < BI; ++i)
#pragma unroll
              for (int j = 0; j < VAL_J; ++j)
#pragma unroll
                for (int part = 0; part < (LO ? 2 : 1); ++part) {
                  _Float16* p =
                      out + part * lo_at<SPLIT>(a.C) +
                      place<SPLIT>(a.C.ld, r0 + 16 * i + (lane & 3), cv + 16 * j - (lane & 3));
                  *(u32x2*)p = quad_transpose(packed(val[i][j], part), lane);
                }
          }
        }
      }
    });
  }
  // no copy outlives the workgroup's LDS, and what was written can be read behind a barrier
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <int MODE, bool SPLIT, class T>
__global__ void __launch_bounds__(64 * T::WAVES)
    __attribute__((amdgpu_waves_per_eu(T::EU_WAVES, T::EU_WAVES))) ns_product_kernel(Args a) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::NST * T::STAGE];
  // workgroups go to the 8 XCDs in turn: each XCD takes a contiguous run of the tiles, its
  // workgroups neighbours in it, whose panels its L2 then holds
  const int items = a.count << (a.sub_m_log + a.sub_n_log);
  int item = blockIdx.x, end = item + 1, stride = 1;
  if (gridDim.x >= 8) {
    const int xcd = blockIdx.x & 7, share = items >> 3, extra = items & 7;
    item = xcd * share + min(xcd, extra) + (blockIdx.x >> 3);
    end = xcd * share + min(xcd, extra) + share + (xcd < extra ? 1 : 0);
    stride = (gridDim.x - xcd + 7) >> 3;         // workgroups on this XCD
  }
  if (item >= end) return;
  product<MODE, SPLIT, T>(a, item, end, stride, smem);
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
constexpr int PRE = 256;

typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// Eight neighbours in a row, `n` of them there (rows start at any element).
__device__ __forceinline__ void load8(const void* p, bool f32, int64_t at, int n, float (&v)[8]) {
  if (n >= 8 && f32) {
    const f32x4 a = *(const f32x4_any*)((const float*)p + at);
    const f32x4 b = *(const f32x4_any*)((const float*)p + at + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = a[k], v[k + 4] = b[k];
  } else if (n >= 8) {
    const u32x4 a = *(const u32x4_any*)((const uint16_t*)p + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(a[k] << 16);
      v[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = k >= n ? 0.0f
             : f32  ? ((const float*)p)[at + k]
                    : bf16_bits_to_f32(((const uint16_t*)p)[at + k]);
  }
}

// Sum over the workgroup in every thread of wave 0, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
  return v;
}

// What is orthogonalised, of a gradient g and the momentum m that has taken it in.
__device__ __forceinline__ float momentum_u(const Source& s, float m, float g) {
  return s.nesterov ? fmaf(s.mu, m, g) : m;
}

// Run j of 8 entries of row i of the matrix at `base`: the momentum takes it in, sum += u^2.
__device__ __forceinline__ void source_run(const Source& s, int64_t base, float* mom, int64_t i,
                                           int j, double (&sum)[2]) {
  const int n = s.cols - 8 * j;
  float u[8];
  load8(s.g, s.f32, base + i * s.ld + 8 * j, n, u);
  if (mom) {
    float* const p = mom + i * s.cols + 8 * j;
    float m[8];
    load8(p, true, 0, n, m);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = fmaf(s.mu, m[k], u[k]);
      u[k] = momentum_u(s, m[k], u[k]);
    }
    if (n >= 8) {
      *(f32x4_any*)p = f32x4{m[0], m[1], m[2], m[3]};
      *(f32x4_any*)(p + 4) = f32x4{m[4], m[5], m[6], m[7]};
    } else {
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (k < n) p[k] = m[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k & 1] = fma((double)u[k], (double)u[k], sum[k & 1]);
}

// S / (|u| + eps) as factor 2^exponent: in one fp32 number it would be infinite for a norm below
// 1.2e-35, which a zero matrix with a small eps has (and 0 times it NaN), and short of bits for one
// beyond 3e41.  The exponent is applied first: |u| 2^exponent is at most 1.
struct Scale {
  float factor;
  int exponent;
};
__device__ __forceinline__ Scale scale_of(double sum_of_squares, float eps) {
  int e;
  const double m = frexp(sqrt(sum_of_squares) + (double)eps, &e);
  return Scale{(float)((double)S / m), -e};
}

// Eight neighbours of a row of X, scaled.
template <bool SPLIT>
__device__ __forceinline__ void store_x(const Planes& X, int64_t z, int64_t row, int64_t col,
                                        const float (&v)[8], const Scale& by) {
  f16x8 hi, lo;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const HiLo x = split(ldexpf(v[k], by.exponent) * by.factor);
    hi[k] = x.hi, lo[k] = x.lo;
  }
  _Float16* p = X.at + z * X.matrix + place<SPLIT>(X.ld, row, col);
  *(f16x8*)p = hi;
  *(f16x8*)(p + lo_at<SPLIT>(X)) = lo;
}

// Runs of 8 entries, `runs` of them a row.
__global__ void __launch_bounds__(NORM_THREADS) ns_norm_kernel(Source s, double* part) {
  const int64_t z = blockIdx.y;
  const int runs = (s.cols + 7) / 8;
  const int64_t all = (int64_t)s.rows * runs, step = (int64_t)gridDim.x * NORM_THREADS;
  float* const mom = s.m ? s.m + z * s.rows * s.cols : nullptr;
  const int64_t step_i = step / runs;
  const int step_j = (int)(step - step_i * runs);
  int64_t e = (int64_t)blockIdx.x * NORM_THREADS + threadIdx.x;
  int64_t i = e / runs;
  int j = (int)(e - i * runs);
  double sum[2] = {0.0, 0.0};
  for (; e < all; e += step) {
    source_run(s, z * s.matrix, mom, i, j, sum);
    i += step_i;
    j += step_j;
    if (j >= runs) j -= runs, ++i;
  }
  __shared__ double red[NORM_THREADS / 64];
  const double total = block_sum<NORM_THREADS>(sum[0] + sum[1], red);
  if (threadIdx.x == 0) part[z * gridDim.x + blockIdx.x] = total;
}

// X [r_pad, k_pad] by tiles of 64 x 64, through LDS where the matrix is tall.
template <bool SPLIT>
__global__ void __launch_bounds__(PRE)
    ns_start_kernel(Source s, const double* part, int n_part, float eps, int tall, Planes X) {
  __shared__ double red[PRE / 64];
  __shared__ float tile[64][65];
  const int64_t z = blockIdx.z;
  const int t = threadIdx.x;
  const int64_t i0 = (int64_t)(tall ? blockIdx.x : blockIdx.y) * 64;   // in the matrix
  const int64_t j0 = (int64_t)(tall ? blockIdx.y : blockIdx.x) * 64;
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t i = i0 + (t >> 3) + 32 * h, j = j0 + (t & 7) * 8;
    const int n = i < s.rows ? (int)max((int64_t)0, min((int64_t)8, s.cols - j)) : 0;
    load8(s.g, s.f32, z * s.matrix + i * s.ld + j, n, v[h]);
    if (s.m) {
      float m[8];
      load8(s.m, true, z * s.rows * s.cols + i * s.cols + j, n, m);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[h][k] = momentum_u(s, m[k], v[h][k]);
    }
  }
  const double total = block_sum<PRE>(t < n_part ? part[z * n_part + t] : 0.0, red);
  const Scale by = scale_of(total, eps);
  if (tall) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < 8; ++k) tile[(t >> 3) + 32 * h][(t & 7) * 8 + k] = v[h][k];
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[h][k] = tile[(t & 7) * 8 + k][(t >> 3) + 32 * h];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    store_x<SPLIT>(X, z, (int64_t)blockIdx.y * 64 + (t >> 3) + 32 * h,
                   (int64_t)blockIdx.x * 64 + (t & 7) * 8, v[h], by);
}

struct Steps {
  int32_t n;
  float a, b, c, eps;
};

// A matrix of up to 64 rows and SMALL_K columns: everything in one workgroup, a launch for the whole
// stack.  What the separate launches of such a matrix take is mostly their starts (4 of 6 to 9 us
// each, seventeen of them); one compute unit's matrix cores are enough for its products: 64 x 64 57
// us, in separate launches 110; 64 x 256 84, 105.
using TileOne = Tile<2, 2, 2, 2, 9, 1, true>;
using TileOneX = Tile<2, 2, 4, 2, 4, 1>;      // B X: fewer, wider tiles, one after the other

__global__ void __launch_bounds__(64 * TileOne::WAVES)
    ns_small_kernel(Source s, Steps o, Result res, Planes X0, Planes X1, Planes A, Planes B) {
  constexpr int THREADS = 64 * TileOne::WAVES;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[TileOne::NST * TileOne::STAGE];
  __shared__ double red[THREADS / 64];
  const int z = blockIdx.x;
  const int64_t base = z * s.matrix;
  float* const mom = s.m ? s.m + (int64_t)z * s.rows * s.cols : nullptr;
  const int runs = (s.cols + 7) / 8;
  double sum[2] = {0.0, 0.0};
  for (int e = threadIdx.x; e < s.rows * runs; e += THREADS)
    source_run(s, base, mom, e / runs, e % runs, sum);
  const double total = block_sum<THREADS>(sum[0] + sum[1], red);
  const Scale by = scale_of(total, o.eps);
  // X, zero beyond the matrix
  const int k_runs = (int)X0.ld / 8;
  for (int e = threadIdx.x; e < SMALL_ROWS * k_runs; e += THREADS) {
    const int row = e / k_runs, col = e % k_runs * 8;
    float v[8];
    if (res.tall) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = col + k;
        const bool in = i < s.rows && row < s.cols;
        float u[8] = {};
        load8(s.g, s.f32, in ? base + i * s.ld + row : 0, in ? 1 : 0, u);
        v[k] = u[0];
        if (mom) v[k] = momentum_u(s, in ? mom[i * s.cols + row] : 0.0f, u[0]);
      }
    } else {
      const int n = row < s.rows ? s.cols - col : 0;
      load8(s.g, s.f32, base + row * s.ld + col, n, v);
      if (mom) {
        float m[8];
        load8(mom, true, row * s.cols + col, n, m);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = momentum_u(s, m[k], v[k]);
      }
    }
    store_x<true>(X0, z, row, col, v, by);
  }
  Args a = {};
  a.unit_m = a.unit_n = 64;
  a.res = res;
  const int k_tiles = (int)X0.ld / TileOneX::BM;
  for (int i = 0; i < o.n; ++i) {
    const Planes& X = i & 1 ? X1 : X0;
    __syncthreads();
    a.unit_m = 64, a.units_m = a.units_n = a.units = a.count = 1, a.first = z;
    a.P = a.Q = X, a.K = (int)X0.ld, a.C = A;
    product<GRAM, true, TileOne>(a, 0, 1, 1, smem);
    __syncthreads();
    a.P = a.Q = A, a.K = SMALL_ROWS, a.C = B, a.alpha = o.c, a.beta = o.b, a.shift = 0.0f;
    product<SQUARE, true, TileOne>(a, 0, 1, 1, smem);
    __syncthreads();
    a.unit_m = TileOneX::BM, a.units_m = a.units = a.count = k_tiles, a.first = z * k_tiles;
    a.P = X, a.Q = B, a.C = i & 1 ? X0 : X1, a.beta = o.a;
    if (i == o.n - 1)
      product<RESULT, true, TileOneX>(a, 0, k_tiles, 1, smem);
    else
      product<UPDATE, true, TileOneX>(a, 0, k_tiles, 1, smem);
  }
}

// ---------------------------------------------------------------------------
using Tile64 = TileOne;
using Tile128 = Tile<2, 2, 4, 4, 4, 1, true>;
using Tile128Pair = Tile<2, 2, 4, 4, 2, 2>;
using Tile256 = Tile<2, 2, 8, 4, 3, 1>;
using Tile256Square = Tile<2, 2, 8, 8, 2, 1>;

template <int MODE, class T>
void launch_tile(const Plan& p, Args a, hipStream_t s) {
  while (T::BM << a.sub_m_log < a.unit_m) ++a.sub_m_log;
  while (T::BN << a.sub_n_log < a.unit_n) ++a.sub_n_log;
  const int64_t items = (int64_t)a.count << (a.sub_m_log + a.sub_n_log);
  const int64_t most = (int64_t)device_cu_count() * T::PER_CU;
  const dim3 grid((unsigned)(items < most ? items : most)), block(64 * T::WAVES);
  if constexpr (T::BM <= 128) {       // (a wide tile of two parts does not fit the registers)
    if (p.split) {
      hipLaunchKernelGGL((ns_product_kernel<MODE, true, T>), grid, block, 0, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((ns_product_kernel<MODE, false, T>), grid, block, 0, s, a);
}

template <int MODE>
void launch(const Plan& p, Args a, hipStream_t s) {
  Launch parts[PARTS];
  const int n = product_launches(p, MODE == GRAM ? 0 : MODE == SQUARE ? 1 : 2, parts);
  for (int j = 0; j < n; ++j) {
    const Launch& l = parts[j];
    a.unit_m = l.unit_m, a.unit_n = l.unit_n, a.units_m = l.units_m, a.units_n = l.units_n;
    a.units = l.units, a.first = l.first, a.count = l.count, a.halves_log = l.halves_log;
    if (l.tile == K256_SQUARE)
      launch_tile<MODE, Tile256Square>(p, a, s);
    else if (l.tile == K256)
      launch_tile<MODE, Tile256>(p, a, s);
    else if (l.tile == K128_PAIR)
      launch_tile<MODE, Tile128Pair>(p, a, s);
    else if (l.tile == K128)
      launch_tile<MODE, Tile128>(p, a, s);
    else
      launch_tile<MODE, Tile64>(p, a, s);
  }
}

void run(const Plan& p, const Steps& o, const Source& src, const Result& res, uint8_t* ws,
         hipStream_t s) {
  double* part = (double*)(ws + p.part);
  Planes X[2], A, B;
  const int64_t parts = p.split ? 2 : 1;      // interleaved
  for (int i = 0; i < 2; ++i)
    X[i] = Planes{(_Float16*)(ws + p.x[i]), parts * p.r_pad * p.k_pad, p.x_plane, p.k_pad};
  A = Planes{(_Float16*)(ws + p.a), parts * p.r_pad * p.r_pad, 0, p.r_pad};
  B = Planes{(_Float16*)(ws + p.b), parts * p.r_pad * p.r_pad, 0, p.r_pad};
  if (p.one) {
    hipLaunchKernelGGL(ns_small_kernel, dim3((unsigned)p.batch), dim3(64 * TileOne::WAVES), 0, s, src,
                       o, res, X[0], X[1], A, B);
    return;
  }
  hipLaunchKernelGGL(ns_norm_kernel, dim3(p.n_part, (unsigned)p.batch), dim3(NORM_THREADS), 0, s,
                     src, part);
  const dim3 grid((unsigned)(p.k_pad / 64), (unsigned)(p.r_pad / 64), (unsigned)p.batch);
  if (p.split)
    hipLaunchKernelGGL(ns_start_kernel<true>, grid, dim3(PRE), 0, s, src, part, p.n_part, o.eps,
                       p.tall, X[0]);
  else
    hipLaunchKernelGGL(ns_start_kernel<false>, grid, dim3(PRE), 0, s, src, part, p.n_part, o.eps,
                       p.tall, X[0]);
  for (int i = 0; i < o.n; ++i) {
    Args a = {};
    a.P = a.Q = X[i & 1], a.K = (int32_t)p.k_pad, a.C = A;
    launch<GRAM>(p, a, s);
    // One part: X = (a - sigma) X + (B + sigma I) hi is the same step, but for the rounding of hi,
    // which the second term carries.  Directions whose singular value is still small are spoilt by
    // it times sigma and every later step's growth, those near 1 by it times |b + c + sigma| or so:
    // sigma is 0 as long as there is growth to come, and a in the last step, which then needs no
    // lo at all.  (256 x 1024, equal singular values: 1.7e-3 with 0 throughout, 1.2e-3 so; eight
    // strong directions over 1e-3: 3.5e-4, and 1.0e-3.)
    const bool last = i == o.n - 1, before = i == o.n - 2;
    const float sigma = p.split ? 0.0f : last ? o.a : before ? -0.5f * (o.b + o.c) : 0.0f;
    a.P = a.Q = A, a.K = (int32_t)p.r_pad;
    a.C = B, a.alpha = o.c, a.beta = o.b, a.shift = sigma;
    launch<SQUARE>(p, a, s);
    a.P = X[i & 1], a.Q = B, a.C = X[(i + 1) & 1], a.beta = o.a - sigma;
    a.keep_lo = !before;
    a.res = res;
    if (last)
      launch<RESULT>(p, a, s);
    else
      launch<UPDATE>(p, a, s);
  }
}

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
  run(p, o, src, res, (uint8_t*)ws, s);
  return hip_status(hipGetLastError());
}

// Whether no two rows of a stack share an element: the matrices follow each other, or their rows
// take turns (a stack that is a view of [m, batch, n]).  128 bits: strides are the caller's.
bool rows_apart(int64_t batch, int64_t m, int64_t n, int64_t ld, int64_t stride) {
  typedef __int128 wide;
  return (wide)stride >= (wide)(m - 1) * ld + n ||
         (stride >= n && (wide)ld >= (wide)(batch - 1) * stride + n);
}

int check(const char* fn, int64_t batch, int64_t m, int64_t n, int32_t in_dtype, int64_t ld_in,
          int64_t stride_in, int32_t out_dtype, int64_t ld_out, int64_t stride_out, Plan* p) {
  if ((in_dtype != AGRL_BF16 && in_dtype != AGRL_F32) ||
      (out_dtype != AGRL_BF16 && out_dtype != AGRL_F32))
    return fail(AGRL_E_DTYPE, fn, "dtype must be AGRL_BF16 or AGRL_F32");
  if (batch < 0 || m < 0 || n < 0) return fail(AGRL_E_SHAPE, fn, "negative size");
  if (ld_in < n || ld_out < n) return fail(AGRL_E_SHAPE, fn, "a row stride is smaller than n");
  if (batch == 0 || m == 0 || n == 0) return AGRL_OK;
  if (batch > 1 && (stride_in < 0 || !rows_apart(batch, m, n, ld_out, stride_out)))
    return fail(AGRL_E_SHAPE, fn, "a matrix stride is negative, or rows that are written overlap");
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
