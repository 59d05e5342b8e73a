// Causal attention within each sequence of a packed stream, forward and backward (gfx950).
//
//   S = scale q k^T over the keys of the row's sequence up to the row itself, P = softmax(S),
//   o = P v, lse = log sum exp S;  with do given and D = sum do o of each row and head:
//   P = exp(S - lse), dv = P^T do, dS = P (do v^T - D), dq = scale dS k, dk = scale dS^T q
//
// Query head h reads key head h / (n_head / n_kv); dk and dv are the sums over those heads.
//
// Tiles are cut from the stream as it lies: a row's keys start at its sequence's first token, so a tile
// that holds several sequences masks, one that holds a part of one reads a contiguous range of
// keys, and nothing is padded or planned ahead.
//
// Every product is formed with its long side in the rows of a 32 x 32 matrix-core block and the wave's own 32
// queries (or keys, in the kernel of dk and dv) in the columns, S^T = K Q^T.  A lane then
// holds 16 values of one column: maximum and sum of a softmax are its own but for one exchange
// with the other half-wave, and the block of P, converted, is the operand of the next product as it
// lies (its contraction index may come in any order, so the other operand is read in the order
// the accumulator has: two transposing LDS reads of four rows each).
//
// bf16: v_mfma_f32_32x32x16_bf16, fp32: v_mfma_f32_32x32x2_f32; the same loops on 16-byte fragments.
//
// Kernels: att_fwd, att_dq and att_dkv serve every case with one simple loop; the pipelined ones further down serve bf16
// with heads of whole 16-byte chunks, wherever those can be copied 16 bytes at a time.
//
// P, and dS in the backward, meet v, dout, k and q in the inputs' type, the matrix core's operand: in bf16 each is off by 2^-8 of
// itself at most.  Against 64 bits, of a tensor's norm: o 2.2e-3 to 2.3e-3, with 32-bit weights 1.6e-3 (all of it o's own
// rounding); gradients of packed 16k 2.8e-3 and 2.0e-3, of short sequences 3.2e-3 and 2.6e-3.  Keeping 16 bits of them would
// take two products for one, a third to a half more matrix-core time in kernels that it bounds.
//
// Measured (MI355X, bf16; a large library product reaches 1.6 PFLOP/s; the lower times over hundreds of calls in a row, the
// higher ones in traces of a first dozen, while the clock settles): forward of 32768 tokens, 40 heads over 8 of 128, in
// sequences of 26524 and 6244, 6.4 to 6.9 ms, 1.10 to 1.19 PFLOP/s, matrix cores busy 0.59 at 1.8 GHz (the power limit); of 28
// heads over 4, in ten sequences around 3400, 0.99 to 1.19 ms, 0.9 PFLOP/s at best.  Backward of 16384 tokens of the latter
// in five, 2.0 to 2.1 ms: dk and dv 1.26 to 1.30, dq 0.74 to 0.76 (0.58 PFLOP/s counting five products; seven are formed).
// The simple loops took 17.9, 2.15 and 10.4 ms: their registers spill, and every fragment read is waited for.
#include <math.h>

#include <type_traits>

#include "gemm.hpp"
#include "rows.hpp"

namespace agrl {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// Scores past some 2^24 are many units apart in fp32, and an exponent formed from two roundings of one score is off by as
// much.  Such rows therefore subtract before they scale in the forward (the largest weight is exactly 1), their lse is scale m
// + ln l, rounded once, and the backward takes S with the same rounding: where one key is all of a row,
// S is the lse and the weight 1.  (And a row's largest S is not above its lse: both roundings are of growing functions.)  Up
// to FAR powers of 2 one fused operation does: it is off by 3 FAR 2^-24 = 2^-10.4 of a weight at most, less than a bf16
// weight's rounding.
constexpr float FAR = 4096.0f;
__device__ __forceinline__ float row_lse(float m, float scale, float l) {
  return fmaf(m, scale, LN2 * __builtin_amdgcn_logf(l));
}
__device__ __forceinline__ float weight_log2(float s, float scale, float lse) {
#pragma clang fp contract(off)
  const float S = s * scale;
  return (S - lse) * LOG2E;
}

// [T, n_head, d]: rows `ld`, heads `hs` elements apart
struct Heads {
  const void* p;
  int64_t ld, hs;
};
struct HeadsOut {
  void* p;
  int64_t ld, hs;
};

template <typename T>
struct Mma;
template <>
struct Mma<uint16_t> {
  static constexpr int E = 8;        // elements of a 16-byte fragment
  static constexpr int K = 16;       // contraction of a fragment pair
  static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
  }
  // accumulator rows 8 s .. 8 s + 7 as a fragment
  static __device__ __forceinline__ u32x4 frag(const f32x16& c, int s) {
    return u32x4{pack(c[8 * s], c[8 * s + 1]), pack(c[8 * s + 2], c[8 * s + 3]),
                 pack(c[8 * s + 4], c[8 * s + 5]), pack(c[8 * s + 6], c[8 * s + 7])};
  }
  // largest magnitude bits: at least LIMIT if an element is infinite or NaN
  static __device__ __forceinline__ uint32_t magnitude(uint32_t m, u32x4 f) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m),
                                                                 __builtin_bit_cast(u16x2, f[k] & 0x7fff7fffu)));
    return m;
  }
  static __device__ __forceinline__ bool odd(uint32_t m) {
    return (m & 0xffffu) >= 0x7f80u || m >= 0x7f800000u;
  }
  // the fragment with 0 for infinite and NaN elements, and 1 there and 0 elsewhere
  static __device__ __forceinline__ void split(u32x4 f, u32x4& sane, u32x4& ind) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t lo = (f[k] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u;
      const uint32_t hi = (f[k] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
      sane[k] = f[k] & ~(lo | hi);
      ind[k] = (lo | hi) & 0x3f803f80u;
    }
  }
};
template <>
struct Mma<float> {
  static constexpr int E = 4;
  static constexpr int K = 8;
  static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ u32x4 frag(const f32x16& c, int s) {
    return u32x4{__float_as_uint(c[4 * s]), __float_as_uint(c[4 * s + 1]), __float_as_uint(c[4 * s + 2]),
                 __float_as_uint(c[4 * s + 3])};
  }
  static __device__ __forceinline__ uint32_t magnitude(uint32_t m, u32x4 f) {
#pragma unroll
    for (int k = 0; k < 4; ++k) m = max(m, f[k] & 0x7fffffffu);
    return m;
  }
  static __device__ __forceinline__ bool odd(uint32_t m) { return m >= 0x7f800000u; }
  static __device__ __forceinline__ void split(u32x4 f, u32x4& sane, u32x4& ind) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool bad = (f[k] & 0x7f800000u) == 0x7f800000u;
      sane[k] = bad ? 0u : f[k];
      ind[k] = bad ? 0x3f800000u : 0u;
    }
  }
};

// A tile of rows of DP elements in LDS.  16-byte chunk c of row r sits at c ^ sw(r): the 16 rows that a
// pass of row-wise fragment reads touches lie in 16 distinct bank groups, and so do the four
// rows of a transposing read (its 64-byte windows).
template <typename T, int DP>
struct Tile {
  using M = Mma<T>;
  static constexpr int ROW = DP * (int)sizeof(T);    // bytes
  static constexpr int CPR = ROW / 16;               // chunks of a row
  static constexpr int NS = DP / M::K;               // fragments along a row
  static constexpr int ND = DP / 32;                 // 32-column blocks
  static constexpr int NP = 32 / M::K;               // fragments along 32 rows

  static __device__ __forceinline__ int sw(int r) {
    return CPR == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
  }

  // Lane's byte offsets of its row-wise and transposing reads (the rest is XORs and immediates)
  struct Lane {
    int row, tr;
    __device__ __forceinline__ Lane() {
      const int l = threadIdx.x & 63, r = l & 31, h = l >> 5;
      row = r * ROW + ((sw(r) ^ h) << 4);
      if constexpr (sizeof(T) == 2) {
        // 16-lane group g: columns 16 (g & 1) .., rows 4 h ..; lane s of it points at row s >> 2, columns 4 (s & 3)
        const int s = l & 15, q = s >> 2, k = 4 * h + q, c = ((l >> 4) & 1) * 2 + ((s & 3) >> 1);
        tr = k * ROW + ((c ^ sw(k)) << 4) + (s & 1) * 8;
      } else {
        tr = 4 * h * ROW + (((r >> 2) ^ sw(4 * h)) << 4) + (r & 3) * 4;
      }
    }
  };
  // row operand: rows 32 b .., fragment s
  static __device__ __forceinline__ u32x4 rows(const uint8_t* p, const Lane& L, int b, int s) {
    return *(const u32x4*)(p + b * 32 * ROW + (L.row ^ (s << 5)));
  }
  // transposed operand: columns 32 c .. of the tile are the rows, fragment s of the rows 32 b ..
  static __device__ __forceinline__ u32x4 cols(const uint8_t* p, const Lane& L, int b, int s, int c) {
    if constexpr (sizeof(T) == 2) {
      const uint8_t* q = p + (b * 32 + s * 16) * ROW;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(q + (L.tr ^ (c << 6))));
      const bf16x4 hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(q + 8 * ROW + (L.tr ^ (c << 6) ^ 32)));
      const u32x2 a = __builtin_bit_cast(u32x2, lo), d = __builtin_bit_cast(u32x2, hi);
      return u32x4{a.x, a.y, d.x, d.y};
    } else {
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *(const uint32_t*)(p + (b * 32 + s * 8 + j) * ROW +
                                  (L.tr ^ (j << 6) ^ ((s & 1) << 5) ^ (c << 7)));
      return v;
    }
  }
};

// R rows of a head, from global memory through registers into LDS by NT lanes.  Rows from `end` on are 0.
template <typename T, int DP, int R, int NT, bool FULL>
struct Stage {
  using TL = Tile<T, DP>;
  static constexpr int N = R * TL::CPR / NT, STEP = NT / TL::CPR;
  static_assert(N >= 1 && NT % TL::CPR == 0, "whole chunks a lane");
  u32x4 v[N];
  __device__ __forceinline__ void load(const T* base, int64_t ld, int row0, int end, int d) {
    const int r0 = threadIdx.x / TL::CPR, col = (threadIdx.x & (TL::CPR - 1)) * TL::M::E;
    const T* p = base + (int64_t)(row0 + r0) * ld + col;
#pragma unroll
    for (int i = 0; i < N; ++i, p += STEP * ld) {
      v[i] = u32x4{0, 0, 0, 0};
      if (row0 + r0 + i * STEP < end) v[i] = chunk(p, d - col);
    }
  }
  static __device__ __forceinline__ u32x4 chunk(const T* p, int n) {
    if (FULL || n >= TL::M::E) return sizeof(T) == 2 ? (u32x4) * (const u32x4_a2*)p : (u32x4) * (const u32x4_a4*)p;
    u32x4 w = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < TL::M::E - 1; ++k)
      if (k < n) {
        if constexpr (sizeof(T) == 2)
          w[k >> 1] |= (uint32_t)p[k] << (16 * (k & 1));
        else
          w[k] = __float_as_uint(p[k]);
      }
    return w;
  }
  __device__ __forceinline__ void store(uint8_t* lds) const {
    const int r0 = threadIdx.x / TL::CPR, c = threadIdx.x & (TL::CPR - 1);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * STEP;
      *(u32x4*)(lds + r * TL::ROW + ((c ^ TL::sw(r)) << 4)) = v[i];
    }
  }
};

// A column operand held in registers: 32 rows of a head, lane's row r, as fragments
template <typename T, int DP, bool FULL, int NS>
__device__ __forceinline__ void hold(u32x4 (&f)[NS], const T* row, bool live, int d) {
  using M = Mma<T>;
  static_assert(NS == Tile<T, DP>::NS, "a whole row");
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    f[s] = u32x4{0, 0, 0, 0};
    if (live) f[s] = Stage<T, DP, 32, 64, FULL>::chunk(row + (2 * s + h) * M::E, d - (2 * s + h) * M::E);
  }
}

// ------------------------------------------------------------------ sequences
// The number of offsets that are at most n, by one wave: 64 probes a step
__device__ __forceinline__ int offsets_upto(const int32_t* start, int n_seq, int n) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_seq + 1;
  while (hi - lo > 64) {
    const int step = (hi - lo + 63) >> 6, i = lo + (lane + 1) * step - 1;
    const int c = __popcll(__ballot(i < hi && start[min(i, hi - 1)] <= n));
    lo += c * step;
    hi = min(hi, lo + step);
  }
  const int i = lo + lane;
  return lo + __popcll(__ballot(i < hi && start[min(i, n_seq)] <= n));
}

// A lane's token n and its sequence [begin, end); live: there is one
struct Place {
  int begin, end;
  bool live;
  // lo, hi: offsets up to the first and the last of the wave's tokens; n one of them
  __device__ __forceinline__ Place(const int32_t* start, int n_seq, int T, int lo, int hi, int n) {
    while (lo < hi) {
      const int mid = lo + ((hi - lo) >> 1);
      if (start[mid] <= n)
        lo = mid + 1;
      else
        hi = mid;
    }
    live = n < T && lo >= 1 && lo <= n_seq;
    begin = end = n;
    if (live) {
      begin = min(max(start[lo - 1], 0), n);     // (offsets out of order stay within the stream)
      end = min(max(start[lo], n + 1), T);
    }
  }
};

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o));
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max(int v) { return -wave_min(-v); }

// Offsets that decrease or leave [0, T] set the error word's bit; the grid's workgroups share them.
__device__ __forceinline__ void check_offsets(const int32_t* start, int n_seq, int T, int* err) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i <= n_seq;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int s = start[i];
    if (s < 0 || s > T || (i > 0 && start[i - 1] > s)) set_error(err, ERR_SEQ_START);
  }
}

// ------------------------------------------------------------------ products
// acc += X^T p over the tile's 32 rows of block b; `ok`: which of the lane's 16 rows count.  In masked blocks
// p is 0 where a row does not count, but 0 times an infinite or NaN element of X is not: there such
// elements are taken out, and a second product with ones in their places finds who did count them.
template <typename T, int DP, bool MASKED, int ND, int NP>
__device__ __forceinline__ void add_cols(f32x16 (&acc)[ND], const uint8_t* x,
                                         const typename Tile<T, DP>::Lane& L, int b, const u32x4 (&p)[NP],
                                         uint32_t ok) {
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  if constexpr (MASKED) {
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < TL::ND; ++c)
#pragma unroll
      for (int s = 0; s < TL::NP; ++s) m = M::magnitude(m, TL::cols(x, L, b, s, c));
    if (__any(M::odd(m))) {
      f32x16 counts;
#pragma unroll
      for (int r = 0; r < 16; ++r) counts[r] = ok >> r & 1 ? 1.0f : 0.0f;
#pragma unroll
      for (int c = 0; c < TL::ND; ++c) {
        f32x16 hit = {};
#pragma unroll
        for (int s = 0; s < TL::NP; ++s) {
          u32x4 sane, ind;
          M::split(TL::cols(x, L, b, s, c), sane, ind);
          acc[c] = M::mma(sane, p[s], acc[c]);
          hit = M::mma(ind, M::frag(counts, s), hit);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = hit[r] > 0.0f ? NAN : acc[c][r];
      }
      return;
    }
  }
#pragma unroll
  for (int c = 0; c < TL::ND; ++c)
#pragma unroll
    for (int s = 0; s < TL::NP; ++s) acc[c] = M::mma(TL::cols(x, L, b, s, c), p[s], acc[c]);
}

// acc = X f over the tile's 32 rows of block b
template <typename T, int DP, int NS>
__device__ __forceinline__ f32x16 mul_rows(const uint8_t* x, const typename Tile<T, DP>::Lane& L, int b,
                                           const u32x4 (&f)[NS]) {
  f32x16 acc = {};
#pragma unroll
  for (int s = 0; s < NS; ++s) acc = Mma<T>::mma(Tile<T, DP>::rows(x, L, b, s), f[s], acc);
  return acc;
}

// The same of a padded head of whole chunks, for the second pass of the pipelines.  Past d their tiles repeat the last chunk,
// and the zeros that it meets there would make a NaN of an infinite element: taken as 0.
template <typename T, int DP, bool FULL, int NS>
__device__ __forceinline__ f32x16 mul_rows_upto(const uint8_t* x, const typename Tile<T, DP>::Lane& L, int b,
                                                const u32x4 (&f)[NS], int d) {
  if constexpr (FULL) return mul_rows<T, DP>(x, L, b, f);
  const int h = (threadIdx.x & 63) >> 5;
  f32x16 acc = {};
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const u32x4 v = Tile<T, DP>::rows(x, L, b, s);
    acc = Mma<T>::mma((2 * s + h) * Mma<T>::E < d ? v : u32x4{0, 0, 0, 0}, f[s], acc);
  }
  return acc;
}

// row of accumulator element r within its block
__device__ __forceinline__ int acc_row(int r) { return 8 * (r >> 2) + (r & 3) + 4 * ((threadIdx.x & 63) >> 5); }

__device__ __forceinline__ float other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// The column's DP values times f to a row of the output, eight (fp32: four) adjacent ones a lane
template <typename T, int DP, bool FULL, int ND>
__device__ __forceinline__ void put_row(T* row, const f32x16 (&acc)[ND], float f, bool zero, bool live, int d) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int c = 0; c < ND; ++c) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = zero ? 0u : Mma<T>::pack(acc[c][4 * g + 2 * k] * f, acc[c][4 * g + 2 * k + 1] * f);
        const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        const u32x4 v = {a[0], b[0], a[1], b[1]};
        const int col = 32 * c + 8 * (g + h);
        if (!live) continue;
        if (FULL || col + 8 <= d) {
          *(u32x4_a2*)(row + col) = v;
        } else {
#pragma unroll
          for (int k = 0; k < 7; ++k)
            if (col + k < d) row[col + k] = (T)(v[k >> 1] >> (16 * (k & 1)));
        }
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = zero ? 0.0f : acc[c][4 * g + k] * f;
        const int col = 32 * c + 8 * g + 4 * h;
        typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
        if (!live) continue;
        if (FULL || col + 4 <= d) {
          *(f32x4_a4*)(row + col) = v;
        } else {
#pragma unroll
          for (int k = 0; k < 3; ++k)
            if (col + k < d) row[col + k] = v[k];
        }
      }
    }
  }
}

// ------------------------------------------------------------------ forward
constexpr int WAVES = 4, THREADS = 64 * WAVES, BM = 32 * WAVES;   // own rows of a workgroup
template <typename T>
constexpr int BN = sizeof(T) == 2 ? 64 : 32;                      // rows of a tile that goes through LDS

struct AttArgs {
  int32_t T, n_seq, n_head, n_kv, rep, d;
  Heads q, k, v;
  const int32_t* start;
  float scale;
  HeadsOut o;
  float* lse;
  int* err;
  // backward
  Heads dout;
  const float *lse_in, *lse2, *delta;      // [n_head, T]: the forward's lse, in powers of 2, sum do o
  const int32_t* order;          // key tiles in the order they are taken
  const uint8_t* far;            // [FLAGS] whether some row's lse is past FAR: not 0 anywhere
  HeadsOut dq, dk, dv;
  int32_t splits;                // parts that a group's heads are dealt to, each a workgroup's
  float* part;                   // more than one: [splits][2][T, n_kv, d] sums of dk and dv
};

// What a wave's 32 columns need: its range of the other side
struct Span {
  int lo, hi;              // [lo, hi): rows that some column counts
  int full_lo, full_hi;    // [full_lo, full_hi): rows that every column counts
};
// the workgroup's range
__device__ __forceinline__ void join(const Span& s, int (&lds)[2][WAVES], int& lo, int& hi) {
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    lds[0][wave] = s.lo;
    lds[1][wave] = s.hi;
  }
  __syncthreads();
  lo = 0x7fffffff;
  hi = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    lo = min(lo, lds[0][w]);
    hi = max(hi, lds[1][w]);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
}

// Queries in the columns: a row of the stream counts the keys begin .. itself
__device__ __forceinline__ Span query_span(const Place& at, int n) {
  const int lo = wave_min(at.live ? at.begin : 0x7fffffff), last = wave_max(at.live ? n : -1);
  const bool all = __all(at.live);
  const int full_lo = wave_max(at.begin), full_hi = wave_min(n) + 1;
  return Span{lo, last + 1, full_lo, all ? full_hi : 0};
}

template <typename T, int DP, bool FULL>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 ? 2 : 1) att_fwd_kernel(AttArgs a) {
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  constexpr int R = BN<T>, NB = R / 32;
  __shared__ __align__(16) uint8_t lds_k[2][R * TL::ROW], lds_v[2][R * TL::ROW];
  __shared__ int lds_span[2][WAVES];
  if (a.err) check_offsets(a.start, a.n_seq, a.T, a.err);
  // the stream's last tiles first (of one sequence: the longest ranges); a key head's query heads on one XCD (8 in turn) as far
  // as the numbers allow
  const int tiles = (a.T + BM - 1) / BM;
  const int tile = tiles - 1 - blockIdx.x / a.n_head, j = blockIdx.x % a.n_head;
  const int kv = j % a.n_kv, head = kv * a.rep + j / a.n_kv;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = tile * BM + wave * 32, n = first + (lane & 31);
  const Place at(a.start, a.n_seq, a.T, offsets_upto(a.start, a.n_seq, first),
                 offsets_upto(a.start, a.n_seq, first + 31), n);
  const Span span = query_span(at, n);
  const uint32_t len = at.live ? n - at.begin + 1 : 0;
  int lo, hi;
  join(span, lds_span, lo, hi);

  const typename TL::Lane L;
  u32x4 q[TL::NS];
  hold<T, DP, FULL>(q, (const T*)a.q.p + head * a.q.hs + (int64_t)n * a.q.ld, at.live, a.d);
  const T* kp = (const T*)a.k.p + kv * a.k.hs;
  const T* vp = (const T*)a.v.p + kv * a.v.hs;
  const float sl2 = a.scale * LOG2E;
  f32x16 o[TL::ND] = {};
  float m = -INFINITY, l = 0.0f;
  Stage<T, DP, R, THREADS, FULL> sk, sv;
  const int kt0 = lo / R * R;
  if (lo < hi) {
    sk.load(kp, a.k.ld, kt0, a.T, a.d);
    sv.load(vp, a.v.ld, kt0, a.T, a.d);
    sk.store(lds_k[0]);
    sv.store(lds_v[0]);
  }
  __syncthreads();
  int buf = 0;
  for (int k0 = kt0; k0 < hi; k0 += R, buf ^= 1) {
    const bool more = k0 + R < hi;
    if (more) {
      sk.load(kp, a.k.ld, k0 + R, a.T, a.d);
      sv.load(vp, a.v.ld, k0 + R, a.T, a.d);
    }
    auto step = [&](auto masked_c) {
      constexpr bool MASKED = decltype(masked_c)::value;
      f32x16 s[NB];
      uint32_t ok[NB];
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        s[b] = mul_rows<T, DP>(lds_k[buf], L, b, q);
        ok[b] = 0;
        if constexpr (MASKED) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool in = (uint32_t)(k0 + 32 * b + acc_row(r) - at.begin) < len;
            ok[b] |= in ? 1u << r : 0u;
            s[b][r] = in ? s[b][r] : -INFINITY;
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
      }
      top = fmaxf(top, other_half(top));
      // a column's reference moves only when the maximum has left it 2^8 behind: any reference gives the same
      // quotient (and a column's own, so no other row's values change its roundings)
      const bool far = (top - m) * sl2 > 8.0f;
      if (__any(far)) {
        const float to = far ? top : m;
        const float f = far ? __builtin_amdgcn_exp2f((m - to) * sl2) : 1.0f;
        l *= f;
#pragma unroll
        for (int c = 0; c < TL::ND; ++c) o[c] *= f;
        m = to;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        u32x4 p[TL::NP];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[b][r] = __builtin_amdgcn_exp2f((s[b][r] - ref) * sl2);
          l += s[b][r];
        }
#pragma unroll
        for (int i = 0; i < TL::NP; ++i) p[i] = M::frag(s[b], i);
        add_cols<T, DP, MASKED>(o, lds_v[buf], L, b, p, ok[b]);
      }
    };
    if (k0 + R > span.lo && k0 < span.hi) {
      if (k0 >= span.full_lo && k0 + R <= span.full_hi)
        step(std::false_type{});
      else
        step(std::true_type{});
    }
    if (more) {
      sk.store(lds_k[buf ^ 1]);
      sv.store(lds_v[buf ^ 1]);
    }
    __syncthreads();
  }
  l += other_half(l);
  if (a.lse && n < a.T && lane < 32)
    a.lse[(int64_t)head * a.T + n] = at.live ? row_lse(m, a.scale, l) : 0.0f;
  put_row<T, DP, FULL>((T*)a.o.p + head * a.o.hs + (int64_t)n * a.o.ld, o, 1.0f / l, !at.live, n < a.T, a.d);
}

// ------------------------------------------------------------------ forward, pipelined
// 64 queries a wave (two column blocks), one wave a SIMD: half the LDS reads per product, and registers for a
// pipeline in which nothing waits.  Keys go by halves of 32: while the exponentials of one half run on the
// vector ALU, the matrix cores form the next half's scores and the previous half's share of o.  A phase
// has a slot per MFMA (32 cycles of the matrix core); each carries two of the half's 64 columns' values, and
// every other one an LDS fragment read, seven fragments ahead (three with heads of 64).  K and V go
// straight from global memory into rings of three tiles of 64, K a tile ahead of V.
//
// The softmax's reference is the row's own score q k, which is one of those that count: the sum is at least 1, and
// there is no running maximum to follow.  Weights may grow to 2^96 before that fails (scores 66 above the row's own);
// then, or where a result is not finite (a NaN or infinite element of V met a weight of 0, or a weight times a large one
// left the range), the workgroup goes through its tile again step by step, masked elements taken out.  There a row whose
// sum had left its range, or whose own score is past FAR, follows its maximum.  Any other keeps its reference: its results have
// the bits of the first pass, and where they were not finite its weights are taken down by the power of 2 of its sum, which
// changes no mantissa.
constexpr int PIPE_ROWS = 64 * WAVES;

template <int N, class F>
__device__ __forceinline__ void slots(F&& f) {
  static_for<N>(f);
}

// Copies of 64-row tiles of a head into LDS, 1 KiB an instruction; rows past the end repeat the last one
template <int DP>
struct Copy {
  using TL = Tile<uint16_t, DP>;
  static constexpr int RPI = 1024 / TL::ROW, PER = 64 / RPI / WAVES, BYTES = 64 * TL::ROW;
  const uint8_t* p;
  int64_t ldb;
  uint32_t r, c, off;        // lane's row and byte of the first copy, its offset
  uint32_t lds;
  int T;
  // (the places past a head of d elements get its last chunk again: they meet zeros, or are not stored; where that chunk is not
  // finite the second pass takes them out)
  __device__ __forceinline__ void init(const void* head, int64_t ld, uint32_t lds_base, int wave, int rows, int d) {
    const int lane = threadIdx.x & 63;
    p = (const uint8_t*)head;
    ldb = ld * 2;
    T = rows;
    r = wave * RPI + lane / TL::CPR;
    c = min((lane & (TL::CPR - 1)) ^ TL::sw(r), d / 8 - 1) << 4;
    off = r * (uint32_t)ldb + c;
    lds = __builtin_amdgcn_readfirstlane(lds_base + wave * 1024);
  }
  // rows row0 .. row0 + 63 of the head `head` bytes on, to byte `at` of the ring
  __device__ __forceinline__ void tile(int row0, int at, int64_t head = 0) const {
    const uint8_t* base = p + head + (int64_t)row0 * ldb;
    const uint32_t to = lds + at;
    if (row0 + 64 <= T) {
      slots<PER>([&](auto i) {
        bf16k::copy16<i.value * WAVES * 1024>(base + (int64_t)(i.value * WAVES * RPI) * ldb, off, to);
      });
    } else {
      slots<PER>([&](auto i) {
        const uint32_t row = min(r + i.value * WAVES * RPI, (uint32_t)(T - 1 - row0));
        bf16k::copy16<i.value * WAVES * 1024>(base, row * (uint32_t)ldb + c, to);
      });
    }
  }
};

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p;
}

template <int DP, bool FULL>
__global__ void __launch_bounds__(THREADS, 1) att_fwd_pipe_kernel(AttArgs a) {
  using T = uint16_t;
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  constexpr int NS = TL::NS, ND = TL::ND, NP = TL::NP, ROW = TL::ROW, RING = 3 * Copy<DP>::BYTES;
  __shared__ __align__(16) uint8_t lds_k[RING], lds_v[RING];
  __shared__ int lds_span[2][WAVES];
  if (a.err) check_offsets(a.start, a.n_seq, a.T, a.err);
  const int tiles = (a.T + PIPE_ROWS - 1) / PIPE_ROWS;
  const int tile = tiles - 1 - blockIdx.x / a.n_head, j = blockIdx.x % a.n_head;
  const int kv = j % a.n_kv, head = kv * a.rep + j / a.n_kv;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = tile * PIPE_ROWS + wave * 64;
  const int nA = first + (lane & 31), nB = nA + 32;
  const int upto0 = offsets_upto(a.start, a.n_seq, first), upto1 = offsets_upto(a.start, a.n_seq, first + 63);
  const Place at[2] = {Place(a.start, a.n_seq, a.T, upto0, upto1, nA),
                       Place(a.start, a.n_seq, a.T, upto0, upto1, nB)};
  const Span part[2] = {query_span(at[0], nA), query_span(at[1], nB)};
  const Span span = {min(part[0].lo, part[1].lo), max(part[0].hi, part[1].hi),
                     max(part[0].full_lo, part[1].full_lo), min(part[0].full_hi, part[1].full_hi)};
  int lo, hi;
  join(span, lds_span, lo, hi);

  const typename TL::Lane L;
  u32x4 q[2][NS];
  Copy<DP> ck, cv;
  ck.init((const T*)a.k.p + kv * a.k.hs, a.k.ld, lds_address(lds_k), wave, a.T, a.d);
  cv.init((const T*)a.v.p + kv * a.v.hs, a.v.ld, lds_address(lds_v), wave, a.T, a.d);
  const float sl2 = a.scale * LOG2E;
  f32x16 o[2][ND] = {};
  float l[2] = {0.0f, 0.0f}, m[2];
  const uint32_t len[2] = {at[0].live ? nA - at[0].begin + 1u : 0u, at[1].live ? nB - at[1].begin + 1u : 0u};
  float ref[2];
  const int t0 = lo / 64, t1 = lo < hi ? (hi + 63) / 64 : t0;
  // the wave's tiles, and those of them that all its columns count whole
  const int w0 = span.lo < span.hi ? span.lo / 64 : t1, w1 = span.lo < span.hi ? (span.hi + 63) / 64 : t0;
  const int f0 = (span.full_lo + 63) / 64, f1 = span.full_hi / 64;
  // what passes from phase to phase
  constexpr int AHEAD = DP == 128 ? 7 : 3, FR = AHEAD + 1;
  static_assert(AHEAD <= NS, "what is read ahead of a phase is K");
  f32x16 s0[2], s1[2];
  u32x4 p0[2][NP], p1[2][NP], fr[FR];
  int ko[NS], vo[ND][2];
#pragma unroll
  for (int s = 0; s < NS; ++s) ko[s] = 0;
#pragma unroll
  for (int c = 0; c < ND; ++c) vo[c][0] = vo[c][1] = 0;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    s0[b] = s1[b] = f32x16{};
#pragma unroll
    for (int i = 0; i < NP; ++i) p0[b][i] = p1[b][i] = u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < FR; ++i) fr[i] = u32x4{0, 0, 0, 0};

  auto read_v = [&](int half, int s, int c) {
    const uint8_t* x = lds_v + (half * 32 + s * 16) * ROW;
    const u32x2 u = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + vo[c][0])));
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + vo[c][1] + 8 * ROW)));
    return u32x4{u.x, u.y, w.x, w.y};
  };
  // The weights of `cur` into `pn`, the next half's scores (rows 32 KH of the tile that ko points at) into `nxt`, the
  // previous half's weights `pp` times V (rows 32 VH of vo's tile).  `move`: what ko (behind its last read for this
  // phase) or vo (before its first) advance by.
  auto phase = [&](auto first_c, auto masked_c, f32x16 (&cur)[2], f32x16 (&nxt)[2], u32x4 (&pp)[2][NP], u32x4 (&pn)[2][NP],
                   int move, int key0) {
    constexpr bool FIRST = decltype(first_c)::value;      // of a tile
    constexpr bool MASKED = decltype(masked_c)::value;
    // keys counted from the lane's first row of the half to its columns' first key
    const int from[2] = {key0 + 4 * (lane >> 5) - at[0].begin, key0 + 4 * (lane >> 5) - at[1].begin};
    constexpr int KH = FIRST ? 1 : 0, VH = FIRST ? 1 : 0;
    constexpr int NQ = 2 * NS, NM = NQ + 2 * NP * ND, NF = NM / 2;
    slots<NM>([&](auto slot) {
      constexpr int i = slot.value, fi = i / 2, b = i & 1;
      if constexpr (b == 0) {
        constexpr int n = fi + AHEAD;
        if constexpr (n < NS)
          fr[n % FR] = *(const u32x4*)(lds_k + KH * 32 * ROW + ko[n]);
        else if constexpr (n < NF)
          fr[n % FR] = read_v(VH, (n - NS) / ND, (n - NS) % ND);
        else
          fr[n % FR] = *(const u32x4*)(lds_k + (KH ^ 1) * 32 * ROW + ko[n - NF]);
      }
      if constexpr (i < NQ) {
        nxt[b] = M::mma(fr[fi % FR], q[b][fi], fi == 0 ? f32x16{} : nxt[b]);
      } else {
        constexpr int s = (fi - NS) / ND, c = (fi - NS) % ND;
        o[b][c] = M::mma(fr[fi % FR], pp[b][s], o[b][c]);
      }
      if constexpr (FIRST && i >= NQ && i < NQ + NS) ko[i - NQ] += move;
      if constexpr (!FIRST && i < 2 * ND) vo[i >> 1][i & 1] += move;
      // a value takes three slots: its exponent, the exponential, the sum and the conversion
      constexpr int EPS = 32 / NM, last = i + 1 == NM ? 32 : 0;
      slots<32>([&](auto e_c) {
        constexpr int e = e_c.value, cb = e >> 4, r = e & 15;
        float x = cur[cb][r];
        if constexpr (e / EPS == i) {
          if constexpr (MASKED) {
            const bool in = (uint32_t)(from[cb] + 8 * (r >> 2) + (r & 3)) < len[cb];
            x = in ? x : -INFINITY;
          }
          x = fmaf(x, sl2, -ref[cb]);
        }
        if constexpr (e / EPS == i - 1 || (last && e / EPS == i)) x = __builtin_amdgcn_exp2f(x);
        if constexpr (e / EPS == i - 2 || (last && e / EPS >= i - 1)) {
          l[cb] += x;
          if constexpr (r & 1) {
            uint32_t w = M::pack(cur[cb][r - 1], x);
            asm volatile("" : "+v"(w), "+v"(l[cb]));          // (here, not where it is used)
            pn[cb][r >> 3][(r & 7) >> 1] = w;
          }
        }
        cur[cb][r] = x;
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  constexpr int TB = Copy<DP>::BYTES;
  int slot = 0;        // of tile t in both rings
  auto begin = [&]() {
    slot = 0;
    if (t0 >= t1) return;
    ck.tile(t0 * 64, 0);
    if (t0 + 1 < t1) ck.tile(t0 * 64 + 64, TB);
    cv.tile(t0 * 64, 0);
  };
  // tile t has landed, the next ones are on their way
  auto arrive = [&](int t) {
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    const int next = slot == 2 ? 0 : slot + 1;
    if (t + 2 < t1) ck.tile(t * 64 + 128, (next == 2 ? 0 : next + 1) * TB);
    if (t + 1 < t1) cv.tile(t * 64 + 64, next * TB);
  };
  begin();
  const T* qp = (const T*)a.q.p + head * a.q.hs;
  hold<T, DP, FULL>(q[0], qp + (int64_t)nA * a.q.ld, at[0].live, a.d);
  hold<T, DP, FULL>(q[1], qp + (int64_t)nB * a.q.ld, at[1].live, a.d);
  // the reference: the row's own score
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    u32x4 own[NS];
    hold<T, DP, FULL>(own, (const T*)a.k.p + kv * a.k.hs + (int64_t)(cb ? nB : nA) * a.k.ld, at[cb].live, a.d);
    float dot = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = q[cb][s][e], y = own[s][e];
        dot = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), dot, false);
      }
    ref[cb] = (dot + other_half(dot)) * sl2;
  }
  int t = t0;
  for (; t < min(w0, t1); ++t) {
    arrive(t);
    slot = slot == 2 ? 0 : slot + 1;
  }
  if (t < w1) {
    arrive(t);
    // the first half's scores; no weights are pending yet (V's first half meets weights of 0)
    const int at_k = slot * TB;
#pragma unroll
    for (int s = 0; s < NS; ++s) ko[s] = (L.row ^ (s << 5)) + at_k;
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      vo[c][0] = (L.tr ^ (c << 6)) + at_k;
      vo[c][1] = (L.tr ^ (c << 6) ^ 32) + at_k;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s0[b] = mul_rows<T, DP>(lds_k + at_k, L, 0, q[b]);
#pragma unroll
      for (int i = 0; i < NP; ++i) p1[b][i] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fr[i] = *(const u32x4*)(lds_k + 32 * ROW + ko[i]);
    static_assert((NS + NP * ND) % FR == 0, "a phase starts at the ring's first fragment");
    int vmove = 0;
    auto through = [&](auto masked_c, int until) {
      while (t < until) {
        const int kmove = slot == 2 ? -2 * TB : TB;
        phase(std::true_type{}, masked_c, s0, s1, p1, p0, kmove, t * 64);
        phase(std::false_type{}, masked_c, s1, s0, p0, p1, vmove, t * 64 + 32);
        vmove = kmove;
        slot = slot == 2 ? 0 : slot + 1;
        if (++t < w1) arrive(t);
      }
    };
    through(std::true_type{}, min(f0, w1));
    through(std::false_type{}, min(f1, w1));
    through(std::true_type{}, w1);
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
      for (int c = 0; c < ND; ++c) {
        const u32x4 v = read_v(1, s, c);
        o[0][c] = M::mma(v, p1[0][s], o[0][c]);
        o[1][c] = M::mma(v, p1[1][s], o[1][c]);
      }
  }
  for (; t < t1; ++t) {
    arrive(t);
    slot = slot == 2 ? 0 : slot + 1;
  }
  bool lost = false, follow[2];
  float up[2] = {1.0f, 1.0f};            // what the weights of the second pass are smaller by
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    l[cb] += other_half(l[cb]);
    follow[cb] = !(l[cb] > 0.5f && l[cb] < 0x1p96f && fabsf(ref[cb]) <= FAR);
    m[cb] = follow[cb] ? -INFINITY : ref[cb];
    float z = 0.0f;
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) z = fmaf(o[cb][c][r], 0.0f, z);
    z += other_half(z);                  // 0 or NaN
    lost = lost || (at[cb].live && (follow[cb] || z != 0.0f));
    if (!follow[cb] && z != 0.0f && l[cb] > 1.0f) up[cb] = __uint_as_float(__float_as_uint(l[cb]) & 0x7f800000u);
  }
  if (__syncthreads_or(lost)) {
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) {
      l[cb] = 0.0f;
#pragma unroll
      for (int c = 0; c < ND; ++c) o[cb][c] = f32x16{};
    }
    begin();
    for (t = t0; t < t1; ++t) {
      arrive(t);
      const int at_k = slot * TB;
#pragma unroll
      for (int cb = 0; cb < 2; ++cb) {
        if (t * 64 + 64 <= part[cb].lo || t * 64 >= part[cb].hi) continue;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          f32x16 s = mul_rows_upto<T, DP, FULL>(lds_k + at_k, L, b, q[cb], a.d);
          uint32_t ok = 0;
          float top = -INFINITY;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool in = (uint32_t)(t * 64 + 32 * b + acc_row(r) - at[cb].begin) < len[cb];
            ok |= in ? 1u << r : 0u;
            s[r] = in ? s[r] : -INFINITY;
            top = fmaxf(top, s[r]);
          }
          top = fmaxf(top, other_half(top));
          const bool far = follow[cb] && top > m[cb];         // (m: a score; of the others, the reference in powers of 2)
          const float to = far ? top : m[cb], f = far ? __builtin_amdgcn_exp2f((m[cb] - to) * sl2) : 1.0f;
          const float down = __uint_as_float(0x7f000000u - __float_as_uint(up[cb]));        // 1 / up
          m[cb] = to;
          l[cb] *= f;
#pragma unroll
          for (int c = 0; c < ND; ++c) o[cb][c] *= f;
          const float from = to == -INFINITY ? 0.0f : to;
          u32x4 p[NP];
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(follow[cb] ? (s[r] - from) * sl2 : fmaf(s[r], sl2, -from)) * down;
            l[cb] += s[r];
          }
#pragma unroll
          for (int i = 0; i < NP; ++i) p[i] = M::frag(s, i);
          add_cols<T, DP, true>(o[cb], lds_v + at_k, L, b, p, ok);
        }
      }
      slot = slot == 2 ? 0 : slot + 1;
    }
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) l[cb] += other_half(l[cb]);
  }
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const int n = cb ? nB : nA;
    if (a.lse && n < a.T && lane < 32)
      a.lse[(int64_t)head * a.T + n] = !at[cb].live  ? 0.0f
                                       : follow[cb] ? row_lse(m[cb], a.scale, l[cb])
                                                    : LN2 * (m[cb] + __builtin_amdgcn_logf(l[cb] * up[cb]));
    put_row<T, DP, FULL>((T*)a.o.p + head * a.o.hs + (int64_t)n * a.o.ld, o[cb], 1.0f / l[cb], !at[cb].live,
                         n < a.T, a.d);
  }
}

// ------------------------------------------------------------------ backward
// lse in powers of 2 and D = sum do o, [n_head, T].  A wave takes a token's heads in turn, 16 lanes a head.
struct DeltaArgs {
  int32_t T, n_head, d, n_seq;
  Heads o, dout;
  const float* lse;
  float *lse2, *delta;
  const int32_t* start;
  int32_t* order;       // [tiles of BM keys], those with the most rows first
  uint8_t* far;         // [FLAGS] whether a workgroup met a row whose lse is past FAR
};
constexpr int FLAGS = 16 * THREADS;

// The key tiles by the rows that count them, in 256 classes (the order within one does not matter: each tile's
// results are its own).  One workgroup.
__device__ __forceinline__ void order_tiles(const DeltaArgs& a) {
  constexpr int CLASSES = 256;
  __shared__ int from[CLASSES], widest;
  const int tiles = (a.T + BM - 1) / BM;
  // rows from the tile's first key to the end of its last one's sequence
  auto rows = [&](int t) {
    const int last = min(t * BM + BM, a.T) - 1;
    int lo = 0, hi = a.n_seq + 1;
    while (lo < hi) {
      const int mid = lo + ((hi - lo) >> 1);
      if (a.start[mid] <= last)
        lo = mid + 1;
      else
        hi = mid;
    }
    return min(max(lo <= a.n_seq ? a.start[lo] : 0, last), a.T) - t * BM;
  };
  from[threadIdx.x] = 0;
  if (threadIdx.x == 0) widest = 1;
  __syncthreads();
  for (int t = threadIdx.x; t < tiles; t += CLASSES) atomicMax(&widest, rows(t));
  __syncthreads();
  auto of = [&](int t) { return CLASSES - 1 - (int)((int64_t)rows(t) * (CLASSES - 1) / widest); };
  for (int t = threadIdx.x; t < tiles; t += CLASSES) atomicAdd(&from[of(t)], 1);
  __syncthreads();
  int before = 0;
  for (int c = 0; c < (int)threadIdx.x; ++c) before += from[c];
  __syncthreads();
  from[threadIdx.x] = before;
  __syncthreads();
  for (int t = threadIdx.x; t < tiles; t += CLASSES) a.order[atomicAdd(&from[of(t)], 1)] = t;
}

template <typename T>
__global__ void __launch_bounds__(256) att_delta_kernel(DeltaArgs a) {
  if (blockIdx.x == gridDim.x - 1) {
    for (int i = gridDim.x - 1 + threadIdx.x; i < FLAGS; i += 256) a.far[i] = 0;
    return order_tiles(a);
  }
  const int l = threadIdx.x & 15, team = threadIdx.x >> 4;
  bool far = false;
  for (int64_t i = (int64_t)blockIdx.x * 16 + team; i < (int64_t)a.T * a.n_head; i += (int64_t)(gridDim.x - 1) * 16) {
    const int n = (int)(i / a.n_head), h = (int)(i - (int64_t)n * a.n_head);
    const T* o = (const T*)a.o.p + (int64_t)n * a.o.ld + h * a.o.hs;
    const T* g = (const T*)a.dout.p + (int64_t)n * a.dout.ld + h * a.dout.hs;
    float sum = 0.0f;
    for (int c = l * CH; c < a.d; c += 16 * CH) {
      Chunk<T> x, y;
      if (c + CH <= a.d) {
        x.load(o + c);
        y.load(g + c);
      } else {
        x.load_some(o + c, a.d - c);
        y.load_some(g + c, a.d - c);
      }
#pragma unroll
      for (int k = 0; k < CH; ++k) sum = fmaf(x.get(k), y.get(k), sum);
    }
    sum = dpp_add<0xb1>(sum);
    sum = dpp_add<0x4e>(sum);
    sum = dpp_add<0x141>(sum);
    sum = dpp_add<0x140>(sum);
    if (l == 0) {
      a.delta[(int64_t)h * a.T + n] = sum;
      const float z = a.lse[(int64_t)h * a.T + n] * LOG2E;
      a.lse2[(int64_t)h * a.T + n] = z;
      far = far || fabsf(z) > FAR;
    }
  }
  far = __syncthreads_or(far);
  if (threadIdx.x == 0) a.far[blockIdx.x] = far;
}

// dq: queries in the columns as in the forward; dS^T is the operand that meets K^T.
template <typename T, int DP, bool FULL>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 ? 2 : 1) att_dq_kernel(AttArgs a) {
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  constexpr int R = BN<T>, NB = R / 32;
  __shared__ __align__(16) uint8_t lds_k[2][R * TL::ROW], lds_v[2][R * TL::ROW];
  __shared__ int lds_span[2][WAVES];
  if (a.err) check_offsets(a.start, a.n_seq, a.T, a.err);
  const int tiles = (a.T + BM - 1) / BM;
  const int tile = tiles - 1 - blockIdx.x / a.n_head, j = blockIdx.x % a.n_head;
  const int kv = j % a.n_kv, head = kv * a.rep + j / a.n_kv;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = tile * BM + wave * 32, n = first + (lane & 31);
  const Place at(a.start, a.n_seq, a.T, offsets_upto(a.start, a.n_seq, first),
                 offsets_upto(a.start, a.n_seq, first + 31), n);
  const Span span = query_span(at, n);
  const uint32_t len = at.live ? n - at.begin + 1 : 0;
  int lo, hi;
  join(span, lds_span, lo, hi);

  const typename TL::Lane L;
  u32x4 q[TL::NS], g[TL::NS];
  hold<T, DP, FULL>(q, (const T*)a.q.p + head * a.q.hs + (int64_t)n * a.q.ld, at.live, a.d);
  hold<T, DP, FULL>(g, (const T*)a.dout.p + head * a.dout.hs + (int64_t)n * a.dout.ld, at.live, a.d);
  const float lse = at.live ? a.lse_in[(int64_t)head * a.T + n] : 0.0f;
  const float delta = at.live ? a.delta[(int64_t)head * a.T + n] : 0.0f;
  const T* kp = (const T*)a.k.p + kv * a.k.hs;
  const T* vp = (const T*)a.v.p + kv * a.v.hs;
  f32x16 dq[TL::ND] = {};
  Stage<T, DP, R, THREADS, FULL> sk, sv;
  const int kt0 = lo / R * R;
  if (lo < hi) {
    sk.load(kp, a.k.ld, kt0, a.T, a.d);
    sv.load(vp, a.v.ld, kt0, a.T, a.d);
    sk.store(lds_k[0]);
    sv.store(lds_v[0]);
  }
  __syncthreads();
  int buf = 0;
  for (int k0 = kt0; k0 < hi; k0 += R, buf ^= 1) {
    const bool more = k0 + R < hi;
    if (more) {
      sk.load(kp, a.k.ld, k0 + R, a.T, a.d);
      sv.load(vp, a.v.ld, k0 + R, a.T, a.d);
    }
    auto step = [&](auto masked_c) {
      constexpr bool MASKED = decltype(masked_c)::value;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x16 s = mul_rows<T, DP>(lds_k[buf], L, b, q);
        const f32x16 dp = mul_rows<T, DP>(lds_v[buf], L, b, g);
        uint32_t ok = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = __builtin_amdgcn_exp2f(weight_log2(s[r], a.scale, lse)) * (dp[r] - delta);
          if constexpr (MASKED) {
            const bool in = (uint32_t)(k0 + 32 * b + acc_row(r) - at.begin) < len;
            ok |= in ? 1u << r : 0u;
            s[r] = in && len > 1 ? s[r] : 0.0f;      // (a row's only key: P is 1 whatever the scores are)
          }
        }
        u32x4 p[TL::NP];
#pragma unroll
        for (int i = 0; i < TL::NP; ++i) p[i] = M::frag(s, i);
        add_cols<T, DP, MASKED>(dq, lds_k[buf], L, b, p, ok);
      }
    };
    if (k0 + R > span.lo && k0 < span.hi) {
      if (k0 >= span.full_lo && k0 + R <= span.full_hi)
        step(std::false_type{});
      else
        step(std::true_type{});
    }
    if (more) {
      sk.store(lds_k[buf ^ 1]);
      sv.store(lds_v[buf ^ 1]);
    }
    __syncthreads();
  }
  put_row<T, DP, FULL>((T*)a.dq.p + head * a.dq.hs + (int64_t)n * a.dq.ld, dq, a.scale, !at.live, n < a.T, a.d);
}

// The key tile, key head and query heads of a workgroup; the first ranks' first
struct KeyTile {
  int rank, kv, split, head, heads;
  __device__ __forceinline__ KeyTile(const AttArgs& a, int b) {
    const int each = a.n_kv * a.splits, j = b % each;
    rank = b / each;
    kv = j % a.n_kv;
    split = j / a.n_kv;
    const int h0 = split * a.rep / a.splits;
    head = kv * a.rep + h0;
    heads = (split + 1) * a.rep / a.splits - h0;
  }
};

// dk and dv of the lane's key, or its part of them
template <typename T, int DP, bool FULL, int ND>
__device__ __forceinline__ void put_keys(const AttArgs& a, const KeyTile& w, int n, const f32x16 (&dk)[ND],
                                         const f32x16 (&dv)[ND], bool live) {
  if (a.splits > 1) {
    const int64_t all = (int64_t)a.T * a.n_kv * a.d;
    float* p = a.part + 2 * w.split * all + ((int64_t)n * a.n_kv + w.kv) * a.d;
    put_row<float, DP, FULL>(p, dk, a.scale, !live, n < a.T, a.d);
    put_row<float, DP, FULL>(p + all, dv, 1.0f, !live, n < a.T, a.d);
  } else {
    put_row<T, DP, FULL>((T*)a.dk.p + w.kv * a.dk.hs + (int64_t)n * a.dk.ld, dk, a.scale, !live, n < a.T, a.d);
    put_row<T, DP, FULL>((T*)a.dv.p + w.kv * a.dv.hs + (int64_t)n * a.dv.ld, dv, 1.0f, !live, n < a.T, a.d);
  }
}

// The parts of dk and dv in order, 8 elements a lane
template <typename T>
__global__ void __launch_bounds__(256) att_join_kernel(AttArgs a) {
  const int per = (a.d + CH - 1) / CH;
  const int64_t rows = (int64_t)a.T * a.n_kv, all = rows * a.d;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per, n = row / a.n_kv;
    const int c = (int)(i - row * per) * CH, kv = (int)(row - n * a.n_kv), some = a.d - c;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const float* p = a.part + which * all + row * a.d + c;
      float f[CH] = {};
      for (int s = 0; s < a.splits; ++s, p += 2 * all) {
        Chunk<float> x;
        if (some >= CH)
          x.load(p);
        else
          x.load_some(p, some);
#pragma unroll
        for (int k = 0; k < CH; ++k) f[k] += x.get(k);
      }
      const HeadsOut& o = which ? a.dv : a.dk;
      T* to = (T*)o.p + n * o.ld + kv * o.hs + c;
      if (some >= CH)
        Chunk<T>::store(to, f);
      else
        Chunk<T>::store_some(to, f, some);
    }
  }
}

// dk and dv: keys in the columns, the rows of Q and do go through LDS, head after head of the group.
template <typename T, int DP, bool FULL>
__global__ void __launch_bounds__(THREADS, 1) att_dkv_kernel(AttArgs a) {
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  constexpr int R = BN<T>, NB = R / 32;
  __shared__ __align__(16) uint8_t lds_q[2][R * TL::ROW], lds_g[2][R * TL::ROW];
  __shared__ __align__(16) float lds_s[2][2][R];     // lse and D of the tile's rows
  __shared__ int lds_span[2][WAVES];
  const KeyTile w(a, blockIdx.x);
  const int tile = a.order[w.rank], kv = w.kv;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = tile * BM + wave * 32, n = first + (lane & 31);
  const Place at(a.start, a.n_seq, a.T, offsets_upto(a.start, a.n_seq, first),
                 offsets_upto(a.start, a.n_seq, first + 31), n);
  // a key is counted by the rows from itself to its sequence's end
  const Span span = {wave_min(at.live ? n : 0x7fffffff), wave_max(at.live ? at.end : 0),
                     wave_max(n), __all(at.live) ? wave_min(at.end) : 0};
  const uint32_t len = at.live ? at.end - n : 0;
  const bool head_of = at.live && at.begin == n;     // the sequence's first token
  int lo, hi;
  join(span, lds_span, lo, hi);

  const typename TL::Lane L;
  u32x4 k[TL::NS], v[TL::NS];
  hold<T, DP, FULL>(k, (const T*)a.k.p + kv * a.k.hs + (int64_t)n * a.k.ld, at.live, a.d);
  hold<T, DP, FULL>(v, (const T*)a.v.p + kv * a.v.hs + (int64_t)n * a.v.ld, at.live, a.d);
  f32x16 dk[TL::ND] = {}, dv[TL::ND] = {};
  Stage<T, DP, R, THREADS, FULL> sq, sg;
  float stat = 0.0f;
  const int t0 = lo / R * R, per = lo < hi ? (hi - t0 + R - 1) / R : 0, steps = per * w.heads;
  auto load = [&](int i) {
    const int head = w.head + i / per, q0 = t0 + (i - i / per * per) * R;
    sq.load((const T*)a.q.p + head * a.q.hs, a.q.ld, q0, a.T, a.d);
    sg.load((const T*)a.dout.p + head * a.dout.hs, a.dout.ld, q0, a.T, a.d);
    const int r = q0 + (threadIdx.x & (R - 1));
    if (threadIdx.x < 2 * R && r < a.T)
      stat = (threadIdx.x < R ? a.lse_in : a.delta)[(int64_t)head * a.T + r];
  };
  auto store = [&](int buf) {
    sq.store(lds_q[buf]);
    sg.store(lds_g[buf]);
    if (threadIdx.x < 2 * R) lds_s[buf][threadIdx.x / R][threadIdx.x & (R - 1)] = stat;
  };
  if (steps > 0) {
    load(0);
    store(0);
  }
  __syncthreads();
  int buf = 0;
  for (int i = 0; i < steps; ++i, buf ^= 1) {
    const int q0 = t0 + (i % per) * R;
    if (i + 1 < steps) load(i + 1);
    auto step = [&](auto masked_c) {
      constexpr bool MASKED = decltype(masked_c)::value;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x16 s = mul_rows<T, DP>(lds_q[buf], L, b, k);
        f32x16 ds = mul_rows<T, DP>(lds_g[buf], L, b, v);
        uint32_t ok = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 z = *(const f32x4*)&lds_s[buf][0][32 * b + acc_row(4 * g)];
          const f32x4 del = *(const f32x4*)&lds_s[buf][1][32 * b + acc_row(4 * g)];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * g + e;
            s[r] = __builtin_amdgcn_exp2f(weight_log2(s[r], a.scale, z[e]));
            ds[r] = s[r] * (ds[r] - del[e]);
            if constexpr (MASKED) {
              const uint32_t after = q0 + 32 * b + acc_row(r) - n;
              const bool in = after < len;
              ok |= in ? 1u << r : 0u;
              s[r] = in ? s[r] : 0.0f;
              ds[r] = in && !(head_of && after == 0) ? ds[r] : 0.0f;   // (the first row's only key)
            }
          }
        }
        u32x4 p[TL::NP], dp[TL::NP];
#pragma unroll
        for (int i2 = 0; i2 < TL::NP; ++i2) {
          p[i2] = M::frag(s, i2);
          dp[i2] = M::frag(ds, i2);
        }
        add_cols<T, DP, MASKED>(dv, lds_g[buf], L, b, p, ok);
        add_cols<T, DP, MASKED>(dk, lds_q[buf], L, b, dp, ok);
      }
    };
    if (q0 + R > span.lo && q0 < span.hi) {
      if (q0 >= span.full_lo && q0 + R <= span.full_hi)
        step(std::false_type{});
      else
        step(std::true_type{});
    }
    if (i + 1 < steps) store(buf ^ 1);
    __syncthreads();
  }
  put_keys<T, DP, FULL>(a, w, n, dk, dv, at.live);
}

// ------------------------------------------------------------------ backward, pipelined
// As in the forward: a slot per MFMA, the vector ALU's share of a half of 32 rows spread over the slots of a phase,
// fragments read AHEAD of their use, tiles of 64 rows copied into rings.  Weights are at most 1, so nothing needs
// a reference; a result that is not finite, or a row whose lse is past FAR, sends the workgroup through its tile again, step by
// step with masked elements taken out.

// lane R of the lane's group of 16, as an operand
template <int R>
__device__ __forceinline__ float row_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x150 + R, 0xf, 0xf, false));
}

// log2 of a weight as the pipeline of dk and dv forms it, from the forward's lse
__device__ __forceinline__ float near_log2(float s, float lse, float sl2) {
#pragma clang fp contract(off)
  const float lse2 = lse * LOG2E, z = lse2 * (1.0f / sl2);
  return (s - z) * sl2;
}

// dk, dv: 32 keys a wave.  A phase forms the next half's S and dP, the previous half's shares of dv and dk, and on the
// vector ALU this half's P and dS.  A ring of four tiles: Q's and do's rows are read a half ahead, their
// columns a half behind.
template <int DP, bool FULL>
__global__ void __launch_bounds__(THREADS, 1) att_dkv_pipe_kernel(AttArgs a) {
  using T = uint16_t;
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  constexpr int NS = TL::NS, ND = TL::ND, NP = TL::NP, ROW = TL::ROW, TB = Copy<DP>::BYTES;
  constexpr int SLOT = 2 * TB, RING = 4 * SLOT, STAT = 2 * 64 * 4;
  __shared__ __align__(16) uint8_t lds[RING];                 // [4][Q, do]
  __shared__ __align__(16) uint8_t lds_s[4 * STAT];           // [4][lse, D][64]
  __shared__ int lds_span[2][WAVES];
  const KeyTile w(a, blockIdx.x);
  const int tile = a.order[w.rank], kv = w.kv, reps = w.heads;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = tile * BM + wave * 32, n = first + (lane & 31);
  const Place at(a.start, a.n_seq, a.T, offsets_upto(a.start, a.n_seq, first),
                 offsets_upto(a.start, a.n_seq, first + 31), n);
  const Span span = {wave_min(at.live ? n : 0x7fffffff), wave_max(at.live ? at.end : 0),
                     wave_max(n), __all(at.live) ? wave_min(at.end) : 0};
  const uint32_t len = at.live ? at.end - n : 0;
  const bool head_of = at.live && at.begin == n;
  int lo, hi;
  join(span, lds_span, lo, hi);
  const int t0 = lo / 64, t1 = lo < hi ? (hi + 63) / 64 : t0, per = t1 - t0, steps = per * reps;
  const int w0 = span.lo < span.hi ? span.lo / 64 : t1, w1 = span.lo < span.hi ? (span.hi + 63) / 64 : t0;
  const int f0 = (span.full_lo + 63) / 64, f1 = span.full_hi / 64;

  const typename TL::Lane L;
  u32x4 k[NS], v[NS];
  Copy<DP> cq, cg;
  cq.init((const T*)a.q.p + (int64_t)w.head * a.q.hs, a.q.ld, lds_address(lds), wave, a.T, a.d);
  cg.init((const T*)a.dout.p + (int64_t)w.head * a.dout.hs, a.dout.ld, lds_address(lds) + TB, wave, a.T, a.d);
  const float* stats = (threadIdx.x < 64 ? a.lse2 : a.delta) + (int64_t)w.head * a.T;
  const float sl2 = a.scale * LOG2E;
  f32x16 dk[ND] = {}, dv[ND] = {};
  constexpr int AHEAD = 7, FR = AHEAD + 1;
  f32x16 s0 = {}, s1 = {}, d0 = {}, d1 = {};
  u32x4 p0[NP], p1[NP], e0[NP], e1[NP], fr[FR];
  float zc = 0.0f, gc = 0.0f, zn, gn;      // lse / scale and D of this half and the next one
  int ko[NS], vo[ND][2], so = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) p0[i] = p1[i] = e0[i] = e1[i] = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < FR; ++i) fr[i] = u32x4{0, 0, 0, 0};

  auto read_col = [&](int off, int s, int c) {
    const uint8_t* x = lds + off + s * 16 * ROW;
    const u32x2 u = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + vo[c][0])));
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + vo[c][1] + 8 * ROW)));
    return u32x4{u.x, u.y, w.x, w.y};
  };
  // Row statistics of a half: lane r of a group of 16 reads those of accumulator row r, and the VALU's own broadcast
  // within 16 lanes hands them out (16-byte reads by every lane were a fifth of the LDS's time)
  auto read_stat = [&](int half) {
    zn = *(const float*)(lds_s + so + half * 128);
    gn = *(const float*)(lds_s + so + half * 128 + 256);
  };
  // this half's P and dS from s, d into pn, en; the next half's scores and dP into sn, dn; the previous half's pp, ep
  // into dv and dk.  move: as in the forward, so after its last read of the tile.
  auto phase = [&](auto first_c, auto masked_c, f32x16& s, f32x16& d, f32x16& sn, f32x16& dn, u32x4 (&pp)[NP],
                   u32x4 (&ep)[NP], u32x4 (&pn)[NP], u32x4 (&en)[NP], int move, int smove, int q0) {
    constexpr bool FIRST = decltype(first_c)::value, MASKED = decltype(masked_c)::value;
    constexpr int KH = FIRST ? 1 : 0, NC = NP * ND, NM = 2 * NS + 2 * NC;
    const uint32_t from = q0 + 4 * (lane >> 5) - n;
    slots<NM>([&](auto slot) {
      constexpr int i = slot.value, rd = i + AHEAD;
      if constexpr (rd < 2 * NS)
        fr[rd % FR] = *(const u32x4*)(lds + KH * 32 * ROW + (rd & 1) * TB + ko[rd / 2]);
      else if constexpr (rd < NM) {
        constexpr int c = (rd - 2 * NS) / 2;
        fr[rd % FR] = read_col(KH * 32 * ROW + (rd & 1 ? 0 : TB), c / ND, c % ND);
      } else {
        fr[rd % FR] = *(const u32x4*)(lds + (KH ^ 1) * 32 * ROW + (rd & 1) * TB + ko[(rd - NM) / 2]);
      }
      // (two sums in turn: one behind the other the matrix core waits for each product's result)
      constexpr int c = (i - 2 * NS) / 2;
      if constexpr (i < 2 * NS && i % 2 == 0)
        sn = M::mma(fr[i % FR], k[i / 2], i == 0 ? f32x16{} : sn);
      else if constexpr (i < 2 * NS)
        dn = M::mma(fr[i % FR], v[i / 2], i == 1 ? f32x16{} : dn);
      else if constexpr (i % 2 == 0)
        dv[c % ND] = M::mma(fr[i % FR], pp[c / ND], dv[c % ND]);
      else
        dk[c % ND] = M::mma(fr[i % FR], ep[c / ND], dk[c % ND]);
      if constexpr (FIRST && i >= 2 * NS && i < 3 * NS) ko[i - 2 * NS] += move;
      if constexpr (!FIRST && i == 0)
#pragma unroll
        for (int c = 0; c < ND; ++c) vo[c][0] += move, vo[c][1] += move;
      // a value takes two slots: the exponent, then the exponential and the rest
      slots<16>([&](auto e_c) {
        constexpr int r = e_c.value, sl = r * NM / 16;
        float x = s[r], y = d[r];
        bool in = true;
        if constexpr (MASKED) in = from + 8 * (r >> 2) + (r & 3) < len;
        if constexpr (sl == i) {
          x = (x - row_lane<r>(zc)) * sl2;
          if constexpr (MASKED) x = in ? x : -INFINITY;
        }
        if constexpr (sl + 1 == i || (sl == i && i + 1 == NM)) {
          x = __builtin_amdgcn_exp2f(x);
          y = x * (y - row_lane<r>(gc));
          if constexpr (MASKED) y = in && !(head_of && from + 8 * (r >> 2) + (r & 3) == 0) ? y : 0.0f;
          if constexpr (r & 1) {
            uint32_t w = M::pack(s[r - 1], x), z = M::pack(d[r - 1], y);
            asm volatile("" : "+v"(w), "+v"(z));              // (here, not where it is used)
            pn[r >> 3][(r & 7) >> 1] = w;
            en[r >> 3][(r & 7) >> 1] = z;
          }
        }
        s[r] = x;
        d[r] = y;
      });
      if constexpr (i == NM / 2) {
        if constexpr (!FIRST) so += smove;
        read_stat(FIRST ? 1 : 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    zc = zn;
    gc = gn;
  };

  // Step u of the walk: all heads of the group at one tile, from the last tile to the first.  Key tiles of one sequence
  // then start on the same rows and stay with each other, sharing them through the XCD's L2.
  float stat = 0.0f;
  float to_stat = threadIdx.x < 64 ? 1.0f / sl2 : 1.0f;
  auto load_stat = [&](int u) {
    const int row = (t1 - 1 - u / reps) * 64 + (threadIdx.x & 63);
    if (threadIdx.x < 128 && u < steps && row < a.T) stat = stats[(int64_t)(u % reps) * a.T + row];
  };
  auto put_stat = [&](int u) {
    if (threadIdx.x < 128) *(float*)(lds_s + (u & 3) * STAT + threadIdx.x * 4) = stat * to_stat;
  };
  auto copy = [&](int u) {
    if (u >= steps) return;
    const int up = u / reps, h = u - up * reps, row = (t1 - 1 - up) * 64;
    cq.tile(row, (u & 3) * SLOT, (int64_t)h * a.q.hs * 2);
    cg.tile(row, (u & 3) * SLOT, (int64_t)h * a.dout.hs * 2);
  };
  auto begin = [&]() {
    if (steps == 0) return;
    load_stat(0);
    put_stat(0);
    load_stat(1);
    put_stat(1);
    load_stat(2);
    copy(0);
    copy(1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  // Step u's rows and the next one's have landed, those of the one after are on their way.  Statistics are written two
  // steps ahead: a wave that reads fragments in between has seen its write done before the next barrier,
  // and needs no wait that would drain them; one that does not (idle) waits.
  auto arrive = [&](int u, bool idle) {
    if (idle) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    put_stat(u + 2);
    load_stat(u + 3);
    copy(u + 2);
  };
  begin();
  hold<T, DP, FULL>(k, (const T*)a.k.p + kv * a.k.hs + (int64_t)n * a.k.ld, at.live, a.d);
  hold<T, DP, FULL>(v, (const T*)a.v.p + kv * a.v.hs + (int64_t)n * a.v.ld, at.live, a.d);
  const int ua = w0 < w1 ? (t1 - w1) * reps : steps, ub = w0 < w1 ? (t1 - w0) * reps : steps;
  int u = 0;
  for (; u < ua; ++u) arrive(u, true);
  if (u < ub) {
    arrive(u, true);
    const int at_q = (u & 3) * SLOT;
#pragma unroll
    for (int s = 0; s < NS; ++s) ko[s] = (L.row ^ (s << 5)) + at_q;
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      vo[c][0] = (L.tr ^ (c << 6)) + at_q;
      vo[c][1] = (L.tr ^ (c << 6) ^ 32) + at_q;
    }
    so = (u & 3) * STAT + (8 * ((lane & 15) >> 2) + (lane & 3) + 4 * (lane >> 5)) * 4;
    s0 = mul_rows<T, DP>(lds + at_q, L, 0, k);
    d0 = mul_rows<T, DP>(lds + at_q + TB, L, 0, v);
#pragma unroll
    for (int i = 0; i < NP; ++i) p1[i] = e1[i] = u32x4{0, 0, 0, 0};
    read_stat(0);
    zc = zn;
    gc = gn;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      fr[i] = *(const u32x4*)(lds + 32 * ROW + (i & 1) * TB + ko[i / 2]);
    static_assert((2 * NS + 2 * NP * ND) % FR == 0, "a phase starts at the ring's first fragment");
    int vmove = 0;
    auto through = [&](auto masked_c, int until) {
      while (u < until) {
        const int kmove = (u & 3) == 3 ? -3 * SLOT : SLOT, smove = (u & 3) == 3 ? -3 * STAT : STAT;
        const int q0 = decltype(masked_c)::value ? (t1 - 1 - u / reps) * 64 : 0;
        phase(std::true_type{}, masked_c, s0, d0, s1, d1, p1, e1, p0, e0, kmove, 0, q0);
        phase(std::false_type{}, masked_c, s1, d1, s0, d0, p0, e0, p1, e1, vmove, smove, q0 + 32);
        vmove = kmove;
        if (++u < ub) arrive(u, false);
      }
    };
    through(std::true_type{}, min((t1 - min(f1, t1)) * reps, ub));
    through(std::false_type{}, min((t1 - min(f0, t1)) * reps, ub));
    through(std::true_type{}, ub);
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
      for (int c = 0; c < ND; ++c) {
        dv[c] = M::mma(read_col(32 * ROW + TB, s, c), p1[s], dv[c]);
        dk[c] = M::mma(read_col(32 * ROW, s, c), e1[s], dk[c]);
      }
  }
  for (; u < steps; ++u) arrive(u, true);
  float bad = 0.0f;
#pragma unroll
  for (int c = 0; c < ND; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) bad = fmaf(dk[c][r], 0.0f, fmaf(dv[c][r], 0.0f, bad));
  // Rows past FAR: looked for where some row of the stream is one.  (A maximum kept where the statistics pass by cost the
  // pipeline 4%, a look at all of the tile's rows each time 1.5%.)
  bool far = false;
  const u32x4 some = ((const u32x4*)a.far)[threadIdx.x];
  if (__syncthreads_or((some.x | some.y | some.z | some.w) != 0))
    for (int h = 0; h < reps; ++h) {
      const float* z = a.lse2 + (int64_t)(w.head + h) * a.T;
      for (int r = lo + threadIdx.x; r < hi; r += THREADS) far = far || fabsf(z[r]) > FAR;
    }
  if (__syncthreads_or((at.live && bad != 0.0f) || far)) {
#pragma unroll
    for (int c = 0; c < ND; ++c) dk[c] = dv[c] = f32x16{};
    if (threadIdx.x < 64) stats = a.lse_in + (int64_t)w.head * a.T;
    to_stat = 1.0f;
    begin();
    for (u = 0; u < steps; ++u) {
        arrive(u, true);
        const int t = t1 - 1 - u / reps;
        if (t < w0 || t >= w1) continue;
        const uint8_t* q = lds + (u & 3) * SLOT;
#pragma unroll 1
        for (int b = 0; b < 2; ++b) {
          f32x16 s = mul_rows_upto<T, DP, FULL>(q + b * 32 * ROW, L, 0, k, a.d);
          f32x16 ds = mul_rows_upto<T, DP, FULL>(q + b * 32 * ROW + TB, L, 0, v, a.d);
          const float* st = (const float*)(lds_s + (u & 3) * STAT) + 32 * b;
          uint32_t ok = 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const uint32_t after = t * 64 + 32 * b + acc_row(r) - n;
            const bool in = after < len;
            ok |= in ? 1u << r : 0u;
            const float lse = st[acc_row(r)];
            const float x = fabsf(lse * LOG2E) <= FAR ? near_log2(s[r], lse, sl2) : weight_log2(s[r], a.scale, lse);
            s[r] = __builtin_amdgcn_exp2f(in ? x : -INFINITY);
            ds[r] = in && !(head_of && after == 0) ? s[r] * (ds[r] - st[64 + acc_row(r)]) : 0.0f;
            s[r] = in ? s[r] : 0.0f;
          }
          u32x4 p[NP], e[NP];
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            p[i] = M::frag(s, i);
            e[i] = M::frag(ds, i);
          }
          add_cols<T, DP, true>(dv, q + b * 32 * ROW + TB, L, 0, p, ok);
          add_cols<T, DP, true>(dk, q + b * 32 * ROW, L, 0, e, ok);
        }
      }
  }
  put_keys<T, DP, FULL>(a, w, n, dk, dv, at.live);
}

// dq: 64 queries a wave.  A phase forms the next half's S, this half's dP and the previous half's share of dq; on the
// vector ALU this half's P, then, behind dP, dS.
template <int DP, bool FULL>
__global__ void __launch_bounds__(THREADS, 1) att_dq_pipe_kernel(AttArgs a) {
  using T = uint16_t;
  using TL = Tile<T, DP>;
  using M = Mma<T>;
  constexpr int NS = TL::NS, ND = TL::ND, NP = TL::NP, ROW = TL::ROW, TB = Copy<DP>::BYTES;
  __shared__ __align__(16) uint8_t lds_k[4 * TB], lds_v[2 * TB];
  __shared__ int lds_span[2][WAVES];
  if (a.err) check_offsets(a.start, a.n_seq, a.T, a.err);
  const int tiles = (a.T + PIPE_ROWS - 1) / PIPE_ROWS;
  const int tile = tiles - 1 - blockIdx.x / a.n_head, j = blockIdx.x % a.n_head;
  const int kv = j % a.n_kv, head = kv * a.rep + j / a.n_kv;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = tile * PIPE_ROWS + wave * 64;
  const int nA = first + (lane & 31), nB = nA + 32;
  const int upto0 = offsets_upto(a.start, a.n_seq, first), upto1 = offsets_upto(a.start, a.n_seq, first + 63);
  const Place at[2] = {Place(a.start, a.n_seq, a.T, upto0, upto1, nA),
                       Place(a.start, a.n_seq, a.T, upto0, upto1, nB)};
  const Span part[2] = {query_span(at[0], nA), query_span(at[1], nB)};
  const Span span = {min(part[0].lo, part[1].lo), max(part[0].hi, part[1].hi),
                     max(part[0].full_lo, part[1].full_lo), min(part[0].full_hi, part[1].full_hi)};
  int lo, hi;
  join(span, lds_span, lo, hi);
  const int t0 = lo / 64, t1 = lo < hi ? (hi + 63) / 64 : t0;
  const int w0 = span.lo < span.hi ? span.lo / 64 : t1, w1 = span.lo < span.hi ? (span.hi + 63) / 64 : t0;
  const int f0 = (span.full_lo + 63) / 64, f1 = span.full_hi / 64;

  const typename TL::Lane L;
  u32x4 q[2][NS], g[2][NS];
  float lse2[2], delta[2];
  uint32_t len[2];
  Copy<DP> ck, cv;
  ck.init((const T*)a.k.p + kv * a.k.hs, a.k.ld, lds_address(lds_k), wave, a.T, a.d);
  cv.init((const T*)a.v.p + kv * a.v.hs, a.v.ld, lds_address(lds_v), wave, a.T, a.d);
  const float sl2 = a.scale * LOG2E;
  f32x16 dq[2][ND] = {};
  constexpr int AHEAD = DP == 128 ? 7 : 3, FR = AHEAD + 1;
  static_assert(AHEAD <= NS, "what is read ahead of a phase is K");
  f32x16 s0[2], s1[2], dp[2];
  u32x4 e0[2][NP], e1[2][NP], fr[FR];
  int ko[NS], go[NS], vo[ND][2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    s0[b] = s1[b] = dp[b] = f32x16{};
#pragma unroll
    for (int i = 0; i < NP; ++i) e0[b][i] = e1[b][i] = u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < FR; ++i) fr[i] = u32x4{0, 0, 0, 0};
  auto read_col = [&](int half, int s, int c) {
    const uint8_t* x = lds_k + (half * 32 + s * 16) * ROW;
    const u32x2 u = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + vo[c][0])));
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + vo[c][1] + 8 * ROW)));
    return u32x4{u.x, u.y, w.x, w.y};
  };
  auto phase = [&](auto first_c, auto masked_c, f32x16 (&cur)[2], f32x16 (&nxt)[2], u32x4 (&ep)[2][NP],
                   u32x4 (&en)[2][NP], int move, int gmove, int key0) {
    constexpr bool FIRST = decltype(first_c)::value, MASKED = decltype(masked_c)::value;
    // S reads half KH of ko's tile, dP half GH of go's, dq half KH of vo's
    constexpr int KH = FIRST ? 1 : 0, GH = FIRST ? 0 : 1;
    constexpr int NQ = 2 * NS, NC = 2 * NP * ND, NM = 2 * NQ + NC, NF = NM / 2, LATE = 2 * NQ + NM / 24;
    const int from[2] = {key0 + 4 * (lane >> 5) - at[0].begin, key0 + 4 * (lane >> 5) - at[1].begin};
    slots<NM>([&](auto slot) {
      constexpr int i = slot.value, fi = i / 2, b = i & 1;
      if constexpr (b == 0) {
        constexpr int n = fi + AHEAD;
        if constexpr (n < NS)
          fr[n % FR] = *(const u32x4*)(lds_k + KH * 32 * ROW + ko[n]);
        else if constexpr (n < 2 * NS)
          fr[n % FR] = *(const u32x4*)(lds_v + GH * 32 * ROW + go[n - NS]);
        else if constexpr (n < NF)
          fr[n % FR] = read_col(KH, (n - 2 * NS) / ND, (n - 2 * NS) % ND);
        else
          fr[n % FR] = *(const u32x4*)(lds_k + (KH ^ 1) * 32 * ROW + ko[n - NF]);
      }
      if constexpr (fi < NS)
        nxt[b] = M::mma(fr[fi % FR], q[b][fi], fi == 0 ? f32x16{} : nxt[b]);
      else if constexpr (fi < 2 * NS)
        dp[b] = M::mma(fr[fi % FR], g[b][fi - NS], fi == NS ? f32x16{} : dp[b]);
      else
        dq[b][(fi - 2 * NS) % ND] = M::mma(fr[fi % FR], ep[b][(fi - 2 * NS) / ND], dq[b][(fi - 2 * NS) % ND]);
      if constexpr (FIRST && i >= NQ && i < NQ + NS) ko[i - NQ] += move;
      if constexpr (!FIRST && i < 2 * ND) vo[i >> 1][i & 1] += move;
      if constexpr (!FIRST && i >= 2 * NQ && i < 2 * NQ + NS) go[i - 2 * NQ] += gmove;
      slots<32>([&](auto e_c) {
        constexpr int e = e_c.value, cb = e >> 4, r = e & 15, EPS = 16 / NS;
        constexpr int late = LATE + e * (NM - LATE) / 32;
        if constexpr (e / EPS == i) {
          float x = cur[cb][r];
          if constexpr (MASKED) {
            const bool in = (uint32_t)(from[cb] + 8 * (r >> 2) + (r & 3)) < len[cb];
            x = in ? x : -INFINITY;
          }
          cur[cb][r] = fmaf(x, sl2, -lse2[cb]);
        }
        if constexpr (e / EPS + 1 == i) cur[cb][r] = __builtin_amdgcn_exp2f(cur[cb][r]);
        if constexpr (late == i) {
          float x = cur[cb][r] * (dp[cb][r] - delta[cb]);
          if constexpr (MASKED) {
            const bool in = (uint32_t)(from[cb] + 8 * (r >> 2) + (r & 3)) < len[cb] && len[cb] > 1;
            x = in ? x : 0.0f;
          }
          cur[cb][r] = x;
          if constexpr (r & 1) {
            uint32_t w = M::pack(cur[cb][r - 1], x);
            asm volatile("" : "+v"(w));                       // (here, not where it is used)
            en[cb][r >> 3][(r & 7) >> 1] = w;
          }
        }
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  int u = 0;           // tile t - t0
  auto begin = [&]() {
    u = 0;
    if (t0 >= t1) return;
    ck.tile(t0 * 64, 0);
    if (t0 + 1 < t1) ck.tile(t0 * 64 + 64, TB);
    cv.tile(t0 * 64, 0);
  };
  auto arrive = [&](int t) {
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 2 < t1) ck.tile(t * 64 + 128, (u + 2 & 3) * TB);
    if (t + 1 < t1) cv.tile(t * 64 + 64, (u + 1 & 1) * TB);
  };
  begin();
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const int n = cb ? nB : nA;
    hold<T, DP, FULL>(q[cb], (const T*)a.q.p + head * a.q.hs + (int64_t)n * a.q.ld, at[cb].live, a.d);
    hold<T, DP, FULL>(g[cb], (const T*)a.dout.p + head * a.dout.hs + (int64_t)n * a.dout.ld, at[cb].live, a.d);
    lse2[cb] = at[cb].live ? a.lse2[(int64_t)head * a.T + n] : 0.0f;
    delta[cb] = at[cb].live ? a.delta[(int64_t)head * a.T + n] : 0.0f;
    len[cb] = at[cb].live ? n - at[cb].begin + 1 : 0;
  }
  int t = t0;
  for (; t < min(w0, t1); ++t, ++u) arrive(t);
  if (t < w1) {
    arrive(t);
    const int at_k = (u & 3) * TB;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      ko[s] = (L.row ^ (s << 5)) + at_k;
      go[s] = (L.row ^ (s << 5)) + (u & 1) * TB;
    }
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      vo[c][0] = (L.tr ^ (c << 6)) + at_k;
      vo[c][1] = (L.tr ^ (c << 6) ^ 32) + at_k;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s0[b] = mul_rows<T, DP>(lds_k + at_k, L, 0, q[b]);
#pragma unroll
      for (int i = 0; i < NP; ++i) e1[b][i] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fr[i] = *(const u32x4*)(lds_k + 32 * ROW + ko[i]);
    static_assert((2 * NS + NP * ND) % FR == 0, "a phase starts at the ring's first fragment");
    int vmove = 0;
    auto through = [&](auto masked_c, int until) {
      while (t < until) {
        const int kmove = (u & 3) == 3 ? -3 * TB : TB, gmove = u & 1 ? -TB : TB;
        phase(std::true_type{}, masked_c, s0, s1, e1, e0, kmove, 0, t * 64);
        phase(std::false_type{}, masked_c, s1, s0, e0, e1, vmove, gmove, t * 64 + 32);
        vmove = kmove;
        ++u;
        if (++t < w1) arrive(t);
      }
    };
    through(std::true_type{}, min(f0, w1));
    through(std::false_type{}, min(f1, w1));
    through(std::true_type{}, w1);
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
      for (int c = 0; c < ND; ++c) {
        const u32x4 x = read_col(1, s, c);
        dq[0][c] = M::mma(x, e1[0][s], dq[0][c]);
        dq[1][c] = M::mma(x, e1[1][s], dq[1][c]);
      }
  }
  for (; t < t1; ++t, ++u) arrive(t);
  bool lost = false;
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    float z = 0.0f;
#pragma unroll
    for (int c = 0; c < ND; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) z = fmaf(dq[cb][c][r], 0.0f, z);
    lost = lost || (at[cb].live && (z != 0.0f || !(fabsf(lse2[cb]) <= FAR)));
  }
  if (__syncthreads_or(lost)) {
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
      for (int c = 0; c < ND; ++c) dq[cb][c] = f32x16{};
    begin();
    for (t = t0; t < t1; ++t, ++u) {
      arrive(t);
      const uint8_t *k = lds_k + (u & 3) * TB, *v = lds_v + (u & 1) * TB;
#pragma unroll
      for (int cb = 0; cb < 2; ++cb) {
        if (t * 64 + 64 <= part[cb].lo || t * 64 >= part[cb].hi) continue;
        const float lse = at[cb].live ? a.lse_in[(int64_t)head * a.T + (cb ? nB : nA)] : 0.0f;
#pragma unroll 1
        for (int b = 0; b < 2; ++b) {
          f32x16 s = mul_rows_upto<T, DP, FULL>(k + b * 32 * ROW, L, 0, q[cb], a.d);
          const f32x16 d = mul_rows_upto<T, DP, FULL>(v + b * 32 * ROW, L, 0, g[cb], a.d);
          uint32_t ok = 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool in = (uint32_t)(t * 64 + 32 * b + acc_row(r) - at[cb].begin) < len[cb];
            ok |= in ? 1u << r : 0u;
            s[r] = in ? s[r] : -INFINITY;
            s[r] = __builtin_amdgcn_exp2f(fabsf(lse2[cb]) <= FAR ? fmaf(s[r], sl2, -lse2[cb])
                                                                 : weight_log2(s[r], a.scale, lse));
            s[r] = in && len[cb] > 1 ? s[r] * (d[r] - delta[cb]) : 0.0f;
          }
          u32x4 e[NP];
#pragma unroll
          for (int i = 0; i < NP; ++i) e[i] = M::frag(s, i);
          add_cols<T, DP, true>(dq[cb], k + b * 32 * ROW, L, 0, e, ok);
        }
      }
    }
  }
#pragma unroll
  for (int cb = 0; cb < 2; ++cb) {
    const int n = cb ? nB : nA;
    put_row<T, DP, FULL>((T*)a.dq.p + head * a.dq.hs + (int64_t)n * a.dq.ld, dq[cb], a.scale, !at[cb].live, n < a.T,
                         a.d);
  }
}

constexpr int32_t ATT_MAX_D = 128;
constexpr int64_t ATT_MAX_T = ((int64_t)1 << 31) - 65536;
constexpr int64_t ATT_MAX_TILES = ((int64_t)1 << 24) - 1;      // workgroups of 256: less than the 2^32 lanes that HIP takes

int att_check(const char* fn, int64_t T, int32_t n_seq, int32_t n_head, int32_t n_kv, int32_t d, int32_t dtype,
              float scale) {
  if (dtype != AGRL_BF16 && dtype != AGRL_F32)
    return fail(AGRL_E_DTYPE, fn, "dtype must be AGRL_BF16 or AGRL_F32");
  if (T < 0 || T > ATT_MAX_T || n_seq < 0 || n_seq > (1 << 30))
    return fail(AGRL_E_SHAPE, fn, "bad T or n_seq");
  if (n_head <= 0 || n_kv <= 0 || n_head % n_kv || d <= 0)
    return fail(AGRL_E_SHAPE, fn, "n_head must be a multiple of n_kv, d positive");
  if (cdiv(T, (int64_t)BM) * n_head > ATT_MAX_TILES) return fail(AGRL_E_SHAPE, fn, "T n_head is too large");
  if (d > ATT_MAX_D) return fail(AGRL_E_UNSUPPORTED, fn, "d is larger than 128");
  // (the backward divides lse by it)
  if (!(scale >= 0x1p-60f && scale <= 0x1p60f))
    return fail(AGRL_E_FLAGS, fn, "scale must be in [2^-60, 2^60]");
  return AGRL_OK;
}
int att_strides(const char* fn, int64_t ld, int64_t hs) {
  return ld < 0 || hs < 0 ? fail(AGRL_E_SHAPE, fn, "a stride is negative") : AGRL_OK;
}

// Parts that the heads of a group are dealt to where the key tiles alone do not fill the chip's 256 units.  How long a tile is
// the host does not know: long ones gain, tiles of short sequences have little to share out and pay for the join.  Whole
// backward, by this rule and in one part:
//                                         one sequence      four             of 33 tokens
//   1519 tokens, 4/2 heads of 64 fp32     444 and 671 us    259 and 392      75 and 97
//   2048, 16/2 of 128 bf16 (8 parts)      171 and 518       118 and 283      77 and 104
//   4096, 28/4 of 128 (2 parts)           636 and 919       348 and 487      136 and 138
//   7168, 28/4 of 128 (2 parts)           1352 and 1790     659 and 887      241 and 200
// Where the tiles do fill it a part costs more than it evens out: 8191 tokens of 16 heads over 4 in short sequences, 256 key
// tiles, dk and dv 45 us in one, 91 in four.
int att_splits(int64_t T, int32_t n_head, int32_t n_kv) {
  const int64_t items = cdiv(T, (int64_t)BM) * n_kv, want = cdiv((int64_t)256, items), rep = n_head / n_kv;
  return (int)(want < rep ? want : rep);
}

struct AttSpace {
  size_t delta, order, far, part, total;
};
AttSpace att_space(int64_t T, int32_t n_head, int32_t n_kv, int32_t d) {
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  const int splits = att_splits(T, n_head, n_kv);
  AttSpace s;
  s.delta = up((size_t)T * n_head * 4);
  s.order = 2 * s.delta;
  s.far = s.order + up((size_t)cdiv(T, (int64_t)BM) * 4);
  s.part = s.far + FLAGS;
  s.total = s.part + (splits > 1 ? (size_t)splits * 2 * T * n_kv * d * 4 : 0);
  return s;
}

// Whether 16-byte copies reach every row of a bf16 operand, 64 rows within 32-bit offsets
bool copies(const Heads& h) {
  return (uintptr_t)h.p % 16 == 0 && h.ld % 8 == 0 && h.hs % 8 == 0 && h.ld < (1 << 24);
}

// f(padded head size, whether it is the head size)
template <class F>
void att_size(int32_t d, F&& f) {
  if (d == 128)
    f(std::integral_constant<int, 128>{}, std::true_type{});
  else if (d == 64)
    f(std::integral_constant<int, 64>{}, std::true_type{});
  else if (d > 64)
    f(std::integral_constant<int, 128>{}, std::false_type{});
  else
    f(std::integral_constant<int, 64>{}, std::false_type{});
}
// f(element type, padded head size, whether it is the head size)
template <class F>
void att_pick(int32_t dtype, int32_t d, F&& f) {
  att_size(d, [&](auto dp, auto full) {
    if (dtype == AGRL_BF16)
      f(uint16_t{}, dp, full);
    else
      f(float{}, dp, full);
  });
}

}  // namespace
}  // namespace agrl

extern "C" int agrl_attention_fwd(int64_t T, int32_t n_seq, int32_t n_head, int32_t n_kv, int32_t d,
                                  int32_t dtype, const void* q, int64_t ld_q, int64_t head_q,
                                  const void* k, int64_t ld_k, int64_t head_k, const void* v,
                                  int64_t ld_v, int64_t head_v, const int32_t* seq_start, float scale,
                                  void* o, int64_t ld_o, int64_t head_o, float* lse, void* stream) {
  using namespace agrl;
  const char* fn = "agrl_attention_fwd";
  int rc = att_check(fn, T, n_seq, n_head, n_kv, d, dtype, scale);
  if (!rc) rc = att_strides(fn, ld_q, head_q);
  if (!rc) rc = att_strides(fn, ld_k, head_k);
  if (!rc) rc = att_strides(fn, ld_v, head_v);
  if (rc) return rc;
  if (!heads_apart(T, n_head, d, ld_o, head_o)) return fail(AGRL_E_SHAPE, fn, "the heads of o overlap");
  if (T == 0) return AGRL_OK;
  if (!q || !k || !v || !o || !seq_start) return fail(AGRL_E_NULL, fn, "q, k, v, o or seq_start is NULL");
  AttArgs a = {};
  a.T = (int32_t)T, a.n_seq = n_seq, a.n_head = n_head, a.n_kv = n_kv, a.rep = n_head / n_kv, a.d = d;
  a.q = {q, ld_q, head_q}, a.k = {k, ld_k, head_k}, a.v = {v, ld_v, head_v};
  a.start = seq_start, a.scale = scale, a.o = {o, ld_o, head_o}, a.lse = lse, a.err = device_error_ptr();
  if (dtype == AGRL_BF16 && d % 8 == 0 && copies(a.k) && copies(a.v)) {
    const dim3 grid((unsigned)(cdiv(T, (int64_t)PIPE_ROWS) * n_head));
    att_size(d, [&](auto dp, auto full) {
      hipLaunchKernelGGL((att_fwd_pipe_kernel<decltype(dp)::value, decltype(full)::value>), grid, dim3(THREADS), 0,
                         (hipStream_t)stream, a);
    });
    return hip_status(hipGetLastError());
  }
  att_pick(dtype, d, [&](auto z, auto dp, auto full) {
    hipLaunchKernelGGL((att_fwd_kernel<decltype(z), decltype(dp)::value, decltype(full)::value>),
                       dim3((unsigned)(cdiv(T, (int64_t)BM) * n_head)), dim3(THREADS), 0, (hipStream_t)stream, a);
  });
  return hip_status(hipGetLastError());
}

extern "C" size_t agrl_attention_bwd_workspace_size(int64_t T, int32_t n_head, int32_t n_kv, int32_t d,
                                                    int32_t dtype) {
  using namespace agrl;
  if ((dtype != AGRL_BF16 && dtype != AGRL_F32) || T <= 0 || T > ATT_MAX_T || n_head <= 0 || n_kv <= 0 ||
      n_head % n_kv || d <= 0 || d > ATT_MAX_D || cdiv(T, (int64_t)BM) * n_head > ATT_MAX_TILES)
    return 0;
  return att_space(T, n_head, n_kv, d).total;
}

extern "C" int agrl_attention_bwd(int64_t T, int32_t n_seq, int32_t n_head, int32_t n_kv, int32_t d,
                                  int32_t dtype, const void* q, int64_t ld_q, int64_t head_q,
                                  const void* k, int64_t ld_k, int64_t head_k, const void* v,
                                  int64_t ld_v, int64_t head_v, const int32_t* seq_start, float scale,
                                  const void* o, int64_t ld_o, int64_t head_o, const float* lse,
                                  const void* dout, int64_t ld_do, int64_t head_do, void* workspace,
                                  size_t ws_bytes, void* dq, int64_t ld_dq, int64_t head_dq, void* dk,
                                  int64_t ld_dk, int64_t head_dk, void* dv, int64_t ld_dv,
                                  int64_t head_dv, void* stream) {
  using namespace agrl;
  const char* fn = "agrl_attention_bwd";
  int rc = att_check(fn, T, n_seq, n_head, n_kv, d, dtype, scale);
  if (!rc) rc = att_strides(fn, ld_q, head_q);
  if (!rc) rc = att_strides(fn, ld_k, head_k);
  if (!rc) rc = att_strides(fn, ld_v, head_v);
  if (!rc) rc = att_strides(fn, ld_o, head_o);
  if (!rc) rc = att_strides(fn, ld_do, head_do);
  if (rc) return rc;
  if (!heads_apart(T, n_head, d, ld_dq, head_dq) || !heads_apart(T, n_kv, d, ld_dk, head_dk) ||
      !heads_apart(T, n_kv, d, ld_dv, head_dv))
    return fail(AGRL_E_SHAPE, fn, "the heads of dq, dk or dv overlap");
  if (T == 0) return AGRL_OK;
  if (!q || !k || !v || !seq_start || !o || !lse || !dout)
    return fail(AGRL_E_NULL, fn, "q, k, v, seq_start, o, lse or dout is NULL");
  if (!dq || !dk || !dv) return fail(AGRL_E_NULL, fn, "dq, dk or dv is NULL");
  if (!workspace || ws_bytes < agrl_attention_bwd_workspace_size(T, n_head, n_kv, d, dtype))
    return fail(AGRL_E_WORKSPACE, fn, "workspace missing or too small");
  if ((uintptr_t)workspace % 256 != 0)
    return fail(AGRL_E_UNSUPPORTED, fn, "workspace must be 256-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const AttSpace sp = att_space(T, n_head, n_kv, d);
  uint8_t* ws = (uint8_t*)workspace;
  float* lse2 = (float*)ws;
  float* delta = (float*)(ws + sp.delta);
  int32_t* order = (int32_t*)(ws + sp.order);
  uint8_t* far = ws + sp.far;
  const DeltaArgs de = {(int32_t)T, n_head, d, n_seq, {o, ld_o, head_o}, {dout, ld_do, head_do}, lse, lse2, delta,
                        seq_start, order, far};
  const int64_t need = cdiv(T * n_head, (int64_t)16), most = (int64_t)device_cu_count() * 16;
  const int64_t dwork = need < most ? need : most;
  const dim3 dgrid((unsigned)(dwork < FLAGS ? dwork : FLAGS) + 1);
  if (dtype == AGRL_BF16)
    hipLaunchKernelGGL(att_delta_kernel<uint16_t>, dgrid, dim3(256), 0, s, de);
  else
    hipLaunchKernelGGL(att_delta_kernel<float>, dgrid, dim3(256), 0, s, de);
  AttArgs a = {};
  a.T = (int32_t)T, a.n_seq = n_seq, a.n_head = n_head, a.n_kv = n_kv, a.rep = n_head / n_kv, a.d = d;
  a.q = {q, ld_q, head_q}, a.k = {k, ld_k, head_k}, a.v = {v, ld_v, head_v};
  a.start = seq_start, a.scale = scale, a.err = device_error_ptr();
  a.dout = {dout, ld_do, head_do}, a.lse_in = lse, a.lse2 = lse2, a.delta = delta, a.order = order, a.far = far;
  a.splits = att_splits(T, n_head, n_kv), a.part = (float*)(ws + sp.part);
  a.dq = {dq, ld_dq, head_dq}, a.dk = {dk, ld_dk, head_dk}, a.dv = {dv, ld_dv, head_dv};
  const int64_t tiles = cdiv(T, (int64_t)BM);
  const bool pipe = dtype == AGRL_BF16 && d % 8 == 0 && copies(a.q) && copies(a.k) && copies(a.v) && copies(a.dout);
  const dim3 kgrid((unsigned)(tiles * n_kv * a.splits)), block(THREADS);
  if (pipe) {
    const dim3 qgrid((unsigned)(cdiv(T, (int64_t)PIPE_ROWS) * n_head));
    att_size(d, [&](auto dp, auto full) {
      constexpr int DP = decltype(dp)::value;
      constexpr bool FULL = decltype(full)::value;
      hipLaunchKernelGGL((att_dkv_pipe_kernel<DP, FULL>), kgrid, block, 0, s, a);
      hipLaunchKernelGGL((att_dq_pipe_kernel<DP, FULL>), qgrid, block, 0, s, a);
    });
  } else {
    att_pick(dtype, d, [&](auto z, auto dp, auto full) {
      using E = decltype(z);
      constexpr int DP = decltype(dp)::value;
      constexpr bool FULL = decltype(full)::value;
      hipLaunchKernelGGL((att_dkv_kernel<E, DP, FULL>), kgrid, block, 0, s, a);
      hipLaunchKernelGGL((att_dq_kernel<E, DP, FULL>), dim3((unsigned)(tiles * n_head)), block, 0, s, a);
    });
  }
  if (a.splits > 1) {
    const int64_t want = cdiv(T * n_kv * cdiv(d, CH), (int64_t)256), top = (int64_t)device_cu_count() * 8;
    const dim3 jgrid((unsigned)(want < top ? want : top));
    if (dtype == AGRL_BF16)
      hipLaunchKernelGGL(att_join_kernel<uint16_t>, jgrid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL(att_join_kernel<float>, jgrid, dim3(256), 0, s, a);
  }
  return hip_status(hipGetLastError());
}
