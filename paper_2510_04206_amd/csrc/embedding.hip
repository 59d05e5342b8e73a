// Embedding of a packed stream of token ids, and its gradient by sorted tokens (gfx950).
//
//   forward   y[n] = scale W[id[n]]
//   backward  dW[v] (+)= scale * sum over tokens n with id[n] = v of dy[n], in an order that depends on the ids alone
//
// Forward: a wave copies up to 2048 elements of a row.  Memory bounds it.
//
// Backward, three launches, no floating-point atomics:
//   sort  A workgroup owns `range` neighbouring ids and reads all T ids twice.  First it counts
//         (its ids, a counter per id and wave, and how many ids lie below its own: so it knows
//         where its tokens start without asking another workgroup), then it places its
//         tokens in order.  A wave has a run of consecutive tokens and its own counters,
//         so the order within an id is the tokens'.
//   rows  The sorted tokens in chunks of 32 (few: of 8), each row's run of tokens added up in registers.
//         A run that lies within its chunk goes to dW, a piece of one that crosses into
//         another chunk to a partial sum (a separator's run is thousands of tokens: it
//         is added by as many workgroups).  The rows of ids that do not occur are cleared by
//         further workgroups of the same launch.
//   join  adds the pieces of each crossing run: every fourth one in turn, then the four sums.
// Up to 256 tokens one launch does it all (embed_few_kernel).
//
// Measured (MI355X; a copy of 2 GiB moves 4.9 TB/s, a fill 6.9): forward of 65536 x 5120 bf16 out of [152064, 5120]
// 213 us (6.2 TB/s of rows, the repeated ones from the caches).  Backward of the same, the whole gradient written,
// 806 us: rows 712 (3.8 GB), sort 54, join 36; 3823 x 1001 fp32 onto a [4096, 1001] 31 us: three launches of 11, 10 and 9.
#include <math.h>

#include "rows.hpp"

namespace agrl {
namespace {

constexpr int SEG = 64 * CH * 4;       // elements of a row that a wave takes at a time (forward)
constexpr int64_t MAX_TOKENS = ((int64_t)1 << 31) - 1024;

struct EmbedArgs {
  int64_t T;
  int32_t d, V, segs;
  const void* w;
  const int32_t* id;
  const uint8_t* live;
  float scale;
  void* y;
  int64_t ld_y;
  int* err;
};

template <typename W, typename Y>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t first = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t items = a.T * a.segs;
  for (int64_t it = first; it < items; it += (int64_t)gridDim.x * 4) {
    const int64_t n = it / a.segs;
    const int c0 = (int)(it - n * a.segs) * SEG + lane * CH;
    const bool live = !a.live || a.live[n] != 0;
    const int id = live ? a.id[n] : 0;
    const bool bad = id < 0 || id >= a.V;
    if (bad && c0 == 0) set_error(a.err, ERR_TOKEN_ID);
    const W* row = (const W*)a.w + (int64_t)(bad ? 0 : id) * a.d;
    Y* y = (Y*)a.y + n * a.ld_y;
    Chunk<W> x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = c0 + k * 64 * CH;
      if (!live || c >= a.d)
        x[k].zero();
      else if (c + CH <= a.d)
        x[k].load(row + c);
      else
        x[k].load_some(row + c, a.d - c);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = c0 + k * 64 * CH;
      float f[CH];
#pragma unroll
      for (int e = 0; e < CH; ++e) f[e] = bad ? NAN : live ? x[k].get(e) * a.scale : 0.0f;
      if (c + CH <= a.d)
        Chunk<Y>::store(y + c, f);
      else if (c < a.d)
        Chunk<Y>::store_some(y + c, f, a.d - c);
    }
  }
}

// ------------------------------------------------------------------ backward
constexpr int SORT_WAVES = 16;
constexpr int MAX_RANGE = 512;         // ids per workgroup: 32 KiB of counters
constexpr int MAX_CHUNK = 32;          // sorted tokens per chunk, and of a small call
constexpr int MIN_CHUNK = 8;
constexpr int SLAB = 1024;             // columns per workgroup, four a lane
constexpr int ZROWS = 8;               // rows that a clearing workgroup looks at

struct SortArgs {
  int64_t T;
  int32_t V, range;
  const int32_t* id;
  const uint8_t* live;
  int2* sorted;          // [T] token, id
  int32_t* row_start;    // [V + 1] first sorted token of each id
  int32_t* crossing;     // number of runs that cross into another chunk: cleared here
  int* err;
};

__global__ void __launch_bounds__(64 * SORT_WAVES) embed_sort_kernel(SortArgs a) {
  extern __shared__ int cnt[];                       // [SORT_WAVES][range]
  __shared__ int below_of[SORT_WAVES], ids_of[SORT_WAVES];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lo = blockIdx.x * a.range, hi = min(lo + a.range, a.V);
  for (int i = threadIdx.x; i < SORT_WAVES * a.range; i += 64 * SORT_WAVES) cnt[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.crossing = 0;
  __syncthreads();
  int* own = cnt + wave * a.range;
  const int64_t per = cdiv(cdiv(a.T, (int64_t)SORT_WAVES), (int64_t)64) * 64;
  const int64_t t0 = wave * per, t1 = min(a.T, t0 + per);
  constexpr int NONE = 0x7fffffff;
  constexpr int AHEAD = 16;                          // loads in flight
  // the ids of tokens t, t + 64, ..: NONE for dead tokens and ids out of range.  (All loads first, from
  // clamped places: behind a branch each would wait for the one before)
  auto fetch = [&](int64_t t, int (&id)[AHEAD]) {
    // whole batches without a mask, the usual ones: nothing but the loads and a look at the largest (the vector ALU
    // is what bounds this kernel: every workgroup sees every id)
    if (!a.live && t - lane + 64 * AHEAD <= t1) {
      uint32_t most = 0;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) id[k] = (a.id + t)[64 * k];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) most = max(most, (uint32_t)id[k]);
      if (!__any(most >= (uint32_t)a.V)) return;
    }
    uint8_t live[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int64_t at = min(t + 64 * k, a.T - 1);
      id[k] = a.id[at];
      live[k] = a.live ? a.live[at] : 1;
    }
    bool bad = false;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const bool in = t + 64 * k < t1 && live[k] != 0, ok = id[k] >= 0 && id[k] < a.V;
      bad = bad || (in && !ok);
      id[k] = in && ok ? id[k] : NONE;
    }
    if (bad && blockIdx.x == 0) set_error(a.err, ERR_TOKEN_ID);
  };
  int below = 0, id[AHEAD];                          // (few tokens stay in registers for the second pass)
  for (int64_t t = t0 + lane; t < t1 + lane; t += 64 * AHEAD) {
    fetch(t, id);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      below += __popcll(__ballot(id[k] < lo));
      const uint32_t v = id[k] - lo;
      if (v < (uint32_t)(hi - lo)) atomicAdd(&own[v], 1);
    }
  }
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  // where each id and wave starts: ids in order, within an id the waves in order
  const int i = threadIdx.x;
  int mine = 0, sum;
  int each[SORT_WAVES];                              // the id's tokens in each wave's run
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) each[w] = i < a.range ? cnt[w * a.range + i] : 0;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) mine += each[w];
  sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 63) ids_of[wave] = sum;
  __syncthreads();
  int start = sum - mine;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) start += below_of[w] + (w < wave ? ids_of[w] : 0);
  if (i < a.range) {
    if (lo + i <= a.V) a.row_start[lo + i] = start;
    if (lo + i == a.V - 1) a.row_start[a.V] = start + mine;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) {
      cnt[w * a.range + i] = start;
      start += each[w];
    }
  }
  __syncthreads();
  for (int64_t t = t0 + lane; t < t1 + lane; t += 64 * AHEAD) {
    if (per > 64 * AHEAD) fetch(t, id);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int v = id[k] - lo;
      const bool in = (uint32_t)v < (uint32_t)(hi - lo);
      uint64_t same = __ballot(in);
      if (!same) continue;
      // the wave's tokens with the lane's id: those that agree in each of its bits
      for (int b = 0; 1 << b < a.range; ++b) {
        const uint64_t set = __ballot(v >> b & 1);
        same &= v >> b & 1 ? set : ~set;
      }
      if (in) {
        const int at = own[v], rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        a.sorted[at + rank] = make_int2((int)(t + 64 * k), id[k]);
        if (rank == 0) own[v] = at + __popcll(same);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // (the wave's LDS accesses are in order)
    }
  }
}

typedef float f32x4_a4v __attribute__((aligned(4), ext_vector_type(4)));
typedef uint32_t u32x2_a2v __attribute__((aligned(2), ext_vector_type(2)));

// four elements of a row, those past its end 0
__device__ __forceinline__ f32x4 load4(const float* p, int n) {
  if (n >= 4) return *(const f32x4_a4v*)p;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int k = 0; k < 3; ++k)
    if (k < n) v[k] = p[k];
  return v;
}
__device__ __forceinline__ f32x4 load4(const uint16_t* p, int n) {
  if (n >= 4) {
    const u32x2_a2v v = *(const u32x2_a2v*)p;
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                 __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
  }
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int k = 0; k < 3; ++k)
    if (k < n) v[k] = bf16_bits_to_f32(p[k]);
  return v;
}
__device__ __forceinline__ void store4(float* p, f32x4 v, int n) {
  if (n >= 4) {
    *(f32x4_a4v*)p = v;
  } else {
    for (int k = 0; k < 3; ++k)
      if (k < n) p[k] = v[k];
  }
}

struct RowsArgs {
  int32_t d, V, slabs, accumulate, chunk;
  int64_t chunks;
  const void* dy;
  int64_t ld_dy;
  float scale;
  const int2* sorted;
  const int32_t* row_start;
  float* part;           // [chunks][2][d]: the piece that comes in, the piece that goes out
  int32_t* crossing;     // number of runs that go on in another chunk, and each's first chunk (in any order)
  float* dw;
};

template <typename Y, bool ADD>
__global__ void __launch_bounds__(256) embed_rows_kernel(RowsArgs a) {
  const int64_t adding = a.chunks * a.slabs;
  if (blockIdx.x >= adding) {
    const int v0 = (int)(blockIdx.x - adding) * ZROWS;
    for (int v = v0; v < min(v0 + ZROWS, a.V); ++v) {
      if (a.row_start[v] != a.row_start[v + 1]) continue;
      float* p = a.dw + (int64_t)v * a.d;
      for (int c = threadIdx.x * 4; c < a.d; c += 1024) store4(p + c, f32x4{0, 0, 0, 0}, a.d - c);
    }
    return;
  }
  const int64_t c = blockIdx.x / a.slabs;
  const int col = (int)(blockIdx.x - c * a.slabs) * SLAB + threadIdx.x * 4;
  const int total = a.row_start[a.V];
  const int64_t p0 = c * a.chunk;
  if (p0 >= total) return;
  const int n = (int)min((int64_t)a.chunk, total - p0);
  __shared__ int tok[MAX_CHUNK], ids[MAX_CHUNK + 2];         // ids[k + 1]: of the chunk's token k
  if (threadIdx.x < a.chunk + 2) {
    const int64_t p = p0 + threadIdx.x - 1;
    const int2 s = p >= 0 && p < total ? a.sorted[p] : make_int2(0, -1);
    ids[threadIdx.x] = s.y;
    if (threadIdx.x >= 1 && threadIdx.x <= a.chunk) tok[threadIdx.x - 1] = s.x;
  }
  __syncthreads();
  auto id = [&](int k) { return __builtin_amdgcn_readfirstlane(ids[k + 1]); };
  if (col == 0 && id(n - 1) == id(n) && a.row_start[id(n)] >= p0)
    a.crossing[1 + atomicAdd(a.crossing, 1)] = (int)c;
  const int left = a.d - col;
  if (left <= 0) return;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  bool in = id(-1) == id(0);                         // the run came in from the chunk before
  for (int k0 = 0; k0 < n; k0 += 8) {
    f32x4 x[8], old[8];
    // (the rows that the sums are added to come with them, not one after another when a run ends)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t t = __builtin_amdgcn_readfirstlane(tok[min(k0 + k, n - 1)]);
      x[k] = load4((const Y*)a.dy + t * a.ld_dy + col, left);
      old[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (ADD)
        if (k0 + k < n && id(k0 + k) != id(k0 + k + 1))
          old[k] = load4(a.dw + (int64_t)id(k0 + k) * a.d + col, left);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k0 + k >= n) break;
      sum += x[k];
      const bool same = id(k0 + k) == id(k0 + k + 1);
      if (same && k0 + k + 1 < n) continue;
      if (!in && !same)
        store4(a.dw + (int64_t)id(k0 + k) * a.d + col, old[k] + sum * a.scale, left);
      else
        store4(a.part + (2 * c + (in ? 0 : 1)) * a.d + col, sum, left);
      in = false;
      sum = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
}

// The runs that cross, 256 columns a workgroup: each of its four waves every fourth piece in order, then the four sums.
__global__ void __launch_bounds__(256) embed_join_kernel(RowsArgs a) {
  constexpr int COLS = 256;
  __shared__ f32x4 sums[3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cols = (a.d + COLS - 1) / COLS;
  const int64_t items = (int64_t)*a.crossing * cols;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const int64_t c = a.crossing[1 + i / cols];
    const int col = (int)(i % cols) * COLS + lane * 4, left = a.d - col;
    const int v = a.sorted[(c + 1) * a.chunk].y;
    const int64_t last = ((int64_t)a.row_start[v + 1] - 1) / a.chunk;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f}, old = sum;
    if (left > 0) {
      if (wave == 0 && a.accumulate) old = load4(a.dw + (int64_t)v * a.d + col, left);
#pragma unroll 4
      for (int64_t k = c + wave; k <= last; k += 4)
        sum += load4(a.part + (2 * k + (k == c ? 1 : 0)) * a.d + col, left);
    }
    if (wave) sums[wave - 1][lane] = sum;
    __syncthreads();
    if (wave == 0 && left > 0) {
      sum = (sum + sums[0][lane]) + (sums[1][lane] + sums[2][lane]);
      store4(a.dw + (int64_t)v * a.d + col, old + sum * a.scale, left);
    }
    __syncthreads();
  }
}

// Tokens per chunk: few tokens in chunks of 8, so that they fill the chip (3823 x 1001: rows 23 us in chunks of 32, 9 in
// chunks of 8)
int chunk_of(int64_t T, int32_t d) {
  return cdiv(T, (int64_t)MAX_CHUNK) * cdiv(d, SLAB) < 1024 ? MIN_CHUNK : MAX_CHUNK;
}

// Few tokens: one launch, no sort.  A workgroup per token and slab of columns looks all ids over: the first token of an
// id adds up those that follow, the others leave.  Workgroups behind them clear the rows of absent ids.
// Added to [V, d] in bf16, here and by the sort: a text's ids, [4096, 256] 64 tokens 7.3 and 13.6 us, 256 7.7 and 15.4, 512
// 16.5 and 16.7; [4096, 1001] 256 10.6 and 17.5, 512 26 and 19; [4096, 8192] 256 8.9 and 16, 512 19 and 18.  What it is slow at is
// one id in every token, whose rows one workgroup a slab adds up: 64 tokens 14 to 20 and 15 us, 256 47 to 76 and 15 to 18
// (512: 150 and 21).
constexpr int FEW = 256;
template <typename Y, bool ADD>
__global__ void __launch_bounds__(256) embed_few_kernel(SortArgs t, RowsArgs a) {
  const int T = (int)t.T, adding = T * a.slabs, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto live = [&](int n) { return !t.live || t.live[n] != 0; };
  if (blockIdx.x >= adding) {
    __shared__ int here[ZROWS];
    const int v0 = (int)(blockIdx.x - adding) * ZROWS;
    if (threadIdx.x < ZROWS) here[threadIdx.x] = 0;
    __syncthreads();
    for (int n = threadIdx.x; n < T; n += 256)
      if (live(n) && t.id[n] >= v0 && t.id[n] < v0 + ZROWS) here[t.id[n] - v0] = 1;
    __syncthreads();
    for (int v = v0; v < min(v0 + ZROWS, a.V); ++v) {
      if (here[v - v0]) continue;
      float* p = a.dw + (int64_t)v * a.d;
      for (int c = threadIdx.x * 4; c < a.d; c += 1024) store4(p + c, f32x4{0, 0, 0, 0}, a.d - c);
    }
    return;
  }
  const int n = blockIdx.x / a.slabs, col = (int)(blockIdx.x - n * a.slabs) * SLAB + threadIdx.x * 4, left = a.d - col;
  if (!live(n)) return;
  const int v = t.id[n];
  if (v < 0 || v >= a.V) {
    if (threadIdx.x == 0) set_error(t.err, ERR_TOKEN_ID);
    return;
  }
  __shared__ uint64_t same[FEW / 64];          // the tokens with this id, a bit each
#pragma unroll
  for (int k = 0; k < FEW / 256; ++k) {
    const int m = k * 256 + threadIdx.x;
    const uint64_t bits = __ballot(m < T && t.id[min(m, T - 1)] == v && live(min(m, T - 1)));
    if (lane == 0) same[k * 4 + wave] = bits;
  }
  __syncthreads();
  for (int k = 0; k <= n >> 6; ++k)
    if (same[k] & (k < n >> 6 ? ~(uint64_t)0 : ((uint64_t)1 << (n & 63)) - 1)) return;
  if (left <= 0) return;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f}, old = sum;
  if (ADD) old = load4(a.dw + (int64_t)v * a.d + col, left);
  for (int k = n >> 6; k < FEW / 64; ++k) {
    uint64_t todo = same[k];
    todo = (uint64_t)__builtin_amdgcn_readfirstlane((int)(todo >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)todo);
    while (todo) {
      f32x4 x[8];
      int many = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!todo) continue;
        x[e] = load4((const Y*)a.dy + (int64_t)(k * 64 + __builtin_ctzll(todo)) * a.ld_dy + col, left);
        todo &= todo - 1;
        many = e + 1;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < many) sum += x[e];
    }
  }
  store4(a.dw + (int64_t)v * a.d + col, old + sum * a.scale, left);
}

struct Space {
  size_t sorted, starts, crossing, part, total;
};
Space embed_space(int64_t T, int32_t d, int32_t V) {
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  Space s;
  s.sorted = 0;
  s.starts = up((size_t)T * sizeof(int2));
  s.crossing = s.starts + up(((size_t)V + 1) * 4);
  s.part = s.crossing + up(((size_t)cdiv(T, (int64_t)chunk_of(T, d)) + 1) * 4);
  s.total = s.part + (size_t)cdiv(T, (int64_t)chunk_of(T, d)) * 2 * d * 4;
  return s;
}

bool embed_sizes(int64_t T, int32_t d, int32_t V) {
  return T >= 0 && T <= MAX_TOKENS && d > 0 && d <= (1 << 20) && V > 0 && V < 0x7fffffff;
}
// The gradient's: a range of ids or rows past the last one still counts in 32 bits, and every launch has less than the 2^32
// lanes that HIP takes: workgroups of 256 that add, and with `clear` others that clear (the sort's have 1024 lanes and up to
// 512 ids)
constexpr int32_t MAX_IDS = 0x7fffffff - 1023;
constexpr int64_t MAX_GROUPS = ((int64_t)1 << 24) - 1;
bool embed_bwd_sizes(int64_t T, int32_t d, int32_t V, bool clear) {
  return embed_sizes(T, d, V) && V <= MAX_IDS &&
         (T <= FEW ? T : cdiv(T, (int64_t)chunk_of(T, d))) * cdiv(d, SLAB) + (clear ? cdiv(V, ZROWS) : 0) <= MAX_GROUPS;
}

}  // namespace
}  // namespace agrl

extern "C" int agrl_token_embed_fwd(int64_t T, int32_t d, int32_t V, int32_t w_dtype, int32_t dtype,
                                    const void* weight, const int32_t* token_id,
                                    const uint8_t* live_mask, float scale, void* y, int64_t ld_y,
                                    void* stream) {
  using namespace agrl;
  const char* fn = "agrl_token_embed_fwd";
  if ((dtype != AGRL_BF16 && dtype != AGRL_F32) || (w_dtype != AGRL_BF16 && w_dtype != AGRL_F32))
    return fail(AGRL_E_DTYPE, fn, "dtype must be AGRL_BF16 or AGRL_F32");
  if (!embed_sizes(T, d, V)) return fail(AGRL_E_SHAPE, fn, "bad T, d or V");
  if (ld_y < d) return fail(AGRL_E_SHAPE, fn, "ld_y is smaller than d");
  if (!isfinite(scale)) return fail(AGRL_E_FLAGS, fn, "scale must be finite");
  if (T == 0) return AGRL_OK;
  if (!weight || !token_id || !y) return fail(AGRL_E_NULL, fn, "weight, token_id or y is NULL");
  const EmbedArgs a = {T, d, V, cdiv(d, SEG), weight, token_id, live_mask, scale, y, ld_y,
                       device_error_ptr()};
  const int64_t need = cdiv(T * a.segs, (int64_t)4), most = (int64_t)device_cu_count() * 8;
  const dim3 grid((unsigned)(need < most ? need : most)), block(256);
  hipStream_t s = (hipStream_t)stream;
  if (w_dtype == AGRL_BF16 && dtype == AGRL_BF16)
    hipLaunchKernelGGL((embed_fwd_kernel<uint16_t, uint16_t>), grid, block, 0, s, a);
  else if (w_dtype == AGRL_BF16)
    hipLaunchKernelGGL((embed_fwd_kernel<uint16_t, float>), grid, block, 0, s, a);
  else if (dtype == AGRL_BF16)
    hipLaunchKernelGGL((embed_fwd_kernel<float, uint16_t>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((embed_fwd_kernel<float, float>), grid, block, 0, s, a);
  return hip_status(hipGetLastError());
}

extern "C" size_t agrl_token_embed_bwd_workspace_size(int64_t T, int32_t d, int32_t V) {
  return agrl::embed_bwd_sizes(T, d, V, false) ? agrl::embed_space(T, d, V).total : 0;
}

extern "C" int agrl_token_embed_bwd(int64_t T, int32_t d, int32_t V, int32_t dy_dtype,
                                    const int32_t* token_id, const uint8_t* live_mask,
                                    const void* dy, int64_t ld_dy, float scale, int32_t accumulate,
                                    void* workspace, size_t ws_bytes, float* dweight, void* stream) {
  using namespace agrl;
  const char* fn = "agrl_token_embed_bwd";
  if (dy_dtype != AGRL_BF16 && dy_dtype != AGRL_F32)
    return fail(AGRL_E_DTYPE, fn, "dy_dtype must be AGRL_BF16 or AGRL_F32");
  if (!embed_bwd_sizes(T, d, V, !accumulate)) return fail(AGRL_E_SHAPE, fn, "bad T, d or V");
  if (ld_dy < d) return fail(AGRL_E_SHAPE, fn, "ld_dy is smaller than d");
  if (!isfinite(scale)) return fail(AGRL_E_FLAGS, fn, "scale must be finite");
  if (accumulate != 0 && accumulate != 1) return fail(AGRL_E_FLAGS, fn, "accumulate must be 0 or 1");
  if (T == 0 && accumulate) return AGRL_OK;
  if (!dweight || (T > 0 && (!token_id || !dy)))
    return fail(AGRL_E_NULL, fn, "token_id, dy or dweight is NULL");
  const Space sp = embed_space(T, d, V);
  if (!workspace || ws_bytes < sp.total)
    return fail(AGRL_E_WORKSPACE, fn, "workspace missing or too small");
  if ((uintptr_t)workspace % 256 != 0)
    return fail(AGRL_E_UNSUPPORTED, fn, "workspace must be 256-byte aligned");
  uint8_t* ws = (uint8_t*)workspace;
  int2* sorted = (int2*)(ws + sp.sorted);
  int32_t* starts = (int32_t*)(ws + sp.starts);
  hipStream_t s = (hipStream_t)stream;
  // an id range a compute unit, as far as the counters fit: what a workgroup places one after
  // another is then as little as can be
  const int fair = cdiv(V, device_cu_count());
  const SortArgs so = {T, V, fair < MAX_RANGE ? fair : MAX_RANGE, token_id, live_mask, sorted, starts,
                       (int32_t*)(ws + sp.crossing), device_error_ptr()};
  const int chunk = chunk_of(T, d);
  const RowsArgs r = {d, V, cdiv(d, SLAB), accumulate, chunk, cdiv(T, (int64_t)chunk), dy, ld_dy, scale,
                      sorted, starts, (float*)(ws + sp.part), so.crossing, dweight};
  if (T <= FEW) {
    const dim3 few((unsigned)(T * r.slabs + (accumulate ? 0 : cdiv(V, ZROWS)))), lanes(256);
    if (dy_dtype == AGRL_BF16 && accumulate)
      hipLaunchKernelGGL((embed_few_kernel<uint16_t, true>), few, lanes, 0, s, so, r);
    else if (dy_dtype == AGRL_BF16)
      hipLaunchKernelGGL((embed_few_kernel<uint16_t, false>), few, lanes, 0, s, so, r);
    else if (accumulate)
      hipLaunchKernelGGL((embed_few_kernel<float, true>), few, lanes, 0, s, so, r);
    else
      hipLaunchKernelGGL((embed_few_kernel<float, false>), few, lanes, 0, s, so, r);
    return hip_status(hipGetLastError());
  }
  hipLaunchKernelGGL(embed_sort_kernel, dim3(cdiv(V, so.range)), dim3(64 * SORT_WAVES),
                     SORT_WAVES * so.range * 4, s, so);
  const dim3 grid((unsigned)(r.chunks * r.slabs + (accumulate ? 0 : cdiv(V, ZROWS)))), block(256);
  if (dy_dtype == AGRL_BF16 && accumulate)
    hipLaunchKernelGGL((embed_rows_kernel<uint16_t, true>), grid, block, 0, s, r);
  else if (dy_dtype == AGRL_BF16)
    hipLaunchKernelGGL((embed_rows_kernel<uint16_t, false>), grid, block, 0, s, r);
  else if (accumulate)
    hipLaunchKernelGGL((embed_rows_kernel<float, true>), grid, block, 0, s, r);
  else
    hipLaunchKernelGGL((embed_rows_kernel<float, false>), grid, block, 0, s, r);
  if (r.chunks > 1) {
    const int64_t most = (int64_t)device_cu_count() * 4, need = (r.chunks - 1) * cdiv(d, 256);
    hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(need < most ? need : most)), block, 0, s, r);
  }
  return hip_status(hipGetLastError());
}
