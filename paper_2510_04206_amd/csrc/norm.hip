// Layer and RMS norm over token rows, forward and backward (gfx950).
//
//   layer: mu = (1/d) sum x, v = (1/d) sum (x - mu)^2, r = 1/sqrt(v + eps),
//          y = (x - mu) r w + b
//   RMS:   v = (1/d) sum x^2, r = 1/sqrt(v + eps), y = x r w + b
//   with xh = (x - mu) r and g = dy w:
//          dx = r (g - c1 - xh c2), c1 = (1/d) sum g (layer; 0 for RMS),
//          c2 = (1/d) sum g xh, dw = sum over rows dy xh, db = sum over rows dy
//
// Memory bounds all of it, so each row is read once: a team of TEAM lanes holds a row in
// registers, NC chunks of 8 elements per lane (lane t has chunks t, t + TEAM, ...: every load
// of a wave is consecutive), and the weight, the bias and the backward's sums over rows
// stay in the registers of the lane that owns their columns while the team walks its rows.
// The next live row is loaded before the current one is reduced.  Rows whose mask is 0 are
// not read; their outputs are written after the live rows of a group of 64, so that no load
// waits behind their stores.
//
// Statistics in fp32: a wave's variance is taken about the wave's own mean (two passes over
// registers, the second also finding what the rounded mean is off by) and the waves' means
// are joined as differences from the first one's, so a row far from zero loses nothing to
// cancellation.  One LDS exchange and one barrier per row and team.
//
// Measured (MI355X; a copy of 2 GiB moves 4.9 TB/s): forward of 65536 x 5120 bf16 RMS with a third
// of the rows live 190 us, 4.7 TB/s; of 3823 x 1001, no row aligned, 7.4 us, where a copy's rate would
// take 3.1 (a row a team: nothing is loaded ahead, and the parameters come first); backward of 32768 x
// 3584 bf16 with fp32 dy, a third live, 117 us, 4.0 TB/s (5 us of it the second launch, which
// adds the workgroups' partial sums); of 65536 x 4096, all live, dy bf16, 294 us, 5.5 TB/s.  Past d =
// 8192 the backward's sums do not fit the 128 registers that 1024 lanes leave each and go to
// scratch memory: 16384 x 12288 725 us, 2.2 TB/s (of 16384 x 8192 205 us, 5.2).  Small calls are
// one or two launches: one row of 256 takes 2.3 us on the GPU.
#include <math.h>

#include "../../include/agrl.h"
#include "common.hpp"
#include "rows.hpp"

namespace agrl {
namespace {

template <int TEAM>
struct Shape {
  static constexpr int BLOCK = TEAM < 256 ? 256 : TEAM;
  static constexpr int TEAMS = BLOCK / TEAM;     // rows in flight per workgroup
  static constexpr int WAVES = TEAM / 64;        // waves per team
};

// A lane's place: its team's row sequence and its chunks of a row.
template <int TEAM, int NC>
struct Lane {
  int t;                 // lane within the team
  int64_t first, step;   // rows first, first + step, ...
  int d;

  __device__ __forceinline__ Lane(int d_) : d(d_) {
    t = threadIdx.x & (TEAM - 1);
    const int team = __builtin_amdgcn_readfirstlane((int)threadIdx.x / TEAM);
    first = (int64_t)blockIdx.x * Shape<TEAM>::TEAMS + team;
    step = (int64_t)gridDim.x * Shape<TEAM>::TEAMS;
  }
  __device__ __forceinline__ int col(int c) const { return (t + TEAM * c) * CH; }
  // valid elements of chunk c: 8, 0, or some in the row's last chunk
  __device__ __forceinline__ int valid(int c) const { return min(max(d - col(c), 0), CH); }

  template <typename T>
  __device__ __forceinline__ void load(Chunk<T> (&x)[NC], const T* row) const {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (col(c) + CH <= d)
        x[c].load(row + col(c));
      else if (col(c) < d)
        x[c].load_some(row + col(c), d - col(c));
      else
        x[c].zero();
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, int c, const float (&f)[CH]) const {
    if (col(c) + CH <= d)
      Chunk<T>::store(row + col(c), f);
    else if (col(c) < d)
      Chunk<T>::store_some(row + col(c), f, d - col(c));
  }
  template <typename T>
  __device__ __forceinline__ void store_zero(T* row) const {
    const float z[CH] = {};
#pragma unroll
    for (int c = 0; c < NC; ++c) store(row, c, z);
  }
  // a parameter vector of either type, `none` where there is none
  __device__ __forceinline__ void param(float (&w)[NC][CH], const void* p, int dtype,
                                        float none) const {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int k = 0; k < CH; ++k) w[c][k] = none;
    if (!p) return;
    if (dtype == AGRL_BF16)
      param_as(w, (const uint16_t*)p);
    else
      param_as(w, (const float*)p);
  }
  template <typename T>
  __device__ __forceinline__ void param_as(float (&w)[NC][CH], const T* p) const {
    Chunk<T> x[NC];
    load(x, p);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int k = 0; k < CH; ++k) w[c][k] = x[c].get(k);   // (past the row: 0, used by no one)
  }
};

// Rows of a team in groups of 64: bit k is row k of the group, 1 where it is live.
__device__ __forceinline__ uint64_t live_rows(const uint8_t* mask, int64_t r0, int64_t step,
                                              int64_t T) {
  const int64_t r = r0 + (int64_t)(threadIdx.x & 63) * step;
  return __ballot(r < T && (!mask || mask[r] != 0));
}

struct FwdArgs {
  int64_t T;
  int32_t d, layer, w_dtype;
  const void* x;
  int64_t ld_x;
  const void *w, *b;
  const uint8_t* mask;
  float eps;
  void* y;
  int64_t ld_y;
  float *mean, *rstd;
};

template <typename X, int TEAM, int NC>
__global__ void __launch_bounds__(Shape<TEAM>::BLOCK) norm_fwd_kernel(FwdArgs a) {
  constexpr int W = Shape<TEAM>::WAVES;
  __shared__ f32x4 part[2][W];
  const Lane<TEAM, NC> L(a.d);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x & (TEAM - 1)) >> 6);
  float w[NC][CH], b[NC][CH];
  L.param(w, a.w, a.w_dtype, 1.0f);
  L.param(b, a.b, a.w_dtype, 0.0f);
  const float inv_d = 1.0f / (float)a.d;
  // elements of a row that wave v of the team holds
  auto held = [&](int v) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) n += min(max(a.d - (v * 64 + TEAM * c) * CH, 0), 64 * CH);
    return (float)n;
  };
  const float n_own = held(wave), inv_own = n_own > 0.0f ? 1.0f / n_own : 0.0f;
  int par = 0;
  for (int64_t r0 = L.first; r0 < a.T; r0 += 64 * L.step) {
    const uint64_t live = live_rows(a.mask, r0, L.step, a.T);
    uint64_t todo = live;
    Chunk<X> nx[NC];
    int k = todo ? __builtin_ctzll(todo) : 64;
    if (k < 64) L.load(nx, (const X*)a.x + (r0 + k * L.step) * a.ld_x);
    while (k < 64) {
      const int64_t r = r0 + k * L.step;
      Chunk<X> x[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) x[c] = nx[c];
      todo &= todo - 1;
      k = todo ? __builtin_ctzll(todo) : 64;
      if (k < 64) L.load(nx, (const X*)a.x + (r0 + k * L.step) * a.ld_x);

      float mean = 0.0f, ss = 0.0f;
      if (a.layer) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < CH; ++e) s += x[c].get(e);
        const float about = wave_sum(s) * inv_own;
        float off = 0.0f;        // what the rounding of `about` left
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int nv = L.valid(c);
#pragma unroll
          for (int e = 0; e < CH; ++e) {
            const float u = e < nv ? x[c].get(e) - about : 0.0f;
            off += u;
            ss = fmaf(u, u, ss);
          }
        }
        off = wave_sum(off) * inv_own;
        mean = about + off;
        ss = fmaf(-n_own * off, off, wave_sum(ss));
        if constexpr (W > 1) {
          if ((threadIdx.x & 63) == 0) part[par][wave] = f32x4{about, off, ss, 0.0f};
          __syncthreads();
          const float base = part[par][0].x;
          off = ss = 0.0f;
#pragma unroll
          for (int v = 0; v < W; ++v) {
            const f32x4 p = part[par][v];
            const float n = held(v), u = n > 0.0f ? (p.x - base) + p.y : 0.0f;
            off = fmaf(n, u, off);
            ss += fmaf(n * u, u, p.z);
          }
          off *= inv_d;
          mean = base + off;
          ss = fmaf(-(float)a.d * off, off, ss);
        }
        ss = ss < 0.0f ? 0.0f : ss;    // (a constant row's rounds to either side of 0; NaN stays)
      } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < CH; ++e) ss = fmaf(x[c].get(e), x[c].get(e), ss);
        ss = wave_sum(ss);
        if constexpr (W > 1) {
          if ((threadIdx.x & 63) == 0) part[par][wave].z = ss;
          __syncthreads();
          ss = 0.0f;
#pragma unroll
          for (int v = 0; v < W; ++v) ss += part[par][v].z;
        }
      }
      par ^= 1;    // (the next row's partial sums go to the other half: one barrier a row)
      // infinite: an infinite element (RMS), or squares beyond fp32's range.  1 / sqrt would be 0 and
      // the row a finite one, its bias
      const float var = fmaf(ss, inv_d, a.eps);
      const float rstd = var < INFINITY ? 1.0f / sqrtf(var) : NAN;
      X* y = (X*)a.y + r * a.ld_y;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float f[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e)
          f[e] = fmaf((x[c].get(e) - mean) * rstd, w[c][e], b[c][e]);
        L.store(y, c, f);
      }
      if (L.t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
      }
    }
    // rows that no one reads
    for (int q = 0; q < 64; ++q) {
      const int64_t r = r0 + q * L.step;
      if (r >= a.T) break;
      if (live >> q & 1) continue;
      L.store_zero((X*)a.y + r * a.ld_y);
      if (L.t == 0) {
        if (a.mean) a.mean[r] = 0.0f;
        if (a.rstd) a.rstd[r] = 0.0f;
      }
    }
  }
}

struct BwdArgs {
  int64_t T;
  int32_t d, layer, w_dtype;
  const void* x;
  int64_t ld_x;
  const void* w;
  const uint8_t* mask;
  const void* dy;
  int64_t ld_dy;
  const float *mean, *rstd;
  void* dx;
  int64_t ld_dx;
  float* part;     // [gridDim.x][2][d] sums of dy xh and of dy
};

template <typename X, typename Y, int TEAM, int NC>
__global__ void __launch_bounds__(Shape<TEAM>::BLOCK) norm_bwd_kernel(BwdArgs a) {
  constexpr int W = Shape<TEAM>::WAVES, TEAMS = Shape<TEAM>::TEAMS;
  __shared__ f32x2 part[2][W];
  const Lane<TEAM, NC> L(a.d);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x & (TEAM - 1)) >> 6);
  float w[NC][CH], dw[NC][CH], db[NC][CH];
  L.param(w, a.w, a.w_dtype, 1.0f);
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < CH; ++e) dw[c][e] = db[c][e] = 0.0f;
  const float inv_d = 1.0f / (float)a.d;
  int par = 0;
  for (int64_t r0 = L.first; r0 < a.T; r0 += 64 * L.step) {
    const uint64_t live = live_rows(a.mask, r0, L.step, a.T);
    uint64_t todo = live;
    Chunk<X> nx[NC];
    Chunk<Y> ny[NC];
    float nmean = 0.0f, nrstd = 0.0f;
    auto fetch = [&](int k) {
      const int64_t r = r0 + k * L.step;
      L.load(nx, (const X*)a.x + r * a.ld_x);
      L.load(ny, (const Y*)a.dy + r * a.ld_dy);
      if (a.layer) nmean = a.mean[r];
      nrstd = a.rstd[r];
    };
    int k = todo ? __builtin_ctzll(todo) : 64;
    if (k < 64) fetch(k);
    while (k < 64) {
      const int64_t r = r0 + k * L.step;
      Chunk<X> x[NC];
      Chunk<Y> dy[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        x[c] = nx[c];
        dy[c] = ny[c];
      }
      const float mean = nmean, rstd = nrstd;
      todo &= todo - 1;
      k = todo ? __builtin_ctzll(todo) : 64;
      if (k < 64) fetch(k);

      float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int nv = L.valid(c);
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          // (past the row dy is 0, x a stand-in of 0: a finite xh, nothing is added)
          const float xh = (x[c].get(e) - mean) * rstd, g0 = dy[c].get(e);
          const float g = g0 * w[c][e];
          const bool in = e < nv;
          c1 += in ? g : 0.0f;
          c2 = in ? fmaf(g, xh, c2) : c2;
          dw[c][e] = fmaf(g0, xh, dw[c][e]);
          db[c][e] += g0;
        }
      }
      c1 = wave_sum(c1);
      c2 = wave_sum(c2);
      if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) part[par][wave] = f32x2{c1, c2};
        __syncthreads();
        c1 = c2 = 0.0f;
#pragma unroll
        for (int v = 0; v < W; ++v) {
          c1 += part[par][v].x;
          c2 += part[par][v].y;
        }
      }
      par ^= 1;
      c1 = a.layer ? c1 * inv_d : 0.0f;
      c2 *= inv_d;
      X* dx = (X*)a.dx + r * a.ld_dx;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float f[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          const float xh = (x[c].get(e) - mean) * rstd;
          f[e] = rstd * fmaf(-xh, c2, fmaf(dy[c].get(e), w[c][e], -c1));
        }
        L.store(dx, c, f);
      }
    }
    for (int q = 0; q < 64; ++q) {
      const int64_t r = r0 + q * L.step;
      if (r >= a.T) break;
      if (!(live >> q & 1)) L.store_zero((X*)a.dx + r * a.ld_dx);
    }
  }
  if (!a.part) return;
  float* out = a.part + (int64_t)blockIdx.x * 2 * a.d;
  if constexpr (TEAMS > 1) {
    // the workgroup's teams in order
    __shared__ float sum[2][TEAM * NC * CH];
    const int team = threadIdx.x / TEAM;
    for (int q = 0; q < TEAMS; ++q) {
      if (team == q) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < CH; ++e) {
            const int i = e * TEAM * NC + c * TEAM + L.t;
            dw[c][e] += q ? sum[0][i] : 0.0f;
            db[c][e] += q ? sum[1][i] : 0.0f;
            sum[0][i] = dw[c][e];
            sum[1][i] = db[c][e];
          }
      }
      __syncthreads();
    }
    if (team != TEAMS - 1) return;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    L.store(out, c, dw[c]);
    L.store(out + a.d, c, db[c]);
  }
}

// dw, db: the workgroups' sums in a fixed order.  64 columns per workgroup, 16 waves, wave v
// takes rows v, v + 16, ...
constexpr int RED_WAVES = 16;
__global__ void __launch_bounds__(64 * RED_WAVES)
    norm_param_reduce_kernel(const float* part, int rows, int d, float* dw, float* db,
                             int accumulate) {
  __shared__ float sum[RED_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float* out = blockIdx.y ? db : dw;
  if (!out) return;
  float s = 0.0f;
  if (col < d) {
    const float* p = part + (int64_t)blockIdx.y * d + col;
#pragma unroll 8
    for (int r = wave; r < rows; r += RED_WAVES) s += p[(int64_t)r * 2 * d];
  }
  sum[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < d) {
    s = 0.0f;
#pragma unroll
    for (int v = 0; v < RED_WAVES; ++v) s += sum[v][lane];
    out[col] = accumulate ? out[col] + s : s;
  }
}

// The team that holds a row of d elements: f(TEAM, NC) as integral constants
template <int V>
struct Int {
  static constexpr int value = V;
};
template <class F>
void with_team(int d, F&& f) {
  if (d <= 512) return f(Int<64>{}, Int<1>{});
  if (d <= 1024) return f(Int<64>{}, Int<2>{});
  if (d <= 2048) return f(Int<256>{}, Int<1>{});
  if (d <= 4096) return f(Int<256>{}, Int<2>{});
  if (d <= 6144) return f(Int<256>{}, Int<3>{});
  if (d <= 8192) return f(Int<512>{}, Int<2>{});
  return f(Int<1024>{}, Int<2>{});
}
constexpr int MAX_D = 16384;
constexpr int64_t MAX_T = (int64_t)1 << 40;

// Workgroups of the backward: each leaves a partial sum of 2 d floats, so their number is bounded:
// two a compute unit, with two rows each in flight.  65536 x 4096 dense 294 us (three 320, four
// 343), 32768 x 3584 with a third of the rows live 120 (119, 124).
constexpr int BWD_GROUPS = 512;
int teams_per_group(int d) { return d <= 1024 ? 4 : 1; }
int bwd_groups(int64_t T, int d) {
  const int64_t g = cdiv(T, (int64_t)teams_per_group(d));
  return (int)(g < BWD_GROUPS ? g : BWD_GROUPS);
}

int check(const char* fn, int64_t T, int32_t d, int32_t kind, int32_t dtype, int32_t w_dtype,
          int64_t ld_x) {
  if ((dtype != AGRL_BF16 && dtype != AGRL_F32) || (w_dtype != AGRL_BF16 && w_dtype != AGRL_F32))
    return fail(AGRL_E_DTYPE, fn, "dtype must be AGRL_BF16 or AGRL_F32");
  if (T < 0 || T > MAX_T || d <= 0) return fail(AGRL_E_SHAPE, fn, "bad T or d");
  if (ld_x < d) return fail(AGRL_E_SHAPE, fn, "ld_x is smaller than d");
  if (kind != AGRL_NORM_LAYER && kind != AGRL_NORM_RMS)
    return fail(AGRL_E_FLAGS, fn, "kind must be AGRL_NORM_LAYER or AGRL_NORM_RMS");
  if (d > MAX_D) return fail(AGRL_E_UNSUPPORTED, fn, "d is larger than 16384");
  return AGRL_OK;
}

}  // namespace
}  // namespace agrl

extern "C" int agrl_token_norm_fwd(int64_t T, int32_t d, int32_t kind, int32_t dtype,
                                   int32_t w_dtype, const void* x, int64_t ld_x,
                                   const void* weight, const void* bias,
                                   const uint8_t* action_mask, float eps, void* y, int64_t ld_y,
                                   float* mean, float* rstd, void* stream) {
  using namespace agrl;
  const char* fn = "agrl_token_norm_fwd";
  int rc = check(fn, T, d, kind, dtype, w_dtype, ld_x);
  if (rc) return rc;
  if (ld_y < d) return fail(AGRL_E_SHAPE, fn, "ld_y is smaller than d");
  if (!(eps >= 0.0f) || !isfinite(eps)) return fail(AGRL_E_FLAGS, fn, "eps must be finite and >= 0");
  if (T == 0) return AGRL_OK;
  if (!x || !y) return fail(AGRL_E_NULL, fn, "x or y is NULL");
  const FwdArgs a = {T, d, kind == AGRL_NORM_LAYER, w_dtype, x, ld_x, weight, bias, action_mask,
                     eps, y, ld_y, kind == AGRL_NORM_LAYER ? mean : nullptr, rstd};
  hipStream_t s = (hipStream_t)stream;
  with_team(d, [&](auto team, auto nc) {
    constexpr int TEAM = decltype(team)::value, NC = decltype(nc)::value;
    // 1024 lanes on a compute unit, each team several rows: 65536 x 5120 189 us (2048 lanes 192,
    // 512 192), 100000 x 512 44 (50, 57)
    constexpr int PER = 1024 / Shape<TEAM>::BLOCK;
    const int64_t need = cdiv(T, (int64_t)Shape<TEAM>::TEAMS);
    const int64_t most = (int64_t)device_cu_count() * PER;
    const dim3 grid((unsigned)(need < most ? need : most)), block(Shape<TEAM>::BLOCK);
    if (dtype == AGRL_BF16)
      hipLaunchKernelGGL((norm_fwd_kernel<uint16_t, TEAM, NC>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((norm_fwd_kernel<float, TEAM, NC>), grid, block, 0, s, a);
  });
  return hip_status(hipGetLastError());
}

extern "C" size_t agrl_token_norm_bwd_workspace_size(int64_t T, int32_t d) {
  if (T <= 0 || T > agrl::MAX_T || d <= 0 || d > agrl::MAX_D) return 0;
  return (size_t)agrl::bwd_groups(T, d) * 2 * d * sizeof(float);
}

extern "C" int agrl_token_norm_bwd(int64_t T, int32_t d, int32_t kind, int32_t dtype,
                                   int32_t w_dtype, int32_t dy_dtype, const void* x, int64_t ld_x,
                                   const void* weight, const uint8_t* action_mask, const void* dy,
                                   int64_t ld_dy, const float* mean, const float* rstd,
                                   int32_t accumulate, void* workspace, size_t ws_bytes, void* dx,
                                   int64_t ld_dx, float* dweight, float* dbias, void* stream) {
  using namespace agrl;
  const char* fn = "agrl_token_norm_bwd";
  int rc = check(fn, T, d, kind, dtype, w_dtype, ld_x);
  if (rc) return rc;
  if (dy_dtype != AGRL_BF16 && dy_dtype != AGRL_F32)
    return fail(AGRL_E_DTYPE, fn, "dy_dtype must be AGRL_BF16 or AGRL_F32");
  if (ld_dy < d || ld_dx < d) return fail(AGRL_E_SHAPE, fn, "ld_dy or ld_dx is smaller than d");
  if (accumulate != 0 && accumulate != 1)
    return fail(AGRL_E_FLAGS, fn, "accumulate must be 0 or 1");
  const bool params = dweight || dbias;
  if (T > 0) {
    if (!x || !dy || !dx || !rstd) return fail(AGRL_E_NULL, fn, "x, dy, dx or rstd is NULL");
    if (kind == AGRL_NORM_LAYER && !mean) return fail(AGRL_E_NULL, fn, "mean is NULL");
    if (params && (!workspace || ws_bytes < agrl_token_norm_bwd_workspace_size(T, d)))
      return fail(AGRL_E_WORKSPACE, fn, "workspace missing or too small");
  }
  if ((uintptr_t)workspace % 4 != 0)
    return fail(AGRL_E_UNSUPPORTED, fn, "workspace must be 4-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const int groups = T > 0 ? bwd_groups(T, d) : 0;
  if (T > 0) {
    const BwdArgs a = {T, d, kind == AGRL_NORM_LAYER, w_dtype, x, ld_x, weight, action_mask, dy,
                       ld_dy, mean, rstd, dx, ld_dx, params ? (float*)workspace : nullptr};
    with_team(d, [&](auto team, auto nc) {
      constexpr int TEAM = decltype(team)::value, NC = decltype(nc)::value;
      const dim3 grid(groups), block(Shape<TEAM>::BLOCK);
      static_assert(Shape<TEAM>::TEAMS == (TEAM * NC <= 128 ? 4 : 1), "teams_per_group");
      if (dtype == AGRL_BF16 && dy_dtype == AGRL_BF16)
        hipLaunchKernelGGL((norm_bwd_kernel<uint16_t, uint16_t, TEAM, NC>), grid, block, 0, s, a);
      else if (dtype == AGRL_BF16)
        hipLaunchKernelGGL((norm_bwd_kernel<uint16_t, float, TEAM, NC>), grid, block, 0, s, a);
      else if (dy_dtype == AGRL_BF16)
        hipLaunchKernelGGL((norm_bwd_kernel<float, uint16_t, TEAM, NC>), grid, block, 0, s, a);
      else
        hipLaunchKernelGGL((norm_bwd_kernel<float, float, TEAM, NC>), grid, block, 0, s, a);
    });
  }
  if (params)
    hipLaunchKernelGGL(norm_param_reduce_kernel, dim3(cdiv(d, 64), 2), dim3(64 * RED_WAVES), 0, s,
                       (const float*)workspace, groups, d, dweight, dbias, accumulate);
  return hip_status(hipGetLastError());
}
