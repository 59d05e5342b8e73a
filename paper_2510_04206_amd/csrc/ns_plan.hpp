// Which tiles and launches the Newton-Schulz products take, and their workspace: host arithmetic only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/agrl.h"

namespace agrl {
namespace ns {

constexpr int SPLIT_ROWS = 128;                     // bf16 results of up to so many rows take two parts, too
constexpr int SMALL_ROWS = 64, SMALL_K = 256;       // a matrix that one workgroup takes whole
constexpr int NORM_GROUPS = 256;   // workgroups of a matrix's sum of squares, at most
constexpr int NORM_THREADS = 1024;

constexpr int64_t MAX_SIDE = (int64_t)1 << 20, MAX_SHORT = (int64_t)1 << 16, MAX_BATCH = 65535;

// A launch of a product: `units` of the product's numbering (see Args) by tile `tile`.
struct Part {
  int32_t tile, units;
};
constexpr int PARTS = 3;

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Sizes and the workspace of a stack of matrices
struct Plan {
  int64_t batch;
  int32_t r, k, tall, one;                  // one: ns_small_kernel's
  Part part_of[3][PARTS];                   // of A, B and X; the first one's tile is the unit
  int64_t r_pad, k_pad;
  int32_t split, n_part;
  int64_t x_plane, a_plane;                 // elements
  size_t part, x[2], a, b, total;           // bytes
};

// The tiles that a launch can take, and the time of one, in microseconds: a round of workgroups
// lasts its stages and its end, a launch's start comes on top.  Fitted to launches that were
// measured; in two parts a last round that fills part of the chip runs faster (the compute units
// in it share less power and bandwidth), which the wide tiles' own figures hold already.
struct Kind {
  int rows, cols, round;      // round: workgroups that the chip holds
  double one, two, start;     // a stage of one part, of two; a launch
  double end[2];              // a round's end in A and A A, and in B X
  double part;                // what of a round's time is left as its share of the chip goes to 0
};
constexpr int K64 = 0, K128 = 1, K128_PAIR = 2, K256 = 3, K256_SQUARE = 4;
constexpr Kind KINDS[] = {
    {64, 64, 256, 0.24, 0.30, 6.0, {0.0, 0.0}, 1.0},      // nine stages in flight: few, small matrices
    {128, 128, 256, 0.62, 1.00, 6.0, {0.0, 0.0}, 0.7},    // four, one workgroup a compute unit
    {128, 128, 512, 0.95, 1.30, 6.0, {0.0, 0.0}, 1.0},    // two, two workgroups
    {256, 128, 256, 0.79, 0.0, 6.0, {3.0, 14.0}, 1.0},    // (the sums of two parts would not fit
    {256, 256, 256, 1.20, 0.0, 4.0, {18.0, 10.0}, 1.0},   // the registers of these two)
};
// e.g. B X of 1024 x 1024: 9.5 us with the first, 18 and 24 us with the third and fourth; of 8 of
// them 42, 32 and 29; of 2048 x 2048 36 us, 26 with the second, 33, 37; of 4096 x 4096 254, 137
// (third), 125 to 135 and, with the fifth, 114.  In two parts: of 1024 x 1024 16 us, third 36; of
// 8 of them 95, 57; of 4096 x 4096 557, 342; five steps of 2048 x 2048 900 us with the third, 797
// with the second where it fits.
inline double launch_us(const Kind& k, bool split, bool update, int64_t items, double stages) {
  const int64_t whole = items / k.round, rest = items % k.round;
  const double part = split ? k.part : 1.0;
  const double rounds = whole + (rest ? part + (1.0 - part) * rest / k.round : 0.0);
  return rounds * (stages * (split ? k.two : k.one) + k.end[update]) + k.start;
}

// Each product takes the tile that is done first; where its last round would leave most of the
// chip idle, that round's units go to a launch of smaller tiles, and so on (B X of 14336 x 3584: 784
// tiles of 256 x 256 are three rounds of 256 and 16 units more, which go by 64 x 64).  The time of
// `units` of unit kind `of` by tile t and smaller ones; out: the launches, `left` of them at most.
inline double plan_parts(bool split, bool update, double stages, int of, int t, int64_t units,
                         int left, Part* out) {
  const Kind& k = KINDS[t];
  const int64_t per = (int64_t)(KINDS[of].rows / k.rows) * (KINDS[of].cols / k.cols);
  double best = launch_us(k, split, update, units * per, stages);
  out[0] = Part{t, (int32_t)units};
  if (left > 1) out[1].units = 0;
  const int64_t whole = units * per / k.round * k.round / per;
  if (left == 1 || whole == 0 || whole == units) return best;
  const double first = launch_us(k, split, update, whole * per, stages);
  for (int next = K64; next < t; ++next) {
    if (KINDS[next].rows * KINDS[next].cols >= k.rows * k.cols) continue;
    Part rest[PARTS] = {};
    const double us =
        first + plan_parts(split, update, stages, of, next, units - whole, left - 1, rest);
    if (us >= best) continue;
    best = us;
    out[0].units = (int32_t)whole;
    for (int i = 1; i < left; ++i) out[i] = rest[i - 1];
  }
  return best;
}

inline void choose_tiles(Plan* p) {
  for (int i = 0; i < 3; ++i) {
    double best = 0.0;
    const double stages = (i == 0 ? p->k : p->r) / (p->split ? 32.0 : 64.0);
    for (int t = K64; t <= (p->split ? K128_PAIR : K256_SQUARE); ++t) {
      const Kind& k = KINDS[t];
      const int64_t r = ceil_div(p->r, k.rows), x = ceil_div(p->k, k.rows);
      const int64_t units = p->batch * (i == 2 ? r * x : r * (r + 1) / 2) * (k.rows / k.cols);
      Part parts[PARTS] = {};
      const double us = plan_parts(p->split, i == 2, stages, t, t, units, PARTS, parts);
      if (t > K64 && us >= best) continue;
      best = us;
      for (int j = 0; j < PARTS; ++j) p->part_of[i][j] = parts[j];
    }
  }
}

inline bool make_plan(int64_t batch, int64_t m, int64_t n, int32_t out_dtype, Plan* p) {
  if (batch <= 0 || batch > MAX_BATCH || m <= 0 || n <= 0 || m > MAX_SIDE || n > MAX_SIDE)
    return false;
  const int64_t r = m < n ? m : n, k = m < n ? n : m;
  if (r > MAX_SHORT) return false;
  p->batch = batch, p->r = (int32_t)r, p->k = (int32_t)k, p->tall = m > n;
  p->split = out_dtype == AGRL_F32 || r <= SPLIT_ROWS;
  choose_tiles(p);
  p->one = p->r <= SMALL_ROWS && p->k <= SMALL_K;
  int64_t pad = 128;
  for (const auto& parts : p->part_of)
    if (KINDS[parts[0].tile].rows > pad) pad = KINDS[parts[0].tile].rows;
  p->r_pad = p->one ? 64 : ceil_div(r, pad) * pad;
  p->k_pad = ceil_div(k, pad) * pad;
  const int64_t per = ceil_div(m * ceil_div(n, (int64_t)8), (int64_t)NORM_THREADS);
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

// The launches of product i (A, A A, B X), as they are made: `count` units of unit_m x unit_n from
// `first` on, by tiles of kind `tile`.
struct Launch {
  int32_t tile, first, count;
  int32_t unit_m, unit_n, units_m, units_n, units;   // units: of a matrix
  int32_t halves_log;                                // units of a square
};
inline int product_launches(const Plan& p, int i, Launch* out) {
  const Kind& k = KINDS[p.part_of[i][0].tile];
  Launch l = {};
  l.unit_m = k.rows, l.unit_n = k.cols;
  l.units_m = (int32_t)((i == 2 ? p.k_pad : p.r_pad) / l.unit_m);
  l.units_n = (int32_t)(p.r_pad / l.unit_n);
  l.halves_log = k.rows == 2 * k.cols;
  l.units = i == 2 ? l.units_m * l.units_n
                   : l.units_m * (l.units_m + 1) / 2 * (l.unit_m / l.unit_n);
  const int32_t all = (int32_t)(l.units * p.batch);
  int n = 0;
  for (int j = 0; j < PARTS && l.first < all; ++j) {
    const Part* const part = &p.part_of[i][j];
    // (the padding may hold more units than were counted: the last launch takes all that is left)
    const bool last = j == PARTS - 1 || part[1].units == 0;
    l.tile = part->tile;
    l.count = last || part->units > all - l.first ? all - l.first : part->units;
    out[n++] = l;
    l.first += l.count;
  }
  return n;
}

}  // namespace ns
}  // namespace agrl
