"""Sizes that take every launch that the Newton-Schulz products can take, and the plans behind them.

A launch's class is (product 0 A, 1 A A, 2 B X; parts 1 or 2; the unit's tile; the launch's own tile;
its place among the launches of the product; whether its workgroups run on from tile to tile).
"""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (batch, rows, columns, result in fp32): found by search among cheap ragged sizes
SIZES = [
    (26, 2194, 2194, False), (20, 2246, 2246, False), (1, 6027, 6657, False), (5, 2473, 3952, False),
    (6, 2177, 2177, False), (2, 2946, 2946, False), (21, 1186, 1186, False), (5, 1679, 2565, False),
    (53, 276, 4282, False), (13, 1026, 1026, False), (49, 643, 643, False), (47, 515, 515, True),
    (2, 818, 9983, False), (41, 516, 516, True), (52, 449, 449, False), (55, 386, 397, True),
    (50, 129, 714, False), (52, 195, 195, False), (52, 193, 193, True), (53, 130, 257, False),
    (57, 65, 536, False), (26, 129, 129, True), (17, 129, 130, False), (1, 129, 129, False),
    (1, 16, 257, False),
]

_MAIN = r"""
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include "ns_plan.hpp"
using namespace agrl::ns;
static void classes(long b, long m, long n, int out) {
  Plan p;
  if (!make_plan(b, m, n, out, &p) || p.one) return;
  for (int i = 0; i < 3; ++i) {
    Launch l[PARTS];
    const int count = product_launches(p, i, l);
    long covered = 0;
    for (int j = 0; j < count; ++j) {
      const Kind& k = KINDS[l[j].tile];
      const long items = (long)l[j].count * (l[j].unit_m / k.rows) * (l[j].unit_n / k.cols);
      printf("%d %d %d %d %d %d\n", i, p.split ? 2 : 1, p.part_of[i][0].tile, l[j].tile, j,
             items > k.round);
      if (l[j].first != covered || l[j].count <= 0 || l[j].unit_m % k.rows || l[j].unit_n % k.cols) abort();
      covered += l[j].count;
    }
    if (covered != (long)l[0].units * b) abort();
  }
}
int main(int argc, char** argv) {
  if (argc == 5) return classes(atol(argv[1]), atol(argv[2]), atol(argv[3]), atoi(argv[4])), 0;
  // a sweep, over the logarithm of the sizes: up to 2e14 operations a step, half of them ragged
  unsigned long long s = strtoull(argv[1], 0, 10);
  auto u = [&]() {
    s = s * 6364136223846793005ull + 1442695040888963407ull;
    return (double)(s >> 11) / 9007199254740992.0;
  };
  for (long t = atol(argv[2]); t > 0; --t) {
    const double r0 = exp(log(16) + u() * log(20000 / 16.0));
    long r = (long)r0, k = (long)(r0 * exp(u() * log(u() < 0.5 ? 16.0 : 1.3)));
    if (u() < 0.3) r = (r + 63) / 64 * 64, k = (k + 63) / 64 * 64;
    if (u() < 0.1 || k < r) k = r;
    const long b = u() < 0.5 ? 1 : (long)exp(u() * log(64.0));
    const int out = u() < 0.7 ? AGRL_BF16 : AGRL_F32;
    if ((double)b * r * r * (3.0 * k + r) <= 2e14) classes(b, r, k, out);
  }
}
"""


def compiled(folder):
    """The program that prints plans' classes, from the host's own planning code; None without g++."""
    import shutil
    gxx = shutil.which("g++")
    if gxx is None:
        return None
    src, exe = os.path.join(folder, "plans.cpp"), os.path.join(folder, "plans")
    with open(src, "w") as f:
        f.write(_MAIN)
    subprocess.run([gxx, "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2510_04206_amd", "csrc"),
                    src, "-o", exe], check=True)
    return exe


def classes(exe, *args):
    out = subprocess.run([exe, *map(str, args)], check=True, capture_output=True, text=True).stdout
    return {tuple(map(int, line.split())) for line in out.splitlines()}
