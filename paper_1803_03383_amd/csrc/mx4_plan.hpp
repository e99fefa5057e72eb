// How an MX4 product is made, plain C++: the launcher and the test of the choice use the same text.
#pragma once

#include <cmath>
#include <cstdint>

namespace halp {

// The edge of its tiles (256, 128, 64: one, two, three workgroups to a CU) and the parts that K is cut in.
struct ProductPlan {
  int tile, cuts;
};

// Small tiles fill the CUs where there are few, at the price of more reads; parts cost a pass over
// them.  The choice is the least of an estimate in microseconds fitted to timings of 21 sizes on this GPU (its choices take
// 1 % longer than the best there, the worst 10 %): a stage takes 1.9 with 256-tiles on every CU (1.0 with a few: the
// power limit), 0.77 and 1.27 with one and two 128-tiles on a CU, 0.42 to 0.8 with one to three 64-tiles; beginning and
// ending a tile 10.5, 4 and 3.4.  On both sides of its borders (measured, us): 4096 x 4096 x 2048 28 / 29 / 44 with
// 256 / 128 / 64, 4096 x 2048 x 4096 31 / 26 / 42, 300 x 4096 x 4096 27 / 13.3 / 13.0; 1000 x 784 x 60000 with 128 in
// 1, 2, 4, 8, 16 parts 152, 82, 50, 49, 57.
inline double product_us(int64_t M, int64_t N, int64_t K, int cus, ProductPlan p) {
  const int most = p.tile == 256 ? 1 : p.tile == 128 ? 2 : 3;
  const auto stage_us = [&](double per_cu) {  // workgroups per CU
    const int n = (int)std::ceil(per_cu);
    if (p.tile == 256) return 1.0 + 0.9 * (per_cu < 1 ? per_cu : 1);
    if (p.tile == 128) return n == 1 ? 0.77 : 1.27;
    return n == 1 ? 0.42 : n == 2 ? 0.61 : 0.8;
  };
  const int64_t stages = (K + 255) / 256;
  const double blocks = (double)((M + p.tile - 1) / p.tile) * ((N + p.tile - 1) / p.tile) * p.cuts / cus;  // per CU
  const double ends = p.tile == 256 ? 10.5 : p.tile == 128 ? 4 : 3.4, full = std::floor(blocks / most), rest = blocks - full * most;
  const double length = (double)((stages + p.cuts - 1) / p.cuts);
  double us = full * (length * stage_us(most) + ends);
  if (rest > 0) us += length * stage_us(rest) + ends;
  if (p.cuts > 1) us += 4.4 + (double)p.cuts * M * N * 8 / 8.5e6;
  return us;
}

// the best plan of at most so many parts, each of four stages of 256 values or more
inline ProductPlan product_plan(int64_t M, int64_t N, int64_t K, int cus, int most_cuts) {
  const int64_t stages = (K + 255) / 256;
  ProductPlan best{128, 1};
  double least = 1e300;
  for (int tile = 256; tile >= 64; tile /= 2)
    for (int cuts = 1; cuts == 1 || (cuts <= most_cuts && stages / cuts >= 4); cuts *= 2) {
      const double us = product_us(M, N, K, cus, {tile, cuts});
      if (us < least) least = us, best = {tile, cuts};
    }
  return best;
}

constexpr int kMostCuts = 16;

inline int64_t parts_stride(int64_t N) { return (N + 3) / 4 * 4; }

// bytes that the parts of a plan take
inline int64_t plan_workspace(int64_t M, int64_t N, ProductPlan p) {
  return p.cuts > 1 ? (int64_t)sizeof(float) * p.cuts * M * parts_stride(N) : 0;
}

// The plan of a product with this much workspace.  Where the parts do not fit, the tiles are chosen again: those that are best
// in parts may leave CUs idle alone.  Uncut, in the tiles that are best in parts and in those taken here, us: 1000 x 784 x 60000
// 153 and 100, 2000 x 2000 x 30000 185 and 96, 1024 x 1024 x 16384 40 and 31, 3000 x 500 x 10000 33 and 35.
inline ProductPlan product_plan_within(int64_t M, int64_t N, int64_t K, int cus, int64_t workspace_bytes) {
  const ProductPlan p = product_plan(M, N, K, cus, kMostCuts);
  return workspace_bytes < plan_workspace(M, N, p) ? product_plan(M, N, K, cus, 1) : p;
}

}  // namespace halp
