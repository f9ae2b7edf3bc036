// Which kernel a product of microscaled matrices runs on (k_mx.hip).  Plain C++, so
// that the choice can be looked at without a GPU.
#pragma once

#include <algorithm>
#include <cstddef>

namespace msd {

constexpr int MX_GROUP = 512;   // columns of a group of scales
constexpr int SPLIT_WAVES = 8;  // waves that share K in the split kernel

// How a product runs: the split kernel over tiles of 16 MT rows x 16 CT columns, or
// (CT = 0) the tile kernel over BM x BN.
struct ProductPlan {
  int MT, CT, BM, BN;
};

// Picks the kernel with the least estimated time (us), from the workgroups W on 256
// CUs and the groups g of 512 columns of K:
//  split  1.5 + the longer of l and, for W > 256, the CU with most workgroups times its
//         256 c: l, what a workgroup takes alone, goes by the rounds of g over its eight
//         waves (less for fewer groups than waves) and the pieces n that it loads per tile
//         along K; c is its share of the memory path;
//  tile   f + rounds of W x 4 g steps of s + the output's writing, or W's bytes at the
//         5 TB/s that these kernels read (4.6 to 4.9 measured, the split kernel 5.8).
// On the 377 products that the constants were fitted to (15 weights of 512 x 8192 to
// 152064 x 3584, 1 to 12288 rows, one and two terms) the choice costs 0.8% over the best
// kernel on average, 18% at worst (1536 x 4096 x 11008, one term: 59 us for 50; before the
// 64 x 128 kernel became up to 6% faster, for which its two rates are 4% lower).  With W
// itself in place of the fullest CU's workgroups and no limit on the tile kernels' reading
// (on 285 of them) it was 1.9% and 36%.
inline ProductPlan plan_product(int M, int N, int g, int terms) {
  ProductPlan best{};
  float best_us = 0.f;
  const auto take = [&](float us, const ProductPlan& p) {
    if (best_us == 0.f || us < best_us) best_us = us, best = p;
  };
  const int MT = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  for (int CT : {1, 2, 4}) {
    const size_t W = (size_t)((M + 16 * MT - 1) / (16 * MT)) * ((N + 16 * CT - 1) / (16 * CT));
    const int n = MT * terms + CT;
    const float rounds = g >= SPLIT_WAVES ? (g + SPLIT_WAVES - 1) / SPLIT_WAVES
                                          : 0.4f + 0.6f * g / SPLIT_WAVES;
    const float l = rounds * (0.24f * n + 0.76f * CT + 0.52f) + 0.13f * MT * CT;
    const float c = 1e-3f * (g * (0.26f * n + 0.155f * CT + 0.08f) + 0.69f * MT * CT);
    take(1.5f + (W <= 256 ? l : std::max(l, (float)((W + 255) / 256) * 256.f * c)), {MT, CT, 0, 0});
  }
  const struct {
    int BM, BN;
    float f, s[2];
  } tiles[] = {{64, 128, 4.f, {0.205f, 0.268f}},
               {128, 256, 10.8f, {0.522f, 0.748f}},
               {256, 256, 5.9f, {1.09f, 1.49f}}};
  const float read = 2.f + (float)N * g * MX_GROUP * (0.53125e-6f / 5.f);
  for (const auto& t : tiles) {
    const size_t W = (size_t)((M + t.BM - 1) / t.BM) * ((N + t.BN - 1) / t.BN);
    const float us = t.f + (float)((W + 255) / 256) * 4 * g * t.s[terms - 1] + (float)M * N * 0.35e-6f;
    take(std::max(us, read), {0, 0, t.BM, t.BN});
  }
  return best;
}

}  // namespace msd
