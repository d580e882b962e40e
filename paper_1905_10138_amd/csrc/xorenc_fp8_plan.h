// Which kernel a block-scaled product takes (host code, without HIP).
#ifndef XORENC_FP8_PLAN_H
#define XORENC_FP8_PLAN_H

#include <cstdint>

namespace xorenc_fp8_detail {

// The kernels, and what they take: `start` + rounds * (`tile` + steps * (`step` + `load` * share of the chip in use)), in us, with
// as many tiles side by side as `slots` says and a block of the reduction a step (its `split`-th part where groups of a workgroup's
// waves take the blocks in turn).  Fitted to 190 shapes of 1 .. 8192 x 64 .. 16384 x 64 .. 9216 for either type of results;
// taking the one that this says is the fastest costs 1.4 % (fp32 1.0 %) over taking the one that was.  Some of the times it goes
// by (us, bf16, in the order of the list):
//   8192 x 1000 x 770    23   16   20   34   27  145  113   75   49   19   23
//   4096 x 4096 x 4096   64   78   97  162  144  619  382  258  189   97  107
//   3000 x 3000 x 3000   47   56   52   74   68  277  198  136   96   41   63
//   1024 x 2048 x 2048   31   18   15   11   13   44   31   23   15   27   16
//   700 x 4096 x 4096    56   32   29   30   25   80   54   47   34   48   27
//   512 x 4096 x 9216   117   66   57   35   48  128   72   60   46  101   54
//   250 x 6000 x 3000    46   26   21   16   20   44   31   24   21   39   22
//   64 x 16384 x 4096    55   32   28   18   24   35   23   19   14   48   27
//   128 x 4096 x 4096    55   32   27   16   23   19   12  9.5   12   48   26
//   16 x 4096 x 4096     54   32   27   15   23  5.6  6.5  9.0   12   48   26
//   1 x 4096 x 9216     116   66   56   29   48  8.1  9.9   15   22  101   53
struct Cost {
  int bn, bm, slots, split;
  float start, tile, step, load;
};
constexpr int kKernels = 11;
constexpr Cost kCosts[2][kKernels] = {
    {{256, 256, 256, 1, 2.55f, 6.96f, 1.48f, 0.28f},   // 0: tiles of 256 x 256, two stages in halves
     {128, 128, 512, 1, 1.60f, 3.84f, 0.78f, 0.34f},   // 1: of 128 x 128
     {128, 64, 768, 1, 1.62f, 2.07f, 0.63f, 0.41f},    // 2: of 128 x 64
     {64, 64, 512, 2, 1.84f, 2.08f, 0.59f, 0.49f},     // 3: rings of two stages: of 64 x 64, two groups of four waves
     {64, 64, 1024, 1, 0.59f, 2.52f, 0.51f, 0.47f},    // 4: of 64 x 64, one group
     {16, 16, 512, 8, 2.87f, 1.11f, 0.24f, 0.42f},     // 5: of 16 x 16, eight waves that split the reduction
     {32, 32, 256, 8, 2.50f, 1.86f, 0.41f, 0.36f},     // 6: of 32 x 32, the same
     {64, 32, 256, 4, 2.11f, 2.54f, 0.55f, 0.19f},     // 7: of three stages: of 64 x 32, four groups of two waves
     {64, 64, 256, 2, 1.88f, 2.25f, 0.50f, 0.13f},     // 8: of 64 x 64, two groups of four waves
     {256, 192, 256, 1, 2.00f, 5.75f, 1.27f, 0.19f},   // 9: as 0, of 256 x 192
     {128, 128, 256, 1, 1.77f, 2.85f, 0.67f, 0.08f}},  // 10: as 8, of 128 x 128, one group of eight waves
    // fp32 results (those of 0 and 9 do not fit in LDS, nor the operands of 0 in registers; 8 and 10 would be taken for no size; of 3
    // two workgroups fit on a CU, but 256 slots are nearer to its times)
    {{},
     {128, 128, 512, 1, 0.81f, 5.84f, 1.23f, 0.45f},
     {128, 64, 768, 1, 1.45f, 3.22f, 0.88f, 0.63f},
     {64, 64, 256, 2, 3.24f, 0.91f, 0.70f, 0.00f},
     {64, 64, 768, 1, 0.99f, 2.44f, 0.60f, 0.38f},
     {16, 16, 512, 8, 2.58f, 1.27f, 0.33f, 0.38f},
     {32, 32, 256, 8, 2.17f, 2.40f, 0.62f, 0.20f},
     {64, 32, 256, 4, 1.95f, 2.81f, 0.75f, 0.16f},
     {},
     {},
     {}}};

inline int cheapest(int64_t M, int64_t N, int64_t blocks, bool exact) {
  int best = -1;
  float least = 0.f;
  for (int i = 0; i < kKernels; ++i) {
    const Cost &c = kCosts[exact][i];
    if (!c.bn) continue;
    const int64_t tiles = ((N + c.bn - 1) / c.bn) * ((M + c.bm - 1) / c.bm), steps = (blocks + c.split - 1) / c.split;
    if (tiles >= (1 << 22)) continue;
    const int64_t rounds = (tiles + c.slots - 1) / c.slots;
    const float use = tiles < c.slots ? (float)tiles / (float)c.slots : 1.f;
    const float t = c.start + (float)rounds * (c.tile + (float)steps * (c.step + c.load * use));
    if (best < 0 || t < least) best = i, least = t;
  }
  return best;
}

}  // namespace xorenc_fp8_detail

#endif
