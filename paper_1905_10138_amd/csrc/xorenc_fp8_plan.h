// Which kernel a block-scaled product takes (host code, without HIP).
#ifndef XORENC_FP8_PLAN_H
#define XORENC_FP8_PLAN_H

#include <cmath>
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

inline bool takes(const Cost &c, int64_t M, int64_t N, int64_t blocks, float *us) {
  if (!c.bn) return false;
  const int64_t tiles = ((N + c.bn - 1) / c.bn) * ((M + c.bm - 1) / c.bm), steps = (blocks + c.split - 1) / c.split;
  if (tiles >= (1 << 22)) return false;
  const int64_t rounds = (tiles + c.slots - 1) / c.slots;
  const float use = tiles < c.slots ? (float)tiles / (float)c.slots : 1.f;
  *us = c.start + (float)rounds * (c.tile + (float)steps * (c.step + c.load * use));
  return true;
}

inline int cheapest(int64_t M, int64_t N, int64_t blocks, bool exact) {
  int best = -1;
  float least = 0.f, t;
  for (int i = 0; i < kKernels; ++i)
    if (takes(kCosts[exact][i], M, N, blocks, &t) && (best < 0 || t < least)) best = i, least = t;
  return best;
}

// The products with an epilogue have one kernel more: rings of two stages, of 32 x 16, four waves that split the reduction (11).  Of 1363 shapes of 1 .. 64 x
// 128 .. 16384 x 128 .. 9216 it is the fastest of 560 (fp32 530); the choice costs 1.9 % (0.6 %) over the fastest kernel's times, without it 3.4 %
// (3.1 %).  (us, with a bias, this and the fastest of the others: 1 x 9216 x 4096 9.1 and 10.3, 1 x 16384 x 4096 12.0 and 13.4, 32 x 9216 x 4096 10.1
// and 10.7, 16 x 4096 x 4096 8.2 and 5.8.)
constexpr Cost kFewRows[2] = {{32, 16, 768, 4, 3.52f, 0.33f, 0.35f, 0.75f}, {32, 16, 768, 4, 3.41f, 0.39f, 0.40f, 0.78f}};
constexpr int kFewRowsKernel = 11;
inline int cheapest_for_linear(int64_t M, int64_t N, int64_t blocks, bool exact) {
  const int best = cheapest(M, N, blocks, exact);
  float few, least;
  return M <= 64 && best >= 0 && takes(kFewRows[exact], M, N, blocks, &few) && takes(kCosts[exact][best], M, N, blocks, &least) && few < least
             ? kFewRowsKernel : best;
}

// The products of rows sorted by expert.  Their tiles come in all degrees of emptiness, and their weights from memory: the kernels take
//   start + (rounds + `tail`) * (`tile` + steps * (`step` + `load` * share of the chip in use)) + `byte` * (MB of the weights of experts that have rows),
// with rounds not rounded, and no tail up to one.  Fitted to 2815 shapes of 1 .. 8192 tokens, 1 .. 8 picks of 2 .. 128 experts of 128 .. 9216 x
// 128 .. 9216, 1200 of them of 15 to 500 G products, with experts that differ in their shares by a factor of four; taking the one that this says is the
// fastest costs 2.1 % (fp32 0.9 %) over taking the one that was, on the quarter of them that was not fitted to.
// Some of the times it goes by (us, bf16, in the order of the list; tokens x picks x experts x outputs x inputs):
//   4096x2x8x8192x4096     332  390  458  763  630 3150 1030  359 1950 1190
//   2048x8x64x1024x2048     80   84   86  133  108  599  186   72  300  181
//   512x2x8x4096x4096       73   57   56   75    -    -    -   66  135  110
//   256x8x64x1024x2048      41   33   32   46   44  109   58   37   57   47
//   64x2x8x4096x4096        70   48   44   33   42   50   42   63   37   39
//   64x6x64x2048x1024        -    -   35   43    -   76   65    -   36   31
//   4x2x8x4096x4096          -    -   38   25    -   25   35    -   20   36
//   1x6x64x2048x1024         -    -   11  8.2    -  9.4  8.3    -  6.6   11
struct ExpertsCost {
  int bn, bm, slots, split;
  float start, tile, step, load, byte, tail;
};
constexpr int kExpertsKernels = 13;  // 0 .. 10 as above, of which 6, 7 and 10 would be the fastest for hardly any size
constexpr ExpertsCost kExpertsCosts[2][kExpertsKernels] = {
    {{256, 256, 256, 1, 18.66f, 2.12f, 1.37f, 0.18f, 0.002f, 0.90f},
     {128, 128, 512, 1, 0.24f, 7.85f, 1.09f, 0.15f, 0.012f, 0.44f},
     {128, 64, 768, 1, 3.57f, 0.99f, 0.84f, 0.30f, 0.070f, 1.37f},
     {64, 64, 512, 2, 2.18f, 6.09f, 0.71f, 0.28f, 0.082f, 1.00f},
     {64, 64, 1024, 1, 0.67f, 2.00f, 0.73f, 1.11f, 0.205f, 0.74f},
     {16, 16, 512, 8, 0.99f, 3.48f, 0.03f, 1.45f, 0.006f, 0.35f},
     {},
     {},
     {64, 64, 256, 2, 1.76f, 3.63f, 0.65f, 0.03f, 0.072f, 1.17f},
     {256, 192, 256, 1, 1.18f, 7.77f, 1.47f, 0.05f, 0.008f, 0.74f},
     {},
     {32, 16, 768, 4, 0.23f, 2.47f, 0.73f, 0.59f, 0.037f, 0.68f},    // 11: rings of two stages: of 32 x 16, four waves that split the reduction
     {64, 32, 1024, 1, 1.38f, 2.07f, 0.76f, 0.40f, 0.021f, 2.97f}},  // 12: of three: of 64 x 32, one group of two waves
    {{},
     {128, 128, 512, 1, 12.12f, 5.45f, 1.49f, 0.22f, 0.020f, 0.46f},
     {128, 64, 768, 1, 3.71f, 3.09f, 1.09f, 0.79f, 0.012f, 0.25f},
     {64, 64, 512, 2, 0.61f, 5.36f, 0.56f, 0.99f, 0.086f, 0.24f},
     {64, 64, 768, 1, 0.35f, 2.63f, 1.06f, 0.39f, 0.186f, 1.02f},
     {16, 16, 512, 8, 1.63f, 3.42f, 0.08f, 1.38f, 0.013f, 0.25f},
     {},
     {},
     {},
     {},
     {},
     {32, 16, 768, 4, 0.53f, 2.74f, 0.82f, 0.37f, 0.023f, 0.68f},
     {64, 32, 1024, 1, 0.41f, 3.35f, 1.12f, 0.19f, 0.019f, 1.07f}}};

// `rows` rows sorted by expert: at most this many tiles of bm rows, whatever the experts' shares (one row each for as many as there
// are, the rest in whole tiles).
inline int64_t most_tiles_of_experts(int64_t rows, int64_t experts, int bm) {
  const int64_t some = rows < experts ? rows : experts;
  return some + (rows - some) / bm;
}

// Experts' weights of 96 MB and more, which a last cache of 256 MB would not keep until the next call, are read past the caches where one tile of bm rows
// takes an expert's (us: 64 tokens, two of eight experts of 4096 x 4096 36.5 and 33.4, 128 tokens 37.1 and 34.1, 30 tokens of 9216 x 4096 71 and 57; 256
// tokens, eight of 64 of 1024 x 2048, 34.2 and 32.6; 512 of the first, two tiles an expert, 74.8 and 77.3).
inline bool streams_weights(int64_t rows, int64_t experts, int64_t bytes_of_one, int bm) {
  return bytes_of_one >= ((int64_t)96 << 20) / (rows < experts ? rows : experts) && rows <= experts * bm;
}

// What streams_weights counts of each expert: the bytes of its matrix, whatever lies between its rows, and none where experts share some of them (one matrix
// for all, w_stride 0, or strides that let them overlap), as what one expert has read is there for the next.  Matrices are apart one after the other, or in
// turn, a row of each.  (us, past the caches and through them: 128 tokens, two of eight experts that are one matrix of 4096 x 4096 32.0 and 25.1; that are
// 4096 x 1024 in rows of 8192 15.3 and 11.3.)
inline int64_t bytes_of_one_expert(int64_t experts, int64_t N, int64_t K, int64_t ldw, int64_t w_stride) {
  const bool apart = experts == 1 || w_stride >= (N - 1) * ldw + K || (w_stride >= K && (experts - 1) * w_stride + K <= ldw);
  return apart ? N * ((K + 15) / 16 * 16) : 0;
}

inline int cheapest_for_experts(int64_t rows, int64_t experts, int64_t N, int64_t blocks, bool exact) {
  const float all = (float)rows, used = (float)experts * (1.f - expf(-all / (float)experts));  // (experts that have rows)
  const float weights = used * (float)N * (float)blocks * 128e-6f;
  int best = -1;
  float least = 0.f;
  for (int i = 0; i < kExpertsKernels; ++i) {
    const ExpertsCost &c = kExpertsCosts[exact][i];
    if (!c.bn) continue;
    const int64_t n_tiles = (N + c.bn - 1) / c.bn, steps = (blocks + c.split - 1) / c.split;
    if (n_tiles * most_tiles_of_experts(rows, experts, c.bm) >= (1 << 22)) continue;
    const float more = all - used * 0.5f * (float)c.bm;  // an expert's last tile is half empty
    const float rounds = (float)n_tiles * (used + (more > 0.f ? more / (float)c.bm : 0.f)) / (float)c.slots;
    const float use = rounds < 1.f ? rounds : 1.f, in_turn = rounds > 1.f ? rounds + c.tail : 1.f;
    const float t = c.start + in_turn * (c.tile + (float)steps * (c.step + c.load * use)) + c.byte * weights;
    if (best < 0 || t < least) best = i, least = t;
  }
  return best;
}

}  // namespace xorenc_fp8_detail

#endif
