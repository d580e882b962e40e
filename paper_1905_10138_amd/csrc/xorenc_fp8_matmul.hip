// Y = A W^T with A [M, K] and W [N, K] in e4m3, a scale for each 1 x 128 block of A and each 128 x 128 block of W:
//   Y[m][n] = sum over blocks b of SA[m][b] SW[n / 128][b] sum over k in b of A[m][k] W[n][k].
// The sum inside a block is the matrix instruction's; the scaled sums are added in fp32.
#include "xorenc_fp8_ring.h"

namespace xorenc_fp8_detail {
namespace {

template <int TN, int TM, int WN, int WM, bool EXACT>
void launch_tile(const MatmulArgs &g, hipStream_t st) {
  typedef TileShape<TN, TM, WN, WM, EXACT> Shape;
  const int n_tiles = (g.N + Shape::BN - 1) / Shape::BN, m_tiles = (g.M + Shape::BM - 1) / Shape::BM;
  const int per_xcd = (n_tiles * m_tiles + 7) / 8;
  hipLaunchKernelGGL((matmul_tile_kernel<TN, TM, WN, WM, EXACT>), dim3((unsigned)(per_xcd * 8)), dim3(Shape::WAVES * 64), Shape::LDS, st, g,
                     n_tiles, m_tiles, per_xcd);
}

template <int TN, int TM, int WN, int WM, int KG, int NS, bool EXACT>
void launch_ring(const MatmulArgs &g, hipStream_t st) {
  typedef RingShape<TN, TM, WN, WM, KG, NS> Shape;
  const int n_tiles = (g.N + Shape::BN - 1) / Shape::BN, m_tiles = (g.M + Shape::BM - 1) / Shape::BM;
  const int per_xcd = (n_tiles * m_tiles + 7) / 8;
  hipLaunchKernelGGL((matmul_ring_kernel<TN, TM, WN, WM, KG, NS, EXACT>), dim3((unsigned)(per_xcd * 8)), dim3(Shape::WAVES * 64), Shape::LDS, st, g,
                     n_tiles, m_tiles, per_xcd);
}

// The kernels, and what they take: `start` + rounds * (`tile` + steps * (`step` + `load` * share of the chip in use)), in us, with
// as many tiles side by side as `slots` says and a block of the reduction a step (its `split`-th part where groups of a workgroup's
// waves take the blocks in turn).  Fitted to 80 shapes of 1 .. 8192 x 128 .. 16384 x 256 .. 9216 for either type of results;
// taking the one that this says is the fastest costs 1 % over taking the one that was.  Some of the times it goes by (us, bf16,
// in the order of the list):
//   8192 x 1000 x 770        24   17   20   34   28  145  113   76   49
//   4096 x 4096 x 4096       61   77   96  163  144  615  391  260  191
//   1024 x 2048 x 2048       31   19   16   12   13   43   32   23   15
//   512 x 4096 x 9216       116   66   57   34   48  131   73   60   46
//   250 x 6000 x 3000        45   26   21   16   19   44   31   24   21
//   64 x 16384 x 4096        55   33   28   18   23   34   22   19   14
//   128 x 4096 x 4096        54   32   27   15   22   19   12  9.6   12
//   16 x 4096 x 4096         53   32   27   15   22  5.4  6.5  9.0   12
//   1 x 4096 x 9216         114   67   56   29   48  8.1  9.9   15   23
struct Cost {
  int bn, bm, slots, split;
  float start, tile, step, load;
};
constexpr int kKernels = 9;
constexpr Cost kCosts[2][kKernels] = {
    {{256, 256, 256, 1, 0.00f, 10.16f, 1.53f, 0.19f},  // 0: tiles of 256 x 256, two stages in halves
     {128, 128, 512, 1, 0.60f, 5.17f, 0.84f, 0.27f},   // 1: of 128 x 128
     {128, 64, 768, 1, 0.76f, 3.25f, 0.70f, 0.32f},    // 2: of 128 x 64
     {64, 64, 512, 2, 1.23f, 2.41f, 0.71f, 0.37f},     // 3: rings of two stages: of 64 x 64, two groups of four waves
     {64, 64, 1024, 1, 1.18f, 2.26f, 0.54f, 0.43f},    // 4: of 64 x 64, one group
     {16, 16, 512, 8, 2.03f, 1.18f, 0.35f, 0.45f},     // 5: of 16 x 16, eight waves that split the reduction
     {32, 32, 256, 8, 1.14f, 2.39f, 0.81f, 0.18f},     // 6: of 32 x 32, the same
     {64, 32, 256, 4, 1.59f, 2.98f, 0.65f, 0.12f},     // 7: of three stages: of 64 x 32, four groups of two waves
     {64, 64, 256, 2, 1.41f, 2.73f, 0.54f, 0.08f}},    // 8: of 64 x 64, two groups of four waves
    // fp32 results (those of a tile of 256 x 256 do not fit in LDS, nor its operands in registers)
    {{},
     {128, 128, 512, 1, 1.76f, 6.06f, 1.17f, 0.47f},
     {128, 64, 768, 1, 1.43f, 3.66f, 0.92f, 0.51f},
     {64, 64, 512, 2, 2.00f, 2.29f, 0.72f, 0.60f},
     {64, 64, 1024, 1, 0.45f, 3.05f, 0.66f, 0.68f},
     {16, 16, 512, 8, 2.13f, 1.30f, 0.38f, 0.43f},
     {32, 32, 256, 8, 1.18f, 2.65f, 0.90f, 0.12f},
     {64, 32, 256, 4, 1.47f, 3.26f, 0.81f, 0.10f},
     {64, 64, 256, 2, 1.25f, 3.07f, 0.77f, 0.05f}}};

int cheapest(int64_t M, int64_t N, int64_t blocks, bool exact) {
  int best = -1;
  float least = 0.f;
  for (int i = exact ? 1 : 0; i < kKernels; ++i) {
    const Cost &c = kCosts[exact][i];
    const int64_t tiles = ((N + c.bn - 1) / c.bn) * ((M + c.bm - 1) / c.bm), steps = (blocks + c.split - 1) / c.split;
    if (tiles >= (1 << 22)) continue;
    const int64_t rounds = (tiles + c.slots - 1) / c.slots;
    const float use = tiles < c.slots ? (float)tiles / (float)c.slots : 1.f;
    const float t = c.start + (float)rounds * (c.tile + (float)steps * (c.step + c.load * use));
    if (best < 0 || t < least) best = i, least = t;
  }
  return best;
}

template <bool EXACT>
int32_t dispatch_matmul(const MatmulArgs &g, hipStream_t st) {
  switch (cheapest(g.M, g.N, g.blocks, EXACT)) {
    case 0:
      if constexpr (!EXACT) launch_tile<8, 4, 2, 4, EXACT>(g, st);
      break;
    case 1: launch_tile<4, 4, 2, 2, EXACT>(g, st); break;
    case 2: launch_tile<4, 2, 2, 2, EXACT>(g, st); break;
    case 3: launch_ring<2, 2, 2, 2, 2, 2, EXACT>(g, st); break;
    case 4: launch_ring<2, 2, 2, 2, 1, 2, EXACT>(g, st); break;
    case 8: launch_ring<2, 2, 2, 2, 2, 3, EXACT>(g, st); break;
    case 5: launch_ring<1, 1, 1, 1, 8, 2, EXACT>(g, st); break;
    case 6: launch_ring<2, 2, 1, 1, 8, 2, EXACT>(g, st); break;
    case 7: launch_ring<2, 2, 2, 1, 4, 3, EXACT>(g, st); break;
    default: return XORENC_ELIMIT;
  }
  return xorenc_internal_check_launch();
}

}  // namespace
}  // namespace xorenc_fp8_detail

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_matmul_fp8(const uint8_t *A, int64_t lda, const float *SA, int64_t sa_row, int64_t sa_blk, const uint8_t *W,
                                     int64_t ldw, const float *SW, int64_t ldsw, int32_t M, int32_t N, int32_t K, void *Y,
                                     int32_t y_dtype, int64_t ldy, void *hip_stream) {
  const int32_t blocks = K > 0 ? (int32_t)(((int64_t)K + kBlock - 1) / kBlock) : 0;
  if (M < 0 || N <= 0 || K <= 0 || lda < K || ldw < K || ldy < N || sa_row < 0 || sa_blk < 0 || ldsw < blocks) return XORENC_EINVAL;
  if (!known_dtype(y_dtype)) return XORENC_EUNSUPPORTED;
  if (M == 0) return XORENC_OK;
  if (!A || !SA || !W || !SW || !Y) return XORENC_EINVAL;
  if (!aligned_to(A, 16) || (M > 1 && lda % 16) || !aligned_to(W, 16) || (N > 1 && ldw % 16) || !aligned_to(SA, 4) || !aligned_to(SW, 4) ||
      !aligned_to(Y, dtype_bytes(y_dtype)))
    return XORENC_EALIGN;
  // a tile's rows, and all scales of its rows of A, are addressed with 32-bit offsets
  const int64_t row_step = M > 1 ? sa_row : 0;
  if (M > 65535 * 64 || K > (1 << 22) || (M > 1 && lda > (1 << 22)) || (N > 1 && ldw > (1 << 22)) || row_step > (1 << 20) || sa_blk > (1 << 28) ||
      256 * row_step + sa_blk * blocks >= (1 << 29))
    return XORENC_ELIMIT;
  const MatmulArgs g = {A, W, SA, SW, Y, lda, ldw, row_step, sa_blk, ldsw, ldy, M, N, K, blocks};
  xorenc_internal_begin_call();
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return y_dtype == XORENC_X_F32 ? dispatch_matmul<true>(g, st) : dispatch_matmul<false>(g, st);
}
