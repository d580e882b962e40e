// Y = A W^T with A [M, K] and W [N, K] in e4m3, a scale for each 1 x 128 block of A and each 128 x 128 block of W:
//   Y[m][n] = sum over blocks b of SA[m][b] SW[n / 128][b] sum over k in b of A[m][k] W[n][k].
// The sum inside a block is the matrix instruction's; the scaled sums are added in fp32.
#include "xorenc_fp8_plan.h"
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
    case 5: launch_ring<1, 1, 1, 1, 8, 2, EXACT>(g, st); break;
    case 6: launch_ring<2, 2, 1, 1, 8, 2, EXACT>(g, st); break;
    case 7: launch_ring<2, 2, 2, 1, 4, 3, EXACT>(g, st); break;
    case 8:
      if constexpr (!EXACT) launch_ring<2, 2, 2, 2, 2, 3, EXACT>(g, st);
      break;
    case 9:
      if constexpr (!EXACT) launch_tile<8, 3, 2, 4, EXACT>(g, st);
      break;
    case 10:
      if constexpr (!EXACT) launch_ring<4, 2, 2, 4, 1, 3, EXACT>(g, st);
      break;
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
