// Y = A W^T with A [M, K] and W [N, K] in e4m3, a scale for each 1 x 128 block of A and each 128 x 128 block of W:
//   Y[m][n] = sum over blocks b of SA[m][b] SW[n / 128][b] sum over k in b of A[m][k] W[n][k].
// The sum inside a block is the matrix instruction's; the scaled sums are added in fp32.
#include "xorenc_fp8_dispatch.h"

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_matmul_fp8(const uint8_t *A, int64_t lda, const float *SA, int64_t sa_row, int64_t sa_blk, const uint8_t *W,
                                     int64_t ldw, const float *SW, int64_t ldsw, int32_t M, int32_t N, int32_t K, void *Y,
                                     int32_t y_dtype, int64_t ldy, void *hip_stream) {
  const int32_t rc = check_product(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, M, M, N, K, Y, y_dtype, ldy);
  if (rc != XORENC_OK || M == 0) return rc;
  const MatmulArgs g = arguments_of(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, M, M, N, K, Y, ldy);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return y_dtype == XORENC_X_F32 ? dispatch_matmul<true>(cheapest(M, N, g.blocks, true), g, Plain(), st)
                                 : dispatch_matmul<false>(cheapest(M, N, g.blocks, false), g, Plain(), st);
}
