// The block-scaled product with an epilogue: Y = residual + f(A W^T + bias).  The kernels are those of the product alone, and so is the rule between them,
// but for one kernel more: the epilogue is a few instructions a result, and the residual as many bytes as Y.
#include "xorenc_fp8_dispatch.h"

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_linear_fp8(const uint8_t *A, int64_t lda, const float *SA, int64_t sa_row, int64_t sa_blk, const uint8_t *W,
                                     int64_t ldw, const float *SW, int64_t ldsw, int32_t M, int32_t N, int32_t K, const xorenc_epilogue *epilogue,
                                     void *Y, int32_t y_dtype, int64_t ldy, void *hip_stream) {
  int32_t rc = check_product(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, M, M, N, K, Y, y_dtype, ldy);
  if (rc != XORENC_OK) return rc;
  Linear job;
  rc = read_epilogue(epilogue, N, y_dtype, true, &job.epilogue);
  if (rc != XORENC_OK || M == 0) return rc;
  if (job.epilogue.residual && job.epilogue.residual == Y && job.epilogue.ld_residual != ldy && M > 1) return XORENC_EINVAL;
  if (job.epilogue.none()) return xorenc_matmul_fp8(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, M, N, K, Y, y_dtype, ldy, hip_stream);
  const MatmulArgs g = arguments_of(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, M, M, N, K, Y, ldy);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return y_dtype == XORENC_X_F32 ? dispatch_matmul<true>(cheapest_for_linear(M, N, g.blocks, true), g, job, st)
                                 : dispatch_matmul<false>(cheapest_for_linear(M, N, g.blocks, false), g, job, st);
}
