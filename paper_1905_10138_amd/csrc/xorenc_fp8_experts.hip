// Products of rows that are sorted by expert with their own expert's matrix: Y[i] = f(A[r(i)] W_e^T + bias_e).  The kernels are those of one product; where
// each expert's rows begin is known on the GPU alone, so the grid is as large as it may have to be, and a workgroup finds its
// expert from the offsets.
#include "xorenc_fp8_dispatch.h"

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_experts_fp8(const uint8_t *A, int64_t lda, const float *SA, int64_t sa_row, int64_t sa_blk, int32_t a_rows,
                                      const int32_t *rows, const int32_t *offsets, int32_t experts, const uint8_t *W, int64_t ldw, int64_t w_stride,
                                      const float *SW, int64_t ldsw, int64_t sw_stride, int32_t N, int32_t K, const xorenc_epilogue *epilogue,
                                      void *Y, int32_t y_dtype, int64_t ldy, int32_t y_rows, void *hip_stream) {
  if (experts <= 0 || w_stride < 0 || sw_stride < 0) return XORENC_EINVAL;
  int32_t rc = check_product(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, y_rows, a_rows, N, K, Y, y_dtype, ldy);
  if (rc != XORENC_OK) return rc;
  Experts job;
  rc = read_epilogue(epilogue, N, y_dtype, false, &job.epilogue);
  if (rc != XORENC_OK) return rc;
  job.bias_stride = epilogue ? epilogue->bias_stride : 0;
  if (job.epilogue.bias && experts > 1 && job.bias_stride < 0) return XORENC_EINVAL;
  if (experts > XORENC_MOE_MAX_EXPERTS) return XORENC_ELIMIT;
  if (y_rows == 0) return XORENC_OK;
  if (!offsets || a_rows == 0 || (!rows && a_rows != y_rows)) return XORENC_EINVAL;
  if (!aligned_to(offsets, 4) || !aligned_to(rows, 4) || (experts > 1 && w_stride % 16)) return XORENC_EALIGN;
  const MatmulArgs g = arguments_of(A, lda, SA, sa_row, sa_blk, W, ldw, SW, ldsw, y_rows, a_rows, N, K, Y, ldy);
  // with `rows` every row of A and its scales are addressed with 32-bit offsets from the first, and what is past the descriptors' extent reads as zero
  if (rows && (a_rows * lda > kMostTileBytes || a_rows * g.sa_row + sa_blk * g.blocks >= kMostTileBytes / 4)) return XORENC_ELIMIT;
  job.offsets = offsets, job.rows = rows, job.w_stride = w_stride, job.sw_stride = sw_stride;
  job.experts = experts, job.a_rows = a_rows, job.y_rows = y_rows;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  const bool exact = y_dtype == XORENC_X_F32;
  const int kernel = cheapest_for_experts(y_rows, experts, N, g.blocks, exact);
  return exact ? dispatch_matmul<true>(kernel, g, job, st) : dispatch_matmul<false>(kernel, g, job, st);
}
