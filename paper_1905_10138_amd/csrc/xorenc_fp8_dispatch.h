// The launches of the block-scaled product's kernels, for one job (xorenc_fp8_job.h) each source.
#ifndef XORENC_FP8_DISPATCH_H
#define XORENC_FP8_DISPATCH_H

#include "xorenc_fp8_plan.h"
#include "xorenc_fp8_ring.h"

namespace xorenc_fp8_detail {

// How many tiles of bm rows there can be at most.
template <class Job>
int64_t most_row_tiles(const Job &job, const MatmulArgs &g, int bm) {
  if constexpr (Job::ROWS) {
    return most_tiles_of_experts(job.y_rows, job.experts, bm);
  } else {
    return (g.M + bm - 1) / bm;
  }
}

inline bool streams_weights(const Experts &job, const MatmulArgs &g, int bm) {
  return streams_weights(job.y_rows, job.experts, bytes_of_one_expert(job.experts, g.N, g.K, g.ldw, job.w_stride), bm);
}

// STREAMS: it may be that experts' weights are read past the caches.
template <int TN, int TM, int WN, int WM, bool EXACT, bool STREAMS = false, bool STREAM = false, class Job>
void launch_tile(const MatmulArgs &g, const Job &job, hipStream_t st) {
  typedef TileShape<TN, TM, WN, WM, EXACT> Shape;
  if constexpr (STREAMS && !STREAM) {
    if (streams_weights(job, g, Shape::BM)) return launch_tile<TN, TM, WN, WM, EXACT, STREAMS, true>(g, job, st);
  }
  const int n_tiles = (g.N + Shape::BN - 1) / Shape::BN, m_tiles = (int)most_row_tiles(job, g, Shape::BM);
  const int per_xcd = (n_tiles * m_tiles + 7) / 8;
  hipLaunchKernelGGL((matmul_tile_kernel<TN, TM, WN, WM, EXACT, Job, STREAM>), dim3((unsigned)(per_xcd * 8)), dim3(Shape::WAVES * 64), Shape::LDS, st, g,
                     n_tiles, m_tiles, per_xcd, job);
}

template <int TN, int TM, int WN, int WM, int KG, int NS, bool EXACT, bool STREAMS = false, bool STREAM = false, class Job>
void launch_ring(const MatmulArgs &g, const Job &job, hipStream_t st) {
  typedef RingShape<TN, TM, WN, WM, KG, NS> Shape;
  if constexpr (STREAMS && !STREAM) {
    if (streams_weights(job, g, Shape::BM)) return launch_ring<TN, TM, WN, WM, KG, NS, EXACT, STREAMS, true>(g, job, st);
  }
  const int n_tiles = (g.N + Shape::BN - 1) / Shape::BN, m_tiles = (int)most_row_tiles(job, g, Shape::BM);
  const int per_xcd = (n_tiles * m_tiles + 7) / 8;
  hipLaunchKernelGGL((matmul_ring_kernel<TN, TM, WN, WM, KG, NS, EXACT, Job, STREAM>), dim3((unsigned)(per_xcd * 8)), dim3(Shape::WAVES * 64), Shape::LDS, st,
                     g, n_tiles, m_tiles, per_xcd, job);
}

template <bool EXACT, class Job>
int32_t dispatch_matmul(int kernel, const MatmulArgs &g, const Job &job, hipStream_t st) {
  switch (kernel) {
    case 0:
      if constexpr (!EXACT) launch_tile<8, 4, 2, 4, EXACT>(g, job, st);
      break;
    case 1: launch_tile<4, 4, 2, 2, EXACT>(g, job, st); break;
    case 2: launch_tile<4, 2, 2, 2, EXACT, Job::ROWS>(g, job, st); break;
    case 3: launch_ring<2, 2, 2, 2, 2, 2, EXACT, Job::ROWS>(g, job, st); break;
    case 4: launch_ring<2, 2, 2, 2, 1, 2, EXACT>(g, job, st); break;
    case 5: launch_ring<1, 1, 1, 1, 8, 2, EXACT>(g, job, st); break;
    case 6:
      if constexpr (!Job::ROWS) launch_ring<2, 2, 1, 1, 8, 2, EXACT>(g, job, st);
      break;
    case 7:
      if constexpr (!Job::ROWS) launch_ring<2, 2, 2, 1, 4, 3, EXACT>(g, job, st);
      break;
    case 8:
      if constexpr (!EXACT) launch_ring<2, 2, 2, 2, 2, 3, EXACT>(g, job, st);
      break;
    case 9:
      if constexpr (!EXACT) launch_tile<8, 3, 2, 4, EXACT>(g, job, st);
      break;
    case 10:
      if constexpr (!EXACT && !Job::ROWS) launch_ring<4, 2, 2, 4, 1, 3, EXACT>(g, job, st);
      break;
    case 11:
      if constexpr (Job::EPILOGUE) launch_ring<2, 1, 1, 1, 4, 2, EXACT, Job::ROWS>(g, job, st);
      break;
    case 12:
      if constexpr (Job::ROWS) launch_ring<2, 2, 2, 1, 1, 3, EXACT, true>(g, job, st);
      break;
    default: return XORENC_ELIMIT;
  }
  return xorenc_internal_check_launch();
}

// Host checks that the entry points share: the matrices of a product with M rows of Y.  `a_rows` of A, which `rows` picks from.
inline int32_t check_product(const uint8_t *A, int64_t lda, const float *SA, int64_t sa_row, int64_t sa_blk, const uint8_t *W, int64_t ldw,
                             const float *SW, int64_t ldsw, int32_t M, int32_t a_rows, int32_t N, int32_t K, const void *Y, int32_t y_dtype, int64_t ldy) {
  const int32_t blocks = K > 0 ? (int32_t)(((int64_t)K + kBlock - 1) / kBlock) : 0;
  if (M < 0 || a_rows < 0 || N <= 0 || K <= 0 || lda < K || ldw < K || ldy < N || sa_row < 0 || sa_blk < 0 || ldsw < blocks) return XORENC_EINVAL;
  if (!known_dtype(y_dtype)) return XORENC_EUNSUPPORTED;
  if (M == 0) return XORENC_OK;
  if (!A || !SA || !W || !SW || !Y) return XORENC_EINVAL;
  if (!aligned_to(A, 16) || (a_rows > 1 && lda % 16) || !aligned_to(W, 16) || (N > 1 && ldw % 16) || !aligned_to(SA, 4) || !aligned_to(SW, 4) ||
      !aligned_to(Y, dtype_bytes(y_dtype)))
    return XORENC_EALIGN;
  // a tile's rows, and all scales of its rows of A, are addressed with 32-bit offsets
  const int64_t row_step = a_rows > 1 ? sa_row : 0;
  if (M > 65535 * 64 || K > (1 << 22) || (a_rows > 1 && lda > (1 << 22)) || (N > 1 && ldw > (1 << 22)) || row_step > (1 << 20) || sa_blk > (1 << 28) ||
      256 * row_step + sa_blk * blocks >= (1 << 29))
    return XORENC_ELIMIT;
  return XORENC_OK;
}

inline MatmulArgs arguments_of(const uint8_t *A, int64_t lda, const float *SA, int64_t sa_row, int64_t sa_blk, const uint8_t *W, int64_t ldw,
                               const float *SW, int64_t ldsw, int32_t M, int32_t a_rows, int32_t N, int32_t K, void *Y, int64_t ldy) {
  return MatmulArgs{A, W, SA, SW, Y, lda, ldw, a_rows > 1 ? sa_row : 0, sa_blk, ldsw, ldy, M, N, K, (K + kBlock - 1) / kBlock};
}

// The epilogue of a call whose Y has rows of N values of y_dtype; `residual`: whether it may have one.
inline int32_t read_epilogue(const xorenc_epilogue *given, int32_t N, int32_t y_dtype, bool residual, Epilogue *out) {
  *out = Epilogue{nullptr, nullptr, 0, 0, XORENC_NO_ACTIVATION};
  if (!given) return XORENC_OK;
  if (given->struct_size != sizeof(xorenc_epilogue)) return XORENC_EINVAL;
  if (given->activation < XORENC_NO_ACTIVATION || given->activation > XORENC_GELU_TANH || (given->bias && !known_dtype(given->bias_dtype)))
    return XORENC_EUNSUPPORTED;
  if (given->residual && (!residual || given->ld_residual < N)) return XORENC_EINVAL;
  if ((given->bias && !aligned_to(given->bias, dtype_bytes(given->bias_dtype))) || !aligned_to(given->residual, dtype_bytes(y_dtype))) return XORENC_EALIGN;
  *out = Epilogue{given->bias, given->residual, given->ld_residual, given->bias_dtype == XORENC_X_BF16, given->activation};
  return XORENC_OK;
}

}  // namespace xorenc_fp8_detail

#endif
