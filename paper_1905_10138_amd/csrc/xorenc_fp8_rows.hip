// Operators that end in 8-bit rows: quantisation, the RMS norm with the residual's addition, the gated activation.
//
// All of them read every value once, keep it in registers, and write it in 8 bits; the bytes moved bound them.  Sixteen
// lanes hold a block of 128 columns, eight values each (one 16-byte load of bf16, two of fp32, one 8-byte store of
// e4m3), so that a block's largest magnitude is one maximum over a DPP row and needs no LDS.
#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

// Y = x (or silu(x) * up) by blocks of one row x 128.  Sixteen lanes per block, blocks numbered row by row.
template <class T, bool GATED>
__global__ __launch_bounds__(256) void quant_rows_kernel(const typename T::Elem *__restrict__ X,
                                                         const typename T::Elem *__restrict__ up, int64_t ldx, int64_t blocks,
                                                         int cols, int per_row, int wide, uint8_t *__restrict__ Q, int64_t ldq,
                                                         float *__restrict__ S, int64_t s_row, int64_t s_blk) {
  const int64_t b = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (b >= blocks) return;
  const int64_t r = blocks <= 0x7fffffff ? (int64_t)((uint32_t)b / (uint32_t)per_row) : b / per_row;
  const int kb = (int)(b - r * per_row), l = threadIdx.x & 15;
  const int c = kb * kBlock + l * 8;
  float v[8];
  load_piece<T>(X + r * ldx, c, cols, wide, v);
  if constexpr (GATED) {
    float u[8];
    load_piece<T>(up + r * ldx, c, cols, wide, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = silu(v[i]) * u[i];
  }
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, magnitude_bits(v[i]));
  const float s = block_scale(max_of_16_lanes(a));
  store_e4m3_piece(Q + r * ldq, c, cols, v, 1.f / s);
  if (l == 0) S[r * s_row + kb * s_blk] = s;
}

// Blocks of 128 x 128: a workgroup holds one, 16 rows a pass.
template <class T>
__global__ __launch_bounds__(256) void quant_square_kernel(const typename T::Elem *__restrict__ X, int64_t ldx, int64_t x_mat,
                                                           int rows, int cols, int per_row, int wide, uint8_t *__restrict__ Q,
                                                           int64_t ldq, int64_t q_mat, float *__restrict__ S, int64_t s_row,
                                                           int64_t s_blk, int64_t s_mat) {
  __shared__ uint32_t wave_max[4];
  const int rb = blockIdx.x / per_row, kb = blockIdx.x - rb * per_row;
  X += blockIdx.y * x_mat;
  Q += blockIdx.y * q_mat;
  const int l = threadIdx.x & 15, c = kb * kBlock + l * 8;
  const int r0 = rb * kBlock + (threadIdx.x >> 4);
  float v[8][8];
  uint32_t a = 0;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int r = r0 + 16 * p;
    if (r < rows) {
      load_piece<T>(X + r * ldx, c, cols, wide, v[p]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[p][i] = 0.f;
    }
  }
#pragma unroll
  for (int p = 0; p < 8; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, magnitude_bits(v[p][i]));
  a = max_of_16_lanes(a);
  a = max(a, (uint32_t)__shfl_xor((int)a, 16));
  a = max(a, (uint32_t)__shfl_xor((int)a, 32));
  if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = a;
  __syncthreads();
  a = max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3]));
  const float s = block_scale(a), inv = 1.f / s;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int r = r0 + 16 * p;
    if (r < rows) store_e4m3_piece(Q + r * ldq, c, cols, v[p], inv);
  }
  if (threadIdx.x == 0) S[blockIdx.y * s_mat + rb * s_row + kb * s_blk] = s;
}

// One workgroup per row: s = x + residual, y = s / sqrt(mean s^2 + eps) * w.  PASSES > 0: the row's sums stay in registers, eight
// per thread and pass.  PASSES = 0, rows that do not fit: x and the residual are read once more for the second half
// (from the caches; a `total` that is stored over one of them is not read back, it may be rounded).
template <class T, int THREADS, int PASSES>
__global__ __launch_bounds__(THREADS) void rmsnorm_kernel(const typename T::Elem *X, int64_t ldx,
                                                          const typename T::Elem *R, int64_t ldr, const void *__restrict__ w,
                                                          int w_bf16, int wide, int w_wide, int cols, int per_row, float eps,
                                                          typename T::Elem *total, int64_t ldt, typename T::Elem *Y, int64_t y_row,
                                                          int64_t y_col, int y_wide, uint8_t *__restrict__ Q, int64_t ldq,
                                                          float *__restrict__ S, int64_t s_row, int64_t s_blk) {
  constexpr int STEP = THREADS * 8, WAVES = THREADS / 64;
  __shared__ float wave_sum[WAVES];
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x;
  X += r * ldx;
  if (R) R += r * ldr;
  if (total) total += r * ldt;
  auto sums = [&](int c, float *s) {
    load_piece<T>(X, c, cols, wide, s);
    if (R) {
      float u[8];
      load_piece<T>(R, c, cols, wide, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += u[i];
    }
  };
  constexpr int HELD = PASSES > 0 ? PASSES : 1;
  float s[HELD][8];
  float sq = 0.f;
  if constexpr (PASSES > 0) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) sums(p * STEP + t * 8, s[p]);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sq += s[p][i] * s[p][i];
      if (total) store_piece<T>(total, p * STEP + t * 8, cols, wide, s[p]);
    }
  } else {
    for (int c = t * 8; c < cols; c += STEP) {
      sums(c, s[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sq += s[0][i] * s[0][i];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sq += __shfl_xor(sq, o);
  if constexpr (WAVES > 1) {
    if ((t & 63) == 0) wave_sum[t >> 6] = sq;
    __syncthreads();
    sq = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) sq += wave_sum[i];
  }
  const float rstd = 1.f / sqrtf(sq / (float)cols + eps);
  auto finish = [&](int c, float *v) {
    float g[8];
    if (w_bf16)
      load_piece<BF16>(static_cast<const uint16_t *>(w), c, cols, w_wide, g);
    else
      load_piece<F32>(static_cast<const float *>(w), c, cols, w_wide, g);
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = v[i] * rstd * g[i];
      a = max(a, magnitude_bits(v[i]));
    }
    const float sc = block_scale(max_of_16_lanes(a));
    if (c >= cols) return;
    store_e4m3_piece(Q + r * ldq, c, cols, v, 1.f / sc);
    if ((t & 15) == 0) S[r * s_row + (int64_t)(c / kBlock) * s_blk] = sc;
    if (Y) {
      if (y_col == 1) {
        store_piece<T>(Y + r * y_row, c, cols, y_wide, v);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) T::store(Y + r * y_row + (c + i) * y_col, v[i]);
      }
    }
  };
  if constexpr (PASSES > 0) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
      if (p * STEP < cols) finish(p * STEP + t * 8, s[p]);
  } else {
    for (int c0 = 0; c0 < cols; c0 += STEP) {  // uniform: whole rows of 16 lanes take part in a block's maximum
      const int c = c0 + t * 8;
      sums(c, s[0]);
      if (total) store_piece<T>(total, c, cols, wide, s[0]);
      finish(c, s[0]);
    }
  }
}

template <class T, bool GATED>
int32_t launch_rows(const void *X, const void *up, int64_t ldx, int64_t rows, int32_t cols, bool wide, uint8_t *Q, int64_t ldq,
                    float *S, int64_t s_row, int64_t s_blk, hipStream_t st) {
  const int per_row = (cols + kBlock - 1) / kBlock;
  const int64_t blocks = rows * per_row;
  hipLaunchKernelGGL((quant_rows_kernel<T, GATED>), dim3((unsigned)((blocks + 15) / 16)), dim3(256), 0, st,
                     static_cast<const typename T::Elem *>(X), static_cast<const typename T::Elem *>(up), ldx, blocks, cols,
                     per_row, (int)wide, Q, ldq, S, s_row, s_blk);
  return xorenc_internal_check_launch();
}

constexpr int64_t kMostBlocks = ((int64_t)1 << 28) - 16;  // a launch has fewer than 2^32 threads

// Checks that the entry points share: an 8-bit result of rows x cols with its scales.
int32_t check_result(int64_t rows, int32_t cols, const uint8_t *Q, int64_t ldq, const float *S, int64_t s_row, int64_t s_blk) {
  if (rows < 0 || cols <= 0 || ldq < cols || s_row < 0 || s_blk < 0) return XORENC_EINVAL;
  if (rows == 0) return XORENC_OK;
  if (!Q || !S) return XORENC_EINVAL;
  if (!aligned_to(Q, 16) || (rows > 1 && ldq % 16) || !aligned_to(S, 4)) return XORENC_EALIGN;
  if (rows * ((cols + (int64_t)kBlock - 1) / kBlock) > kMostBlocks || cols > (1 << 30)) return XORENC_ELIMIT;
  return XORENC_OK;
}

}  // namespace
}  // namespace xorenc_fp8_detail

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_quant_fp8(const void *X, int32_t x_dtype, int64_t ldx, int64_t x_stride, int32_t matrices,
                                    int64_t rows, int32_t cols, int32_t block_rows, uint8_t *Q, int64_t ldq, int64_t q_stride,
                                    float *S, int64_t s_row, int64_t s_blk, int64_t s_stride, void *hip_stream) {
  if (matrices < 0 || ldx < cols) return XORENC_EINVAL;
  if (block_rows != 1 && block_rows != kBlock) return XORENC_EUNSUPPORTED;
  if (!known_dtype(x_dtype)) return XORENC_EUNSUPPORTED;
  const int32_t rc = check_result(rows, cols, Q, ldq, S, s_row, s_blk);
  if (rc != XORENC_OK) return rc;
  if (rows == 0 || matrices == 0) return XORENC_OK;
  if (!X) return XORENC_EINVAL;
  const int esz = dtype_bytes(x_dtype);
  if (matrices > 1 && (x_stride < 0 || q_stride < 0 || s_stride < 0)) return XORENC_EINVAL;
  if (!aligned_to(X, esz) || (matrices > 1 && q_stride % 16)) return XORENC_EALIGN;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int per_row = (cols + kBlock - 1) / kBlock;
  const bool wide = wide_rows(X, ldx, x_dtype) && (matrices == 1 || x_stride * esz % 16 == 0);
  xorenc_internal_begin_call();
  if (block_rows == 1) {
    for (int32_t i = 0; i < matrices; ++i) {
      const void *x = static_cast<const char *>(X) + i * x_stride * esz;
      uint8_t *q = Q + i * q_stride;
      float *s = S + i * s_stride;
      const int32_t rl = x_dtype == XORENC_X_F32 ? launch_rows<F32, false>(x, nullptr, ldx, rows, cols, wide, q, ldq, s, s_row, s_blk, st)
                                                 : launch_rows<BF16, false>(x, nullptr, ldx, rows, cols, wide, q, ldq, s, s_row, s_blk, st);
      if (rl != XORENC_OK) return rl;
    }
    return XORENC_OK;
  }
  const int64_t squares = (rows + kBlock - 1) / kBlock * per_row;
  if (rows > (1 << 30) || squares >= (1 << 24)) return XORENC_ELIMIT;
  for (int32_t at = 0; at < matrices; at += 65535) {  // the grid's second size is limited
    const dim3 grid((unsigned)squares, (unsigned)min(matrices - at, 65535));
    if (x_dtype == XORENC_X_F32)
      hipLaunchKernelGGL((quant_square_kernel<F32>), grid, dim3(256), 0, st, static_cast<const float *>(X) + at * x_stride, ldx,
                         x_stride, (int)rows, cols, per_row, (int)wide, Q + at * q_stride, ldq, q_stride, S + at * s_stride, s_row,
                         s_blk, s_stride);
    else
      hipLaunchKernelGGL((quant_square_kernel<BF16>), grid, dim3(256), 0, st, static_cast<const uint16_t *>(X) + at * x_stride, ldx,
                         x_stride, (int)rows, cols, per_row, (int)wide, Q + at * q_stride, ldq, q_stride, S + at * s_stride, s_row,
                         s_blk, s_stride);
    const int32_t rl = xorenc_internal_check_launch();
    if (rl != XORENC_OK) return rl;
  }
  return XORENC_OK;
}

extern "C" int32_t xorenc_silu_mul_fp8(const void *gate, const void *up, int32_t x_dtype, int64_t ldx, int64_t rows, int32_t cols,
                                       uint8_t *Q, int64_t ldq, float *S, int64_t s_row, int64_t s_blk, void *hip_stream) {
  if (ldx < cols) return XORENC_EINVAL;
  if (!known_dtype(x_dtype)) return XORENC_EUNSUPPORTED;
  const int32_t rc = check_result(rows, cols, Q, ldq, S, s_row, s_blk);
  if (rc != XORENC_OK) return rc;
  if (rows == 0) return XORENC_OK;
  if (!gate || !up) return XORENC_EINVAL;
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(gate, esz) || !aligned_to(up, esz)) return XORENC_EALIGN;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool wide = wide_rows(gate, ldx, x_dtype) && wide_rows(up, ldx, x_dtype);
  xorenc_internal_begin_call();
  return x_dtype == XORENC_X_F32 ? launch_rows<F32, true>(gate, up, ldx, rows, cols, wide, Q, ldq, S, s_row, s_blk, st)
                                 : launch_rows<BF16, true>(gate, up, ldx, rows, cols, wide, Q, ldq, S, s_row, s_blk, st);
}

namespace xorenc_fp8_detail {
namespace {
template <class T>
int32_t launch_rmsnorm(const void *X, int64_t ldx, const void *R, int64_t ldr, const void *w, int w_bf16, bool wide, bool w_wide,
                       int64_t rows, int32_t cols, float eps, void *total, int64_t ldt, void *Y, int64_t y_row, int64_t y_col,
                       bool y_wide, uint8_t *Q, int64_t ldq, float *S, int64_t s_row, int64_t s_blk, hipStream_t st) {
  typedef typename T::Elem E;
  const int per_row = (cols + kBlock - 1) / kBlock;
#define XORENC_RMSNORM(THREADS, PASSES)                                                                                     \
  hipLaunchKernelGGL((rmsnorm_kernel<T, THREADS, PASSES>), dim3((unsigned)rows), dim3(THREADS), 0, st,                      \
                     static_cast<const E *>(X), ldx, static_cast<const E *>(R), ldr, w, w_bf16, (int)wide, (int)w_wide, cols, \
                     per_row, eps, static_cast<E *>(total), ldt, static_cast<E *>(Y), y_row, y_col, (int)y_wide, Q, ldq, S, s_row, s_blk)
  if (cols <= 512)
    XORENC_RMSNORM(64, 1);
  else if (cols <= 2048)
    XORENC_RMSNORM(256, 1);
  else if (cols <= 4096)
    XORENC_RMSNORM(256, 2);
  else if (cols <= 6144)
    XORENC_RMSNORM(256, 3);
  else if (cols <= 8192)
    XORENC_RMSNORM(256, 4);
  else if (cols <= 16384)
    XORENC_RMSNORM(1024, 2);
  else
    XORENC_RMSNORM(1024, 0);
#undef XORENC_RMSNORM
  return xorenc_internal_check_launch();
}
}  // namespace
}  // namespace xorenc_fp8_detail

extern "C" int32_t xorenc_add_rmsnorm_fp8(const void *X, int32_t x_dtype, int64_t ldx, const void *residual, int64_t ldr,
                                          const void *weight, int32_t w_dtype, int64_t rows, int32_t cols, float eps, void *total,
                                          int64_t ldt, void *Y, int64_t y_row, int64_t y_col, uint8_t *Q, int64_t ldq, float *S,
                                          int64_t s_row, int64_t s_blk, void *hip_stream) {
  if (ldx < cols || (residual && ldr < cols) || (total && ldt < cols) || (Y && (y_row < 0 || y_col < 1)) || !(eps >= 0.f))
    return XORENC_EINVAL;
  if (!known_dtype(x_dtype) || !known_dtype(w_dtype)) return XORENC_EUNSUPPORTED;
  const int32_t rc = check_result(rows, cols, Q, ldq, S, s_row, s_blk);
  if (rc != XORENC_OK) return rc;
  if (rows == 0) return XORENC_OK;
  if (!X || !weight) return XORENC_EINVAL;
  if (rows >= (1 << 22)) return XORENC_ELIMIT;
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(X, esz) || !aligned_to(residual, esz) || !aligned_to(total, esz) || !aligned_to(Y, esz) ||
      !aligned_to(weight, dtype_bytes(w_dtype)))
    return XORENC_EALIGN;
  const bool wide = wide_rows(X, ldx, x_dtype) && (!residual || wide_rows(residual, ldr, x_dtype)) &&
                    (!total || wide_rows(total, ldt, x_dtype));
  const bool w_wide = aligned_to(weight, 16), y_wide = wide_rows(Y, y_row, x_dtype);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return x_dtype == XORENC_X_F32
             ? launch_rmsnorm<F32>(X, ldx, residual, ldr, weight, w_dtype == XORENC_X_BF16, wide, w_wide, rows, cols, eps, total, ldt, Y,
                                   y_row, y_col, y_wide, Q, ldq, S, s_row, s_blk, st)
             : launch_rmsnorm<BF16>(X, ldx, residual, ldr, weight, w_dtype == XORENC_X_BF16, wide, w_wide, rows, cols, eps, total, ldt,
                                    Y, y_row, y_col, y_wide, Q, ldq, S, s_row, s_blk, st);
}
