// Operators that end in 8-bit rows: quantisation, the RMS norm with the residual's addition, the gated activation.
//
// All of them read every value once, keep it in registers, and write it in 8 bits; the bytes moved bound them.  Sixteen
// lanes hold a block of 128 columns, eight values each (one 16-byte load of bf16, two of fp32, one 8-byte store of
// e4m3), so that a block's largest magnitude is one maximum over a DPP row and needs no LDS.  Loads start on any element
// (8192 x 1501 with a residual 22 us; value by value, where rows are not on 16-byte boundaries, 52).
//
// us and GB/s read and written (a copy of 1 GB: 5160): rows of 33 x 9216 fp32 5 (the call's time on the host), of 8192 x 5001 bf16
// 26, 4840; squares of 16384 x 4096 bf16 36, 5600; the gates of 8192 x 9216 bf16 65, 5850; the norm of 8192 x 6000 bf16 with a
// residual 66, 5210.
#include <numeric>
#include <type_traits>

#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

// Y = x (or silu(x) * up) by blocks of one row x 128.  Sixteen lanes per block, blocks numbered row by row.
template <class T, bool GATED, bool STREAM>
__global__ __launch_bounds__(256) void quant_rows_kernel(const typename T::Elem *__restrict__ X,
                                                         const typename T::Elem *__restrict__ up, int64_t ldx, uint32_t blocks,
                                                         int cols, uint32_t per_row, uint8_t *__restrict__ Q, int64_t ldq,
                                                         float *__restrict__ S, int64_t s_row, int64_t s_blk) {
  const uint32_t b = blockIdx.x * 16 + (threadIdx.x >> 4);  // (a launch's blocks are fewer than 2^28)
  if (b >= blocks) return;
  const int64_t r = b / per_row;
  const int kb = (int)(b % per_row), l = threadIdx.x & 15;
  const int c = kb * kBlock + l * 8;
  float v[8];
  const typename T::Raw x = load_piece<T, STREAM>(X + r * ldx, c, cols);
  if constexpr (GATED) {
    float u[8];
    const typename T::Raw y = load_piece<T, STREAM>(up + r * ldx, c, cols);
    piece_of<T>(x, c, cols, v);
    piece_of<T>(y, c, cols, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = silu(v[i]) * u[i];
  } else {
    piece_of<T>(x, c, cols, v);
  }
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, magnitude_bits(v[i]));
  const float s = block_scale(max_of_16_lanes(a));
  store_e4m3_piece<STREAM>(Q + r * ldq, c, cols, v, 1.f / s);
  if (l == 0) S[r * s_row + kb * s_blk] = s;
}

// Blocks of 128 x 128: a workgroup holds one, 16 rows a pass, as it was read: all eight loads of a lane are on their way together
// (16384 x 4096 bf16 41.7 -> 35.3 us), and the values are made from them twice.
template <class T, bool STREAM>
__global__ __launch_bounds__(256) void quant_square_kernel(const typename T::Elem *__restrict__ X, int64_t ldx, int64_t x_mat,
                                                           int rows, int cols, int per_row, uint8_t *__restrict__ Q,
                                                           int64_t ldq, int64_t q_mat, float *__restrict__ S, int64_t s_row,
                                                           int64_t s_blk, int64_t s_mat) {
  __shared__ uint32_t wave_max[4];
  const int rb = blockIdx.x / per_row, kb = blockIdx.x - rb * per_row;
  X += blockIdx.y * x_mat;
  Q += blockIdx.y * q_mat;
  const int l = threadIdx.x & 15, c = kb * kBlock + l * 8;
  const int r0 = rb * kBlock + (threadIdx.x >> 4);
  typename T::Raw x[8];  // (rows past the last: the last one again)
  float v[8];
  uint32_t a = 0;
#pragma unroll
  for (int p = 0; p < 8; ++p) x[p] = load_piece<T, STREAM>(X + min(r0 + 16 * p, rows - 1) * ldx, c, cols);
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    piece_of<T>(x[p], c, cols, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, magnitude_bits(v[i]));
  }
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
    piece_of<T>(x[p], c, cols, v);
    if (r < rows) store_e4m3_piece<STREAM>(Q + r * ldq, c, cols, v, inv);
  }
  if (threadIdx.x == 0) S[blockIdx.y * s_mat + rb * s_row + kb * s_blk] = s;
}

// THREADS per row, ROWS rows a workgroup (more than one only where a row is a wave's): s = x + residual, y = s / sqrt(mean s^2 +
// eps) * w.  PASSES > 0: the row's sums stay in registers, eight per thread and pass.  PASSES = 0, rows that do not fit: x and the
// residual are read once more for the second half (from the caches; a `total` that is stored over one of them is not read
// back, it may be rounded).  A row is wider than all passes but the last, which alone has to look where it ends: its code is four times
// as long, and a single row waits for code (one token of 9216 5.4 -> 5.1 us, and where its end is in brief code 4.7).
//
// Up to 1536 columns a wave holds a row: no barrier, and a quarter of the workgroups (8192 x 600 15.4 -> 12.0 us, 8192 x 1200
// without a residual 14.9 -> 11.0; 8192 x 2000 a wave a row 32.8, four 29.4).  Beyond, 256 threads: several rows a CU hide each
// other's loads (8192 x 9216 without a residual 54 us; 1024 threads 76).  Up to 512 rows there are no others, and more threads a row
// are faster: 512 for 9216 columns of one token 6.6 -> 5.4 us (1024 5.5), of 64 6.6 -> 5.6, of 1000 15.3 and 15.2; 1024 for 16000
// columns of one token 7.8 -> 5.0, of 500 14.9 -> 12.9; 256, not a wave, for 500 x 1500 5.6 -> 4.2.
template <class T, int THREADS, int PASSES, int ROWS, bool STREAM>
__global__ __launch_bounds__(THREADS *ROWS) void rmsnorm_kernel(const typename T::Elem *X, int64_t ldx,
                                                          const typename T::Elem *R, int64_t ldr, const void *__restrict__ w,
                                                          int w_bf16, int rows, int cols, float eps,
                                                          typename T::Elem *total, int64_t ldt, typename T::Elem *Y, int64_t y_row,
                                                          int64_t y_col, uint8_t *__restrict__ Q, int64_t ldq,
                                                          float *__restrict__ S, int64_t s_row, int64_t s_blk) {
  static_assert(ROWS == 1 || THREADS == 64, "a barrier is for the row's threads");
  constexpr int STEP = THREADS * 8, WAVES = THREADS / 64;
  constexpr bool BRIEF = THREADS >= 512;  // (few rows)
  __shared__ float chunk_sum[WAVES * (PASSES > 0 ? PASSES : 1)];
  const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
  const int t = threadIdx.x % THREADS;
  if (ROWS > 1 && r >= rows) return;
  X += r * ldx;
  if (R) R += r * ldr;
  if (total) total += r * ldt;
  struct Pair {
    typename T::Raw x, r;
  };
  auto load = [&](int c, bool whole) {
    Pair p;
    p.x = load_piece<T, STREAM>(X, c, cols, whole);
    if (R) p.r = load_piece<T, STREAM>(R, c, cols, whole);
    return p;
  };
  auto sums = [&](const Pair &p, int c, float *s, bool whole) {
    piece_of<T>(p.x, c, cols, s, whole, BRIEF);
    if (R) {
      float u[8];
      piece_of<T>(p.r, c, cols, u, whole, BRIEF);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += u[i];
    }
  };
  constexpr int HELD = PASSES > 0 ? PASSES : 1;
  float s[HELD][8];
  float sq = 0.f;
  if constexpr (PASSES > 0) {
    Pair held[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) held[p] = load(p * STEP + t * 8, p + 1 < PASSES);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      sums(held[p], p * STEP + t * 8, s[p], p + 1 < PASSES);
      float of_pass = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) of_pass += s[p][i] * s[p][i];
      of_pass = sum_of_wave(of_pass);
      if constexpr (WAVES > 1) {
        if ((t & 63) == 0) chunk_sum[p * WAVES + (t >> 6)] = of_pass;
      } else {
        sq += of_pass;
      }
      if (total) store_piece<T>(total, p * STEP + t * 8, cols, s[p], p + 1 < PASSES);
    }
  } else {
    for (int c = t * 8; c < cols; c += STEP) {
      sums(load(c, false), c, s[0], false);
      float of_pass = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) of_pass += s[0][i] * s[0][i];
      sq += of_pass;
    }
  }
  // A row's sum is that of its chunks of 512 columns (a wave and pass each), one after the other, however many threads it has.
  if constexpr (PASSES == 0) {
    sq = sum_of_wave(sq);
    if ((t & 63) == 0) chunk_sum[t >> 6] = sq;
  }
  if constexpr (WAVES > 1) {
    __syncthreads();
    sq = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES * (PASSES > 0 ? PASSES : 1); ++i) sq += chunk_sum[i];
  }
  const float rstd = 1.f / sqrtf(sq / (float)cols + eps);
  auto finish = [&](int c, float *v, bool whole) {
    float g[8];
    if (w_bf16)
      piece_of<BF16>(load_piece<BF16>(static_cast<const uint16_t *>(w), c, cols, whole), c, cols, g, whole, BRIEF);
    else
      piece_of<F32>(load_piece<F32>(static_cast<const float *>(w), c, cols, whole), c, cols, g, whole, BRIEF);
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = v[i] * rstd * g[i];
      a = max(a, magnitude_bits(v[i]));
    }
    const float sc = block_scale(max_of_16_lanes(a));
    if (!whole && c >= cols) return;
    store_e4m3_piece<STREAM>(Q + r * ldq, c, cols, v, 1.f / sc, whole);
    if ((t & 15) == 0) S[r * s_row + (int64_t)(c / kBlock) * s_blk] = sc;
    if (Y) {
      if (y_col == 1) {
        store_piece<T>(Y + r * y_row, c, cols, v, whole);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (whole || c + i < cols) T::store(Y + r * y_row + (c + i) * y_col, v[i]);
      }
    }
  };
  if constexpr (PASSES > 0) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
      finish(p * STEP + t * 8, s[p], p + 1 < PASSES);
  } else {
    for (int c0 = 0; c0 < cols; c0 += STEP) {  // uniform: whole rows of 16 lanes take part in a block's maximum
      const int c = c0 + t * 8;
      sums(load(c, false), c, s[0], false);
      if (total) store_piece<T>(total, c, cols, s[0]);
      finish(c, s[0], false);
    }
  }
}

template <class T, bool GATED, bool STREAM>
int32_t launch_rows(const void *X, const void *up, int64_t ldx, int64_t rows, int32_t cols, uint8_t *Q, int64_t ldq,
                    float *S, int64_t s_row, int64_t s_blk, hipStream_t st) {
  const uint32_t per_row = (uint32_t)((cols + kBlock - 1) / kBlock), blocks = (uint32_t)(rows * per_row);
  hipLaunchKernelGGL((quant_rows_kernel<T, GATED, STREAM>), dim3((unsigned)((blocks + 15) / 16)), dim3(256), 0, st,
                     static_cast<const typename T::Elem *>(X), static_cast<const typename T::Elem *>(up), ldx, blocks, cols,
                     per_row, Q, ldq, S, s_row, s_blk);
  return xorenc_internal_check_launch();
}

// Calls that move more than half of what the memory-side cache holds (256 MB) would find little there when they run again, and read
// and write their 8 bits past it (into two outputs in turn): 8192 x 6000 with a residual 66 us and, with plain loads, 71; 2500 x 9216 34
// and 37; the gates of 8192 x 9216 65 and 69; 16384 x 4096 to squares 36 and 39.  Below, such loads cost (4096 x 4096 with a residual
// 23.9 and 23.1, 8192 x 4096 to squares 19.5 and 18.2), and where two of them share a line: rows of fp32, of which a lane takes 32 bytes (8192 x
// 9216 with a residual 202 and 185; a square's other rows hide it, 162 and 181).
inline bool streams(int64_t values, int64_t bytes) { return values > ((int64_t)128 << 20) / bytes; }

// f(type, whether to stream)
template <class F>
int32_t for_type(int32_t x_dtype, bool stream, F f) {
  if (x_dtype == XORENC_X_F32) return stream ? f(F32(), std::true_type()) : f(F32(), std::false_type());
  return stream ? f(BF16(), std::true_type()) : f(BF16(), std::false_type());
}
template <class T, bool STREAM>
constexpr bool kStreamsRows = STREAM && sizeof(typename T::Elem) == 2;

constexpr int64_t kMostBlocks = ((int64_t)1 << 28) - 16, kMostSquares = (1 << 24) - 1;  // a launch has fewer than 2^32 threads

// Whether two elements of rows x cols, at r * row + c * col, are one: r * row = c * col for differences r and c below rows and cols,
// the least of which are col / g and row / g with g the strides' greatest common divisor.
bool overlaps(int64_t rows, int64_t cols, int64_t row, int64_t col) {
  if (rows <= 1 || cols <= 1) return (rows > 1 && row == 0) || (cols > 1 && col == 0);
  const int64_t g = std::gcd(row, col);
  return g == 0 || (col / g < rows && row / g < cols);
}

// Checks that the entry points share: an 8-bit result of rows x cols with its scales, a launch's blocks of block_rows x 128.
int32_t check_result(int64_t rows, int32_t cols, const uint8_t *Q, int64_t ldq, const float *S, int64_t s_row, int64_t s_blk, int32_t block_rows = 1) {
  if (rows < 0 || cols <= 0 || ldq < cols || s_row < 0 || s_blk < 0) return XORENC_EINVAL;
  if (rows == 0) return XORENC_OK;
  if (!Q || !S) return XORENC_EINVAL;
  if (!aligned_to(Q, 16) || (rows > 1 && ldq % 16) || !aligned_to(S, 4)) return XORENC_EALIGN;
  const int64_t per_row = (cols + (int64_t)kBlock - 1) / kBlock;  // (divisions: products may not fit)
  if (cols > (1 << 30) || (block_rows == 1 ? rows > kMostBlocks / per_row : rows > (1 << 30) || (rows + kBlock - 1) / kBlock > kMostSquares / per_row))
    return XORENC_ELIMIT;
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
  const int32_t rc = check_result(rows, cols, Q, ldq, S, s_row, s_blk, block_rows);
  if (rc != XORENC_OK) return rc;
  if (rows == 0 || matrices == 0) return XORENC_OK;
  if (!X) return XORENC_EINVAL;
  const int esz = dtype_bytes(x_dtype);
  if (matrices > 1 && (x_stride < 0 || q_stride < 0 || s_stride < 0)) return XORENC_EINVAL;
  if (!aligned_to(X, esz) || (matrices > 1 && q_stride % 16)) return XORENC_EALIGN;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int per_row = (cols + kBlock - 1) / kBlock;
  if (overlaps(block_rows == 1 ? rows : (rows + kBlock - 1) / kBlock, per_row, s_row, s_blk) || (matrices > 1 && (q_stride == 0 || s_stride == 0)))
    return XORENC_EINVAL;
  xorenc_internal_begin_call();
  if (block_rows == 1) {
    for (int32_t i = 0; i < matrices; ++i) {
      const void *x = static_cast<const char *>(X) + i * x_stride * esz;
      uint8_t *q = Q + i * q_stride;
      float *s = S + i * s_stride;
      const int32_t rl = x_dtype == XORENC_X_F32 ? launch_rows<F32, false, false>(x, nullptr, ldx, rows, cols, q, ldq, s, s_row, s_blk, st)
                                                 : launch_rows<BF16, false, false>(x, nullptr, ldx, rows, cols, q, ldq, s, s_row, s_blk, st);
      if (rl != XORENC_OK) return rl;
    }
    return XORENC_OK;
  }
  for (int64_t at = 0; at < matrices; at += 65535) {  // the grid's second size is limited
    const dim3 grid((unsigned)((rows + kBlock - 1) / kBlock * per_row), (unsigned)min(matrices - at, (int64_t)65535));
    const int32_t rl = for_type(x_dtype, streams(rows * cols, (int64_t)(esz + 1) * matrices), [&](auto type, auto stream) {
      typedef typename decltype(type)::Elem E;
      hipLaunchKernelGGL((quant_square_kernel<decltype(type), decltype(stream)::value>), grid, dim3(256), 0, st,
                         static_cast<const E *>(X) + at * x_stride, ldx, x_stride, (int)rows, cols, per_row, Q + at * q_stride, ldq, q_stride,
                         S + at * s_stride, s_row, s_blk, s_stride);
      return xorenc_internal_check_launch();
    });
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
  if (overlaps(rows, (cols + kBlock - 1) / kBlock, s_row, s_blk)) return XORENC_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return for_type(x_dtype, streams(rows * cols, 2 * esz + 1), [&](auto type, auto stream) {
    return launch_rows<decltype(type), true, kStreamsRows<decltype(type), decltype(stream)::value>>(gate, up, ldx, rows, cols, Q, ldq, S, s_row, s_blk, st);
  });
}

namespace xorenc_fp8_detail {
namespace {
template <class T, bool STREAM>
int32_t launch_rmsnorm(const void *X, int64_t ldx, const void *R, int64_t ldr, const void *w, int w_bf16,
                       int64_t rows, int32_t cols, float eps, void *total, int64_t ldt, void *Y, int64_t y_row, int64_t y_col,
                       uint8_t *Q, int64_t ldq, float *S, int64_t s_row, int64_t s_blk, hipStream_t st) {
  typedef typename T::Elem E;
#define XORENC_RMSNORM(THREADS, PASSES, ROWS)                                                                                     \
  hipLaunchKernelGGL((rmsnorm_kernel<T, THREADS, PASSES, ROWS, (STREAM && PASSES > 0)>), dim3((unsigned)((rows + ROWS - 1) / ROWS)), dim3(THREADS * ROWS), 0, st, \
                     static_cast<const E *>(X), ldx, static_cast<const E *>(R), ldr, w, w_bf16, (int)rows, cols, \
                     eps, static_cast<E *>(total), ldt, static_cast<E *>(Y), y_row, y_col, Q, ldq, S, s_row, s_blk)
  if (cols > 16384)
    XORENC_RMSNORM(1024, 0, 1);
  else if (cols <= 512)
    XORENC_RMSNORM(64, 1, 4);
  else if (rows <= 512) {  // two a CU: what counts is how long a row takes
    if (cols <= 2048)
      XORENC_RMSNORM(256, 1, 1);
    else if (cols <= 4096)
      XORENC_RMSNORM(512, 1, 1);
    else if (cols <= 8192)
      XORENC_RMSNORM(1024, 1, 1);
    else if (cols <= 12288)
      XORENC_RMSNORM(512, 3, 1);
    else
      XORENC_RMSNORM(1024, 2, 1);
  } else if (cols <= 1024)
    XORENC_RMSNORM(64, 2, 4);
  else if (cols <= 1536)
    XORENC_RMSNORM(64, 3, 4);
  else if (cols <= 2048)
    XORENC_RMSNORM(256, 1, 1);
  else if (cols <= 4096)
    XORENC_RMSNORM(256, 2, 1);
  else if (cols <= 6144)
    XORENC_RMSNORM(256, 3, 1);
  else if (cols <= 8192)
    XORENC_RMSNORM(256, 4, 1);
  else if (cols <= 10240)
    XORENC_RMSNORM(256, 5, 1);
  else if (cols <= 12288)
    XORENC_RMSNORM(256, 6, 1);
  else if (cols <= 14336)
    XORENC_RMSNORM(256, 7, 1);
  else
    XORENC_RMSNORM(256, 8, 1);
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
  if (overlaps(rows, (cols + kBlock - 1) / kBlock, s_row, s_blk) || (Y && overlaps(rows, cols, y_row, y_col))) return XORENC_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  const int moved = 1 + esz * (1 + (residual != nullptr) + (total != nullptr) + (Y != nullptr));
  return for_type(x_dtype, streams(rows * cols, moved), [&](auto type, auto stream) {
    return launch_rmsnorm<decltype(type), kStreamsRows<decltype(type), decltype(stream)::value>>(
        X, ldx, residual, ldr, weight, w_dtype == XORENC_X_BF16, rows, cols, eps, total, ldt, Y, y_row, y_col, Q, ldq, S, s_row, s_blk, st);
  });
}
