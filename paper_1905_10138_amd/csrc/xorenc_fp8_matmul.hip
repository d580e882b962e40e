// Y = A W^T with A [M, K] and W [N, K] in e4m3, a scale for each 1 x 128 block of A and each 128 x 128 block of W:
//   Y[m][n] = sum over blocks b of SA[m][b] SW[n / 128][b] sum over k in b of A[m][k] W[n][k].
// The sum inside a block is the matrix instruction's; the scaled sums are added in fp32.
#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

struct MatmulArgs {
  const uint8_t *A, *W;
  const float *SA, *SW;
  void *Y;
  int64_t lda, ldw, sa_row, sa_blk, ldsw, ldy;
  int M, N, K, blocks;
};

template <bool EXACT>
__device__ inline void store_result(const MatmulArgs &g, int m, int n, f32x4 v, bool wide) {
  if (m >= g.M) return;
  if constexpr (EXACT) {
    float *const y = static_cast<float *>(g.Y) + m * g.ldy + n;
    if (wide && n + 4 <= g.N) {
      *reinterpret_cast<f32x4 *>(y) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < g.N) y[i] = v[i];
    }
  } else {
    uint16_t *const y = static_cast<uint16_t *>(g.Y) + m * g.ldy + n;
    if (wide && n + 4 <= g.N) {
      *reinterpret_cast<u32x2 *>(y) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < g.N) y[i] = to_bf16(v[i]);
    }
  }
}

// Few rows of A: a workgroup owns 16 rows of W and 16 MT rows of A, its waves take the blocks of the reduction in turn and
// their sums meet in LDS, in the order of the waves.  Operands go from memory to registers.
template <int MT, int WAVES, bool EXACT>
__global__ __launch_bounds__(WAVES * 64) void matmul_rows_kernel(MatmulArgs g, int wide) {
  __shared__ f32x4 part[WAVES][MT][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MT);
  const int r = lane & 15;
  const uint8_t *const w_row = g.W + (int64_t)min(n0 + r, g.N - 1) * g.ldw;
  const uint8_t *a_row[MT];
  const float *sa[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = min(m0 + 16 * i + r, g.M - 1);
    a_row[i] = g.A + m * g.lda;
    sa[i] = g.SA + m * g.sa_row;
  }
  const float *const sw = g.SW + (int64_t)(n0 / kBlock) * g.ldsw;
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int b = wave; b < g.blocks; b += WAVES) {
    const int c0 = b * kBlock + piece_column(lane, 0), c1 = b * kBlock + piece_column(lane, 1);
    E4m3Operand w;
    w.piece[0] = load_e4m3_piece(w_row, c0, g.K);
    w.piece[1] = load_e4m3_piece(w_row, c1, g.K);
    const float s = sw[b];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      E4m3Operand a;
      a.piece[0] = load_e4m3_piece(a_row[i], c0, g.K);
      a.piece[1] = load_e4m3_piece(a_row[i], c1, g.K);
      const float f = s * sa[i][b * g.sa_blk];
      const f32x4 d = product_128<EXACT>(w, a);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] += f * d[j];
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < MT; i += WAVES) {
    f32x4 v = part[0][i][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += part[w][i][lane];
    store_result<EXACT>(g, m0 + 16 * i + r, n0 + 4 * (lane >> 4), v, wide);
  }
}

template <bool EXACT>
int32_t dispatch_matmul(const MatmulArgs &g, bool wide, hipStream_t st) {
  const dim3 grid((unsigned)((g.N + 15) / 16), (unsigned)((g.M + 63) / 64));
  if (g.M <= 16)
    hipLaunchKernelGGL((matmul_rows_kernel<1, 8, EXACT>), grid, dim3(512), 0, st, g, (int)wide);
  else
    hipLaunchKernelGGL((matmul_rows_kernel<4, 8, EXACT>), grid, dim3(512), 0, st, g, (int)wide);
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
  if (M > 65535 * 64 || N > (1 << 24) || K > (1 << 24)) return XORENC_ELIMIT;
  const MatmulArgs g = {A, W, SA, SW, Y, lda, ldw, sa_row, sa_blk, ldsw, ldy, M, N, K, blocks};
  const bool wide = aligned_to(Y, y_dtype == XORENC_X_F32 ? 16 : 8) && ldy % 4 == 0;
  xorenc_internal_begin_call();
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return y_dtype == XORENC_X_F32 ? dispatch_matmul<true>(g, wide, st) : dispatch_matmul<false>(g, wide, st);
}
