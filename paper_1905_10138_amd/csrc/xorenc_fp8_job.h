// What a block-scaled product does beside the product itself: which rows it takes, and what becomes of its results.
#ifndef XORENC_FP8_JOB_H
#define XORENC_FP8_JOB_H

#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {

struct MatmulArgs {
  const uint8_t *A, *W;
  const float *SA, *SW;
  void *Y;
  int64_t lda, ldw, sa_row, sa_blk, ldsw, ldy;
  int M, N, K, blocks;
};

// y = residual + f(z + bias), in fp32 and before the only rounding.
struct Epilogue {
  const void *bias, *residual;
  int64_t ld_residual;
  int bias_bf16, activation;
  __device__ bool none() const { return !bias && !residual && activation == XORENC_NO_ACTIVATION; }
};

// The jobs.  ROWS: rows of A and Y belong to experts.
struct Plain {
  static constexpr bool EPILOGUE = false, ROWS = false;
};
struct Linear {
  static constexpr bool EPILOGUE = true, ROWS = false;
  Epilogue epilogue;
};
struct Experts {
  static constexpr bool EPILOGUE = true, ROWS = true;
  Epilogue epilogue;
  const int *offsets, *rows;
  int64_t w_stride, sw_stride, bias_stride;
  int experts, a_rows, y_rows;
};

// ---------------------------------------------------------------------------------------------- results

// x / (1 + exp(-u)), as silu().
__device__ inline float times_logistic(float x, float u) {
  const float e = __builtin_amdgcn_exp2f(u * -1.44269504f);
  return x * (__builtin_amdgcn_rcpf(fmaf(e, 0.0625f, 0.0625f)) * 0.0625f);
}

__device__ inline float activated(float x, int f) {
  switch (f) {
    case XORENC_RELU: return x < 0.f ? 0.f : x;
    case XORENC_SILU: return silu(x);
    case XORENC_GELU: return 0.5f * x * erfcf(x * -0.70710678f);
    case XORENC_GELU_TANH: return times_logistic(x, 1.59576912f * fmaf(0.044715f * x * x, x, x));
    default: return x;
  }
}

// A wave's 16 TN x 16 TM results with the epilogue.  Sixteen rows at a time change places in LDS in fp32 (`out`, the wave's own; 16-byte chunks of row m
// at chunk ^ m), so that a lane has as many neighbours of a row as 16 bytes of Y hold, and always the same columns: their bias is read once,
// the residual and Y in whole runs.
template <int TN, int TM, bool EXACT>
__device__ inline void store_tile_with(const Epilogue &epilogue, const MatmulArgs &g, const f32x4 (&acc)[TN][TM], uint8_t *out, int m_first, int n_first,
                                       int lane) {
  typedef typename std::conditional<EXACT, F32, BF16>::type T;
  typedef typename T::Elem Out;
  constexpr int WIDTH = 16 * TN, CHUNKS = WIDTH / 4, PER = 16 / (int)sizeof(Out), LANES = WIDTH / PER, SWIZZLE = (CHUNKS < 16 ? CHUNKS : 16) - 1;
  constexpr int STEPS = (16 * LANES + 63) / 64;
  f32x4 *const chunks = reinterpret_cast<f32x4 *>(out);
  const int c = lane % LANES, n = n_first + c * PER;
  const bool whole = n + PER <= g.N;
  float bias[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    bias[e] = 0.f;
    if (epilogue.bias && n + e < g.N)
      bias[e] = epilogue.bias_bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(epilogue.bias)[n + e] << 16)
                                   : static_cast<const float *>(epilogue.bias)[n + e];
  }
  Out *const Y = static_cast<Out *>(g.Y);
  const Out *const residual = static_cast<const Out *>(epilogue.residual);
#pragma unroll
  for (int j = 0; j < TM; ++j) {
#pragma unroll
    for (int i = 0; i < TN; ++i) chunks[(lane & 15) * CHUNKS + ((4 * i + (lane >> 4)) ^ (lane & SWIZZLE))] = acc[i][j];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int m = k * (64 / LANES) + lane / LANES, row = m_first + 16 * j + m;
      if (m >= 16 || row >= g.M) continue;
      float y[PER], old[PER];
#pragma unroll
      for (int e = 0; e < PER; e += 4) {
        const f32x4 v = chunks[m * CHUNKS + ((c * (PER / 4) + e / 4) ^ (m & SWIZZLE))];
#pragma unroll
        for (int q = 0; q < 4; ++q) y[e + q] = activated(v[q] + bias[e + q], epilogue.activation), old[e + q] = 0.f;
      }
      Out *const to = Y + (int64_t)row * g.ldy + n;
      if (residual) {
        const Out *const from = residual + (int64_t)row * epilogue.ld_residual + n;
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (n + e < g.N) {
            if constexpr (EXACT)
              old[e] = from[e];
            else
              old[e] = __uint_as_float((uint32_t)from[e] << 16);
          }
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) y[e] += old[e];
      if (whole) {
        if constexpr (EXACT)
          __builtin_nontemporal_store(f32x4{y[0], y[1], y[2], y[3]}, reinterpret_cast<f32x4_anywhere *>(to));
        else
          __builtin_nontemporal_store(u32x4{to_bf16x2(y[0], y[1]), to_bf16x2(y[2], y[3]), to_bf16x2(y[4 % PER], y[5 % PER]), to_bf16x2(y[6 % PER], y[7 % PER])},
                                      reinterpret_cast<u32x4_anywhere *>(to));
      } else {
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (n + e < g.N) T::store(to + e, y[e]);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------- rows of experts

// Which of all experts' tiles of BM rows (times n_tiles) is this workgroup's: the expert's rows and matrix in g, and its tile.  Tiles of one expert follow each
// other, and each XCD (workgroup i runs on XCD i % 8) takes a run of them, so that they share W in its L2.  Every wave finds out
// by itself: a lane has up to four neighbouring experts, and a scan over the lanes says how many tiles come before.
template <int BM, class Elem>
__device__ inline bool take_tile(const Experts &job, MatmulArgs &g, Epilogue &epilogue, int n_tiles, int lane, int &local, int &m_tiles, int &first_row) {
  constexpr int PER = (XORENC_MOE_MAX_EXPERTS + 63) / 64;
  const int per = (job.experts + 63) / 64;
  int first[PER], rows[PER], sum = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int e = lane * per + k;
    first[k] = rows[k] = 0;
    if (k < per && e < job.experts) {
      first[k] = min(max(job.offsets[e], 0), job.y_rows);  // (whatever they hold, rows stay within Y)
      rows[k] = min(max(job.offsets[e + 1], first[k]), job.y_rows) - first[k];
    }
    sum += (rows[k] + BM - 1) / BM;
  }
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int other = __shfl_up(upto, d);
    if (lane >= d) upto += other;
  }
  const int total = __builtin_amdgcn_readlane(upto, 63) * n_tiles, per_xcd = (total + 7) / 8;
  const int in_run = blockIdx.x >> 3, tile = (blockIdx.x & 7) * per_xcd + in_run;
  if (in_run >= per_xcd || tile >= total) return false;
  const int unit = tile / n_tiles;
  const int owner = __ffsll((unsigned long long)__ballot(upto > unit)) - 1;
  int before = upto - sum, e = lane * per, r = rows[0], f = first[0];
#pragma unroll
  for (int k = 1; k < PER; ++k) {
    const int tiles = (r + BM - 1) / BM;
    if (k < per && unit >= before + tiles) before += tiles, e = lane * per + k, r = rows[k], f = first[k];
  }
  before = __builtin_amdgcn_readlane(before, owner);
  e = __builtin_amdgcn_readlane(e, owner);
  g.M = __builtin_amdgcn_readlane(r, owner);
  first_row = __builtin_amdgcn_readlane(f, owner);
  local = tile - before * n_tiles;
  m_tiles = (g.M + BM - 1) / BM;
  g.W += e * job.w_stride;
  g.SW += e * job.sw_stride;
  g.Y = static_cast<Elem *>(g.Y) + first_row * g.ldy;
  if (!job.rows) g.A += first_row * g.lda, g.SA += first_row * g.sa_row;
  if (epilogue.bias)
    epilogue.bias = static_cast<const uint8_t *>(epilogue.bias) + e * job.bias_stride * (epilogue.bias_bf16 ? 2 : 4);
  return true;
}

// The rows of A of a tile from row m0 on: where they are counted from, and the number there of the tile's row m.
template <class Job>
struct RowsOfA {
  const uint8_t *A;
  const float *SA;
  __device__ RowsOfA(const Job &, const MatmulArgs &g, int m0, int) : A(g.A + m0 * g.lda), SA(g.SA + m0 * g.sa_row) {}
  __device__ int64_t operator()(int m) const { return m; }
};
template <>
struct RowsOfA<Experts> {
  const uint8_t *A;
  const float *SA;
  const int *rows;
  uint32_t last;
  __device__ RowsOfA(const Experts &job, const MatmulArgs &g, int m0, int first_row)
      : A(job.rows ? g.A : g.A + m0 * g.lda), SA(job.rows ? g.SA : g.SA + m0 * g.sa_row), rows(job.rows ? job.rows + first_row + m0 : nullptr),
        last((uint32_t)job.a_rows - 1u) {}
  __device__ int64_t operator()(int m) const { return rows ? (int64_t)min((uint32_t)rows[m], last) : (int64_t)m; }
};

}  // namespace xorenc_fp8_detail

#endif
