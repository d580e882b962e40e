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
  __host__ __device__ __forceinline__ bool none() const { return !bias && !residual && activation == XORENC_NO_ACTIVATION; }
};

// The jobs.  ROWS: rows of A and Y belong to experts.
struct Plain {
  static constexpr bool EPILOGUE = false, ROWS = false;
};
struct Linear {
  static constexpr bool EPILOGUE = true, ROWS = false;  // (there is something to do)
  Epilogue epilogue;
};
struct Experts {
  static constexpr bool EPILOGUE = true, ROWS = true;
  Epilogue epilogue;
  const int *offsets, *rows;
  int64_t w_stride, sw_stride, bias_stride;
  int experts, a_rows, y_rows;
};

template <class Job>
__device__ __forceinline__ Epilogue epilogue_of(const Job &job) {
  if constexpr (Job::EPILOGUE)
    return job.epilogue;
  else
    return Epilogue();
}

// ---------------------------------------------------------------------------------------------- results

// x / (1 + exp(-u)), as silu().
__device__ inline float times_logistic(float x, float u) {
  const float e = __builtin_amdgcn_exp2f(u * -1.44269504f);
  return x * (__builtin_amdgcn_rcpf(fmaf(e, 0.0625f, 0.0625f)) * 0.0625f);
}

// x times the normal distribution function, erfc(-x / sqrt 2) / 2.  For z >= 0, erfc(z) exp(z^2) is t Q(t) with t = 1 / (1 + p z); Q and p were fitted to the
// function's values for 0 <= z <= 10 so that the largest relative error of the fit is least: 5.2e-6 (results of 16 bits, 0.1 % of their half step) and 2e-8.
// In fp32 arithmetic results of 32 bits are off by 5.5e-7 for x >= -2, and below by what rounding the exponential's argument makes, which grows with x^2: 1e-6
// down to -4, 2.1e-6 to -6, 3.4e-6 to -9, 8e-6 to -13 (measured; results of 1e-37 there).  1 + erf, a difference, would leave no digit from -6 on.
// Beyond, exp(-z^2) is 0.  (8192 x 16384 x 4096: 51 us beside a bias alone, with the library's erfcf 145.)
template <bool EXACT>
__device__ inline float gelu(float x) {
  const float e = __builtin_amdgcn_exp2f(x * (x * -0.72134752f));
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), EXACT ? 0.212132037f : 0.311126977f, 1.f));
  float q;
  if constexpr (EXACT) {
    q = fmaf(fmaf(fmaf(fmaf(-0.0647613779f, t, 0.242781237f), t, -0.256138295f), t, 0.273859143f), t, -0.0473247766f);
    q = fmaf(fmaf(fmaf(fmaf(q, t, 0.107462786f), t, 0.0741696507f), t, 0.0853576064f), t, 0.0845940039f);
  } else {
    q = fmaf(fmaf(fmaf(fmaf(fmaf(-0.0730531067f, t, 0.175327033f), t, 0.0203646906f), t, 0.131793633f), t, 0.121284649f), t, 0.12428052f);
  }
  q *= t * e;
  return x * (x > 0.f ? 1.f - q : q);
}

template <int F, bool EXACT>
__device__ inline float activated(float x) {
  if constexpr (F == XORENC_RELU) return x < 0.f ? 0.f : x;
  if constexpr (F == XORENC_SILU) return silu(x);
  if constexpr (F == XORENC_GELU) return gelu<EXACT>(x);
  if constexpr (F == XORENC_GELU_TANH) return times_logistic(x, 1.59576912f * fmaf(0.044715f * x * x, x, x));
  return x;
}

// A wave's 16 TN x 16 TM results with the epilogue, from row n_first of W and m_first of A on.  Sixteen rows at a time change places in LDS in fp32 (the wave's
// own; 16-byte chunks of row m at chunk ^ m), so that a lane has as many neighbours of a row as 16 bytes of Y hold, and always the same columns:
// their bias is read once, the residual and Y in whole runs.
// RESIDUAL: there may be one (rows of experts have none; 17576 of them by 2746 x 71 with SiLU 57.5 -> 53.4 us, 15396 by 335 x 256 in fp32 15.6 -> 13.6).
template <int TN, int TM, bool EXACT, bool RESIDUAL>
struct EpilogueTile {
  typedef typename std::conditional<EXACT, F32, BF16>::type T;
  typedef typename T::Elem Out;
  static constexpr int WIDTH = 16 * TN, CHUNKS = WIDTH / 4, PER = 16 / (int)sizeof(Out), LANES = WIDTH / PER, SWIZZLE = (CHUNKS < 16 ? CHUNKS : 16) - 1;
  static constexpr int STEPS = (16 * LANES + 63) / 64, LDS = 16 * WIDTH * 4;

  int M, N, lane, c, n, m_first;
  int64_t ldy;
  Out *Y;
  bool whole;
  float bias[PER];
  u32x4 old[TM][STEPS];  // the residual, of lanes whose columns are all there

  __device__ __forceinline__ EpilogueTile(const MatmulArgs &g, int m_first_, int n_first, int lane_)
      : M(g.M), N(g.N), lane(lane_), c(lane_ % LANES), n(n_first + lane_ % LANES * PER), m_first(m_first_), ldy(g.ldy), Y(static_cast<Out *>(g.Y)),
        whole(n + PER <= g.N) {}
  __device__ int row_of(int j, int k) const { return 16 * j + k * (64 / LANES) + lane / LANES; }
  __device__ static float widen(Out v) {
    if constexpr (EXACT)
      return v;
    else
      return __uint_as_float((uint32_t)v << 16);
  }

  // What comes from memory, wherever there is time to wait for it.
  __device__ __forceinline__ void load(const Epilogue &epilogue) {
#pragma unroll
    for (int e = 0; e < PER; ++e) bias[e] = 0.f;
    if (epilogue.bias) {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (n + e < N)
          bias[e] = epilogue.bias_bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t *>(epilogue.bias)[n + e] << 16)
                                       : static_cast<const float *>(epilogue.bias)[n + e];
    }
    const Out *const residual = static_cast<const Out *>(epilogue.residual);
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        old[j][k] = u32x4{0u, 0u, 0u, 0u};
        if (RESIDUAL && residual && whole)  // (rows past the last: the last one again)
          old[j][k] = *reinterpret_cast<const u32x4_anywhere *>(residual + (int64_t)min(m_first + row_of(j, k), M - 1) * epilogue.ld_residual + n);
      }
  }

  template <int F>
  __device__ __forceinline__ void store_as(const Epilogue &epilogue, const f32x4 (&acc)[TN][TM], uint8_t *out) {
    f32x4 *const chunks = reinterpret_cast<f32x4 *>(out);
    const Out *const residual = static_cast<const Out *>(epilogue.residual);
#pragma unroll
    for (int j = 0; j < TM; ++j) {
#pragma unroll
      for (int i = 0; i < TN; ++i) chunks[(lane & 15) * CHUNKS + ((4 * i + (lane >> 4)) ^ (lane & SWIZZLE))] = acc[i][j];
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const int in_tile = row_of(j, k), m = in_tile - 16 * j, row = m_first + in_tile;
        if (m >= 16 || row >= M) continue;
        float y[PER];
#pragma unroll
        for (int e = 0; e < PER; e += 4) {
          const f32x4 v = chunks[m * CHUNKS + ((c * (PER / 4) + e / 4) ^ (m & SWIZZLE))];
#pragma unroll
          for (int q = 0; q < 4; ++q) y[e + q] = activated<F, EXACT>(v[q] + bias[e + q]);
        }
        Out *const to = Y + (int64_t)row * ldy + n;
        if (whole) {
          if constexpr (EXACT) {
            const u32x4 r = old[j][k];
            f32x4 v = {y[0], y[1], y[2], y[3]};
            if constexpr (RESIDUAL) v += f32x4{__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[2]), __uint_as_float(r[3])};
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4_anywhere *>(to));
          } else {
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              v[q] = RESIDUAL ? to_bf16x2(y[2 * q] + bf16_lo(old[j][k][q]), y[2 * q + 1] + bf16_hi(old[j][k][q])) : to_bf16x2(y[2 * q], y[2 * q + 1]);
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4_anywhere *>(to));
          }
        } else {
          const Out *const from = RESIDUAL && residual ? residual + (int64_t)row * epilogue.ld_residual + n : nullptr;
#pragma unroll
          for (int e = 0; e < PER; ++e)
            if (n + e < N) T::store(to + e, RESIDUAL && from ? y[e] + widen(from[e]) : y[e]);
        }
      }
    }
  }

  __device__ __forceinline__ void store(const Epilogue &epilogue, const f32x4 (&acc)[TN][TM], uint8_t *out) {
    switch (epilogue.activation) {  // (once, not for each result: a branch each takes longer than what it chooses)
      case XORENC_RELU: return store_as<XORENC_RELU>(epilogue, acc, out);
      case XORENC_SILU: return store_as<XORENC_SILU>(epilogue, acc, out);
      case XORENC_GELU: return store_as<XORENC_GELU>(epilogue, acc, out);
      case XORENC_GELU_TANH: return store_as<XORENC_GELU_TANH>(epilogue, acc, out);
      default: return store_as<XORENC_NO_ACTIVATION>(epilogue, acc, out);
    }
  }
};

// ---------------------------------------------------------------------------------------------- rows of experts

// Which of all experts' tiles of BM rows (times n_tiles) is this workgroup's: the expert's rows and matrix in g, and its tile.  Each XCD (workgroup i runs on XCD
// i % 8) takes a run of tiles.  Where rows are few (COLUMNS 0) an expert's tiles follow each other, and those that share rows of W first.  Large tiles
// come by groups of COLUMNS column tiles of all experts, so that every XCD has rows of all of them, heavy ones and light ones, and finishes with the
// others (4096 tokens, two of eight experts of 8192 x 4096 346 -> 332 us, 8192, four of 32 of 2048 x 2048 198 -> 191; 512 columns, with 1024 329 and 191, and
// 4096 tokens, two of eight of 4096 x 9216 411 and 430).  Every wave finds out by itself: a lane has up to four neighbouring experts, and a scan over the
// lanes says how many tiles come before.
template <int BM, int COLUMNS, class Elem>
__device__ __forceinline__ bool take_tile(const Experts &job, MatmulArgs &g, Epilogue &epilogue, int n_tiles, int lane, int &tile_m, int &tile_n, int &first_row) {
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
  const int units = __builtin_amdgcn_readlane(upto, 63), total = units * n_tiles, per_xcd = (total + 7) / 8;
  const int in_run = blockIdx.x >> 3, tile = (blockIdx.x & 7) * per_xcd + in_run;
  if (in_run >= per_xcd || tile >= total) return false;
  const int columns = COLUMNS ? COLUMNS : n_tiles, group = tile / (columns * units), in_group = tile - group * (columns * units);
  const int wide = min(columns, n_tiles - group * columns), unit = in_group / wide;
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
  const int local = in_group - before * wide, m_tiles = (g.M + BM - 1) / BM;
  if constexpr (COLUMNS) {
    tile_m = local / wide;
    tile_n = group * columns + local - tile_m * wide;
  } else {
    tile_n = local / m_tiles;
    tile_m = local - tile_n * m_tiles;
  }
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
  __device__ __forceinline__ RowsOfA(const Job &, const MatmulArgs &g, int m0, int) : A(g.A + m0 * g.lda), SA(g.SA + m0 * g.sa_row) {}
  __device__ __forceinline__ int64_t operator()(int m) const { return m; }
};
template <>
struct RowsOfA<Experts> {
  const uint8_t *A;
  const float *SA;
  const int *rows;
  uint32_t last;
  __device__ __forceinline__ RowsOfA(const Experts &job, const MatmulArgs &g, int m0, int first_row)
      : A(job.rows ? g.A : g.A + m0 * g.lda), SA(job.rows ? g.SA : g.SA + m0 * g.sa_row), rows(job.rows ? job.rows + first_row + m0 : nullptr),
        last((uint32_t)job.a_rows - 1u) {}
  __device__ __forceinline__ int64_t operator()(int m) const { return rows ? (int64_t)min((uint32_t)rows[m], last) : (int64_t)m; }
};

}  // namespace xorenc_fp8_detail

#endif
