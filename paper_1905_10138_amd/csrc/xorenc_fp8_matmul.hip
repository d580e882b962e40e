// Y = A W^T with A [M, K] and W [N, K] in e4m3, a scale for each 1 x 128 block of A and each 128 x 128 block of W:
//   Y[m][n] = sum over blocks b of SA[m][b] SW[n / 128][b] sum over k in b of A[m][k] W[n][k].
// The sum inside a block is the matrix instruction's; the scaled sums are added in fp32.
#include "xorenc_fp8_ring.h"

namespace xorenc_fp8_detail {
namespace {

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

// Few rows of A, or few tiles: a workgroup owns 16 NT rows of W and 16 MT rows of A.  Its waves take the blocks of the reduction
// in turn, each with all of the tile, and operands go from memory to the registers of the wave that multiplies them, the next
// block's while this one's are multiplied; the sums meet in LDS, in the order of the waves.  Every CU so has work of its own
// where tiles of the other kernel would be too few, and no barrier stands between a load and its use.
template <int MT, int NT, int WAVES, int AHEAD, bool EXACT>
__global__ __launch_bounds__(WAVES * 64) void matmul_rows_kernel(MatmulArgs g, int wide, int n_tiles) {
  constexpr int TILES = MT * NT, PASS = TILES < 8 ? TILES : 8;  // tiles whose sums are in LDS at a time
  __shared__ f32x4 part[WAVES][PASS][64];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tile_m = blockIdx.x / n_tiles, tile_n = blockIdx.x - tile_m * n_tiles;
  const int n0 = tile_n * (16 * NT), m0 = tile_m * (16 * MT);
  const uint8_t *const w_base = g.W + n0 * g.ldw, *const a_base = g.A + m0 * g.lda;
  const float *const sa_base = g.SA + m0 * g.sa_row;
  uint32_t w_at[NT], a_at[MT], sa_at[MT];
#pragma unroll
  for (int i = 0; i < NT; ++i) w_at[i] = (uint32_t)(min(16 * i + r, g.N - n0 - 1) * g.ldw);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = min(16 * i + r, g.M - m0 - 1);
    a_at[i] = (uint32_t)(m * g.lda);
    sa_at[i] = (uint32_t)(m * g.sa_row);
  }
  const float *const sw = g.SW + (int64_t)(n0 / kBlock) * g.ldsw;
  struct Operands {
    E4m3Operand w[NT], a[MT];
    float sa[MT], sw;
  };
  const int zero = vector_zero();
  auto load_scales = [&](int b, Operands &o) {
    const float *const sb = sa_base + b * g.sa_blk;
    o.sw = sw[b + zero];
#pragma unroll
    for (int i = 0; i < MT; ++i) o.sa[i] = sb[sa_at[i]];
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](int, const Operands &o) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float f = o.sa[i] * o.sw;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const f32x4 d = product_128<EXACT>(o.w[j], o.a[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][j][k] += f * d[k];
      }
    }
  };
  const int whole = g.K / kBlock;
  pipeline<AHEAD, Operands>((whole - wave + WAVES - 1) / WAVES, [&](int s, Operands &o) {
    const int b = wave + s * WAVES;
#pragma unroll
    for (int i = 0; i < NT; ++i) load_block(w_base + (int64_t)b * kBlock + w_at[i], lane, o.w[i]);
#pragma unroll
    for (int i = 0; i < MT; ++i) load_block(a_base + (int64_t)b * kBlock + a_at[i], lane, o.a[i]);
    load_scales(b, o);
  }, multiply);
  if (whole < g.blocks && whole % WAVES == wave) {  // the last block, a short one
    const int c = whole * kBlock, left = g.K - c;
    Operands o;
#pragma unroll
    for (int i = 0; i < NT; ++i) load_last_block(w_base + c + w_at[i], lane, left, o.w[i]);
#pragma unroll
    for (int i = 0; i < MT; ++i) load_last_block(a_base + c + a_at[i], lane, left, o.a[i]);
    load_scales(whole, o);
    multiply(0, o);
  }
#pragma unroll
  for (int t0 = 0; t0 < TILES; t0 += PASS) {
    if (t0) __syncthreads();
#pragma unroll
    for (int t = 0; t < PASS; ++t) part[wave][t][lane] = acc[(t0 + t) / NT][(t0 + t) % NT];
    __syncthreads();
    for (int t = wave; t < PASS; t += WAVES) {
      f32x4 v = part[0][t][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v += part[w][t][lane];
      store_result<EXACT>(g, m0 + 16 * ((t0 + t) / NT) + r, n0 + 16 * ((t0 + t) % NT) + 4 * (lane >> 4), v, wide);
    }
  }
}

template <int TN, int TM, int WN, int WM, bool EXACT>
void launch_tile(const MatmulArgs &g, bool wide, hipStream_t st) {
  typedef TileShape<TN, TM, WN, WM, EXACT> Shape;
  const int n_tiles = (g.N + Shape::BN - 1) / Shape::BN, m_tiles = (g.M + Shape::BM - 1) / Shape::BM;
  const int per_xcd = (n_tiles * m_tiles + 7) / 8;
  hipLaunchKernelGGL((matmul_tile_kernel<TN, TM, WN, WM, EXACT>), dim3((unsigned)(per_xcd * 8)), dim3(Shape::WAVES * 64), Shape::LDS, st, g,
                     (int)wide, n_tiles, m_tiles, per_xcd);
}

template <int MT, int NT, int WAVES, int AHEAD, bool EXACT>
void launch_rows_of_a(const MatmulArgs &g, bool wide, hipStream_t st) {
  const int n_tiles = (g.N + 16 * NT - 1) / (16 * NT), m_tiles = (g.M + 16 * MT - 1) / (16 * MT);
  hipLaunchKernelGGL((matmul_rows_kernel<MT, NT, WAVES, AHEAD, EXACT>), dim3((unsigned)(n_tiles * m_tiles)), dim3(WAVES * 64), 0, st, g, (int)wide, n_tiles);
}

template <int TN, int TM, int WN, int WM, int KG, int NS, bool EXACT>
void launch_ring(const MatmulArgs &g, bool wide, hipStream_t st) {
  typedef RingShape<TN, TM, WN, WM, KG, NS> Shape;
  const int n_tiles = (g.N + Shape::BN - 1) / Shape::BN, m_tiles = (g.M + Shape::BM - 1) / Shape::BM;
  const int per_xcd = (n_tiles * m_tiles + 7) / 8;
  hipLaunchKernelGGL((matmul_ring_kernel<TN, TM, WN, WM, KG, NS, EXACT>), dim3((unsigned)(per_xcd * 8)), dim3(Shape::WAVES * 64), Shape::LDS, st, g,
                     (int)wide, n_tiles, m_tiles, per_xcd);
}

// The kernels, and what they take: `start` + rounds * (`tile` + steps * (`step` + `load` * share of the chip in use)), in us, with
// as many tiles side by side as `slots` says and a block of the reduction a step (its `split`-th part where the waves of a
// workgroup split it).  Fitted to 70 shapes of 1 .. 8192 x 64 .. 16384 x 64 .. 9216, bf16 results; taking the one that this
// says is the fastest costs 3 % over taking the one that was.  Some of the times it goes by (us: in the order of the list):
//   4096 x 4096 x 4096       61   76   95  116  131    -  >400
//   1347 x 9216 x 4170       65   84  107  125  128    -     -
//   443 x 12632 x 1979       33   23   23   30   30    -     -
//   1710 x 1024 x 6626       92   51   43   30   44    -     -
//   250 x 6000 x 3000        45   25   21   16   20   38    26
//   1361 x 907 x 256         21   11    7  6.4  5.8    -     -
//   514 x 748 x 1343         34   17    -  8.3    -    -   5.6
//   24 x 144 x 3891          50   26    -   11    -  5.1   7.3
struct Cost {
  int bn, bm, slots, split;
  float start, tile, step, load;
};
constexpr Cost kCosts[] = {
    {256, 256, 256, 1, 0.00f, 8.97f, 1.53f, 0.53f},  // 0: tiles of 256 x 256
    {128, 128, 512, 1, 2.51f, 3.69f, 0.72f, 0.50f},  // 1: of 128 x 128
    {128, 64, 768, 1, 2.73f, 2.37f, 0.55f, 0.58f},   // 2: of 128 x 64
    {64, 64, 512, 2, 2.00f, 2.47f, 0.50f, 0.49f},    // 3: of 64 x 64, two groups of waves, two stages of two blocks
    {64, 64, 1024, 1, 1.68f, 2.17f, 0.49f, 0.47f},   // 4: of 64 x 64, two stages of one block
    {16, 16, 512, 8, 1.49f, 0.00f, 0.69f, 0.48f},    // 5: of 16 x 16, from memory to registers
    {32, 32, 512, 8, 1.70f, 0.03f, 1.02f, 1.74f},    // 6: of 32 x 32
};
constexpr int kKernels = sizeof(kCosts) / sizeof(kCosts[0]);

int cheapest(int64_t M, int64_t N, int64_t blocks, bool exact) {
  int best = -1;
  float least = 0.f;
  for (int i = exact ? 1 : 0; i < kKernels; ++i) {  // (fp32 results of a tile of 256 x 256 do not fit in LDS, nor their operands in registers)
    const Cost &c = kCosts[i];
    const int64_t tiles = ((N + c.bn - 1) / c.bn) * ((M + c.bm - 1) / c.bm), steps = (blocks + c.split - 1) / c.split;
    if (tiles >= (1 << 22)) continue;
    const int64_t rounds = (tiles + c.slots - 1) / c.slots;
    const float use = tiles < c.slots ? (float)tiles / (float)c.slots : 1.f;
    const float t = c.start + (float)rounds * (c.tile + (float)steps * (c.step + c.load * use));
    if (best < 0 || t < least) best = i, least = t;
  }
  return best;
}

template <bool EXACT>
int32_t dispatch_matmul(const MatmulArgs &g, bool wide, hipStream_t st) {
  switch (cheapest(g.M, g.N, g.blocks, EXACT)) {
    case 0:
      if constexpr (!EXACT) launch_tile<8, 4, 2, 4, EXACT>(g, wide, st);
      break;
    case 1: launch_tile<4, 4, 2, 2, EXACT>(g, wide, st); break;
    case 2: launch_tile<4, 2, 2, 2, EXACT>(g, wide, st); break;
    case 3: launch_ring<2, 2, 2, 2, 2, 2, EXACT>(g, wide, st); break;
    case 4: launch_ring<2, 2, 2, 2, 1, 2, EXACT>(g, wide, st); break;
    case 5: launch_rows_of_a<1, 1, 8, 2, EXACT>(g, wide, st); break;
    case 6: launch_rows_of_a<2, 2, 8, 1, EXACT>(g, wide, st); break;
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
  const bool wide = wide_rows(Y, ldy, y_dtype);
  xorenc_internal_begin_call();
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return y_dtype == XORENC_X_F32 ? dispatch_matmul<true>(g, wide, st) : dispatch_matmul<false>(g, wide, st);
}
