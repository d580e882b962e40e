// The block-scaled product with tiles that several waves share (many rows of A).
//
// A workgroup owns BN = 16 TN WN rows of W and BM = 16 TM WM rows of A; its WN x WM waves hold 16 TN x 16 TM results each,
// in registers that vector instructions reach: every block of 128 columns ends in one fused multiply-add per result.  A
// block of both operands (128 bytes a row) goes from memory to one of two LDS buffers without passing through registers;
// a row's eight 16-byte chunks are stored at chunk ^ (row / 2 % 8), so that the 16 rows of an operand read spread over
// all banks.
//
// Two barriers a block.  At the first, halfway through its row tiles, every wave has read the block's rows of A and the
// lower half of its rows of W, so that those of the next block but one can be fetched into their place (group 1), and the
// upper half of this block's W has landed; at the second, before the last row tile, all of the block has been read (the
// upper half is fetched, group 2) and the next block's group 1 has landed.  A fetch so has 1.4 blocks' time to land, not one
// (8192 x 16384 x 4096: 624 -> 570 us), and the matrix instructions of the row tile behind a barrier cover its wait and the
// operand reads behind it.
#ifndef XORENC_FP8_TILE_H
#define XORENC_FP8_TILE_H

#include <type_traits>

#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {

struct MatmulArgs {
  const uint8_t *A, *W;
  const float *SA, *SW;
  void *Y;
  int64_t lda, ldw, sa_row, sa_blk, ldsw, ldy;
  int M, N, K, blocks;
};

// A wave's 16 TN x 16 TM results, from row n_first of W and m_first of A on.  A lane holds four neighbours of a row of Y in
// each 16 x 16 tile.  They change places in LDS (`out`, the wave's own; 16-byte chunks of row m at chunk ^ m), so that a store
// writes 16 bytes a lane and whole runs of 16 TN results (8192 x 16384 x 4096 bf16: 569 -> 539 us).  Stores that pass the caches
// by leave them to A and W, and are not waited for by the next tile's loads: the same shape 547 -> 486 us, 4096 x 2048 x 512 11.2 ->
// 9.4, 4096 x 1024 x 1024 12.1 -> 11.5; 4096 x 8192 x 1024 42.1 -> 42.8.  (What reads Y next finds less of it in the caches: the
// product and the gate behind it 609 -> 599 us for 8192 x 16384 x 4096, 301 -> 306 for 4096, 154 -> 151 for 2048 tokens, 17.3 -> 16.2 for
// 4096 x 2048 x 512.)
template <int TN, int TM, bool EXACT>
__device__ inline void store_tile(const MatmulArgs &g, const f32x4 (&acc)[TN][TM], uint8_t *out, int m_first, int n_first, int lane) {
  typedef typename std::conditional<EXACT, float, uint16_t>::type Out;
  constexpr int WIDTH = 16 * TN, ROW = WIDTH * (int)sizeof(Out), CHUNKS = ROW / 16, PER_CHUNK = 16 / (int)sizeof(Out);
  const int r = lane & 15;
#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      const int m = 16 * j + r, byte = (16 * i + 4 * (lane >> 4)) * (int)sizeof(Out);
      uint8_t *const p = out + m * ROW + ((byte / 16) ^ (m & (CHUNKS - 1))) * 16 + byte % 16;
      const f32x4 v = acc[i][j];
      if constexpr (EXACT)
        *reinterpret_cast<f32x4 *>(p) = v;
      else
        *reinterpret_cast<u32x2 *>(p) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
    }
  Out *const Y = static_cast<Out *>(g.Y);
  const int c = lane % CHUNKS, n = n_first + c * PER_CHUNK;
#pragma unroll
  for (int k = 0; k < (16 * TM * CHUNKS + 63) / 64; ++k) {
    const int m = k * (64 / CHUNKS) + lane / CHUNKS;
    if (m >= 16 * TM) break;
    const u32x4 v = *reinterpret_cast<const u32x4 *>(out + m * ROW + (c ^ (m & (CHUNKS - 1))) * 16);
    if (m_first + m >= g.M) continue;
    Out *const y = Y + (int64_t)(m_first + m) * g.ldy + n;
    if (n + PER_CHUNK <= g.N) {
      __builtin_nontemporal_store(v, reinterpret_cast<u32x4_anywhere *>(y));
    } else {
#pragma unroll
      for (int e = 0; e < PER_CHUNK; ++e)
        if (n + e < g.N) y[e] = EXACT ? (Out)__uint_as_float(v[e & 3]) : (Out)(v[(e / 2) & 3] >> (16 * (e & 1)));
    }
  }
}

template <int TN, int TM, int WN, int WM, bool EXACT>
struct TileShape {
  static constexpr int BN = 16 * TN * WN, BM = 16 * TM * WM, WAVES = WN * WM;
  static constexpr int STAGE = (BN + BM) * 128;
  static constexpr int LDS = 2 * STAGE + 2 * BM * 4;
  // 1 KB loads (eight rows) of a wave per block: rows of A and the lower half of each wave's rows of W; the upper half
  static constexpr int GROUP1 = (BM / 8 + BN / 16) / WAVES, GROUP2 = BN / 16 / WAVES;
  static_assert((BM / 8 + BN / 16) % WAVES == 0 && (BN / 16) % WAVES == 0, "the waves load as much each");
  static_assert(BM % 64 == 0 && TN >= 2 && TN % 2 == 0 && 128 % (16 * TN) == 0, "scales");
};

template <int TN, int TM, int WN, int WM, bool EXACT>
__global__ __launch_bounds__(WN *WM * 64, 2) void matmul_tile_kernel(MatmulArgs g, int n_tiles, int m_tiles, int per_xcd) {
  typedef TileShape<TN, TM, WN, WM, EXACT> Shape;
  constexpr int BN = Shape::BN, BM = Shape::BM, STAGE = Shape::STAGE, N1 = Shape::GROUP1, N2 = Shape::GROUP2;
  extern __shared__ __attribute__((aligned(1024))) uint8_t tile_lds[];

  // workgroup i runs on XCD i % 8: each XCD takes a run of tiles, four row tiles of A wide, that share rows in its L2
  const int tile = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (tile >= n_tiles * m_tiles) return;
  constexpr int GROUP = 4;
  const int strip = tile / (GROUP * n_tiles), in_strip = tile - strip * (GROUP * n_tiles);
  const int strip_m = min(GROUP, m_tiles - strip * GROUP);
  // ... and each strip begins where an XCD's 32 CUs end that began with the strip before: rows of W that come from memory, not from
  // the cache behind the L2s, are then waited for by one XCD, and in the first round (8192 x 16384 x 4096, three sets of operands in turn
  // 553 -> 527 us, 4096 x 9216 x 8192 368 -> 344; one set, which that cache holds, 514 and 521)
  const int at_n = in_strip / strip_m, tile_m = strip * GROUP + in_strip - at_n * strip_m;
  const int tile_n = (at_n + strip * (32 / GROUP)) % n_tiles;
  const int n0 = tile_n * BN, m0 = tile_m * BM;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const uint32_t lds0 = lds_address(tile_lds);

  // ---- this wave's loads
  const u32x4 w_desc = descriptor(g.W + n0 * g.ldw), a_desc = descriptor(g.A + m0 * g.lda), s_desc = descriptor(g.SA + m0 * g.sa_row);
  constexpr int HALF = TN * 8;  // rows of half of a wave's row tiles
  // first row of load i of group 1 (rows of A, then lower halves) and of group 2
  auto row1 = [&](int i) {
    const int l = wave * N1 + i;
    return l < BM / 8 ? l * 8 : (l - BM / 8) / TN * (2 * HALF) + (l - BM / 8) % TN * 8;
  };
  auto of_a = [&](int i) { return wave * N1 + i < BM / 8; };
  auto row2 = [&](int i) {
    const int l = wave * N2 + i;
    return l / TN * (2 * HALF) + HALF + l % TN * 8;
  };
  const int lane_row = lane >> 3;
  auto chunk_of = [&](int row) { return e4m3_chunk(lane, row + lane_row) * 16; };  // this lane's column
  uint32_t at1[N1], at2[N2];
#pragma unroll
  for (int i = 0; i < N1; ++i)
    at1[i] = (uint32_t)(min(row1(i) + lane_row, (of_a(i) ? g.M - m0 : g.N - n0) - 1) * (of_a(i) ? g.lda : g.ldw)) + (uint32_t)chunk_of(row1(i));
#pragma unroll
  for (int i = 0; i < N2; ++i) at2[i] = (uint32_t)(min(row2(i) + lane_row, g.N - n0 - 1) * g.ldw) + (uint32_t)chunk_of(row2(i));
  // ---- and of 64 rows' scales of A (the waves beyond BM / 64 fetch what others fetch: all wait for as many loads)
  const int s_rows = wave % (BM / 64) * 64;
  const uint32_t s_at = (uint32_t)(min(s_rows + lane, g.M - m0 - 1) * g.sa_row) * 4u;
  const uint32_t s_step = (uint32_t)(g.sa_blk * 4);
  const int tail = g.K & (kBlock - 1);
  auto fetch1 = [&](int b, int i) {
    fetch_16(lds0 + (b & 1) * STAGE + (of_a(i) ? BN * 128 : 0) + row1(i) * 128, at1[i], of_a(i) ? a_desc : w_desc, (uint32_t)b * kBlock);
  };
  auto fetch2 = [&](int b, int i) { fetch_16(lds0 + (b & 1) * STAGE + row2(i) * 128, at2[i], w_desc, (uint32_t)b * kBlock); };
  auto fetch_scales = [&](int b) { fetch_4(lds0 + 2 * STAGE + (b & 1) * (BM * 4) + s_rows * 4, s_at, s_desc, (uint32_t)b * s_step); };
  // before the last block is fetched: chunks behind column K read as zero
  auto end1 = [&](int b) {
    if (tail == 0 || b != g.blocks - 1) return;
#pragma unroll
    for (int i = 0; i < N1; ++i) at1[i] = chunk_of(row1(i)) >= tail ? kBeyond : at1[i];
  };
  auto end2 = [&](int b) {
    if (tail == 0 || b != g.blocks - 1) return;
#pragma unroll
    for (int i = 0; i < N2; ++i) at2[i] = chunk_of(row2(i)) >= tail ? kBeyond : at2[i];
  };
  // what the last chunk of a row holds behind column K
  auto clear_tail = [&](int b) {
    if ((tail & 15) == 0 || b != g.blocks - 1) return;
    for (int r = tid; r < BN + BM; r += WN * WM * 64) {
      const int in = r < BN ? r : r - BN;
      uint8_t *const p = tile_lds + (b & 1) * STAGE + r * 128 + (((tail >> 4) ^ ((in >> 1) & 7)) * 16);
      *reinterpret_cast<u32x4 *>(p) = first_bytes(*reinterpret_cast<u32x4 *>(p), tail & 15);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };

  // ---- operand reads
  const int r = lane & 15;
  const uint32_t off = e4m3_operand_offset(lane);
  const uint8_t *const w_lds = tile_lds + wn * (TN * 2048), *const a_lds = tile_lds + BN * 128 + wm * (TM * 2048);
  const float *const s_lds = reinterpret_cast<const float *>(tile_lds + 2 * STAGE) + wm * (TM * 16) + r;
  // ---- scales of W: lane i holds those of block i of a run of 64
  const float *const sw_row = g.SW + (int64_t)((n0 + wn * (TN * 16)) / kBlock < (g.N + kBlock - 1) / kBlock ? (n0 + wn * (TN * 16)) / kBlock : 0) * g.ldsw;
  float sw_run = sw_row[min(lane, g.blocks - 1)];

  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  constexpr int IN_FLIGHT = 1 + N1 + N2;  // loads of a block: what may be outstanding behind those that a barrier waits for
  auto wait_for_loads = [&](bool others) {
    if (others)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(IN_FLIGHT) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (b >= g.blocks) break;
    end1(b);
    fetch_scales(b);
#pragma unroll
    for (int i = 0; i < N1; ++i) fetch1(b, i);
    end2(b);
#pragma unroll
    for (int i = 0; i < N2; ++i) fetch2(b, i);
  }
  wait_for_loads(g.blocks > 1);
  clear_tail(0);
  E4m3Operand a[TM], w[2];
  f32x4 d[2][TM];
  float f[TM], sa[TM];  // scales of this block's sums, and the next block's of A
  auto read_scales = [&](int b) {
#pragma unroll
    for (int j = 0; j < TM; ++j) sa[j] = s_lds[(b & 1) * BM + 16 * j];
  };
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    a[j] = read_operand(a_lds + j * 2048, off);
    f[j] = 0.f;
    d[(TN - 1) & 1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  w[0] = read_operand(w_lds, off);
  read_scales(0);
  // A row tile's sums are added while the matrix instructions of the next one run: four of them go with each.
  for (int b = 0; b < g.blocks; ++b) {
    const uint32_t here = (b & 1) * STAGE, there = STAGE - here;
    const bool more = b + 1 < g.blocks, fetches = b + 2 < g.blocks;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      constexpr int LAST = TN - 1, MIDDLE = TN / 2 - 1;
      if (i == MIDDLE) {
        wait_for_loads(more);
        if (fetches) end1(b + 2);
      }
      if (i < LAST) {
        w[(i + 1) & 1] = read_operand(w_lds + here + (i + 1) * 2048, off);
      } else if (more) {
        wait_for_loads(fetches);
        clear_tail(b + 1);
        if (fetches) end2(b + 2);
        w[0] = read_operand(w_lds + there, off);
        read_scales(b + 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      const int before = i ? i - 1 : LAST;
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        d[i & 1][j] = product_128<EXACT>(w[i & 1], a[j]);
        if (i == LAST && more) a[j] = read_operand(a_lds + there + j * 2048, off);
        if (i == MIDDLE && fetches) {
          if (j == 0) fetch_scales(b + 2);
#pragma unroll
          for (int p = j * N1 / TM; p < (j + 1) * N1 / TM; ++p) fetch1(b + 2, p);
        }
        if (i == LAST && fetches) {
#pragma unroll
          for (int p = j * N2 / TM; p < (j + 1) * N2 / TM; ++p) fetch2(b + 2, p);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[before][j][k] += f[j] * d[before & 1][j][k];
        asm volatile("" : "+v"(acc[before][j]));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (i == 0) {  // (the sums of the block before are complete)
        if ((b & 63) == 0 && b) sw_run = sw_row[min(b + lane, g.blocks - 1)];
        const float s = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sw_run), b & 63));
#pragma unroll
        for (int j = 0; j < TM; ++j) f[j] = sa[j] * s;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[TN - 1][j][k] += f[j] * d[(TN - 1) & 1][j][k];
  static_assert(BN * BM * (EXACT ? 4 : 2) <= 2 * STAGE, "the results of a tile fit");
  __syncthreads();
  store_tile<TN, TM, EXACT>(g, acc, tile_lds + wave * (16 * TM * 16 * TN * (EXACT ? 4 : 2)), m0 + wm * (16 * TM), n0 + wn * (16 * TN), lane);
}

}  // namespace xorenc_fp8_detail

#endif
