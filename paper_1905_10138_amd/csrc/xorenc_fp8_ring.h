// The block-scaled product where tiles of 256 x 256 would be too few: a workgroup owns BN = 16 TN WN rows of W and
// BM = 16 TM WM rows of A, and keeps a ring of NS stages of both in LDS, the next ones on their way from memory while one is
// multiplied.  KG groups of WN x WM waves take the blocks of 128 columns in turn (a stage holds a block for each) and add
// up at the end: more bytes on their way, and fewer barriers, for the same tile; groups of one wave need none.
//
// For few tokens the bytes of W bound it.  Operands read straight from memory to registers would be slower (1 x 16384 x 4096
// 16 against 12 us, 32 x 4096 x 4096 10.8 against 6.9): sixteen neighbouring lanes hold sixteen rows then, and an address
// unit that takes four neighbouring lanes' 64 bytes at a time needs 36 cycles for a load instead of 16.  Here eight lanes
// fetch 128 bytes of a row, and change places when they read the operand from LDS.
#ifndef XORENC_FP8_RING_H
#define XORENC_FP8_RING_H

#include "xorenc_fp8_tile.h"

namespace xorenc_fp8_detail {

template <int TN, int TM, int WN, int WM, int KG, int NS>
struct RingShape {
  static constexpr int BN = 16 * TN * WN, BM = 16 * TM * WM, GROUP = WN * WM, WAVES = GROUP * KG;
  static constexpr int SCALES = BM < 64 ? 64 : BM;             // scales of A that are fetched (those of the last row again, past it)
  static constexpr int BLOCK = (BN + BM) * 128 + SCALES * 4;  // one block's rows of W, of A, and the scales of A
  static constexpr int STAGE = KG * BLOCK;
  static constexpr int SUMS = KG > 1 ? (KG - 1) * BN * BM * 4 : 0;
  static constexpr int LDS = NS * STAGE > SUMS ? NS * STAGE : SUMS;
  static constexpr int PER = (BN + BM) / 8 / GROUP;  // 1 KB loads of a wave per block
  static_assert((BN + BM) % (8 * GROUP) == 0 && SCALES % 64 == 0 && 128 % (16 * TN) == 0 && LDS <= 160 * 1024, "shape");
};

template <int TN, int TM, int WN, int WM, int KG, int NS, bool EXACT>
__global__ __launch_bounds__(WN *WM *KG * 64) void matmul_ring_kernel(MatmulArgs g, int n_tiles, int m_tiles, int per_xcd) {
  typedef RingShape<TN, TM, WN, WM, KG, NS> Shape;
  constexpr int BN = Shape::BN, BM = Shape::BM, PER = Shape::PER, BLOCK = Shape::BLOCK, STAGE = Shape::STAGE;
  extern __shared__ __attribute__((aligned(1024))) uint8_t ring_lds[];
  const int tile = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);  // XCDs take runs of tiles that share rows of W
  if (tile >= n_tiles * m_tiles) return;
  const int tile_n = tile / m_tiles, tile_m = tile - tile_n * m_tiles;
  const int n0 = tile_n * BN, m0 = tile_m * BM;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / Shape::GROUP, in_group = wave % Shape::GROUP, wn = in_group % WN, wm = in_group / WN;
  const uint32_t lds0 = lds_address(ring_lds);

  // ---- loads: this wave's part of its group's blocks
  const u32x4 w_desc = descriptor(g.W + n0 * g.ldw), a_desc = descriptor(g.A + m0 * g.lda), s_desc = descriptor(g.SA + m0 * g.sa_row);
  const int lane_row = lane >> 3;
  auto row_of = [&](int i) {  // of W, then of A
    const int row = (in_group * PER + i) * 8;
    return row < BN ? row : row - BN;
  };
  auto of_w = [&](int i) { return (in_group * PER + i) * 8 < BN; };
  auto chunk_of = [&](int i) { return e4m3_chunk(lane, row_of(i) + lane_row) * 16; };
  uint32_t at[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i)
    at[i] = (uint32_t)(min(row_of(i) + lane_row, (of_w(i) ? g.N - n0 : g.M - m0) - 1) * (of_w(i) ? g.ldw : g.lda)) + (uint32_t)chunk_of(i);
  const int s_rows = in_group % (Shape::SCALES / 64) * 64;
  const uint32_t s_at = (uint32_t)(min(s_rows + lane, g.M - m0 - 1) * g.sa_row) * 4u, s_step = (uint32_t)(g.sa_blk * 4);
  const int tail = g.K & (kBlock - 1), stages = (g.blocks + KG - 1) / KG;
  // Load i of stage s of this group's blocks into its slot.  A block past the last one reads as zero, and so do chunks behind
  // column K.
  auto fetch = [&](int s, int i) {
    const int b = s * KG + kg;
    const uint32_t to = lds0 + (uint32_t)(s % NS) * STAGE + kg * BLOCK;
    const int most = b >= g.blocks ? 0 : tail && b == g.blocks - 1 ? tail : kBlock;  // columns of the block
    if (i < PER)
      fetch_16(to + (in_group * PER + i) * 1024, chunk_of(i) >= most ? kBeyond : at[i], of_w(i) ? w_desc : a_desc, most ? (uint32_t)b * kBlock : 0u);
    else
      fetch_4(to + (BN + BM) * 128 + s_rows * 4, most ? s_at : kBeyond, s_desc, most ? (uint32_t)b * s_step : 0u);
  };
  const int w_row = (n0 + wn * (TN * 16)) / kBlock;
  const float *const sw_row = g.SW + (int64_t)(w_row * kBlock < g.N ? w_row : 0) * g.ldsw;
  float sw_run = sw_row[min(lane, g.blocks - 1)];

  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t off = e4m3_operand_offset(lane);
  constexpr int LOADS = PER + 1;  // of a wave per stage
  struct Operands {
    E4m3Operand w[TN], a[TM];
    float sa[TM];
  };
  // The operands of stage s, which has landed.
  auto read = [&](int s, Operands &o) {
    uint8_t *const slot = ring_lds + (uint32_t)(s % NS) * STAGE + kg * BLOCK;
    if ((tail & 15) && s == stages - 1) {  // what the last chunk of a row holds behind column K
      if (s * KG + kg == g.blocks - 1) {
        for (int row = in_group * 64 + lane; row < BN + BM; row += Shape::GROUP * 64) {
          uint8_t *const p = slot + row * 128 + (((tail >> 4) ^ (((row < BN ? row : row - BN) >> 1) & 7)) * 16);
          *reinterpret_cast<u32x4 *>(p) = first_bytes(*reinterpret_cast<u32x4 *>(p), tail & 15);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) o.a[j] = read_operand(slot + (BN + (wm * TM + j) * 16) * 128, off);
#pragma unroll
    for (int i = 0; i < TN; ++i) o.w[i] = read_operand(slot + (wn * TN + i) * 2048, off);
#pragma unroll
    for (int j = 0; j < TM; ++j) o.sa[j] = reinterpret_cast<const float *>(slot + (BN + BM) * 128)[(wm * TM + j) * 16 + r];
  };
  // The products of stage s; between them the loads of stage `next`, where it is not negative.
  auto multiply = [&](int s, const Operands &o, int next) {
    const int b = s * KG + kg;
    if ((b & 63) == kg && b >= 64) sw_run = sw_row[min(b + lane - kg, g.blocks - 1)];
    const float sw = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sw_run), b & 63));
    const bool there = b < g.blocks;  // (else the last stage, for some groups: zeros)
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const float f = there ? o.sa[j] * sw : 0.f;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        const int k = j * TN + i;
        const f32x4 d = product_128<EXACT>(o.w[i], o.a[j]);
        if (next >= 0) {
#pragma unroll
          for (int l = k * LOADS / (TN * TM); l < (k + 1) * LOADS / (TN * TM); ++l) fetch(next, l);
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[i][j][n] += f * d[n];
      }
    }
  };
  auto fetch_all = [&](int s) {  // (stages past the last read as zero: every wave has as many loads on their way)
#pragma unroll
    for (int l = 0; l < LOADS; ++l) fetch(s, l);
  };
  if constexpr (Shape::GROUP > 1 && !(EXACT && KG * NS == 4)) {
    // A stage's operands are in registers before the one before is multiplied, and the loads into its slot go between the
    // products: a wave that issues its loads in a run waits for the address unit, 35 cycles a load, before it may multiply
    // (64 x 16384 x 4096 with three stages 17.2 -> 14.4 us).
    Operands o[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) fetch_all(s);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 1) * LOADS) : "memory");
    read(0, o[0]);
    auto landed = [&]() {  // and every wave has read the stage before, whose slot is filled next
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * LOADS) : "memory");
    };
    for (int s = 0; s < stages; s += 2) {
      landed();
      if (s + 1 < stages) read(s + 1, o[1]);
      multiply(s, o[0], s + NS);
      if (s + 1 == stages) break;
      landed();
      if (s + 2 < stages) read(s + 2, o[0]);
      multiply(s + 1, o[1], s + 1 + NS);
    }
  } else {
    // A stage's loads, its operands, its products, where that leaves registers for more waves: those on their own, which need no
    // barrier (1 x 4096 x 9216 8.1 us; as above 10.1), and two workgroups a CU with operands in bf16 (250 x 6000 x 3000 21, 29).
    Operands o;
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) fetch_all(s);
    for (int s = 0; s < stages; ++s) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * LOADS) : "memory");
      if constexpr (Shape::GROUP > 1) asm volatile("s_barrier" ::: "memory");
      fetch_all(s + NS - 1);
      read(s, o);
      multiply(s, o, -1);
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (no load may land in what follows)
  if constexpr (KG > 1) {  // the groups' sums meet in LDS, in the order of the groups
    f32x4 *const sums = reinterpret_cast<f32x4 *>(ring_lds);
    if (kg > 0) {
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) sums[(((kg - 1) * Shape::GROUP + in_group) * (TN * TM) + i * TM + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (kg == 0) {
#pragma unroll
      for (int k = 1; k < KG; ++k)
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) acc[i][j] += sums[(((k - 1) * Shape::GROUP + in_group) * (TN * TM) + i * TM + j) * 64 + lane];
    }
    __syncthreads();
    if (kg > 0) return;
  }
  store_tile<TN, TM, EXACT>(g, acc, ring_lds + in_group * (16 * TM * 16 * TN * 4), m0 + wm * (16 * TM), n0 + wn * (16 * TN), lane);
}

}  // namespace xorenc_fp8_detail

#endif
