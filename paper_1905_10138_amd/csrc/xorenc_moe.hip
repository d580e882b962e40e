// A mixture-of-experts layer for a few tokens: Y = sum over a token's picks of share * W2_e (silu(G_e x) * (U_e x)), with
// expert weights in e4m3 (a scale per 128 x 128 block) and everything else in 16 or 32 bits.
//
// Five launches: the router's logits; the picks (not for very few tokens, whose picks every workgroup finds by itself); the gated
// activations h of the picked experts; their second product and the sum over picks; the sum of that product's parts (where it
// has any).  The bytes of the picked experts' weights bound the two products (32 tokens, two of eight experts of 4096 x 9216: 183 us,
// 5.0 TB/s over all launches).  Weights go from memory to a ring of stages in LDS (eight lanes fetch 128 bytes of a row; loads to
// registers, where a lane needs 32 bytes of one row of 16, take the address units twice as long: the same call 250 us, 207 by
// rings alone), and so do the activations that multiply them.  e4m3 values become bf16 exactly and multiply bf16 terms of the
// activations (one for bf16 activations, three for fp32, which sum to the value exactly), so that nothing is rounded to 8 bits on
// the way; h is kept as bf16 terms that hold 16 (24) bits.  The tokens that picked an expert are the columns of its matrix
// instructions; rows of tokens that are not there are not loaded.
//
// Terms of x and h lie in the workspace in the order in which they are used: a row is a run of blocks of 128 columns (zero
// behind the last column), a block its terms one after the other, a term the columns 16 g + 64 p + 8 h + 0..7 at 64 p + 32 h + 8 g:
// a quarter (p, h) of them is what the four lanes g of a row give to one matrix instruction.
#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

constexpr int kMostExperts = XORENC_MOE_MAX_EXPERTS, kMostPicks = XORENC_MOE_MAX_PICKS, kMostTokens = XORENC_MOE_MAX_TOKENS;
static_assert(kMostExperts == 256 && kMostTokens == 64 && kMostPicks == 16, "four experts per lane, tokens as bits of 64, a pick a lane");

// Tokens that picked an expert, `count` of them (at most as many as one pass multiplies: an expert that more tokens picked has
// several uses): pairs of a token and an expert that it picked are ordered by expert, then by token, and these are
// the pairs from `first` on.  Row i of h is pair i's.
struct Use {
  uint16_t expert, first, count, unused;
};

struct MoeArgs {
  const uint8_t *W13, *W2;
  const float *S13, *S2;
  int64_t ldw13, w13_stride, lds13, s13_stride, ldw2, w2_stride, lds2, s2_stride;
  int T, H, I, E, top, renormalise;
  int most_uses, pass;      // most_uses of them, the last ones with count 0; tokens that a pass takes at most
  int plans;                // every workgroup of the first product finds the uses by itself
  float *logits;            // [T][E]
  int *n_uses;              // how many
  Use *uses;
  uint8_t *pair_tokens;
  float *shares;            // of the pairs
  float *parts;             // [splits][T][H rounded up to 128]: their sums
  int splits, row_groups;
  uint16_t *x_terms, *h_terms;  // rows of tokens, and of pairs
  int x_row, h_row;             // bytes of a row
};

// Where column c of a block is in each of its terms.
__device__ inline int term_place(int c) { return (c >> 6) * 64 + ((c >> 3) & 1) * 32 + ((c >> 4) & 3) * 8 + (c & 7); }

// What rounding to bf16 leaves of a value; nothing of what is not finite (infinity less infinity would be NaN).
__device__ inline float rest_of_bf16(float v) {
  const float d = v - (float)(__bf16)v;
  return fabsf(d) <= 3.4028235e38f ? d : 0.f;
}

// ---------------------------------------------------------------------------------------------- router

// Logits in fp32: a workgroup per expert and four tokens, its waves share the columns.  The workgroups behind them write the
// bf16 terms of x.
template <class T, int TERMS>
__global__ __launch_bounds__(256) void router_kernel(const typename T::Elem *__restrict__ X, int64_t ldx,
                                                     const typename T::Elem *__restrict__ router, int64_t ldr, int tokens,
                                                     int H, int E, float *__restrict__ logits, uint16_t *__restrict__ terms,
                                                     int logit_groups) {
  __shared__ float part[4][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x >= logit_groups) {  // eight columns a thread
    const int pieces = (H + kBlock - 1) / kBlock * 16;
    const int64_t i = (int64_t)(blockIdx.x - logit_groups) * 256 + threadIdx.x;
    if (i >= (int64_t)tokens * pieces) return;
    const int t = (int)(i / pieces), c = (int)(i - (int64_t)t * pieces) * 8;
    float v[8];
    piece_of<T>(load_piece<T>(X + t * ldx, c, H), c, H, v);
    uint16_t *const dst = terms + ((int64_t)t * (pieces / 16) + c / kBlock) * (TERMS * kBlock) + term_place(c % kBlock);
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
      BF16::store8(dst + k * kBlock, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rest_of_bf16(v[j]);
    }
    return;
  }
  const int token_groups = (tokens + 3) / 4;
  const int e = blockIdx.x / token_groups, t0 = (blockIdx.x - e * token_groups) * 4;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int c = threadIdx.x * 8; c < H; c += 2048) {
    float r[8], v[4][8];
    typename T::Raw raw[5];
    raw[4] = load_piece<T>(router + e * ldr, c, H);
#pragma unroll
    for (int k = 0; k < 4; ++k) raw[k] = load_piece<T>(X + min(t0 + k, tokens - 1) * ldx, c, H);
    piece_of<T>(raw[4], c, H, r);
#pragma unroll
    for (int k = 0; k < 4; ++k) piece_of<T>(raw[k], c, H, v[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[k] += r[j] * v[k][j];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc[k] += __shfl_xor(acc[k], o);
    if (lane == 0) part[wave][k] = acc[k];
  }
  __syncthreads();
  const int k = threadIdx.x;
  if (k < 4 && t0 + k < tokens) logits[(t0 + k) * E + e] = (part[0][k] + part[1][k]) + (part[2][k] + part[3][k]);
}

// ---------------------------------------------------------------------------------------------- picks

// fp32 -> integers in the same order, any NaN above infinity, both zeros as one (-0 + 0 is 0)
__device__ inline uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  if (v != v) return 0xffffffffu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// A token's picks, by 16 neighbouring lanes (all lanes of a wave take part, for four tokens): lane j gets the j-th (`expert`,
// `share`).  A lane holds the keys of KEYS experts, 16 apart; zero, which is no number's key, stands for those that are not there or
// picked already.  (A wave a token, with its maximum by way of scalar registers: 64 tokens, eight of 128 experts 17.7 us and, this
// way, 8.8.)
template <int KEYS>
__device__ inline void picks_among(const MoeArgs &g, int t, int l, int &expert, float &share) {
  const float *const row = g.logits + t * g.E;
  uint32_t key[KEYS];
#pragma unroll
  for (int i = 0; i < KEYS; ++i) key[i] = l + 16 * i < g.E ? ordered(row[l + 16 * i]) : 0u;
  uint32_t own;  // this lane's largest key, and which it is (the first of equals)
  int which;
  auto find = [&]() {
    own = key[0], which = 0;
#pragma unroll
    for (int i = 1; i < KEYS; ++i) {
      which = key[i] > own ? i : which;
      own = max(own, key[i]);
    }
    return max_of_16_lanes(own);
  };
  uint32_t largest = find(), mine = 0u;
  const float most = from_ordered(largest);
  float sum = 0.f;
  if (!g.renormalise) {  // shares of a softmax over all experts
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
      if (key[i]) sum += expf(from_ordered(key[i]) - most);
    sum = sum_of_16_lanes(sum);
  }
  expert = 0;
  for (int j = 0; j < g.top; ++j) {  // the largest that is left; the lowest index of equals
    const int e = (int)(kMostExperts - max_of_16_lanes(own == largest ? (uint32_t)(kMostExperts - (l + 16 * which)) : 0u));
    if (l == j) expert = e, mine = largest;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) key[i] = e == l + 16 * i ? 0u : key[i];
    if (j + 1 < g.top) largest = find();
  }
  share = l < g.top ? expf(from_ordered(mine) - most) : 0.f;
  if (g.renormalise) sum = sum_of_16_lanes(share);
  share /= sum;
}

__device__ inline void picks_of_token(const MoeArgs &g, int t, int l, int &expert, float &share) {
  if (g.E <= 64)
    picks_among<4>(g, t, l, expert, share);
  else if (g.E <= 128)
    picks_among<8>(g, t, l, expert, share);
  else
    picks_among<16>(g, t, l, expert, share);
}

template <int TOKENS>
struct Picks {
  uint64_t tokens[kMostExperts];  // that picked an expert, a bit each
  float share[TOKENS][kMostPicks];
  uint16_t expert[TOKENS][kMostPicks];
  uint16_t first[kMostExperts];  // pair of an expert
};

// The uses in the order of their experts and the pairs in the order of the uses, by a workgroup of WAVES waves, each for four tokens
// at a time: put_count(uses), put_use(index, use), up to most_uses of them, and put_pair(index, token, share).
template <int WAVES, int TOKENS, class PutCount, class PutUse, class PutPair>
__device__ inline void plan_uses(const MoeArgs &g, Picks<TOKENS> &p, PutCount put_count, PutUse put_use, PutPair put_pair) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid < kMostExperts) p.tokens[tid] = 0u;
  __syncthreads();
  for (int t0 = 4 * wave; t0 < g.T; t0 += 4 * WAVES) {
    const int t = t0 + (lane >> 4), l = lane & 15;
    int e;
    float share;
    picks_of_token(g, min(t, g.T - 1), l, e, share);
    if (t < g.T && l < g.top) {
      p.expert[t][l] = (uint16_t)e;
      p.share[t][l] = share;
      atomicOr(reinterpret_cast<unsigned long long *>(&p.tokens[e]), 1ull << t);
    }
  }
  __syncthreads();
  if (wave == 0) {  // four experts a lane
    int n[4], sum = 0;  // uses << 16 | pairs
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = __popcll(p.tokens[4 * lane + i]);
      n[i] = (k + g.pass - 1) / g.pass << 16 | k;
      sum += n[i];
    }
    int before = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(before, o);
      if (lane >= o) before += v;
    }
    const int uses = __shfl(before, 63) >> 16;
    before -= sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 4 * lane + i, first = before & 0xffff, count = n[i] & 0xffff;
      p.first[e] = (uint16_t)first;
      for (int k = 0; k * g.pass < count; ++k)
        put_use((before >> 16) + k, Use{(uint16_t)e, (uint16_t)(first + k * g.pass), (uint16_t)min(g.pass, count - k * g.pass), 0});
      before += n[i];
    }
    if (lane == 0) put_count(uses);
    for (int u = uses + lane; u < g.most_uses; u += 64) put_use(u, Use{0, 0, 0, 0});
  }
  __syncthreads();
  for (int i = tid; i < g.T * g.top; i += WAVES * 64) {
    const int t = i / g.top, j = i - t * g.top, e = p.expert[t][j];
    put_pair(p.first[e] + __popcll(p.tokens[e] & ((1ull << t) - 1ull)), t, p.share[t][j]);
  }
}

// One workgroup.
__global__ __launch_bounds__(1024) void picks_kernel(MoeArgs g) {
  __shared__ Picks<kMostTokens> p;
  plan_uses<16>(
      g, p, [&](int uses) { *g.n_uses = uses; }, [&](int u, Use use) { g.uses[u] = use; },
      [&](int pair, int t, float share) {
        g.pair_tokens[pair] = (uint8_t)t;
        g.shares[pair] = share;
      });
}

// ---------------------------------------------------------------------------------------------- products

// Rows of terms in LDS: 256 bytes each, a row's 16-byte chunks at chunk ^ row % 16.  A load of four rows: lane l takes row l / 16 of
// them and this chunk of it.  Quarter q of a lane's columns is chunk 4 q + l / 16.
__device__ inline int term_chunk(int lane, int row) { return (lane ^ row) & 15; }
__device__ inline bf16x8 read_terms(const uint8_t *rows, int row, int lane, int q) {
  return *reinterpret_cast<const bf16x8 *>(rows + row * 256 + (((4 * q + (lane >> 4)) ^ row) & 15) * 16);
}

// Sums of the products of 16 rows of weights and 16 N rows of TERMS terms over a block; lane l has row l % 16 of the latter and rows 4 (l
// / 16) .. + 3 of the former.  XR rows are there (four: lanes take them in turn, and only the first of a row's counts).
template <int N, int XR, int TERMS>
__device__ inline void block_products(const E4m3Operand &w, const uint8_t *x, int lane, f32x4 (&d)[N]) {
  bf16x8 v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = quarter_as_bf16(w, q);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = XR < 16 ? lane & (XR - 1) : 16 * i + (lane & 15);
    d[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < TERMS; ++k)
#pragma unroll
      for (int q = 0; q < 4; ++q) d[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[q], read_terms(x + k * (XR * 256), row, lane, q), d[i], 0, 0, 0);
  }
}

// A workgroup takes 16 R rows of h of a use: R waves side by side, and S such groups that take the blocks of the reduction in turn.
// XR: rows of x that a pass has room for.
template <int XR, int TERMS, int R, int S, int NS>
struct UpShape {
  static constexpr int X_LOADS = XR * TERMS / 4, PER = (X_LOADS + R - 1) / R;  // 1 KB loads of x per block: of a group, of a wave
  static constexpr int BLOCK = R * 4096 + X_LOADS * 1024 + R * 256;            // gates' and ups' rows, x, scales
  static constexpr int STAGE = S * BLOCK, RING = NS * STAGE;
  static constexpr int N = XR <= 16 ? 1 : XR / 16, SUMS = R * S * 2 * N * 1024;
  static constexpr int LDS = RING > SUMS ? RING : SUMS, LOADS = 4 + PER + 1;
};

template <int XR, int TERMS, int H_TERMS, int R, int S, int NS, bool STREAM>
__global__ __launch_bounds__(R *S * 64) void moe_up_kernel(MoeArgs g) {
  typedef UpShape<XR, TERMS, R, S, NS> Shape;
  constexpr int N = Shape::N, PER = Shape::PER;
  extern __shared__ __attribute__((aligned(1024))) uint8_t up_lds[];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave / R, rt = wave % R;
  const uint32_t lds0 = lds_address(up_lds);
  const int i0 = (blockIdx.x * R + rt) * 16;
  int e, first, count, token = 0;  // token: lane l's is the l-th of the use
  float share;                     // lane l: of the l-th token
  if (XR == 4 && g.T == 1) {       // the picks are the uses, in their order
    int expert;
    picks_of_token(g, 0, lane & 15, expert, share);
    first = blockIdx.y, count = 1;
    e = __builtin_amdgcn_readlane(expert, first);
    share = __shfl(share, first);
    if (blockIdx.x == 0 && tid == 0) {
      g.uses[first] = Use{(uint16_t)e, (uint16_t)first, 1, 0};
      g.pair_tokens[first] = 0;
      if (first == 0) *g.n_uses = g.top;
    }
  } else if (XR == 4 && R == 1 && g.plans) {
    __shared__ struct {
      Picks<XR> p;
      Use mine;
      float share[XR * kMostPicks];
      uint8_t token[XR * kMostPicks];
    } own;
    const bool tells = blockIdx.x == 0 && blockIdx.y == 0;
    plan_uses<R * S>(
        g, own.p,
        [&](int uses) {
          if (tells) *g.n_uses = uses;
        },
        [&](int u, Use use) {
          if (u != (int)blockIdx.y) return;
          own.mine = use;
          if (blockIdx.x == 0) g.uses[u] = use;
        },
        [&](int pair, int t, float share) {
          own.token[pair] = (uint8_t)t;
          own.share[pair] = share;
          if (tells) g.pair_tokens[pair] = (uint8_t)t;
        });
    __syncthreads();
    e = __builtin_amdgcn_readfirstlane(own.mine.expert), first = __builtin_amdgcn_readfirstlane(own.mine.first),
    count = __builtin_amdgcn_readfirstlane(own.mine.count);
    if (count == 0) return;
    const int pair = first + min(lane, count - 1);
    token = own.token[pair];
    share = own.share[pair];
  } else {
    const Use use = g.uses[blockIdx.y];
    e = use.expert, first = use.first, count = use.count;
    if (count == 0) return;
    const int pair = first + min(lane, count - 1);
    token = g.pair_tokens[pair];
    share = g.shares[pair];
  }
  // ---- this wave's loads: 16 gates, 16 ups, its part of x, scales
  const int blocks = (g.H + kBlock - 1) / kBlock, steps = (blocks + S - 1) / S, tail = g.H & (kBlock - 1);
  const int i_row = min(i0, g.I - 1), last_row = g.I - 1 - i_row;
  const uint8_t *const gates = g.W13 + e * g.w13_stride + i_row * g.ldw13;
  const u32x4 gate_desc = descriptor(gates), up_desc = descriptor(gates + g.I * g.ldw13), x_desc = descriptor(g.x_terms),
              s_desc = descriptor(g.S13 + e * g.s13_stride);
  uint32_t w_at[2], x_at[PER];
  int chunk[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int row = 8 * p + (lane >> 3);
    chunk[p] = e4m3_chunk(lane, row) * 16;
    w_at[p] = (uint32_t)(min(row, last_row) * g.ldw13) + chunk[p];
  }
  auto x_load = [&](int j) { return min(rt * PER + j, Shape::X_LOADS - 1); };  // (the last one again, where there are none left)
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int row = x_load(j) / TERMS * 4 + (lane >> 4), t = __shfl(token, row & 63);
    x_at[j] = row < count ? (uint32_t)(t * g.x_row + x_load(j) % TERMS * 256 + term_chunk(lane, row) * 16) : kBeyond;
  }
  // the up rows of a tile lie in two blocks of scales where I is not a multiple of 16
  const int up_first = g.I + i_row, up_last = g.I + min(i_row + 15, g.I - 1), edge = up_last / kBlock * kBlock - up_first;
  const int s_line = (lane & 3) == 0 ? i_row / kBlock : (lane & 3) == 1 ? up_first / kBlock : up_last / kBlock;
  const uint32_t s_at = (uint32_t)(s_line * g.lds13) * 4u;
  auto fetch = [&](int s) {
    const int b = s * S + kg;
    const uint32_t to = lds0 + (uint32_t)(s % NS) * Shape::STAGE + kg * Shape::BLOCK;
    const int most = b >= blocks ? 0 : tail && b == blocks - 1 ? tail : kBlock;  // columns of the block
    const uint32_t at = most ? (uint32_t)b : 0u;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const uint32_t off = chunk[p] >= most ? kBeyond : w_at[p];
      fetch_16<STREAM>(to + rt * 4096 + p * 1024, off, gate_desc, at * kBlock);
      fetch_16<STREAM>(to + rt * 4096 + 2048 + p * 1024, off, up_desc, at * kBlock);
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
      fetch_16(to + R * 4096 + (x_load(j) % TERMS * XR + x_load(j) / TERMS * 4) * 256, most ? x_at[j] : kBeyond, x_desc, at * (TERMS * 256));
    fetch_4(to + R * 4096 + Shape::X_LOADS * 1024 + rt * 256, most ? s_at : kBeyond, s_desc, at * 4);
  };
  f32x4 gate[N], up[N];
#pragma unroll
  for (int i = 0; i < N; ++i) gate[i] = up[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t off = e4m3_operand_offset(lane);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) fetch(s);
  for (int s = 0; s < steps; ++s) {
    // this stage has landed, and every wave that shares x has read the one before, whose slot is filled next
    if constexpr (R > 1)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * Shape::LOADS) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * Shape::LOADS) : "memory");
    fetch(s + NS - 1);
    const int b = s * S + kg;
    if (b >= blocks) continue;  // (uniform in a group; the last step)
    uint8_t *const slot = up_lds + (uint32_t)(s % NS) * Shape::STAGE + kg * Shape::BLOCK;
    uint8_t *const w = slot + rt * 4096;
    if ((tail & 15) && b == blocks - 1) {  // what the last chunk of a row holds behind column H
      if (lane < 32) {
        u32x4 *const p = reinterpret_cast<u32x4 *>(w + lane * 128 + ((tail >> 4) ^ ((r >> 1) & 7)) * 16);
        *p = first_bytes(*p, tail & 15);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    const float *const sc = reinterpret_cast<const float *>(slot + R * 4096 + Shape::X_LOADS * 1024 + rt * 256);
    const float sg = sc[0], su0 = sc[1], su1 = sc[2];
    const uint8_t *const x = slot + R * 4096;
    const E4m3Operand wg = read_operand(w, off), wu = read_operand(w + 2048, off);
    f32x4 dg[N], du[N];
    if (N == 1 || count > 16) {
      block_products<N, XR, TERMS>(wg, x, lane, dg);
      block_products<N, XR, TERMS>(wu, x, lane, du);
    } else {
      f32x4 one[1];
      block_products<1, XR, TERMS>(wg, x, lane, one), dg[0] = one[0];
      block_products<1, XR, TERMS>(wu, x, lane, one), du[0] = one[0];
#pragma unroll
      for (int i = 1; i < N; ++i) dg[i] = du[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gate[i][j] += sg * dg[i][j];
        up[i][j] += (4 * (lane >> 4) + j < edge ? su0 : su1) * du[i][j];
      }
  }
  // ---- the groups' sums meet in LDS, in the order of the groups
  if constexpr (S > 1) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (no load may land in what follows)
    f32x4 *const sums = reinterpret_cast<f32x4 *>(up_lds);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      sums[(wave * 2 * N + 2 * i) * 64 + lane] = gate[i];
      sums[(wave * 2 * N + 2 * i + 1) * 64 + lane] = up[i];
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int k = 1; k < S; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        gate[i] += sums[((k * R + rt) * 2 * N + 2 * i) * 64 + lane];
        up[i] += sums[((k * R + rt) * 2 * N + 2 * i + 1) * 64 + lane];
      }
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nor behind the end)
  }
  if (i0 >= (g.I + kBlock - 1) / kBlock * kBlock) return;
  const int at = i0 + 4 * (lane >> 4);  // this lane's four columns of h; columns from I on fill up the last block
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int col = 16 * i + r;
    const float f = __shfl(share, col & 63);
    if (col >= count) continue;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = at + k < g.I ? silu(gate[i][k]) * up[i][k] * f : 0.f;
    uint16_t *const h = g.h_terms + (int64_t)(first + col) * (g.h_row / 2) + at / kBlock * (H_TERMS * kBlock) + term_place(at % kBlock);
#pragma unroll
    for (int k = 0; k < H_TERMS; ++k) {
      *reinterpret_cast<u32x2 *>(h + k * kBlock) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = rest_of_bf16(v[n]);
    }
  }
}

// A workgroup takes 128 columns of Y (rows of W2) for all tokens, eight waves side by side, and one of `splits` parts of the
// reduction, which runs over the blocks of all uses.  When it leaves a use, its sums go to those of the use's tokens, in LDS.
constexpr int kDownWaves = 8;
template <int XR, int H_TERMS, int NS>
struct DownShape {
  static constexpr int X_LOADS = XR * H_TERMS / 4, PER = (X_LOADS + kDownWaves - 1) / kDownWaves;
  static constexpr int STAGE = kDownWaves * 2048 + X_LOADS * 1024 + kDownWaves * 256, RING = NS * STAGE;
  static constexpr int N = XR <= 16 ? 1 : XR / 16, LOADS = 2 + PER + 1;
};

template <class T, int XR, int H_TERMS, int NS, bool STREAM>
__global__ __launch_bounds__(kDownWaves * 64) void moe_down_kernel(MoeArgs g, typename T::Elem *__restrict__ Y, int64_t ldy) {
  typedef DownShape<XR, H_TERMS, NS> Shape;
  constexpr int N = Shape::N, PER = Shape::PER;
  extern __shared__ __attribute__((aligned(1024))) uint8_t down_lds[];
  __shared__ Use uses[XORENC_MOE_MAX_EXPERTS + kMostTokens * kMostPicks / 16];
  __shared__ uint8_t pair_tokens[kMostTokens * kMostPicks];
  float *const sums = reinterpret_cast<float *>(down_lds + Shape::RING);  // [token][128 rows]
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = lds_address(down_lds);
  const int n_uses = *g.n_uses, n0 = blockIdx.x * 128;
  for (int i = tid; i < g.most_uses; i += kDownWaves * 64) uses[i] = g.uses[i];  // (all of them: not a load behind a load)
  for (int i = tid; i < g.T * g.top; i += kDownWaves * 64) pair_tokens[i] = g.pair_tokens[i];
  for (int i = tid; i < g.T * 128; i += kDownWaves * 64) sums[i] = 0.f;
  const int blocks = (g.I + kBlock - 1) / kBlock, steps = n_uses * blocks, tail = g.I & (kBlock - 1);
  const int s0 = (int)((int64_t)steps * blockIdx.y / g.splits), s1 = (int)((int64_t)steps * (blockIdx.y + 1) / g.splits);
  __syncthreads();
  // ---- this wave's loads: 16 rows of W2, its part of h, scales
  const int row0 = min(n0 + wave * 16, g.H - 1), last_row = g.H - 1 - row0;
  const u32x4 h_desc = descriptor(g.h_terms);
  uint32_t w_at[2];
  int chunk[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int row = 8 * p + (lane >> 3);
    chunk[p] = e4m3_chunk(lane, row) * 16;
    w_at[p] = (uint32_t)(min(row, last_row) * g.ldw2) + chunk[p];
  }
  auto x_load = [&](int j) { return min(wave * PER + j, Shape::X_LOADS - 1); };
  // the use and block of the step to be fetched next
  int fu = s0 / blocks, fb = s0 - fu * blocks;
  u32x4 w_desc = h_desc, s_desc = h_desc;
  uint32_t x_at[PER];
  auto enter = [&]() {
    const int e = __builtin_amdgcn_readfirstlane(uses[fu].expert), first = __builtin_amdgcn_readfirstlane(uses[fu].first),
              count = __builtin_amdgcn_readfirstlane(uses[fu].count);
    w_desc = descriptor(g.W2 + e * g.w2_stride + row0 * g.ldw2);
    s_desc = descriptor(g.S2 + e * g.s2_stride + (int64_t)(row0 / kBlock) * g.lds2);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int row = x_load(j) / H_TERMS * 4 + (lane >> 4);
      x_at[j] = row < count ? (uint32_t)((first + row) * g.h_row + x_load(j) % H_TERMS * 256 + term_chunk(lane, row) * 16) : kBeyond;
    }
  };
  auto fetch = [&](int s) {  // (steps past the last read as zero: every wave has as many loads on their way)
    const uint32_t to = lds0 + (uint32_t)((s - s0) % NS) * Shape::STAGE;
    const int most = s >= s1 ? 0 : tail && fb == blocks - 1 ? tail : kBlock;
    const uint32_t at = most ? (uint32_t)fb : 0u;
#pragma unroll
    for (int p = 0; p < 2; ++p) fetch_16<STREAM>(to + wave * 2048 + p * 1024, chunk[p] >= most ? kBeyond : w_at[p], w_desc, at * kBlock);
#pragma unroll
    for (int j = 0; j < PER; ++j)
      fetch_16(to + kDownWaves * 2048 + (x_load(j) % H_TERMS * XR + x_load(j) / H_TERMS * 4) * 256, most ? x_at[j] : kBeyond, h_desc,
               at * (H_TERMS * 256));
    fetch_4(to + kDownWaves * 2048 + Shape::X_LOADS * 1024 + wave * 256, most ? 0u : kBeyond, s_desc, at * 4);
    if (most && ++fb == blocks) {
      fb = 0;
      if (++fu < n_uses) enter();
    }
  };
  f32x4 acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t off = e4m3_operand_offset(lane);
  int u = fu, b = fb;
  if (s0 < s1) enter();
#pragma unroll
  for (int k = 0; k < NS - 1; ++k) fetch(s0 + k);
  for (int s = s0; s < s1; ++s) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * Shape::LOADS) : "memory");
    fetch(s + NS - 1);
    uint8_t *const slot = down_lds + (uint32_t)((s - s0) % NS) * Shape::STAGE, *const w = slot + wave * 2048;
    if ((tail & 15) && b == blocks - 1) {
      if (lane < 16) {
        u32x4 *const p = reinterpret_cast<u32x4 *>(w + lane * 128 + ((tail >> 4) ^ ((r >> 1) & 7)) * 16);
        *p = first_bytes(*p, tail & 15);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    const int first = __builtin_amdgcn_readfirstlane(uses[u].first), count = __builtin_amdgcn_readfirstlane(uses[u].count);
    const float sc = *reinterpret_cast<const float *>(slot + kDownWaves * 2048 + Shape::X_LOADS * 1024 + wave * 256);
    const E4m3Operand v = read_operand(w, off);
    f32x4 d[N];
    if (N == 1 || count > 16) {
      block_products<N, XR, H_TERMS>(v, slot + kDownWaves * 2048, lane, d);
    } else {
      f32x4 one[1];
      block_products<1, XR, H_TERMS>(v, slot + kDownWaves * 2048, lane, one), d[0] = one[0];
#pragma unroll
      for (int i = 1; i < N; ++i) d[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] += sc * d[i][j];
    if (++b == blocks || s + 1 == s1) {  // the use's sums to its tokens (a token is once in a use, a row of Y in one wave)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int col = 16 * i + r;
        if (col < count) *reinterpret_cast<f32x4 *>(sums + pair_tokens[first + col] * 128 + wave * 16 + 4 * (lane >> 4)) += acc[i];
        acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      b = 0;
      ++u;
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  const int n = n0 + (tid & 127);
  if (g.splits == 1) {
    for (int t = tid >> 7; t < g.T; t += kDownWaves / 2)
      if (n < g.H) T::store(Y + t * ldy + n, sums[t * 128 + (tid & 127)]);
    return;
  }
  const int64_t row = (int64_t)g.row_groups * 128, part = g.T * row;
  for (int i = tid; i < g.T * 32; i += kDownWaves * 64)
    *reinterpret_cast<f32x4 *>(g.parts + blockIdx.y * part + (i >> 5) * row + n0 + (i & 31) * 4) = *reinterpret_cast<const f32x4 *>(sums + i * 4);
}

// Adds the parts, in their order: four columns a thread, eight tokens a workgroup.  (The last workgroup of the parts, which a ticket
// tells that it is the last, takes as long for one token, 36 us with this launch and 37 without for eight of 16 experts of 1024 x 4096,
// and longer for more: 64 tokens, two of 16 of 512 x 512 31.6 and 52.9.)
template <class T>
__global__ __launch_bounds__(256) void moe_join_kernel(MoeArgs g, typename T::Elem *__restrict__ Y, int64_t ldy) {
  const int t = blockIdx.y * 8 + (threadIdx.x >> 5), n = blockIdx.x * 128 + (threadIdx.x & 31) * 4;
  if (t >= g.T) return;
  const int64_t row = (int64_t)g.row_groups * 128, part = g.T * row;
  const float *const p = g.parts + t * row + n;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  int k = 0;
  for (; k + 8 <= g.splits; k += 8) {
    f32x4 q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = *reinterpret_cast<const f32x4 *>(p + (k + j) * part);
#pragma unroll
    for (int j = 0; j < 8; ++j) v += q[j];
  }
  for (; k < g.splits; ++k) v += *reinterpret_cast<const f32x4 *>(p + k * part);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (n + j < g.H) T::store(Y + t * ldy + n + j, v[j]);
}

// The same for at most XR <= 4 tokens and rows enough: a workgroup takes 16 rows of W2, and its eight waves take the blocks of
// all uses in turn, each with a ring of its own, so that no sums cross workgroups.
template <int XR, int H_TERMS, int NS>
struct FewShape {
  static constexpr int X_LOADS = (XR * H_TERMS + 3) / 4, STAGE = 2048 + X_LOADS * 1024 + 256, RING = kDownWaves * NS * STAGE;
  static constexpr int LOADS = 2 + X_LOADS + 1;
};

template <class T, int XR, int H_TERMS, int NS, bool STREAM>
__global__ __launch_bounds__(kDownWaves * 64) void moe_down_few_kernel(MoeArgs g, typename T::Elem *__restrict__ Y, int64_t ldy) {
  typedef FewShape<XR, H_TERMS, NS> Shape;
  constexpr int X_LOADS = Shape::X_LOADS;
  extern __shared__ __attribute__((aligned(1024))) uint8_t few_lds[];
  __shared__ Use uses[4 * kMostPicks];
  __shared__ uint8_t pair_tokens[4 * kMostPicks];
  __shared__ __attribute__((aligned(16))) float sums[kDownWaves][XR][16];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = lds_address(few_lds) + (uint32_t)wave * (NS * Shape::STAGE);
  const int n_uses = *g.n_uses, n0 = blockIdx.x * 16;
  if (tid < g.most_uses) uses[tid] = g.uses[tid];
  if (tid < g.T * g.top) pair_tokens[tid] = g.pair_tokens[tid];
  for (int i = lane; i < XR * 16; i += 64) sums[wave][i / 16][i % 16] = 0.f;
  const int blocks = (g.I + kBlock - 1) / kBlock, steps = n_uses * blocks, tail = g.I & (kBlock - 1);
  __syncthreads();
  const u32x4 h_desc = descriptor(g.h_terms);
  uint32_t w_at[2];
  int chunk[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int row = 8 * p + (lane >> 3);
    chunk[p] = e4m3_chunk(lane, row) * 16;
    w_at[p] = (uint32_t)(min(row, g.H - 1 - n0) * g.ldw2) + chunk[p];
  }
  // the use and block of this wave's step to be fetched next
  int fs = wave, fu = wave / blocks, fb = wave - fu * blocks, slot_of = 0;
  auto fetch = [&]() {  // (steps past the last read as zero: every wave has as many loads on their way)
    const uint32_t to = lds0 + (uint32_t)slot_of * Shape::STAGE;
    if (++slot_of == NS) slot_of = 0;
    const int u = min(fu, n_uses - 1);
    const int e = __builtin_amdgcn_readfirstlane(uses[u].expert), first = __builtin_amdgcn_readfirstlane(uses[u].first),
              count = __builtin_amdgcn_readfirstlane(uses[u].count);
    const u32x4 w_desc = descriptor(g.W2 + e * g.w2_stride + n0 * g.ldw2),
                s_desc = descriptor(g.S2 + e * g.s2_stride + (int64_t)(n0 / kBlock) * g.lds2);
    const int most = fs >= steps ? 0 : tail && fb == blocks - 1 ? tail : kBlock;
    const uint32_t at = most ? (uint32_t)fb : 0u;
#pragma unroll
    for (int p = 0; p < 2; ++p) fetch_16<STREAM>(to + p * 1024, chunk[p] >= most ? kBeyond : w_at[p], w_desc, at * kBlock);
#pragma unroll
    for (int j = 0; j < X_LOADS; ++j) {
      const int line = 4 * j + (lane >> 4), row = line % XR, k = line / XR;
      fetch_16(to + 2048 + j * 1024,
               most && row < count && k < H_TERMS ? (uint32_t)((first + row) * g.h_row + k * 256 + term_chunk(lane, row) * 16) : kBeyond, h_desc,
               at * (H_TERMS * 256));
    }
    fetch_4(to + 2048 + X_LOADS * 1024, most ? 0u : kBeyond, s_desc, at * 4);
    fs += kDownWaves;
    for (fb += kDownWaves; fb >= blocks; fb -= blocks) ++fu;
  };
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t off = e4m3_operand_offset(lane);
  int u = fu, b = fb, slot = 0;
#pragma unroll
  for (int k = 0; k < NS - 1; ++k) fetch();
  for (int s = wave; s < steps; s += kDownWaves) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * Shape::LOADS) : "memory");
    fetch();
    uint8_t *const w = few_lds + (wave * NS + slot) * Shape::STAGE;
    if (++slot == NS) slot = 0;
    if ((tail & 15) && b == blocks - 1) {
      if (lane < 16) {
        u32x4 *const p = reinterpret_cast<u32x4 *>(w + lane * 128 + ((tail >> 4) ^ ((r >> 1) & 7)) * 16);
        *p = first_bytes(*p, tail & 15);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    const int first = __builtin_amdgcn_readfirstlane(uses[u].first), count = __builtin_amdgcn_readfirstlane(uses[u].count);
    const float sc = *reinterpret_cast<const float *>(w + 2048 + X_LOADS * 1024);
    f32x4 d[1];
    block_products<1, XR, H_TERMS>(read_operand(w, off), w + 2048, lane, d);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += sc * d[0][j];
    const int before = u;
    for (b += kDownWaves; b >= blocks; b -= blocks) ++u;
    if (u != before || s + kDownWaves >= steps) {  // the use's sums to its tokens (a token is once in a use)
      if (r < count) *reinterpret_cast<f32x4 *>(&sums[wave][pair_tokens[first + r]][4 * (lane >> 4)]) += acc;
      acc = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (tid < g.T * 16 && n0 + r < g.H) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kDownWaves; ++k) v += sums[k][tid >> 4][r];
    T::store(Y + (tid >> 4) * ldy + n0 + r, v);
  }
}

// ---------------------------------------------------------------------------------------------- host

constexpr int64_t round_up(int64_t n, int64_t d) { return (n + d - 1) / d * d; }

struct MoePlan {
  int64_t logits, n_uses, uses, pair_tokens, shares, parts, x, h, total;  // bytes: where they start, and in all
  int x_row, h_row, most_uses, pass, splits, row_groups;
};

constexpr int pass_of(bool f32) { return f32 ? 16 : 32; }

MoePlan plan_of(int T, int H, int I, int E, int top, int32_t dtype) {
  MoePlan p;
  const bool f32 = dtype == XORENC_X_F32;
  const int terms = f32 ? 3 : 1, h_terms = f32 ? 3 : 2, pairs = T * top, used = E < pairs ? E : pairs;
  p.pass = pass_of(f32);
  p.most_uses = used + pairs / p.pass < pairs ? used + pairs / p.pass : pairs;
  p.x_row = (H + kBlock - 1) / kBlock * terms * (2 * kBlock);
  p.h_row = (I + kBlock - 1) / kBlock * h_terms * (2 * kBlock);
  p.row_groups = (H + 127) / 128;
  // workgroups of the second product: one for each CU (two: 190 against 184 us for 32 tokens and eight experts of 4096 x 9216, 152
  // against 147 for eight tokens and 16 of 4096 x 4096), a block of the reduction each at least, 32 parts at most (64: 29 against 26
  // for 64 tokens and 16 of 512 x 512)
  const int64_t steps = (int64_t)used * ((I + kBlock - 1) / kBlock);
  p.splits = (256 + p.row_groups - 1) / p.row_groups;
  if (p.splits > steps) p.splits = (int)steps;
  if (p.splits > 32) p.splits = 32;
  p.logits = 0;
  p.n_uses = round_up((int64_t)T * E * 4, 16);
  p.uses = p.n_uses + 16;
  p.pair_tokens = p.uses + p.most_uses * (int64_t)sizeof(Use);
  p.shares = round_up(p.pair_tokens + pairs, 16);
  p.parts = round_up(p.shares + pairs * 4, 256);
  p.x = p.parts + (p.splits > 1 ? (int64_t)p.splits * T * p.row_groups * 512 : 0);
  p.h = p.x + (int64_t)T * p.x_row;
  p.total = p.h + (int64_t)pairs * p.h_row;
  return p;
}

template <bool STREAM, int XR, int TERMS, int H_TERMS, int R, int S>
void launch_up(const MoeArgs &g, hipStream_t st) {
  constexpr int NS = R > 1 && UpShape<XR, TERMS, R, S, 3>::RING <= 80 * 1024 ? 3 : 2;  // (two workgroups a CU, three with R = 1)
  typedef UpShape<XR, TERMS, R, S, NS> Shape;
  static_assert(Shape::LDS <= 160 * 1024, "a CU's");
  const int tiles = (g.I + kBlock - 1) / kBlock * (kBlock / 16);
  hipLaunchKernelGGL((moe_up_kernel<XR, TERMS, H_TERMS, R, S, NS, STREAM>), dim3((unsigned)((tiles + R - 1) / R), (unsigned)g.most_uses), dim3(R * S * 64),
                     Shape::LDS, st, g);
}

template <bool STREAM, class T, int XR, int H_TERMS>
void launch_down_few(const MoeArgs &g, void *Y, int64_t ldy, hipStream_t st) {
  constexpr int NS = FewShape<XR, H_TERMS, 4>::RING <= 150 * 1024 ? 4 : 3;
  static_assert(FewShape<XR, H_TERMS, NS>::RING <= 150 * 1024, "a CU's, less what is declared in the kernel");
  hipLaunchKernelGGL((moe_down_few_kernel<T, XR, H_TERMS, NS, STREAM>), dim3((unsigned)((g.H + 15) / 16)), dim3(kDownWaves * 64),
                     (FewShape<XR, H_TERMS, NS>::RING), st, g, static_cast<typename T::Elem *>(Y), ldy);
}

template <bool STREAM, class T, int XR, int TERMS, int H_TERMS>
void launch_products(const MoeArgs &g, void *Y, int64_t ldy, hipStream_t st) {
  // Four waves: side by side where x is wide and they share it, in pairs otherwise, and all on the same 16 rows where there
  // are few of them (us, in this order: 32 tokens, two of eight experts of 4096 x 9216 184, 189, 246; 16 tokens 177, 163,
  // 175; eight tokens, four of 16 experts of 4096 x 4096 156, 147, 159; one token, six of 64 of 2048 x 1024 24, 21, 20)
  const int64_t tiles = (int64_t)((g.I + 15) / 16) * g.most_uses;
  if (tiles < 2048)
    launch_up<STREAM, XR, TERMS, H_TERMS, 1, 4>(g, st);
  else
    launch_up<STREAM, XR, TERMS, H_TERMS, (XR == 32 ? 4 : 2), (XR == 32 ? 1 : 2)>(g, st);
  if constexpr (XR == 4) {
    // No sums across workgroups where each has few steps (us, against the other kernels: one token, six of 64 experts of 2048 x
    // 1024 20.5 and 21.3, two of 16 of 512 x 512 12.1 and 13.9, four of 16 of 2048 x 4096 33.8 and 32.0; four tokens, two of
    // 16 of 512 x 512 15.9 and 17.0, eight of 32 of 1024 x 256 21.5 and 20.2)
    const int64_t steps = (int64_t)(g.E < g.T * g.top ? g.E : g.T * g.top) * ((g.I + kBlock - 1) / kBlock);
    if (g.T == 1 && steps <= 96) return launch_down_few<STREAM, T, 1, H_TERMS>(g, Y, ldy, st);
    if (g.T > 1 && steps <= 48) return launch_down_few<STREAM, T, 4, H_TERMS>(g, Y, ldy, st);
  }
  constexpr int NS = 3;
  typedef DownShape<XR, H_TERMS, NS> Shape;
  static_assert(Shape::RING + kMostTokens * 512 <= 150 * 1024, "a CU's, less what is declared in the kernel");
  hipLaunchKernelGGL((moe_down_kernel<T, XR, H_TERMS, NS, STREAM>), dim3((unsigned)g.row_groups, (unsigned)g.splits), dim3(kDownWaves * 64),
                     (unsigned)(Shape::RING + g.T * 512), st, g, static_cast<typename T::Elem *>(Y), ldy);
  if (g.splits > 1)
    hipLaunchKernelGGL((moe_join_kernel<T>), dim3((unsigned)g.row_groups, (unsigned)((g.T + 7) / 8)), dim3(256), 0, st, g,
                       static_cast<typename T::Elem *>(Y), ldy);
}

template <class T, int TERMS, int H_TERMS>
int32_t launch_moe(const MoeArgs &g, const void *X, int64_t ldx, const void *router, int64_t ldr, void *Y, int64_t ldy, hipStream_t st) {
  typedef typename T::Elem E;
  const int groups = g.E * ((g.T + 3) / 4);
  const int64_t pieces = (int64_t)g.T * ((g.H + kBlock - 1) / kBlock) * 16;
  hipLaunchKernelGGL((router_kernel<T, TERMS>), dim3((unsigned)(groups + (pieces + 255) / 256)), dim3(256), 0, st,
                     static_cast<const E *>(X), ldx, static_cast<const E *>(router), ldr, g.T, g.H, g.E, g.logits,
                     g.x_terms, groups);
  if (!g.plans) hipLaunchKernelGGL(picks_kernel, dim3(1), dim3(1024), 0, st, g);
  int32_t rc = xorenc_internal_check_launch();
  if (rc != XORENC_OK) return rc;
  constexpr int MOST = pass_of(TERMS > 1);
  // From 96 MB of weights on they are read past the caches, which would not hold them until the next call (us: 8 tokens, four of
  // 16 experts of 4096 x 4096 148 and 161, one token 56 and 60, 32 tokens, two of eight of 4096 x 9216 188 and 201, eight tokens, four of
  // 64 of 1024 x 1024 34.9 and 36.3; one token, six of 64 of 2048 x 1024, 38 MB, 21.7 and 21.0)
  const int64_t used = g.E < g.T * g.top ? g.E : g.T * g.top;
  auto products = [&](auto stream) {
    constexpr bool STREAM = decltype(stream)::value;
    if (g.T <= 4)
      launch_products<STREAM, T, 4, TERMS, H_TERMS>(g, Y, ldy, st);
    else if (g.T <= 16)
      launch_products<STREAM, T, 16, TERMS, H_TERMS>(g, Y, ldy, st);
    else
      launch_products<STREAM, T, MOST, TERMS, H_TERMS>(g, Y, ldy, st);
  };
  if (used * g.H * g.I * 3 >= (int64_t)96 << 20)
    products(std::true_type());
  else
    products(std::false_type());
  return xorenc_internal_check_launch();
}

int32_t check_sizes(int32_t T, int32_t H, int32_t I, int32_t E, int32_t top, int32_t dtype) {
  if (T < 0 || H <= 0 || I <= 0 || E <= 0 || top <= 0 || top > E) return XORENC_EINVAL;
  if (!known_dtype(dtype)) return XORENC_EUNSUPPORTED;
  if (T > kMostTokens || E > kMostExperts || top > kMostPicks || H > (1 << 17) || I > (1 << 17)) return XORENC_ELIMIT;
  return XORENC_OK;
}

}  // namespace
}  // namespace xorenc_fp8_detail

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_moe_workspace(int32_t tokens, int32_t hidden, int32_t inner, int32_t experts, int32_t picks,
                                        int32_t x_dtype, int64_t *bytes) {
  if (!bytes) return XORENC_EINVAL;
  const int32_t rc = check_sizes(tokens, hidden, inner, experts, picks, x_dtype);
  if (rc == XORENC_OK) *bytes = plan_of(tokens, hidden, inner, experts, picks, x_dtype).total;
  return rc;
}

extern "C" int32_t xorenc_moe_fp8(const xorenc_moe *L, const void *X, int32_t x_dtype, int64_t ldx, int32_t tokens, int32_t picks,
                                  int32_t renormalise, void *Y, int64_t ldy, void *workspace, int64_t workspace_bytes,
                                  void *hip_stream) {
  if (!L || L->struct_size != sizeof(xorenc_moe)) return XORENC_EINVAL;
  const int32_t rc = check_sizes(tokens, L->hidden, L->inner, L->experts, picks, x_dtype);
  if (rc != XORENC_OK) return rc;
  const int H = L->hidden, I = L->inner, E = L->experts;
  const int64_t h_blocks = ((int64_t)H + kBlock - 1) / kBlock, i_blocks = ((int64_t)I + kBlock - 1) / kBlock;
  if (ldx < H || ldy < H || L->ld_router < H || L->ld_w13 < H || L->ld_w2 < I || L->ld_s13 < h_blocks || L->ld_s2 < i_blocks ||
      L->w13_stride < 0 || L->s13_stride < 0 || L->w2_stride < 0 || L->s2_stride < 0)
    return XORENC_EINVAL;
  if (tokens == 0) return XORENC_OK;
  if (!X || !Y || !L->router || !L->W13 || !L->S13 || !L->W2 || !L->S2 || !workspace) return XORENC_EINVAL;
  const MoePlan p = plan_of(tokens, H, I, E, picks, x_dtype);
  if (workspace_bytes < p.total) return XORENC_EINVAL;
  if (L->ld_w13 > (1 << 24) || L->ld_w2 > (1 << 24) || L->ld_s13 > (1 << 16) || L->ld_s2 > (1 << 16)) return XORENC_ELIMIT;
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(X, esz) || !aligned_to(Y, esz) || !aligned_to(L->router, esz) || !aligned_to(L->W13, 16) || L->ld_w13 % 16 ||
      L->w13_stride % 16 || !aligned_to(L->W2, 16) || L->ld_w2 % 16 || L->w2_stride % 16 || !aligned_to(L->S13, 4) ||
      !aligned_to(L->S2, 4) || !aligned_to(workspace, 16))
    return XORENC_EALIGN;
  unsigned char *const ws = static_cast<unsigned char *>(workspace);
  MoeArgs g;
  g.W13 = L->W13, g.W2 = L->W2, g.S13 = L->S13, g.S2 = L->S2;
  g.ldw13 = L->ld_w13, g.w13_stride = L->w13_stride, g.lds13 = L->ld_s13, g.s13_stride = L->s13_stride;
  g.ldw2 = L->ld_w2, g.w2_stride = L->w2_stride, g.lds2 = L->ld_s2, g.s2_stride = L->s2_stride;
  g.T = tokens, g.H = H, g.I = I, g.E = E, g.top = picks, g.renormalise = renormalise != 0;
  g.logits = reinterpret_cast<float *>(ws + p.logits);
  g.n_uses = reinterpret_cast<int *>(ws + p.n_uses);
  g.uses = reinterpret_cast<Use *>(ws + p.uses);
  g.pair_tokens = ws + p.pair_tokens;
  g.shares = reinterpret_cast<float *>(ws + p.shares);
  g.parts = reinterpret_cast<float *>(ws + p.parts);
  g.x_terms = reinterpret_cast<uint16_t *>(ws + p.x);
  g.h_terms = reinterpret_cast<uint16_t *>(ws + p.h);
  g.x_row = p.x_row, g.h_row = p.h_row, g.most_uses = p.most_uses, g.pass = p.pass, g.splits = p.splits, g.row_groups = p.row_groups;
  // Up to four tokens, up to 1024 workgroups: a launch less for a longer start of each (us: two tokens, four of 16 experts of 1024 x
  // 1024 22.2 and 23.4; four tokens, six of 64 of 2048 x 1024, 1536 workgroups, 45.0 and 43.9)
  g.plans = tokens == 1 || (tokens <= 4 && (int64_t)((I + 15) / 16) * p.most_uses <= 1024);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return x_dtype == XORENC_X_F32
             ? launch_moe<F32, 3, 3>(g, X, ldx, L->router, L->ld_router, Y, ldy, st)
             : launch_moe<BF16, 1, 2>(g, X, ldx, L->router, L->ld_router, Y, ldy, st);
}
