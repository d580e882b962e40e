// A mixture-of-experts layer for a few tokens: Y = sum over a token's picks of share * W2_e (silu(G_e x) * (U_e x)), with
// expert weights in e4m3 (a scale per 128 x 128 block) and everything else in 16 or 32 bits.
//
// Four launches: the router's logits; the picks (not for a single token, whose picks every workgroup finds by itself); the gated
// activations h of the picked experts; their second product and the sum over picks.  The bytes of the picked experts'
// weights bound the last two, so both stream 16 rows of weights per workgroup from memory to registers, its waves taking
// parts of the reduction.  e4m3 values become bf16 exactly and multiply bf16 terms of the activations (one for bf16
// activations, three for fp32, which sum to the value exactly), so that nothing is rounded to 8 bits on the way; h is kept
// as bf16 terms that hold 16 (24) bits.  The tokens that picked an expert are the columns of its matrix instructions, 16 at a
// time; lanes of columns without a token load nothing.
//
// Terms of x and h lie in the workspace in the order in which lanes load them: a row is a run of blocks of 128 columns (zero
// behind the last column), a block its terms one after the other, a term four quarters of 32 columns: those that the
// four lanes of a row take with one load, 64 contiguous bytes.
#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

constexpr int kMostExperts = XORENC_MOE_MAX_EXPERTS, kMostPicks = XORENC_MOE_MAX_PICKS, kMostTokens = XORENC_MOE_MAX_TOKENS;
static_assert(kMostExperts == 256 && kMostTokens == 64, "four experts per lane, four column tiles");

// An expert that some token picked: its tokens are `count` entries of the list of pairs of a token and an expert that it
// picked, from `first` on.  Pairs are ordered by expert, then by token; row i of h is pair i's.
struct Use {
  int expert, first, count, unused;
};

struct MoeArgs {
  const uint8_t *W13, *W2;
  const float *S13, *S2;
  int64_t ldw13, w13_stride, lds13, s13_stride, ldw2, w2_stride, lds2, s2_stride;
  int T, H, I, E, top, renormalise;
  float *logits;            // [T][E]
  Use *uses;                // experts in use, ascending; min(E, T * top) of them, the last ones with count 0
  int *n_used;              // how many
  uint8_t *use_tokens;      // [use][kMostTokens]
  float *shares;            // of the entries
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
__global__ __launch_bounds__(256) void router_kernel(const typename T::Elem *__restrict__ X, int64_t ldx, int wide,
                                                     const typename T::Elem *__restrict__ router, int64_t ldr, int r_wide, int tokens,
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
    load_piece<T>(X + t * ldx, c, H, wide, v);
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
    load_piece<T>(router + e * ldr, c, H, r_wide, r);
#pragma unroll
    for (int k = 0; k < 4; ++k) load_piece<T>(X + min(t0 + k, tokens - 1) * ldx, c, H, wide, v[k]);
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

// fp32 -> integers in the same order (NaN above infinity or below its negative, as the sign says)
__device__ inline uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// A token's picks, by one wave: lane j gets the j-th (`expert`, `share`).
__device__ inline void picks_of_token(const MoeArgs &g, int t, int lane, int &expert, float &share) {
  const float *const row = g.logits + t * g.E;
  uint32_t key[4];
  bool left[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = lane + 64 * i;
    left[i] = e < g.E;
    key[i] = left[i] ? ordered(row[e]) : 0u;
  }
  auto largest = [&]() {  // of the keys that are left, the same on all lanes
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = left[i] ? max(m, key[i]) : m;
    m = max_of_16_lanes(m);
    return max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
               max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
  };
  const float most = from_ordered(largest());
  float sum = 0.f;
  if (!g.renormalise) {  // shares of a softmax over all experts
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (left[i]) sum += expf(from_ordered(key[i]) - most);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  }
  expert = 0, share = 0.f;
  for (int j = 0; j < g.top; ++j) {  // the largest that is left; the lowest index of equals
    const uint32_t m = largest();
    int e = 0;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      const uint64_t at = __ballot(left[i] && key[i] == m);
      if (at) e = 64 * i + __builtin_ctzll(at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) left[i] = left[i] && e != lane + 64 * i;
    const float v = expf(from_ordered(m) - most);
    if (g.renormalise) sum += v;
    if (lane == j) expert = e, share = v;
  }
  share /= sum;
}

// One workgroup; a wave per token at a time.
__global__ __launch_bounds__(1024) void picks_kernel(MoeArgs g) {
  constexpr int WAVES = 16;
  __shared__ struct {
    uint64_t tokens[kMostExperts];  // that picked an expert, a bit each
    float share[kMostTokens][kMostPicks];
    uint16_t expert[kMostTokens][kMostPicks];
    uint16_t place[kMostExperts], first[kMostExperts];  // of an expert among those in use; its first pair
  } p;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid < kMostExperts) p.tokens[tid] = 0u;
  __syncthreads();
  for (int t = wave; t < g.T; t += WAVES) {
    int e;
    float share;
    picks_of_token(g, t, lane, e, share);
    if (lane < g.top) {
      p.expert[t][lane] = (uint16_t)e;
      p.share[t][lane] = share;
      atomicOr(reinterpret_cast<unsigned long long *>(&p.tokens[e]), 1ull << t);
    }
  }
  __syncthreads();
  if (wave == 0) {  // four experts a lane
    int n[4], sum = 0;  // experts in use << 16 | pairs
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = __popcll(p.tokens[4 * lane + i]);
      n[i] = k ? k | 0x10000 : 0;
      sum += n[i];
    }
    int before = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(before, o);
      if (lane >= o) before += v;
    }
    const int used = __shfl(before, 63) >> 16;
    before -= sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n[i]) {
        const int e = 4 * lane + i, at = before >> 16, first = before & 0xffff;
        p.place[e] = (uint16_t)at;
        p.first[e] = (uint16_t)first;
        g.uses[at] = Use{e, first, n[i] & 0xffff, 0};
      }
      before += n[i];
    }
    if (lane == 0) *g.n_used = used;
    for (int u = used + lane; u < min(g.E, g.T * g.top); u += 64) g.uses[u] = Use{0, 0, 0, 0};
  }
  __syncthreads();
  for (int i = tid; i < g.T * g.top; i += WAVES * 64) {
    const int t = i / g.top, j = i - t * g.top, e = p.expert[t][j];
    const int rank = __popcll(p.tokens[e] & ((1ull << t) - 1ull));
    g.use_tokens[p.place[e] * kMostTokens + rank] = (uint8_t)t;
    g.shares[p.first[e] + rank] = p.share[t][j];
  }
}

// ---------------------------------------------------------------------------------------------- products

typedef __amdgpu_buffer_rsrc_t Buffer;
constexpr int kNoColumn = (int)0x80000000u;  // an offset behind every buffer: reads as zero, from nowhere

// Terms of a lane's columns of a block, in quarters: the columns that quarter_as_bf16 gives of weights.
template <int TERMS>
struct TermOperand {
  u32x4 q[TERMS][4];
};
template <int TERMS>
__device__ inline void load_terms(Buffer rows, int at, int block, TermOperand<TERMS> &o) {
#pragma unroll
  for (int k = 0; k < TERMS; ++k)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      o.q[k][q] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at + k * 256 + q * 64, block * (TERMS * 256), 0));
}

// What a wave of the first product needs to know.
struct UpRows {
  const uint8_t *gate, *up;                // this lane's row of weights
  const float *s_gate, *s_up0, *s_up1;     // scales of the gates' rows, of the ups' rows before `edge` and from it on
  int edge;
};

template <int N, int TERMS>
struct UpOperands {
  E4m3Operand gate, up;
  TermOperand<TERMS> x[N];
  float sg, su0, su1;
};

// Blocks b0 .. b1 - 1 of the reduction for N tiles of 16 tokens.
template <int N, int MT, int TERMS>
__device__ inline void up_blocks(const UpRows &w, Buffer x, const int (&x_at)[MT], int H, int lane, int b0, int b1, f32x4 (&gate)[MT],
                                 f32x4 (&up)[MT]) {
  typedef UpOperands<N, TERMS> Operands;
  const int zero = vector_zero();
  auto multiply = [&](int, Operands &o) {
    bf16x8 vg[4], vu[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) vg[q] = quarter_as_bf16(o.gate, q), vu[q] = quarter_as_bf16(o.up, q);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f32x4 dg = {0.f, 0.f, 0.f, 0.f}, du = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < TERMS; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bf16x8 v = __builtin_bit_cast(bf16x8, o.x[i].q[k][q]);
          dg = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vg[q], v, dg, 0, 0, 0);
          du = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vu[q], v, du, 0, 0, 0);
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gate[i][j] += o.sg * dg[j];
        up[i][j] += (4 * (lane >> 4) + j < w.edge ? o.su0 : o.su1) * du[j];
      }
    }
  };
  auto load_others = [&](int b, Operands &o) {
#pragma unroll
    for (int i = 0; i < N; ++i) load_terms<TERMS>(x, x_at[i], b, o.x[i]);
    o.sg = w.s_gate[b + zero], o.su0 = w.s_up0[b + zero], o.su1 = w.s_up1[b + zero];
  };
  const int whole = H / kBlock;
  pipeline<0, Operands>(min(b1, whole) - b0, [&](int s, Operands &o) {
    load_block(w.gate + (b0 + s) * kBlock, lane, o.gate);
    load_block(w.up + (b0 + s) * kBlock, lane, o.up);
    load_others(b0 + s, o);
  }, multiply);
  if (b0 < b1 && b1 > whole) {  // the last block, a short one
    const int c = whole * kBlock;
    Operands o;
    load_last_block(w.gate + c, lane, H - c, o.gate);
    load_last_block(w.up + c, lane, H - c, o.up);
    load_others(whole, o);
    multiply(0, o);
  }
}

// h of 16 rows of an expert for all tokens that picked it.
template <int MT, int TERMS, int H_TERMS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void moe_up_kernel(MoeArgs g) {
  __shared__ f32x4 part[WAVES][2][MT][64];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i0 = blockIdx.x * 16;
  int e, first, count, token;
  float one_share = 0.f;
  if (MT == 1 && g.T == 1) {  // its picks are the experts in use, in their order
    int expert;
    picks_of_token(g, 0, lane, expert, one_share);
    first = blockIdx.y, count = 1, token = 0;
    e = __builtin_amdgcn_readlane(expert, first);
    one_share = __shfl(one_share, first);
    if (blockIdx.x == 0 && tid == 0) {
      g.uses[first] = Use{e, first, 1, 0};
      g.use_tokens[first * kMostTokens] = 0;
      if (first == 0) *g.n_used = g.top;
    }
  } else {
    const Use use = g.uses[blockIdx.y];
    token = g.use_tokens[blockIdx.y * kMostTokens + lane];
    e = use.expert, first = use.first, count = use.count;
    if (count == 0) return;
  }
  const int tiles = (count + 15) / 16;
  const int h_block = i0 / kBlock * (H_TERMS * kBlock) + term_place(i0 % kBlock + 4 * (lane >> 4));  // where this lane's four results go
  uint16_t *const h = g.h_terms + (int64_t)first * (g.h_row / 2) + h_block;
  if (i0 >= g.I) {  // columns that fill up the last block
    for (int col = 16 * wave + r; col < count; col += 16 * WAVES)
#pragma unroll
      for (int k = 0; k < H_TERMS; ++k) *reinterpret_cast<u32x2 *>(h + (int64_t)col * (g.h_row / 2) + k * kBlock) = u32x2{0u, 0u};
    return;
  }
  const uint8_t *const base = g.W13 + e * g.w13_stride;
  const float *const s_base = g.S13 + e * g.s13_stride;
  const int row = min(i0 + r, g.I - 1);
  // the up rows of a tile lie in two blocks of scales where I is not a multiple of 16
  const int up_first = g.I + i0, up_last = g.I + min(i0 + 15, g.I - 1);
  const UpRows w = {base + row * g.ldw13, base + ((int64_t)g.I + row) * g.ldw13, s_base + (int64_t)(i0 / kBlock) * g.lds13,
                    s_base + (int64_t)(up_first / kBlock) * g.lds13, s_base + (int64_t)(up_last / kBlock) * g.lds13,
                    (up_last / kBlock) * kBlock - up_first};
  const Buffer x = __builtin_amdgcn_make_buffer_rsrc(g.x_terms, 0, g.T * g.x_row, 0x00020000);
  int x_at[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int t = __shfl(token, (16 * i + r) & 63);
    x_at[i] = 16 * i + r < count ? t * g.x_row + (lane >> 4) * 16 : kNoColumn;
  }
  f32x4 gate[MT], up[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) gate[i] = up[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int blocks = (g.H + kBlock - 1) / kBlock, b0 = blocks * wave / WAVES, b1 = blocks * (wave + 1) / WAVES;
  if (tiles == 1)
    up_blocks<1, MT, TERMS>(w, x, x_at, g.H, lane, b0, b1, gate, up);
  else if (MT == 2 || tiles == 2)
    up_blocks<(MT < 2 ? 1 : 2), MT, TERMS>(w, x, x_at, g.H, lane, b0, b1, gate, up);
  else
    up_blocks<MT, MT, TERMS>(w, x, x_at, g.H, lane, b0, b1, gate, up);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    part[wave][0][i][lane] = gate[i];
    part[wave][1][i][lane] = up[i];
  }
  __syncthreads();
  for (int i = wave; i < tiles; i += WAVES) {
    f32x4 a = part[0][0][i][lane], c = part[0][1][i][lane];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) {
      a += part[k][0][i][lane];
      c += part[k][1][i][lane];
    }
    const int col = 16 * i + r;
    if (col >= count) continue;
    const float share = MT == 1 && g.T == 1 ? one_share : g.shares[first + col];
    const int at = i0 + 4 * (lane >> 4);
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = at + k < g.I ? silu(a[k]) * c[k] * share : 0.f;
#pragma unroll
    for (int k = 0; k < H_TERMS; ++k) {
      *reinterpret_cast<u32x2 *>(h + (int64_t)col * (g.h_row / 2) + k * kBlock) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = rest_of_bf16(v[n]);
    }
  }
}

template <int N, int H_TERMS>
struct DownOperands {
  E4m3Operand w;
  TermOperand<H_TERMS> h[N];
  float scale;
};

// Blocks b0 .. b1 - 1 of an expert's reduction for N tiles of 16 tokens, from the lane's rows of weights and of h.
template <int N, int MT, int H_TERMS>
__device__ inline void down_blocks(const uint8_t *w_row, const float *s_row, Buffer h, const int (&h_at)[MT], int I, int lane, int b0, int b1,
                                   f32x4 (&acc)[MT]) {
  typedef DownOperands<N, H_TERMS> Operands;
  const int zero = vector_zero();
  auto multiply = [&](int, Operands &o) {
    bf16x8 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = quarter_as_bf16(o.w, q);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < H_TERMS; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[q], __builtin_bit_cast(bf16x8, o.h[i].q[k][q]), d, 0, 0, 0);
#pragma unroll
      for (int n = 0; n < 4; ++n) acc[i][n] += o.scale * d[n];
    }
  };
  auto load_others = [&](int b, Operands &o) {
#pragma unroll
    for (int i = 0; i < N; ++i) load_terms<H_TERMS>(h, h_at[i], b, o.h[i]);
    o.scale = s_row[b + zero];
  };
  const int whole = I / kBlock;
  pipeline<0, Operands>(min(b1, whole) - b0, [&](int s, Operands &o) {
    load_block(w_row + (b0 + s) * kBlock, lane, o.w);
    load_others(b0 + s, o);
  }, multiply);
  if (b0 < b1 && b1 > whole) {
    const int c = whole * kBlock;
    Operands o;
    load_last_block(w_row + c, lane, I - c, o.w);
    load_others(whole, o);
    multiply(0, o);
  }
}

// 16 columns of Y (rows of W2) for all tokens.  The reduction runs over the blocks of all experts in use, ascending; a wave
// takes a run of it, and adds an expert's sums to those of the tokens that picked it, in LDS of its own.
template <class T, int MT, int H_TERMS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void moe_down_kernel(MoeArgs g, typename T::Elem *__restrict__ Y, int64_t ldy) {
  __shared__ f32x4 part[WAVES][16 * MT][4];  // [token][four rows of W2]
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][16 * i + r][lane >> 4] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int n0 = blockIdx.x * 16;
  const uint8_t *const w_row = g.W2 + min(n0 + r, g.H - 1) * g.ldw2;
  const float *const s_row = g.S2 + (int64_t)(n0 / kBlock) * g.lds2;
  const Buffer h = __builtin_amdgcn_make_buffer_rsrc(g.h_terms, 0, g.T * g.top * g.h_row, 0x00020000);
  const int blocks = (g.I + kBlock - 1) / kBlock, steps = *g.n_used * blocks;
  const int s0 = (int)((int64_t)steps * wave / WAVES), s1 = (int)((int64_t)steps * (wave + 1) / WAVES);
  for (int s = s0; s < s1;) {
    const int u = s / blocks, b0 = s - u * blocks, b1 = min(blocks, b0 + s1 - s);
    const Use use = g.uses[u];
    const int token = g.use_tokens[u * kMostTokens + lane];
    int h_at[MT];
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      h_at[i] = 16 * i + r < use.count ? (use.first + 16 * i + r) * g.h_row + (lane >> 4) * 16 : kNoColumn;
      acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint8_t *const w = w_row + use.expert * g.w2_stride;
    const float *const sc = s_row + use.expert * g.s2_stride;
    if (use.count <= 16)
      down_blocks<1, MT, H_TERMS>(w, sc, h, h_at, g.I, lane, b0, b1, acc);
    else if (MT == 2 || use.count <= 32)
      down_blocks<(MT < 2 ? 1 : 2), MT, H_TERMS>(w, sc, h, h_at, g.I, lane, b0, b1, acc);
    else
      down_blocks<MT, MT, H_TERMS>(w, sc, h, h_at, g.I, lane, b0, b1, acc);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int to = __shfl(token, (16 * i + r) & 63);
      if (16 * i + r < use.count) part[wave][to][lane >> 4] += acc[i];
    }
    s += b1 - b0;
  }
  __syncthreads();
  for (int i = tid; i < 16 * g.T; i += WAVES * 64) {
    const int t = i / 16, n = i % 16;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += reinterpret_cast<const float *>(part[w][t])[n];
    if (n0 + n < g.H) T::store(Y + t * ldy + n0 + n, v);
  }
}

// ---------------------------------------------------------------------------------------------- host

constexpr int64_t round_up(int64_t n, int64_t d) { return (n + d - 1) / d * d; }

struct MoePlan {
  int64_t logits, n_used, uses, tokens, shares, x, h, total;  // bytes: where they start, and in all
  int x_row, h_row;  // bytes
};

MoePlan plan_of(int T, int H, int I, int E, int top, int32_t dtype) {
  MoePlan p;
  const int terms = dtype == XORENC_X_F32 ? 3 : 1, h_terms = dtype == XORENC_X_F32 ? 3 : 2;
  const int64_t most_used = E < T * top ? E : T * top;
  p.x_row = (H + kBlock - 1) / kBlock * terms * (2 * kBlock);
  p.h_row = (I + kBlock - 1) / kBlock * h_terms * (2 * kBlock);
  p.logits = 0;
  p.n_used = round_up((int64_t)T * E * 4, 16);
  p.uses = p.n_used + 16;
  p.tokens = p.uses + most_used * (int64_t)sizeof(Use);
  p.shares = p.tokens + most_used * kMostTokens;
  p.x = round_up(p.shares + (int64_t)T * top * 4, 256);
  p.h = p.x + (int64_t)T * p.x_row;
  p.total = p.h + (int64_t)T * top * p.h_row;
  return p;
}

template <int MT, int TERMS, int H_TERMS, int WAVES>
void launch_up(const MoeArgs &g, dim3 grid, hipStream_t st) {
  hipLaunchKernelGGL((moe_up_kernel<MT, TERMS, H_TERMS, WAVES>), grid, dim3(WAVES * 64), 0, st, g);
}

template <class T, int TERMS, int H_TERMS, int MT>
void launch_products(const MoeArgs &g, void *Y, int64_t ldy, hipStream_t st) {
  constexpr int DOWN_WAVES = 8;
  const dim3 grid((unsigned)((g.I + kBlock - 1) / kBlock * (kBlock / 16)), (unsigned)min(g.E, g.T * g.top));
  const int64_t tasks = (int64_t)grid.x * grid.y;
  if (tasks >= 2048)
    launch_up<MT, TERMS, H_TERMS, 4>(g, grid, st);
  else
    launch_up<MT, TERMS, H_TERMS, 8>(g, grid, st);
  hipLaunchKernelGGL((moe_down_kernel<T, MT, H_TERMS, DOWN_WAVES>), dim3((unsigned)((g.H + 15) / 16)), dim3(DOWN_WAVES * 64), 0, st, g,
                     static_cast<typename T::Elem *>(Y), ldy);
}

template <class T, int TERMS, int H_TERMS>
int32_t launch_moe(const MoeArgs &g, const void *X, int64_t ldx, bool wide, const void *router, int64_t ldr, bool r_wide, void *Y, int64_t ldy, hipStream_t st) {
  typedef typename T::Elem E;
  const int groups = g.E * ((g.T + 3) / 4);
  const int64_t pieces = (int64_t)g.T * ((g.H + kBlock - 1) / kBlock) * 16;
  hipLaunchKernelGGL((router_kernel<T, TERMS>), dim3((unsigned)(groups + (pieces + 255) / 256)), dim3(256), 0, st,
                     static_cast<const E *>(X), ldx, (int)wide, static_cast<const E *>(router), ldr, (int)r_wide, g.T, g.H, g.E, g.logits,
                     g.x_terms, groups);
  if (g.T > 1) hipLaunchKernelGGL(picks_kernel, dim3(1), dim3(1024), 0, st, g);
  int32_t rc = xorenc_internal_check_launch();
  if (rc != XORENC_OK) return rc;
  if (g.T <= 16)
    launch_products<T, TERMS, H_TERMS, 1>(g, Y, ldy, st);
  else if (g.T <= 32)
    launch_products<T, TERMS, H_TERMS, 2>(g, Y, ldy, st);
  else
    launch_products<T, TERMS, H_TERMS, 4>(g, Y, ldy, st);
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
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(X, esz) || !aligned_to(Y, esz) || !aligned_to(L->router, esz) || !aligned_to(L->W13, 16) || L->ld_w13 % 16 ||
      L->w13_stride % 16 || !aligned_to(L->W2, 16) || L->ld_w2 % 16 || L->w2_stride % 16 || !aligned_to(L->S13, 4) ||
      !aligned_to(L->S2, 4) || !aligned_to(workspace, 16))
    return XORENC_EALIGN;
  unsigned char *const ws = static_cast<unsigned char *>(workspace);
  const bool wide = wide_rows(X, ldx, x_dtype);
  MoeArgs g;
  g.W13 = L->W13, g.W2 = L->W2, g.S13 = L->S13, g.S2 = L->S2;
  g.ldw13 = L->ld_w13, g.w13_stride = L->w13_stride, g.lds13 = L->ld_s13, g.s13_stride = L->s13_stride;
  g.ldw2 = L->ld_w2, g.w2_stride = L->w2_stride, g.lds2 = L->ld_s2, g.s2_stride = L->s2_stride;
  g.T = tokens, g.H = H, g.I = I, g.E = E, g.top = picks, g.renormalise = renormalise != 0;
  g.logits = reinterpret_cast<float *>(ws + p.logits);
  g.uses = reinterpret_cast<Use *>(ws + p.uses);
  g.n_used = reinterpret_cast<int *>(ws + p.n_used);
  g.use_tokens = ws + p.tokens;
  g.shares = reinterpret_cast<float *>(ws + p.shares);
  g.x_terms = reinterpret_cast<uint16_t *>(ws + p.x);
  g.h_terms = reinterpret_cast<uint16_t *>(ws + p.h);
  g.x_row = p.x_row, g.h_row = p.h_row;
  const bool r_wide = wide_rows(L->router, L->ld_router, x_dtype);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return x_dtype == XORENC_X_F32
             ? launch_moe<F32, 3, 3>(g, X, ldx, wide, L->router, L->ld_router, r_wide, Y, ldy, st)
             : launch_moe<BF16, 1, 2>(g, X, ldx, wide, L->router, L->ld_router, r_wide, Y, ldy, st);
}
