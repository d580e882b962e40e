// A mixture-of-experts layer for a few tokens: Y = sum over a token's picks of share * W2_e (silu(G_e x) * (U_e x)), with
// expert weights in e4m3 (a scale per 128 x 128 block) and everything else in 16 or 32 bits.
//
// Three launches: the router's logits; the gated activations h of the picked experts; their second product and the sum
// over picks.  The bytes of the picked experts' weights bound the last two, so both stream 16 rows of weights per workgroup
// from memory to registers, its waves taking the blocks of the reduction in turn.  e4m3 values become bf16 exactly and
// multiply bf16 terms of the activations (one for bf16 activations, three for fp32, which sum to the value exactly), so that
// nothing is rounded to 8 bits on the way; h is kept as bf16 terms that hold 16 (24) bits.  Tokens are the columns of the
// matrix instruction: an expert multiplies those that picked it, the others' columns are zero.
#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

constexpr int kMostExperts = XORENC_MOE_MAX_EXPERTS, kMostPicks = XORENC_MOE_MAX_PICKS, kMostTokens = XORENC_MOE_MAX_TOKENS;
static_assert(kMostExperts == 256 && kMostTokens == 64, "four experts per lane, four column tiles");

struct MoeArgs {
  const uint8_t *W13, *W2;
  const float *S13, *S2;
  int64_t ldw13, w13_stride, lds13, s13_stride, ldw2, w2_stride, lds2, s2_stride;
  int T, H, I, E, top, renormalise;
  const float *logits;      // [T][E]
  const uint16_t *x_terms;  // bf16 terms of x: [term][T][x_ld], zero from H to the next multiple of 16
  int64_t x_ld, x_term;
  uint16_t *h_terms;        // [term][T * top][h_ld], zero from I to the next multiple of 16
  int64_t h_ld, h_term;
};

// What rounding to bf16 leaves of a value; nothing of what is not finite (infinity less infinity would be NaN).
__device__ inline float rest_of_bf16(float v) {
  const float d = v - (float)(__bf16)v;
  return fabsf(d) <= 3.4028235e38f ? d : 0.f;
}

// ---------------------------------------------------------------------------------------------- router

// Logits in fp32: a wave per expert and four tokens.  The waves behind them write the bf16 terms of x where the products
// cannot read it as it is.
template <class T, int TERMS>
__global__ __launch_bounds__(256) void router_kernel(const typename T::Elem *__restrict__ X, int64_t ldx, int wide,
                                                     const typename T::Elem *__restrict__ router, int64_t ldr, int r_wide, int tokens,
                                                     int H, int E, float *__restrict__ logits, uint16_t *__restrict__ terms,
                                                     int64_t x_ld, int64_t x_term, int logit_groups) {
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= logit_groups) {  // x_ld / 8 pieces per token
    const int pieces = (int)(x_ld / 8);
    const int64_t i = (int64_t)(blockIdx.x - logit_groups) * 256 + threadIdx.x;
    if (i >= (int64_t)tokens * pieces) return;
    const int t = (int)(i / pieces), c = (int)(i - (int64_t)t * pieces) * 8;
    float v[8];
    load_piece<T>(X + t * ldx, c, H, wide, v);
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = v[j];
      BF16::store8(terms + k * x_term + t * x_ld + c, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rest_of_bf16(v[j]);
    }
    return;
  }
  const int token_groups = (tokens + 3) / 4;
  const int w = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (w >= E * token_groups) return;
  const int e = w / token_groups, t0 = (w - e * token_groups) * 4;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int c = lane * 8; c < H; c += 512) {
    float r[8];
    load_piece<T>(router + e * ldr, c, H, r_wide, r);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float v[8];
      load_piece<T>(X + min(t0 + k, tokens - 1) * ldx, c, H, wide, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[k] += r[j] * v[j];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc[k] += __shfl_xor(acc[k], o);
    if (lane == 0 && t0 + k < tokens) logits[(t0 + k) * E + e] = acc[k];
  }
}

// ---------------------------------------------------------------------------------------------- picks

constexpr uint8_t kNotPicked = 0xff;

// What every workgroup works out for itself from the logits: the experts that some token picked, ascending, and which of
// a token's picks each of them is.
template <int MT>
struct Picks {
  float share[16 * MT][kMostPicks];
  uint16_t expert[16 * MT][kMostPicks];
  uint16_t used[kMostExperts];  // experts in use
  uint16_t place[kMostExperts]; // of an expert among them
  uint32_t in_use[kMostExperts / 32];
  int n_used;
  uint8_t slot[kMostExperts * 16 * MT];  // [place][token]: which of the token's picks, or kNotPicked
};

// fp32 -> integers in the same order (NaN above infinity or below its negative, as the sign says)
__device__ inline uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

template <int MT, int WAVES>
__device__ inline void find_picks(const MoeArgs &g, Picks<MT> &p) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int most_used = min(g.E, g.T * g.top);
  if (tid < kMostExperts / 32) p.in_use[tid] = 0u;
  for (int i = tid; i < most_used * (16 * MT) / 4; i += WAVES * 64) reinterpret_cast<uint32_t *>(p.slot)[i] = 0xffffffffu;
  __syncthreads();
  for (int t = wave; t < g.T; t += WAVES) {
    const float *const row = g.logits + t * g.E;
    uint32_t key[4];
    bool left[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      left[i] = e < g.E;
      key[i] = left[i] ? ordered(row[e]) : 0u;
    }
    float first = 0.f, sum = 0.f, mine = 0.f;
    if (!g.renormalise) {  // shares of a softmax over all experts
      uint32_t m = max(max(key[0], key[1]), max(key[2], key[3]));
      m = max_of_16_lanes(m);
      m = max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
              max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
      const float most = from_ordered(m);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (left[i]) sum += expf(from_ordered(key[i]) - most);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    }
    for (int j = 0; j < g.top; ++j) {  // the largest that is left; the lowest index of equals
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = left[i] ? max(m, key[i]) : m;
      m = max_of_16_lanes(m);
      m = max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
              max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
      int e = -1;
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        const uint64_t at = __ballot(left[i] && key[i] == m);
        if (at) e = 64 * i + __builtin_ctzll(at);
      }
      e = __builtin_amdgcn_readfirstlane(e);
#pragma unroll
      for (int i = 0; i < 4; ++i) left[i] = left[i] && e != lane + 64 * i;
      const float l = from_ordered(m);
      if (j == 0) first = l;
      const float v = expf(l - first);
      if (g.renormalise) sum += v;
      if (lane == j) mine = v;
      if (lane == 0) {
        p.expert[t][j] = (uint16_t)e;
        atomicOr(&p.in_use[e >> 5], 1u << (e & 31));
      }
    }
    if (lane < g.top) p.share[t][lane] = mine / sum;
  }
  __syncthreads();
  if (wave == 0) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      const bool in = (p.in_use[e >> 5] >> (e & 31)) & 1u;
      const uint64_t all = __ballot(in);
      if (in) {
        const int at = n + __popcll(all & ((1ull << lane) - 1ull));
        p.used[at] = (uint16_t)e;
        p.place[e] = (uint16_t)at;
      }
      n += __popcll(all);
    }
    if (lane == 0) p.n_used = n;
  }
  __syncthreads();
  for (int i = tid; i < g.T * g.top; i += WAVES * 64) {
    const int t = i / g.top, j = i - t * g.top;
    p.slot[p.place[p.expert[t][j]] * (16 * MT) + t] = (uint8_t)j;
  }
  __syncthreads();
}

// ---------------------------------------------------------------------------------------------- products

// Quarter q of the columns that a lane holds of a row of bf16 values: the columns that quarter_as_bf16 gives of weights.
__device__ inline bf16x8 term_quarter(const uint16_t *row, int c, int q, int cols) {
  const int at = c + (q >> 1) * 64 + (q & 1) * 8;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (at < cols) v = *reinterpret_cast<const u32x4 *>(row + at);  // (rows are zero up to a multiple of 16)
  return __builtin_bit_cast(bf16x8, v);
}

// h of 16 rows of an expert for all tokens that picked it.
template <int MT, int TERMS, int H_TERMS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void moe_up_kernel(MoeArgs g) {
  __shared__ Picks<MT> picks;
  __shared__ f32x4 part[WAVES][2][MT][64];
  find_picks<MT, WAVES>(g, picks);
  const int u = blockIdx.y;
  if (u >= picks.n_used) return;
  const int e = __builtin_amdgcn_readfirstlane(picks.used[u]);
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i0 = blockIdx.x * 16;
  const uint8_t *const base = g.W13 + e * g.w13_stride;
  const int row = min(i0 + r, g.I - 1);
  const uint8_t *const gate_row = base + row * g.ldw13, *const up_row = base + ((int64_t)g.I + row) * g.ldw13;
  // the up rows of a tile lie in two blocks of scales where I is not a multiple of 16
  const int first = g.I + i0, last = g.I + min(i0 + 15, g.I - 1), edge = (last / kBlock) * kBlock - first;
  const float *const s_gate = g.S13 + e * g.s13_stride + (int64_t)(i0 / kBlock) * g.lds13;
  const float *const s_up0 = g.S13 + e * g.s13_stride + (int64_t)(first / kBlock) * g.lds13;
  const float *const s_up1 = g.S13 + e * g.s13_stride + (int64_t)(last / kBlock) * g.lds13;
  const uint16_t *x_row[MT];
  bool picked[MT], any[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int t = 16 * i + r;
    picked[i] = picks.slot[u * (16 * MT) + t] != kNotPicked;
    any[i] = __ballot(picked[i]) != 0;
    x_row[i] = g.x_terms + (picked[i] ? t : 0) * g.x_ld;
  }
  f32x4 gate[MT], up[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) gate[i] = up[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int blocks = (g.H + kBlock - 1) / kBlock;
  for (int b = wave; b < blocks; b += WAVES) {
    const int c = b * kBlock + piece_column(lane, 0);
    E4m3Operand wg, wu;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      wg.piece[k] = load_e4m3_piece(gate_row, c + 64 * k, g.H);
      wu.piece[k] = load_e4m3_piece(up_row, c + 64 * k, g.H);
    }
    const float sg = s_gate[b], su0 = s_up0[b], su1 = s_up1[b];
    f32x4 dg[MT], du[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) dg[i] = du[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bf16x8 vg = quarter_as_bf16(wg, q), vu = quarter_as_bf16(wu, q);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if (!any[i]) continue;
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
          const bf16x8 x = term_quarter(x_row[i] + k * g.x_term, c, q, picked[i] ? g.H : 0);
          dg[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vg, x, dg[i], 0, 0, 0);
          du[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vu, x, du[i], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gate[i][j] += sg * dg[i][j];
        up[i][j] += (4 * (lane >> 4) + j < edge ? su0 : su1) * du[i][j];
      }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    part[wave][0][i][lane] = gate[i];
    part[wave][1][i][lane] = up[i];
  }
  __syncthreads();
  for (int i = wave; i < MT; i += WAVES) {
    f32x4 a = part[0][0][i][lane], b = part[0][1][i][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      a += part[w][0][i][lane];
      b += part[w][1][i][lane];
    }
    const int t = 16 * i + r;
    const uint8_t j = picks.slot[u * (16 * MT) + t];
    if (j == kNotPicked) continue;
    const float share = picks.share[t][j];
    const int at = i0 + 4 * (lane >> 4);
    float h[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) h[k] = at + k < g.I ? silu(a[k]) * b[k] * share : 0.f;
    uint16_t *const dst = g.h_terms + ((int64_t)t * g.top + j) * g.h_ld + at;
#pragma unroll
    for (int k = 0; k < H_TERMS; ++k) {
      *reinterpret_cast<u32x2 *>(dst + k * g.h_term) = u32x2{to_bf16x2(h[0], h[1]), to_bf16x2(h[2], h[3])};
#pragma unroll
      for (int n = 0; n < 4; ++n) h[n] = rest_of_bf16(h[n]);
    }
  }
}

// 16 columns of Y (rows of W2) for all tokens: the reduction runs over the blocks of all experts in use, ascending.
template <class T, int MT, int H_TERMS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void moe_down_kernel(MoeArgs g, typename T::Elem *__restrict__ Y, int64_t ldy) {
  __shared__ Picks<MT> picks;
  __shared__ f32x4 part[WAVES][MT][64];
  find_picks<MT, WAVES>(g, picks);
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int64_t row_off = min(n0 + r, g.H - 1) * g.ldw2, s_off = (int64_t)(n0 / kBlock) * g.lds2;
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int blocks = (g.I + kBlock - 1) / kBlock, steps = picks.n_used * blocks;
  for (int s = wave; s < steps; s += WAVES) {
    const int u = s / blocks, b = s - u * blocks;
    const int e = __builtin_amdgcn_readfirstlane(picks.used[u]);
    const int c = b * kBlock + piece_column(lane, 0);
    const uint8_t *const w_row = g.W2 + e * g.w2_stride + row_off;
    E4m3Operand w;
    w.piece[0] = load_e4m3_piece(w_row, c, g.I);
    w.piece[1] = load_e4m3_piece(w_row, c + 64, g.I);
    const float sc = g.S2[e * g.s2_stride + s_off + b];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int t = 16 * i + r;
      const uint8_t j = picks.slot[u * (16 * MT) + t];
      if (!__ballot(j != kNotPicked)) continue;
      const uint16_t *const h_row = g.h_terms + ((int64_t)t * g.top + (j == kNotPicked ? 0 : j)) * g.h_ld;
      f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x8 v = quarter_as_bf16(w, q);
#pragma unroll
        for (int k = 0; k < H_TERMS; ++k)
          d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, term_quarter(h_row + k * g.h_term, c, q, j == kNotPicked ? 0 : g.I), d, 0, 0, 0);
      }
      // (a weight or scale of this expert that is not finite concerns the tokens that picked it alone)
#pragma unroll
      for (int n = 0; n < 4; ++n) acc[i][n] += j != kNotPicked ? sc * d[n] : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < MT; i += WAVES) {
    f32x4 v = part[0][i][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += part[w][i][lane];
    const int t = 16 * i + r, n = n0 + 4 * (lane >> 4);
    if (t >= g.T) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < g.H) T::store(Y + t * ldy + n + k, v[k]);
  }
}

// ---------------------------------------------------------------------------------------------- host

constexpr int64_t round_up(int64_t n, int64_t d) { return (n + d - 1) / d * d; }

struct MoePlan {
  int64_t logits, x, h, total;  // bytes: where they start, and in all
  int64_t x_ld, h_ld;
};

MoePlan plan_of(int T, int H, int I, int E, int top, int32_t dtype) {
  MoePlan p;
  const int terms = dtype == XORENC_X_F32 ? 3 : 1, h_terms = dtype == XORENC_X_F32 ? 3 : 2;
  p.x_ld = round_up(H, 16);
  p.h_ld = round_up(I, 16);
  p.logits = 0;
  p.x = round_up((int64_t)T * E * 4, 256);
  p.h = p.x + round_up(terms * T * p.x_ld * 2, 256);
  p.total = p.h + h_terms * T * top * p.h_ld * 2;
  return p;
}

template <class T, int TERMS, int H_TERMS, int MT>
void launch_products(const MoeArgs &g, void *Y, int64_t ldy, hipStream_t st) {
  hipLaunchKernelGGL((moe_up_kernel<MT, TERMS, H_TERMS, 4>), dim3((unsigned)((g.I + 15) / 16), (unsigned)min(g.E, g.T * g.top)), dim3(256),
                     0, st, g);
  hipLaunchKernelGGL((moe_down_kernel<T, MT, H_TERMS, 8>), dim3((unsigned)((g.H + 15) / 16)), dim3(512), 0, st, g,
                     static_cast<typename T::Elem *>(Y), ldy);
}

template <class T, int TERMS, int H_TERMS>
int32_t launch_moe(const MoeArgs &g, const void *X, int64_t ldx, bool wide, const void *router, int64_t ldr, bool r_wide, bool staged,
                   float *logits, uint16_t *terms, void *Y, int64_t ldy, hipStream_t st) {
  typedef typename T::Elem E;
  const int groups = (g.E * ((g.T + 3) / 4) + 3) / 4;
  const int64_t pieces = staged ? g.T * (g.x_ld / 8) : 0;
  hipLaunchKernelGGL((router_kernel<T, TERMS>), dim3((unsigned)(groups + (pieces + 255) / 256)), dim3(256), 0, st,
                     static_cast<const E *>(X), ldx, (int)wide, static_cast<const E *>(router), ldr, (int)r_wide, g.T, g.H, g.E, logits,
                     terms, g.x_ld, g.x_term, groups);
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
  if (T > kMostTokens || E > kMostExperts || top > kMostPicks || H > (1 << 24) || I > (1 << 23)) return XORENC_ELIMIT;
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
  const bool staged = x_dtype == XORENC_X_F32 || !wide || H % 16;  // the products read x as bf16 in whole pieces
  MoeArgs g;
  g.W13 = L->W13, g.W2 = L->W2, g.S13 = L->S13, g.S2 = L->S2;
  g.ldw13 = L->ld_w13, g.w13_stride = L->w13_stride, g.lds13 = L->ld_s13, g.s13_stride = L->s13_stride;
  g.ldw2 = L->ld_w2, g.w2_stride = L->w2_stride, g.lds2 = L->ld_s2, g.s2_stride = L->s2_stride;
  g.T = tokens, g.H = H, g.I = I, g.E = E, g.top = picks, g.renormalise = renormalise != 0;
  float *const logits = reinterpret_cast<float *>(ws + p.logits);
  uint16_t *const terms = reinterpret_cast<uint16_t *>(ws + p.x);
  g.logits = logits;
  g.x_terms = staged ? terms : static_cast<const uint16_t *>(X);
  g.x_ld = staged ? p.x_ld : ldx;
  g.x_term = tokens * p.x_ld;
  g.h_terms = reinterpret_cast<uint16_t *>(ws + p.h);
  g.h_ld = p.h_ld;
  g.h_term = (int64_t)tokens * picks * p.h_ld;
  const bool r_wide = wide_rows(L->router, L->ld_router, x_dtype);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return x_dtype == XORENC_X_F32
             ? launch_moe<F32, 3, 3>(g, X, ldx, wide, L->router, L->ld_router, r_wide, staged, logits, terms, Y, ldy, st)
             : launch_moe<BF16, 1, 2>(g, X, ldx, wide, L->router, L->ld_router, r_wide, staged, logits, terms, Y, ldy, st);
}
