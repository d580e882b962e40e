// A mixture of experts over many tokens, around its products: picks, the pairs of tokens and experts sorted by expert, the tokens'
// rows in that order and back, and the gradient of the way back.
//
// Rows are moved in pieces of eight elements, a lane each, every piece of a token read once; the bytes bound these kernels.
#include "xorenc_fp8.h"

namespace xorenc_fp8_detail {
namespace {

constexpr int kMostExperts = XORENC_MOE_MAX_EXPERTS, kMostPicks = XORENC_MOE_MAX_PICKS;
constexpr int64_t kMostPairs = (1 << 24) - 1;

// ---------------------------------------------------------------------------------------------- picks

// The order of the picks as integers: a NaN above all, -0 and 0 equal, 0 for what is never picked (-infinity); and the value that has it.
__device__ inline uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (b == 0xff800000u) return 0u;
  return (b & 0x7fffffffu) == 0u ? 0x80000000u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }

// Sixteen lanes hold a token's logits, V each, and take the largest that is left once per pick: its order first, then the least index of
// those that have it.  Logits of 16 bits leave room for both in one integer, and for one maximum (65536 tokens, 8 of 128 experts: 14.1
// us, in 32 bits 16.9).  Lane p ends up with the p-th pick.
template <class T, int V>
__global__ __launch_bounds__(256) void pick_kernel(const typename T::Elem *__restrict__ logits, int64_t ldl, int tokens, int experts, int picks,
                                                   int renormalise, int *__restrict__ ids, float *__restrict__ shares) {
  constexpr bool NARROW = sizeof(typename T::Elem) == 2;
  const int t = blockIdx.x * 16 + (threadIdx.x >> 4), l = threadIdx.x & 15;
  if (t >= tokens) return;
  const typename T::Elem *const row = logits + t * ldl;
  auto expert = [&](int v) { return V < 8 ? l * V + v : v / 8 * 128 + l * 8 + v % 8; };
  float x[V];
  if constexpr (V < 8) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = -INFINITY;
      if (expert(v) < experts) {
        if constexpr (NARROW)
          x[v] = __uint_as_float((uint32_t)row[expert(v)] << 16);
        else
          x[v] = row[expert(v)];
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; v += 8) {
      piece_of<T>(load_piece<T>(row, min(expert(v), experts), experts), min(expert(v), experts), experts, x + v);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (expert(v + i) >= experts) x[v + i] = -INFINITY;
    }
  }
  uint32_t key[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    key[v] = order_of(x[v]);
    if (NARROW && key[v]) key[v] = (key[v] & 0xffff0000u) | (0xffffu - (uint32_t)expert(v));
  }
  int id = -1;
  float mine = -INFINITY, most = 0.f;
  for (int p = 0; p < picks; ++p) {
    uint32_t best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    best = max_of_16_lanes(best);
    if (best == 0) break;  // (the same on all 16 lanes)
    int first;
    if constexpr (NARROW) {
      first = (int)(0xffffu - (best & 0xffffu));
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = key[v] == best ? 0u : key[v];
      best = best & 0x80000000u ? best & 0xffff0000u : best | 0xffffu;  // (a negative value's lower bits are inverted zeros)
    } else {
      uint32_t least = 0;  // 0xffff less the index
#pragma unroll
      for (int v = V - 1; v >= 0; --v) least = key[v] == best ? 0xffffu - (uint32_t)expert(v) : least;
      first = (int)(0xffffu - max_of_16_lanes(least));
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = expert(v) == first ? 0u : key[v];
    }
    const float value = value_of(best);
    if (p == 0) most = value;
    if (l == p) id = first, mine = value;
  }
  // (nothing to pick: most = 0, and every term is exp(-infinity))
  const float e = id < 0 ? 0.f : expf(mine - most);
  float total;
  if (renormalise) {
    total = sum_of_16_lanes(e);
  } else {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) s += expf(x[v] - most);
    total = sum_of_16_lanes(s);
  }
  if (l < picks) {
    ids[t * picks + l] = id;
    shares[t * picks + l] = id < 0 ? 0.f : e / total;
  }
}

// ---------------------------------------------------------------------------------------------- sort

// A stable counting sort.  A workgroup places a segment of pairs, ROUNDS of 64 a wave: what comes before them, and where each expert's rows begin, it
// counts itself where there are few pairs (one launch); otherwise a launch before has counted every segment.  Long segments where there are many: what a
// workgroup adds up is theirs all (us, in segments of 2048 and of 8192: 2^18 pairs of 128 experts 13.5 and 19.0, 2^20 35 and 25, 8 M of 64 504 and 100; 2^14 of
// 64 in one launch 9.1, 2^15 in two 9.2).
constexpr int kSortWaves = 8, kFewRounds = 4, kManyRounds = 16, kManyPairs = 1 << 19;
constexpr int segment_of(int rounds) { return kSortWaves * rounds * 64; }
constexpr int kBuckets = kMostExperts + 1;  // the last: pairs without an expert
constexpr int kFewPairs = 16384;

template <class Id>
__device__ inline int bucket_of(Id id, int experts) {
  return id >= 0 && id < experts ? (int)id : experts;
}

template <class Id, int ROUNDS>
__global__ __launch_bounds__(kSortWaves * 64) void count_kernel(const Id *__restrict__ ids, int pairs, int experts, int *__restrict__ counts) {
  __shared__ int count[kBuckets];
  for (int e = threadIdx.x; e <= experts; e += kSortWaves * 64) count[e] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int pair = blockIdx.x * segment_of(ROUNDS) + i * (kSortWaves * 64) + threadIdx.x;
    if (pair < pairs) atomicAdd(&count[bucket_of(ids[pair], experts)], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= experts; e += kSortWaves * 64) counts[blockIdx.x * (experts + 1) + e] = count[e];
}

template <class Id, int ROUNDS>
__global__ __launch_bounds__(kSortWaves * 64) void sort_kernel(const Id *__restrict__ ids, int pairs, int picks, int experts,
                                                               const int *__restrict__ counts, int segments, int *__restrict__ places,
                                                               int *__restrict__ rows, int *__restrict__ offsets) {
  __shared__ int before[kBuckets], behind[kBuckets], first[kBuckets];  // pairs of segments before this one, and of it and those behind
  __shared__ int of_wave[kSortWaves][kBuckets];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = kSortWaves * 64;
  const int start = blockIdx.x * segment_of(ROUNDS);
  for (int e = tid; e <= experts; e += threads) {
    before[e] = behind[e] = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) of_wave[w][e] = 0;
  }
  // this wave's pairs, in order
  int bucket[ROUNDS], rank[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int pair = start + (wave * ROUNDS + i) * 64 + lane;
    bucket[i] = pair < pairs ? bucket_of(ids[pair], experts) : -1;
  }
  __syncthreads();
  if (counts) {
    // Groups of threads, a thread an expert, take the segments in turn, eight loads of each on their way together (sums of integers, the same in any order).
    const int width = (experts + 64) & ~63, groups = threads / width, group = tid / width, e = tid - group * width;
    if (group < groups && e <= experts) {
      int b = 0, a = 0;
      for (int s0 = group; s0 < segments; s0 += 8 * groups) {
        int n[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int s = s0 + i * groups;
          n[i] = s < segments ? counts[s * (experts + 1) + e] : 0;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (s0 + i * groups < (int)blockIdx.x) b += n[i]; else a += n[i];
        }
      }
      atomicAdd(&before[e], b);
      atomicAdd(&behind[e], a);
    }
  } else {
    for (int pair = tid; pair < pairs; pair += threads) atomicAdd(pair < start ? &before[bucket_of(ids[pair], experts)] : &behind[bucket_of(ids[pair], experts)], 1);
  }
  // ranks within the wave's pairs: of the same bucket, those on lower lanes and of earlier rounds
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int b = bucket[i];
    uint64_t same = __ballot(b >= 0);
#pragma unroll
    for (int bit = 0; bit < 9; ++bit) {
      const uint64_t set = __ballot((b >> bit) & 1);
      same &= (b >> bit) & 1 ? set : ~set;
    }
    const int below = __popcll(same & ((1ull << lane) - 1));
    int had = 0;
    if (b >= 0 && below == 0) had = atomicAdd(&of_wave[wave][b], __popcll(same));
    rank[i] = below + __shfl(had, b >= 0 ? __ffsll((unsigned long long)same) - 1 : lane);
  }
  __syncthreads();
  if (wave == 0) {  // first[e]: pairs of the experts before e
    constexpr int PER = (kBuckets + 63) / 64;
    int n[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int e = lane * PER + k;
      n[k] = e <= experts ? before[e] + behind[e] : 0;
      sum += n[k];
    }
    int upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(upto, d);
      if (lane >= d) upto += other;
    }
    int at = upto - sum;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int e = lane * PER + k;
      if (e <= experts) first[e] = at;
      at += n[k];
    }
  } else {
    for (int e = tid - 64; e <= experts; e += threads - 64) {
      int at = 0;
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int n = of_wave[w][e];
        of_wave[w][e] = at;
        at += n;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    if (bucket[i] < 0) continue;
    const int pair = start + (wave * ROUNDS + i) * 64 + lane;
    const int place = first[bucket[i]] + before[bucket[i]] + of_wave[wave][bucket[i]] + rank[i];
    places[pair] = place;
    if (rows) rows[place] = pair / picks;
  }
  if (blockIdx.x == 0)
    for (int e = tid; e <= experts; e += threads) offsets[e] = first[e];
}

// ---------------------------------------------------------------------------------------------- rows

struct RowArgs {
  const int *places, *used;
  const float *shares;
  int64_t ldx, ldr, ldo;  // of tokens' rows that are read, of sorted rows, of rows that are written
  int tokens, picks, cols, per_row;
};

// STREAM: past the caches.
template <class T, bool STREAM>
__device__ inline void store_row(typename T::Elem *row, int c, int cols, const float *v) {
  if constexpr (STREAM && sizeof(typename T::Elem) == 2) {
    if (c + 8 <= cols) {
      const u32x4 w = {to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7])};
      __builtin_nontemporal_store(w, reinterpret_cast<u32x4_anywhere *>(row + c));
      return;
    }
  }
  store_piece<T>(row, c, cols, v);
}

template <class T, bool STREAM>
__device__ inline void store_zero(typename T::Elem *row, int c, int cols) {
  const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  store_row<T, STREAM>(row, c, cols, none);
}

// A lane a piece of X, which it stores as often as the token has pairs.
template <class T, bool SHARES, bool STREAM>
__global__ __launch_bounds__(256) void gather_kernel(const typename T::Elem *__restrict__ X, RowArgs g, typename T::Elem *__restrict__ R) {
  const uint32_t piece = blockIdx.x * 256u + threadIdx.x;
  const int t = (int)(piece / (uint32_t)g.per_row), c = (int)(piece % (uint32_t)g.per_row) * 8;
  if (t >= g.tokens) return;
  const int used = max(min(*g.used, g.tokens * g.picks), 0);
  float x[8];
  piece_of<T>(load_piece<T, STREAM>(X + t * g.ldx, c, g.cols), c, g.cols, x);
  for (int p = 0; p < g.picks; ++p) {
    const int place = g.places[t * g.picks + p];
    if ((unsigned)place >= (unsigned)(g.tokens * g.picks)) continue;
    typename T::Elem *const row = R + place * g.ldr;
    if (place >= used) {
      store_zero<T, STREAM>(row, c, g.cols);
    } else if constexpr (SHARES) {
      const float s = g.shares[t * g.picks + p];
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i] * s;
      store_row<T, STREAM>(row, c, g.cols, y);
    } else {
      store_row<T, STREAM>(row, c, g.cols, x);
    }
  }
}

// A lane a piece of Y.  The rows of up to MOST pairs are on their way together.
template <class T, int MOST, bool STREAM>
__global__ __launch_bounds__(256) void combine_kernel(const typename T::Elem *__restrict__ R, RowArgs g, const typename T::Elem *residual,
                                                      typename T::Elem *Y) {
  const uint32_t piece = blockIdx.x * 256u + threadIdx.x;
  const int t = (int)(piece / (uint32_t)g.per_row), c = (int)(piece % (uint32_t)g.per_row) * 8;
  if (t >= g.tokens) return;
  const int used = max(min(*g.used, g.tokens * g.picks), 0);
  typename T::Raw rest;
  if (residual) rest = load_piece<T, STREAM>(residual + t * g.ldx, c, g.cols);
  float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < g.picks; p0 += MOST) {
    typename T::Raw raw[MOST];
    int place[MOST];
    float share[MOST];
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
      const int p = min(p0 + k, g.picks - 1);
      place[k] = p0 + k < g.picks ? g.places[t * g.picks + p] : -1;
      share[k] = g.shares ? g.shares[t * g.picks + p] : 1.f;
    }
#pragma unroll
    for (int k = 0; k < MOST; ++k)
      if ((unsigned)place[k] < (unsigned)used) raw[k] = load_piece<T, STREAM>(R + place[k] * g.ldr, c, g.cols);
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
      if ((unsigned)place[k] >= (unsigned)used) continue;
      float x[8];
      piece_of<T>(raw[k], c, g.cols, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = fmaf(share[k], x[i], y[i]);
    }
  }
  if (residual) {
    float x[8];
    piece_of<T>(rest, c, g.cols, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] += x[i];
  }
  store_row<T, STREAM>(Y + t * g.ldo, c, g.cols, y);
}

// A workgroup a token: every piece of dY is read once, multiplied into each row's sum and written to each row's gradient.
template <class T, int THREADS, int MOST, bool STREAM>
__global__ __launch_bounds__(THREADS) void combine_grad_kernel(const typename T::Elem *__restrict__ dY, RowArgs g, const typename T::Elem *R,
                                                               typename T::Elem *dR, float *__restrict__ dshares) {
  constexpr int WAVES = THREADS / 64;
  __shared__ float sums[WAVES][MOST];
  const int t = blockIdx.x, tid = threadIdx.x, pairs = g.tokens * g.picks;
  const int used = max(min(*g.used, pairs), 0);
  int place[MOST];
  float share[MOST], dot[MOST];
#pragma unroll
  for (int p = 0; p < MOST; ++p) {
    const int q = min(p, g.picks - 1);
    place[p] = p < g.picks ? g.places[t * g.picks + q] : -1;
    share[p] = g.shares[t * g.picks + q];
    dot[p] = 0.f;
  }
  for (int c = tid * 8; c < g.cols; c += THREADS * 8) {
    float dy[8];
    typename T::Raw raw[MOST];
    const typename T::Raw y = load_piece<T, STREAM>(dY + t * g.ldx, c, g.cols);
#pragma unroll
    for (int p = 0; p < MOST; ++p)
      if ((unsigned)place[p] < (unsigned)used) raw[p] = load_piece<T, STREAM>(R + place[p] * g.ldr, c, g.cols);
    piece_of<T>(y, c, g.cols, dy);
#pragma unroll
    for (int p = 0; p < MOST; ++p) {
      if ((unsigned)place[p] >= (unsigned)pairs) continue;
      typename T::Elem *const row = dR + place[p] * g.ldo;
      if (place[p] >= used) {
        store_zero<T, STREAM>(row, c, g.cols);
        continue;
      }
      float x[8];
      piece_of<T>(raw[p], c, g.cols, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot[p] = fmaf(x[i], dy[i], dot[p]), x[i] = dy[i] * share[p];
      store_row<T, STREAM>(row, c, g.cols, x);
    }
  }
#pragma unroll
  for (int p = 0; p < MOST; ++p) {
    const float s = sum_of_wave(dot[p]);
    if ((tid & 63) == 0) sums[tid >> 6][p] = s;
  }
  __syncthreads();
  if (tid < g.picks) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += sums[w][tid];
    dshares[t * g.picks + tid] = s;
  }
}

// ---------------------------------------------------------------------------------------------- host

int32_t check_pairs(int32_t tokens, int32_t picks) {
  if (tokens < 0 || picks <= 0) return XORENC_EINVAL;
  if (picks > kMostPicks || (int64_t)tokens * picks > kMostPairs) return XORENC_ELIMIT;
  return XORENC_OK;
}

int32_t check_rows(int32_t dtype, int32_t tokens, int32_t picks, int32_t cols) {
  if (cols <= 0) return XORENC_EINVAL;
  const int32_t rc = check_pairs(tokens, picks);
  if (rc != XORENC_OK) return rc;
  if (!known_dtype(dtype)) return XORENC_EUNSUPPORTED;
  if (cols > (1 << 20) || (int64_t)tokens * ((cols + 7) / 8) > 0x7fffffff) return XORENC_ELIMIT;
  return XORENC_OK;
}

// f(type), and f(type, whether to stream: rows of 16 bits; those of 32 go through the caches whatever their number)
template <class F>
int32_t for_type(int32_t dtype, F f) {
  return dtype == XORENC_X_F32 ? f(F32()) : f(BF16());
}
template <class F>
int32_t for_rows(int32_t dtype, bool stream, F f) {
  return dtype == XORENC_X_F32 ? f(F32(), std::false_type()) : stream ? f(BF16(), std::true_type()) : f(BF16(), std::false_type());
}
// Whether `rows` rows that a call reads or writes are more than half of what the memory-side cache holds (256 MB).  (8192 x 4096 to two experts 37.4 us through
// the caches, 35.4 past them, back 48.1 and 44.8; the gradient of 4096 x 2048 from eight 60.3 and 58.2.)
inline bool streams(int64_t rows, int64_t cols, int esz) { return rows * cols > ((int64_t)128 << 20) / esz; }

template <class T, int V>
int32_t launch_pick(const void *logits, int64_t ldl, int tokens, int experts, int picks, int renormalise, int32_t *ids, float *shares, hipStream_t st) {
  hipLaunchKernelGGL((pick_kernel<T, V>), dim3((unsigned)((tokens + 15) / 16)), dim3(256), 0, st, static_cast<const typename T::Elem *>(logits), ldl,
                     tokens, experts, picks, renormalise, ids, shares);
  return xorenc_internal_check_launch();
}

int rounds_of(int64_t pairs) { return pairs < kManyPairs ? kFewRounds : kManyRounds; }

int64_t sort_workspace(int64_t pairs, int32_t experts) {
  const int segment = segment_of(rounds_of(pairs));
  return pairs <= kFewPairs ? 0 : (pairs + segment - 1) / segment * (experts + 1) * 4;
}

template <class Id, int ROUNDS>
int32_t launch_sort(const void *ids, int pairs, int picks, int experts, int32_t *places, int32_t *rows, int32_t *offsets, int *counts, hipStream_t st) {
  const int segments = pairs ? (pairs + segment_of(ROUNDS) - 1) / segment_of(ROUNDS) : 1;
  const Id *const id = static_cast<const Id *>(ids);
  if (counts) hipLaunchKernelGGL((count_kernel<Id, ROUNDS>), dim3((unsigned)segments), dim3(kSortWaves * 64), 0, st, id, pairs, experts, counts);
  hipLaunchKernelGGL((sort_kernel<Id, ROUNDS>), dim3((unsigned)segments), dim3(kSortWaves * 64), 0, st, id, pairs, picks, experts, counts, segments, places,
                     rows, offsets);
  return xorenc_internal_check_launch();
}

}  // namespace
}  // namespace xorenc_fp8_detail

using namespace xorenc_fp8_detail;

extern "C" int32_t xorenc_pick_experts(const void *logits, int32_t x_dtype, int64_t ldl, int32_t tokens, int32_t experts, int32_t picks,
                                       int32_t renormalise, int32_t *ids, float *shares, void *hip_stream) {
  if (experts <= 0 || picks > experts || ldl < experts) return XORENC_EINVAL;
  const int32_t rc = check_pairs(tokens, picks);
  if (rc != XORENC_OK) return rc;
  if (!known_dtype(x_dtype)) return XORENC_EUNSUPPORTED;
  if (experts > kMostExperts) return XORENC_ELIMIT;
  if (tokens == 0) return XORENC_OK;
  if (!logits || !ids || !shares) return XORENC_EINVAL;
  if (!aligned_to(logits, dtype_bytes(x_dtype)) || !aligned_to(ids, 4) || !aligned_to(shares, 4)) return XORENC_EALIGN;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return for_type(x_dtype, [&](auto type) {
    typedef decltype(type) T;
    if (experts <= 16) return launch_pick<T, 1>(logits, ldl, tokens, experts, picks, renormalise, ids, shares, st);
    if (experts <= 32) return launch_pick<T, 2>(logits, ldl, tokens, experts, picks, renormalise, ids, shares, st);
    if (experts <= 64) return launch_pick<T, 4>(logits, ldl, tokens, experts, picks, renormalise, ids, shares, st);
    if (experts <= 128) return launch_pick<T, 8>(logits, ldl, tokens, experts, picks, renormalise, ids, shares, st);
    return launch_pick<T, 16>(logits, ldl, tokens, experts, picks, renormalise, ids, shares, st);
  });
}

extern "C" int32_t xorenc_sort_tokens_workspace(int32_t tokens, int32_t picks, int32_t experts, int64_t *bytes) {
  if (!bytes || experts <= 0) return XORENC_EINVAL;
  const int32_t rc = check_pairs(tokens, picks);
  if (rc != XORENC_OK) return rc;
  if (experts > kMostExperts) return XORENC_ELIMIT;
  *bytes = sort_workspace((int64_t)tokens * picks, experts);
  return XORENC_OK;
}

extern "C" int32_t xorenc_sort_tokens(const void *ids, int32_t id_type, int32_t tokens, int32_t picks, int32_t experts, int32_t *places,
                                      int32_t *rows, int32_t *offsets, void *workspace, int64_t workspace_bytes, void *hip_stream) {
  int64_t need;
  const int32_t rc = xorenc_sort_tokens_workspace(tokens, picks, experts, &need);
  if (rc != XORENC_OK) return rc;
  if (id_type != XORENC_I32 && id_type != XORENC_I64) return XORENC_EUNSUPPORTED;
  if (!offsets || (tokens && (!ids || !places)) || (need && (!workspace || workspace_bytes < need))) return XORENC_EINVAL;
  if (!aligned_to(ids, id_type == XORENC_I64 ? 8 : 4) || !aligned_to(places, 4) || !aligned_to(rows, 4) || !aligned_to(offsets, 4) ||
      (need && !aligned_to(workspace, 4)))
    return XORENC_EALIGN;
  int *const counts = need ? static_cast<int *>(workspace) : nullptr;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  auto launch = [&](auto id, auto rounds) {
    return launch_sort<decltype(id), decltype(rounds)::value>(ids, tokens * picks, picks, experts, places, rows, offsets, counts, st);
  };
  typedef std::integral_constant<int, kFewRounds> Few;
  typedef std::integral_constant<int, kManyRounds> Many;
  if (rounds_of((int64_t)tokens * picks) == kFewRounds) return id_type == XORENC_I64 ? launch(int64_t(), Few()) : launch(int32_t(), Few());
  return id_type == XORENC_I64 ? launch(int64_t(), Many()) : launch(int32_t(), Many());
}

extern "C" int32_t xorenc_gather_tokens(const void *X, int32_t x_dtype, int64_t ldx, const int32_t *places, const int32_t *used,
                                        const float *shares, int32_t tokens, int32_t picks, int32_t cols, void *R, int64_t ldr, void *hip_stream) {
  const int32_t rc = check_rows(x_dtype, tokens, picks, cols);
  if (rc != XORENC_OK) return rc;
  if (ldx < cols || ldr < cols) return XORENC_EINVAL;
  if (tokens == 0) return XORENC_OK;
  if (!X || !places || !used || !R) return XORENC_EINVAL;
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(X, esz) || !aligned_to(R, esz) || !aligned_to(places, 4) || !aligned_to(used, 4) || !aligned_to(shares, 4)) return XORENC_EALIGN;
  const RowArgs g = {places, used, shares, ldx, ldr, 0, tokens, picks, cols, (cols + 7) / 8};
  const dim3 grid((unsigned)(((int64_t)tokens * g.per_row + 255) / 256));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return for_rows(x_dtype, streams((int64_t)tokens * (picks + 1), cols, esz), [&](auto type, auto stream) {
    typedef decltype(type) T;
    typedef typename T::Elem E;
    constexpr bool STREAM = decltype(stream)::value;
    if (shares)
      hipLaunchKernelGGL((gather_kernel<T, true, STREAM>), grid, dim3(256), 0, st, static_cast<const E *>(X), g, static_cast<E *>(R));
    else
      hipLaunchKernelGGL((gather_kernel<T, false, STREAM>), grid, dim3(256), 0, st, static_cast<const E *>(X), g, static_cast<E *>(R));
    return xorenc_internal_check_launch();
  });
}

extern "C" int32_t xorenc_combine_tokens(const void *R, int32_t x_dtype, int64_t ldr, const int32_t *places, const int32_t *used,
                                         const float *shares, const void *residual, int64_t ld_residual, int32_t tokens, int32_t picks, int32_t cols,
                                         void *Y, int64_t ldy, void *hip_stream) {
  const int32_t rc = check_rows(x_dtype, tokens, picks, cols);
  if (rc != XORENC_OK) return rc;
  if (ldr < cols || ldy < cols || (residual && ld_residual < cols) || (residual && residual == Y && ld_residual != ldy && tokens > 1)) return XORENC_EINVAL;
  if (tokens == 0) return XORENC_OK;
  if (!R || !places || !used || !Y) return XORENC_EINVAL;
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(R, esz) || !aligned_to(Y, esz) || !aligned_to(residual, esz) || !aligned_to(places, 4) || !aligned_to(used, 4) ||
      !aligned_to(shares, 4))
    return XORENC_EALIGN;
  const RowArgs g = {places, used, shares, ld_residual, ldr, ldy, tokens, picks, cols, (cols + 7) / 8};
  const dim3 grid((unsigned)(((int64_t)tokens * g.per_row + 255) / 256));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return for_rows(x_dtype, streams((int64_t)tokens * (picks + 1 + (residual != nullptr)), cols, esz), [&](auto type, auto stream) {
    typedef decltype(type) T;
    typedef typename T::Elem E;
    auto launch = [&](auto most) {
      hipLaunchKernelGGL((combine_kernel<T, decltype(most)::value, decltype(stream)::value>), grid, dim3(256), 0, st, static_cast<const E *>(R), g,
                         static_cast<const E *>(residual), static_cast<E *>(Y));
    };
    if (picks <= 2)
      launch(std::integral_constant<int, 2>());
    else if (picks <= 4)
      launch(std::integral_constant<int, 4>());
    else
      launch(std::integral_constant<int, 8>());
    return xorenc_internal_check_launch();
  });
}

extern "C" int32_t xorenc_combine_tokens_grad(const void *dY, int32_t x_dtype, int64_t ldy, const void *R, int64_t ldr, const int32_t *places,
                                              const int32_t *used, const float *shares, int32_t tokens, int32_t picks, int32_t cols, void *dR,
                                              int64_t lddr, float *dshares, void *hip_stream) {
  const int32_t rc = check_rows(x_dtype, tokens, picks, cols);
  if (rc != XORENC_OK) return rc;
  if (ldy < cols || ldr < cols || lddr < cols || (dR == R && lddr != ldr)) return XORENC_EINVAL;
  if (tokens == 0) return XORENC_OK;
  if (!dY || !R || !places || !used || !shares || !dR || !dshares) return XORENC_EINVAL;
  const int esz = dtype_bytes(x_dtype);
  if (!aligned_to(dY, esz) || !aligned_to(R, esz) || !aligned_to(dR, esz) || !aligned_to(places, 4) || !aligned_to(used, 4) ||
      !aligned_to(shares, 4) || !aligned_to(dshares, 4))
    return XORENC_EALIGN;
  const RowArgs g = {places, used, shares, ldy, ldr, lddr, tokens, picks, cols, 0};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  xorenc_internal_begin_call();
  return for_rows(x_dtype, streams((int64_t)tokens * (2 * picks + 1), cols, esz), [&](auto type, auto stream) {
    typedef decltype(type) T;
    typedef typename T::Elem E;
    auto launch = [&](auto threads, auto most) {
      constexpr int THREADS = decltype(threads)::value;
      hipLaunchKernelGGL((combine_grad_kernel<T, THREADS, decltype(most)::value, decltype(stream)::value>), dim3((unsigned)tokens), dim3(THREADS), 0, st,
                         static_cast<const E *>(dY), g, static_cast<const E *>(R), static_cast<E *>(dR), dshares);
    };
    auto by_picks = [&](auto threads) {
      if (picks <= 2)
        launch(threads, std::integral_constant<int, 2>());
      else if (picks <= 4)
        launch(threads, std::integral_constant<int, 4>());
      else if (picks <= 8)
        launch(threads, std::integral_constant<int, 8>());
      else
        launch(threads, std::integral_constant<int, 16>());
    };
    if (cols <= 512)
      by_picks(std::integral_constant<int, 64>());
    else
      by_picks(std::integral_constant<int, 256>());
    return xorenc_internal_check_launch();
  });
}
