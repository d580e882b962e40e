// Shared by the kernels for dense layers in 8 bits: e4m3 values (sign, 4 bits of exponent, 3 of mantissa, largest 448, no
// infinities) with one fp32 scale for each block of 128 columns.
#ifndef XORENC_FP8_H
#define XORENC_FP8_H

#include <type_traits>

#include <hip/hip_runtime.h>

#include "xorenc_internal.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

namespace xorenc_fp8_detail {

constexpr int kBlock = XORENC_FP8_BLOCK;
constexpr float kE4m3Most = 448.f;
constexpr float kLeastScale = 1.1754943508222875e-38f;  // 2^-126: its reciprocal is finite

// The scale of a block from the bits of its largest magnitude (taken as integers, so that infinities and NaN come through).
__device__ inline float block_scale(uint32_t amax_bits) {
  const float s = __uint_as_float(amax_bits) / kE4m3Most;
  return s < kLeastScale ? kLeastScale : s;
}

__device__ inline uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Four fp32 values as e4m3, nearest-even.
__device__ inline uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// x / (1 + exp(-x)).  The exponential's argument is rounded in base 2, and so is its constant: 7.5e-8 |x| of relative error beside those
// of two instructions, 1.2e-7 each.  The reciprocal is taken of a sixteenth, where it is a normal number (the instruction
// gives 0 for others) up to exp(-x) = 2^128; from there on the result is -0.
__device__ inline float silu(float x) {
  const float e = __builtin_amdgcn_exp2f(x * -1.44269504f);
  return x * (__builtin_amdgcn_rcpf(fmaf(e, 0.0625f, 0.0625f)) * 0.0625f);
}

// fp32 -> bf16, nearest-even (the compiler takes the conversion instruction; NaN stays NaN)
__device__ inline uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ inline uint32_t to_bf16x2(float a, float b) { return (uint32_t)to_bf16(a) | ((uint32_t)to_bf16(b) << 16); }

// Rows may start on any element: 16 bytes are loaded and stored wherever they start.
typedef f32x4 f32x4_anywhere __attribute__((aligned(4)));
typedef u32x4 u32x4_anywhere __attribute__((aligned(2)));

struct F32 {
  typedef float Elem;
  struct Raw {  // eight elements
    f32x4 a, b;
  };
  template <bool STREAM>
  static __device__ inline Raw load8(const Elem *p) {
    const f32x4_anywhere *const q = reinterpret_cast<const f32x4_anywhere *>(p);
    if constexpr (STREAM) return {__builtin_nontemporal_load(q), __builtin_nontemporal_load(q + 1)};
    return {q[0], q[1]};
  }
  static __device__ inline Raw first_of(const Elem *p, int n) {  // those from the n-th on are zero
    Raw r = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll 1
    for (int k = n - 1; k >= 0; --k) r.b = f32x4{r.a[3], r.b[0], r.b[1], r.b[2]}, r.a = f32x4{p[k], r.a[0], r.a[1], r.a[2]};
    return r;
  }
  static __device__ inline void widen(const Raw &r, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r.a[i], v[4 + i] = r.b[i];
  }
  static __device__ inline void store(Elem *p, float v) { *p = v; }
  static __device__ inline void store8(Elem *p, const float *v) {
    *reinterpret_cast<f32x4_anywhere *>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_anywhere *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};

struct BF16 {
  typedef uint16_t Elem;
  typedef u32x4 Raw;
  template <bool STREAM>
  static __device__ inline Raw load8(const Elem *p) {
    const u32x4_anywhere *const q = reinterpret_cast<const u32x4_anywhere *>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(q);
    return *q;
  }
  static __device__ inline Raw first_of(const Elem *p, int n) {
    Raw r = {0u, 0u, 0u, 0u};
#pragma unroll 1
    for (int k = n - 1; k >= 0; --k)
      r = Raw{r[0] << 16 | p[k], r[1] << 16 | r[0] >> 16, r[2] << 16 | r[1] >> 16, r[3] << 16 | r[2] >> 16};
    return r;
  }
  static __device__ inline void widen(const Raw &r, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(r[i]), v[2 * i + 1] = bf16_hi(r[i]);
  }
  static __device__ inline void store(Elem *p, float v) { *p = to_bf16(v); }
  static __device__ inline void store8(Elem *p, const float *v) {
    *reinterpret_cast<u32x4_anywhere *>(p) =
        u32x4{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7])};
  }
};

// Eight values of a row from column c on; columns from `cols` on are zero.  The load comes first, without a branch (so that
// several are on their way together), and takes the row's last eight elements where fewer are left behind c; the values
// come from it (piece_of).  STREAM: they are not kept in caches.  whole (a constant): c + 8 <= cols is known.
template <class T, bool STREAM = false>
__device__ inline typename T::Raw load_piece(const typename T::Elem *row, int c, int cols, bool whole = false) {
  if (whole) return T::template load8<STREAM>(row + c);
  return cols >= 8 ? T::template load8<STREAM>(row + min(c, cols - 8)) : T::first_of(row, c ? 0 : cols);
}

// Stores of a row's end are short loops, not straight code: a kernel that few waves run waits for its code.
__device__ inline void shift_down(float *v) {
#pragma unroll
  for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
  v[7] = 0.f;
}

// The values of such a load.  brief (a constant): in short code, which takes longer at a row's end.
template <class T>
__device__ inline void piece_of(const typename T::Raw &raw, int c, int cols, float *v, bool whole = false, bool brief = false) {
  T::widen(raw, v);
  const int off = c + 8 - cols;  // elements before column c
  if (!whole && off > 0 && cols >= 8) {
    if (brief) {
#pragma unroll 1
      for (int k = off & 7; k > 0; --k) shift_down(v);
    } else {
#pragma unroll
      for (int d = 1; d < 8; d *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = off & d ? (i + d < 8 ? v[i + d] : 0.f) : v[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = off >= 8 ? 0.f : v[i];
  }
}

template <class T>
__device__ inline void store_piece(typename T::Elem *row, int c, int cols, const float *v, bool whole = false) {
  if (whole || c + 8 <= cols) {
    T::store8(row + c, v);
  } else {
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = v[i];
#pragma unroll 1
    for (; c < cols; ++c) {
      T::store(row + c, u[0]);
      shift_down(u);
    }
  }
}

// Eight values as e4m3 to row[c ..].  Rows of Q start on 16-byte boundaries and c is a multiple of eight.
template <bool STREAM = false>
__device__ inline void store_e4m3_piece(uint8_t *row, int c, int cols, const float *v, float inv, bool whole = false) {
  const u32x2 w = {pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                   pack_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
  if (whole || c + 8 <= cols) {
    if constexpr (STREAM)
      __builtin_nontemporal_store(w, reinterpret_cast<u32x2 *>(row + c));
    else
      *reinterpret_cast<u32x2 *>(row + c) = w;
  } else {
    uint64_t left = __builtin_bit_cast(uint64_t, w);
#pragma unroll 1
    for (; c < cols; ++c, left >>= 8) row[c] = (uint8_t)left;
  }
}

// Largest of 16 neighbouring lanes' values, on all of them: a row of the DPP network.
__device__ inline uint32_t max_of_16_lanes(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));   // quad: 1 0 3 2
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));   // quad: 2 3 0 1
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // half row mirrored
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));  // row mirrored
  return v;
}

// Sum of 16 neighbouring lanes' values, or of a wave's, on all of them: the same tree wherever they are.
__device__ inline float sum_of_16_lanes(float v) {
  auto moved = [&](auto pattern) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(pattern)::value, 0xf, 0xf, true));
  };
  v += moved(std::integral_constant<int, 0xB1>());
  v += moved(std::integral_constant<int, 0x4E>());
  v += moved(std::integral_constant<int, 0x141>());
  return v + moved(std::integral_constant<int, 0x140>());
}
__device__ inline float sum_of_wave(float v) {
  v = sum_of_16_lanes(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// What a row's last 16-byte piece holds behind its last column, `left` bytes from its start (1 .. 15): zero.
__device__ inline u32x4 first_bytes(u32x4 v, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = left - 4 * i;
    v[i] = n >= 4 ? v[i] : n <= 0 ? 0u : v[i] & ((1u << (8 * n)) - 1u);
  }
  return v;
}

// Loads from memory to LDS: lane l's 16 (4) bytes at descriptor + off + more go to to + 16 l (4 l).  The compiler does not know
// of them: who reads the LDS waits for them with s_waitcnt vmcnt, as many later ones left out as it knows of.  Nor does it look
// after the wait states that such a load needs: one behind the instruction that writes m0, and five behind a vector instruction
// that writes a scalar register it reads (the descriptor, `more`: v_readfirstlane, or one that the compiler restores from a vector
// register).  s_mov and s_nop 3 are five (64 x 16384 x 4096 14.5 us; with s_nop 0, for m0 alone, 14.3).
constexpr uint32_t kRawBuffer = 0x00020000u;    // descriptor word 3: untyped data
constexpr uint32_t kBeyond = 0x80000000u;       // an offset past every descriptor's extent: reads as zero, from nowhere
constexpr int64_t kMostTileBytes = 0x7fffff00;  // extent of the descriptors
__device__ inline u32x4 descriptor(const void *p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)), (uint32_t)kMostTileBytes, kRawBuffer};
}
template <bool STREAM = false>
__device__ inline void fetch_16(uint32_t to, uint32_t off, const u32x4 &desc, uint32_t more) {
  if constexpr (STREAM)  // not kept in caches
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off),
                 "s"(desc), "s"(__builtin_amdgcn_readfirstlane(more))
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off),
                 "s"(desc), "s"(__builtin_amdgcn_readfirstlane(more))
                 : "memory", "m0");
}
__device__ inline void fetch_4(uint32_t to, uint32_t off, const u32x4 &desc, uint32_t more) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off),
               "s"(desc), "s"(__builtin_amdgcn_readfirstlane(more))
               : "memory", "m0");
}
__device__ inline uint32_t lds_address(const void *p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) const uint8_t *)p);
}

// Rows of e4m3 in LDS: 128 bytes each, a row's 16-byte chunks at chunk ^ (row / 2 % 8), so that the 16 rows of an operand read
// spread over all banks.  A load of eight rows: lane l takes row l / 8 of them, and this chunk of it.
__device__ inline int e4m3_chunk(int lane, int row) { return (lane & 7) ^ ((row >> 1) & 7); }
__device__ inline uint32_t e4m3_operand_offset(int lane) {  // of the first piece, in 16 rows; the second's is this ^ 64
  return (uint32_t)((lane & 15) * 128 + (((lane >> 4) ^ (((lane & 15) >> 1) & 7)) * 16));
}

// Operands of the matrix instructions for 128 columns of 16 rows.  Lane l holds 32 values of row l % 16: columns
// 16 (l / 16) + 0..15 of the first 64 columns (piece 0), then of the second 64 (piece 1).  Which of the instruction's k a column
// becomes does not matter as long as both operands agree.
struct E4m3Operand {
  u32x4 piece[2];
};

__device__ inline E4m3Operand read_operand(const uint8_t *rows, uint32_t offset) {
  E4m3Operand o;
  o.piece[0] = *reinterpret_cast<const u32x4 *>(rows + offset);
  o.piece[1] = *reinterpret_cast<const u32x4 *>(rows + (offset ^ 64u));
  return o;
}

__device__ inline i32x8 as_operand(const E4m3Operand &o) {
  return i32x8{(int)o.piece[0][0], (int)o.piece[0][1], (int)o.piece[0][2], (int)o.piece[0][3],
               (int)o.piece[1][0], (int)o.piece[1][1], (int)o.piece[1][2], (int)o.piece[1][3]};
}

// Quarter q of a lane's 32 values (columns 8 (q % 2) .. + 7 of piece q / 2) as bf16, which holds every e4m3 value exactly.
__device__ inline bf16x8 quarter_as_bf16(const E4m3Operand &o, int q) {
  const uint32_t w0 = o.piece[q >> 1][2 * (q & 1)], w1 = o.piece[q >> 1][2 * (q & 1) + 1];
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The product of 16 rows of A and 16 of B over 128 columns.  Lane l gets column l % 16 (a row of B), rows 4 (l / 16) .. + 3
// (of A).  The 8-bit instruction adds products aligned to the largest of them, some 14 bits below it: 1.5e-5 of the result for
// Gaussian values (2-norm), less than results of 16 bits are rounded by, unless a block's products cancel to far less than the largest of them.
// Results of 32 bits come from the bf16 instruction, which multiplies e4m3 values exactly and adds in fp32, at half the rate.
template <bool EXACT>
__device__ inline f32x4 product_128(const E4m3Operand &a, const E4m3Operand &b) {
  f32x4 d = {0.f, 0.f, 0.f, 0.f};
  if constexpr (EXACT) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(quarter_as_bf16(a, q), quarter_as_bf16(b, q), d, 0, 0, 0);
  } else {
    d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_operand(a), as_operand(b), d, 0, 0, 0, 0, 0, 0);
  }
  return d;
}

// Host checks shared by the entry points.
inline bool known_dtype(int32_t t) { return t == XORENC_X_F32 || t == XORENC_X_BF16; }
inline int dtype_bytes(int32_t t) { return t == XORENC_X_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace xorenc_fp8_detail

#endif
