// The 8-bit block cache: formats, scales and addresses shared by the kernels that fill it, extend it,
// read it and prune it.
//
// A block holds 64 tokens of `hb` heads.  K codes lie token by token [64, d]; V codes lie dimension by
// dimension [d, 64]: in the product of probabilities and values a lane owns one dimension and 16
// consecutive tokens, which are then one 16-byte load.  A (block, head) has one scale for K and one for V.
//
// Scales are powers of two, the least one under which the largest magnitude still fits the format.
// Dividing by a power of two is exact, so a code is one rounding of the value (halves to even) whatever
// computes it, and a row that moves to a block of the same or a smaller scale keeps its value exactly.
// What that costs against a scale of amax / 127: half a bit of int8 on average; of e4m3, whose steps are
// relative, nothing.
#pragma once

#include "kvc_internal.h"

namespace kvc {

constexpr int CB_TOKENS = 64;          // tokens of a block
constexpr int CB_SCALE_MIN = -100;     // least exponent of a scale: it and its inverse are normal numbers, and code * scale too

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// What the kernels know of a cache (validated on the host).
struct CacheView {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  float* weight;            // may be null
  const int32_t* table;
  int32_t blocks;           // of the pools: a table entry outside [0, blocks) is never followed
  int32_t width;            // entries of a row of the table
  int32_t hb;               // heads of a block: hkv, or 1 where every head has a row of its own
  int32_t hkv;
  int32_t d;
  int32_t layers;
};

// Row of the table that head h of layer l of sequence b lies in, and the head's place in its blocks.
__device__ __forceinline__ int64_t cache_row(const CacheView& c, int b, int l, int h) {
  const int64_t bl = (int64_t)b * c.layers + l;
  return c.hb == 1 ? bl * c.hkv + h : bl;
}
__device__ __forceinline__ int cache_head(const CacheView& c, int h) { return c.hb == 1 ? 0 : h; }

// Tokens of a row that the table can hold.
__device__ __forceinline__ int cache_length(const CacheView& c, int len) {
  const int64_t most = (int64_t)c.width * CB_TOKENS;
  return len < 0 ? 0 : len > most ? (int)most : len;
}

template <int FMT> struct Code;

template <> struct Code<KVC_E4M3> {
  static constexpr int TOP = 8;                     // 448 = 1.75 * 2^8
  static constexpr uint32_t MANTISSA = 0x600000u;
  // four values in units of their scale -> four codes
  static __device__ __forceinline__ uint32_t encode(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
  static __device__ __forceinline__ void decode(uint32_t w, float (&x)[4]) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  }
  // eight codes as bf16, exactly
  static __device__ __forceinline__ bf16x8_t widen(uint32_t a, uint32_t b) {
    const bf16x2_t p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const bf16x2_t r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
  }
};

template <> struct Code<KVC_INT8> {
  static constexpr int TOP = 6;                     // 127 = 1.984375 * 2^6
  static constexpr uint32_t MANTISSA = 0x7e0000u;
  // x + 1.5 * 2^23 holds the nearest integer, halves to even, in its low bits
  static __device__ __forceinline__ uint32_t byte(float x) { return __float_as_uint(x + 12582912.0f); }
  static __device__ __forceinline__ uint32_t encode(float a, float b, float c, float d) {
    const uint32_t lo = __builtin_amdgcn_perm(byte(b), byte(a), 0x0c0c0400u), hi = __builtin_amdgcn_perm(byte(d), byte(c), 0x0c0c0400u);
    return lo | hi << 16;
  }
  static __device__ __forceinline__ void decode(uint32_t w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
  // whole numbers up to 127 are bf16 exactly: the upper halves of their floats
  static __device__ __forceinline__ uint32_t pair(uint32_t w, int i) {
    const float a = (float)(int8_t)(w >> (8 * i)), b = (float)(int8_t)(w >> (8 * i + 8));
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  }
  // (The words are opaque: else codes that a loop carries from one turn to the next are carried as four
  // registers of one byte each.)
  static __device__ __forceinline__ bf16x8_t widen(uint32_t a, uint32_t b) {
    asm("" : "+v"(a), "+v"(b));
    return __builtin_bit_cast(bf16x8_t, u32x4_t{pair(a, 0), pair(a, 2), pair(b, 0), pair(b, 2)});
  }
};

// Scale of a block whose largest magnitude is amax: the least 2^e, e >= CB_SCALE_MIN, with
// amax <= top * 2^e.  amax = 1.m * 2^x fits x - TOP where its mantissa is at most the format's largest.
template <int FMT>
__device__ __forceinline__ float block_scale(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - Code<FMT>::TOP + ((u & 0x7fffffu) > Code<FMT>::MANTISSA ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, CB_SCALE_MIN) + 127) << 23);
}
// 1 / scale of a power of two
__device__ __forceinline__ float inverse_scale(float scale) {
  return __uint_as_float((254u << 23) - __float_as_uint(scale));
}

// Loads from caller memory, which is only element-aligned (the instructions are the 16-byte ones).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_word __attribute__((ext_vector_type(4), aligned(4)));

// Eight consecutive elements as floats.
template <typename T> struct Row8;
template <> struct Row8<uint16_t> {
  u32x4_any w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p)); }
  __device__ __forceinline__ void clear() { w = u32x4_any{0, 0, 0, 0}; }
  __device__ __forceinline__ void opaque() {
#pragma unroll
    for (int i = 0; i < 4; ++i) { uint32_t x = w[i]; asm("" : "+v"(x)); w[i] = x; }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <> struct Row8<float> {
  u32x4_word w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_word*>(p));
    w[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_word*>(p) + 1);
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = u32x4_word{0, 0, 0, 0}; }
  __device__ __forceinline__ void opaque() {}       // already floats
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = __uint_as_float(w[0][i]); x[4 + i] = __uint_as_float(w[1][i]); }
  }
};

// Maximum over the 64 lanes of a wave.
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 32; off; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

}  // namespace kvc
