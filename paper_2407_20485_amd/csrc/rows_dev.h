// Rows of fp32 or bf16 elements, eight at a time, and their 8-bit form.
//
// 8-bit rows: e4m3 values (three bits behind the leading one, largest 448) and a scale per 128 columns, a power of two held as
// its exponent plus 127 in a byte (255: not a number).  The scale is the smallest that brings the block's largest magnitude to
// 448 or below.  A power of two costs the values no precision, unlike a quotient it is exact, and it is what the matrix
// instruction takes as its scale operand, so that a product needs no multiplication of its own for it.
#pragma once
#include "a2sf_dev.h"

namespace a2sf {

constexpr int kBlock = 128;           // columns under one scale
constexpr int kUnit = 8;              // consecutive elements a lane holds: 16 lanes (a DPP row) hold a block
constexpr uint32_t kNoScale = 255;    // the block holds an infinity or a NaN

// Sixteen bytes at an address that only an element's alignment is known of (rows of odd strides): the same single
// instruction as an aligned access, which the memory system splits where it has to.
typedef u32x4_t u32x4_at2_t __attribute__((aligned(2)));
typedef u32x4_t u32x4_at4_t __attribute__((aligned(4)));

__device__ __forceinline__ void load_unit(const bf16_t* p, float* f) {
  const u32x4_t r = *(const u32x4_at2_t*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(r[i] << 16);
    f[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load_unit(const float* p, float* f) {
  const u32x4_t a = *(const u32x4_at4_t*)p, b = *(const u32x4_at4_t*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = __uint_as_float(a[i]);
    f[4 + i] = __uint_as_float(b[i]);
  }
}
__device__ __forceinline__ float load_one(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load_one(const float* p) { return *p; }
// the first `have` elements (0 .. 8), zeros behind them
template <typename T>
__device__ __forceinline__ void load_unit(const T* p, int have, float* f) {
  if (have >= kUnit) {
    load_unit(p, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < kUnit; ++i) f[i] = i < have ? load_one(p + i) : 0.f;
}

__device__ __forceinline__ void store_unit(bf16_t* p, const float* f) {
  u32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  *(u32x4_at2_t*)p = r;
}
__device__ __forceinline__ void store_unit(float* p, const float* f) {
  u32x4_t a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = __float_as_uint(f[i]);
    b[i] = __float_as_uint(f[4 + i]);
  }
  *(u32x4_at4_t*)p = a;
  *(u32x4_at4_t*)(p + 4) = b;
}
__device__ __forceinline__ void store_one(bf16_t* p, float x) { *p = (bf16_t)pack_bf16(x, x); }
__device__ __forceinline__ void store_one(float* p, float x) { *p = x; }
template <typename T>
__device__ __forceinline__ void store_unit(T* p, int have, const float* f) {
  if (have >= kUnit) {
    store_unit(p, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < kUnit; ++i)
    if (i < have) store_one(p + i, f[i]);
}

// Largest magnitude of eight values as its bits: as whole numbers they are ordered like the magnitudes, with infinity
// above the finite ones and NaN above that, so neither is lost in a maximum.
__device__ __forceinline__ uint32_t unit_top(const float* f) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
  return top;
}
// ... over the 16 lanes that hold a block
__device__ __forceinline__ uint32_t block_top(uint32_t top) {
  top = max(top, dpp_move_u32<0xB1>(top));
  top = max(top, dpp_move_u32<0x4E>(top));
  top = max(top, dpp_move_u32<0x141>(top));
  return max(top, dpp_move_u32<0x140>(top));
}
// The byte b of the smallest scale 2^(b - 127), b >= 0, with top <= 448 * 2^(b - 127): 448 = 1.75 * 2^8
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return kNoScale;
  const int b = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
  return (uint32_t)max(b, 0);
}
// Eight values in 8 bits under that scale: rounded to the nearest, ties to even, once.  The reciprocal scale is exact and
// the product below 448 + half a step, so the conversion never overflows.
__device__ __forceinline__ uint2 to_eight_bits(const float* f, uint32_t byte) {
  if (byte == kNoScale) return make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
  const float inv = __uint_as_float((254u - byte) << 23);
  uint32_t lo = 0, hi = 0;
  lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inv, f[1] * inv, (int)lo, false);
  lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inv, f[3] * inv, (int)lo, true);
  hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4] * inv, f[5] * inv, (int)hi, false);
  hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[6] * inv, f[7] * inv, (int)hi, true);
  return make_uint2(lo, hi);
}
// 8-bit rows start at multiples of 16 bytes, so a unit's eight bytes are aligned
__device__ __forceinline__ void store_eight_bits(uint8_t* p, int have, uint2 v) {
  if (have >= kUnit) {
    *(uint2*)p = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < kUnit; ++i)
    if (i < have) p[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
}

}  // namespace a2sf
