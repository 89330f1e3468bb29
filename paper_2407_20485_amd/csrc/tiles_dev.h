// Tiles of 64 rows of bf16 in LDS as the prompt kernels use them: the 32 x 32 matrix instruction, plain and transposing reads, swizzles.
#pragma once
#include "a2sf_dev.h"

namespace a2sf {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;  // keys (attn_fwd) or query rows (col_scores) per LDS tile
constexpr int kPrefetch = 4;  // LDS fragment reads in flight ahead of their matrix op

__device__ __forceinline__ f32x16 mfma_bf16(const uint4& a, const uint4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

__device__ __forceinline__ uint2 lds_read_tr16(const lds_char* p) {
  v4i16_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) v4i16_t*)p);
  return __builtin_bit_cast(uint2, r);
}
__device__ __forceinline__ uint4 lds_read16(const lds_char* p) {
  const u32x4_t r = *reinterpret_cast<const __attribute__((address_space(3))) u32x4_t*>(p);
  return make_uint4(r.x, r.y, r.z, r.w);
}

__device__ __forceinline__ void lds_write8(lds_char* p, const uint2& v) {
  const u32x2_t x = {v.x, v.y};
  *reinterpret_cast<__attribute__((address_space(3))) u32x2_t*>(p) = x;
}

// Chunk swizzles (16-byte chunks of a row; the LDS has 64 four-byte banks, i.e. 16 chunks side by
// side: one row of d = 128, two of d = 64).  K and Q are read 16 rows x one chunk column per 16
// lanes: XOR with the row (d = 64: row pair) spreads them over all 16 places.  V is read by 32
// lanes as 4 rows x 4 chunk columns x 2 halves: XOR with 4 * (row % 4) (d = 64: 4 * (row / 2 % 2))
// sends the rows to disjoint groups of four places.  Both measure zero LDS bank conflicts
// (SQ_LDS_BANK_CONFLICT).
template <int D = 128>
__device__ __forceinline__ int k_swizzle(int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); }
template <int D = 128>
__device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }

// Geometry of a tile fetch: a wave's load u fills the rows (4 u + wave) * kRowsPerLoad ..
template <int D> constexpr int kRowsPerLoad = 512 / D;
template <int D> constexpr int kLoadsPerWave = kTile / (4 * kRowsPerLoad<D>);

template <int D, bool V_LAYOUT>
__device__ __forceinline__ void tile_place(int u, int& lrow, int& chunk) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
  lrow = (u * 4 + wave) * kRowsPerLoad<D> + lane / (D / 8);
  chunk = (lane % (D / 8)) ^ (V_LAYOUT ? v_swizzle<D>(lrow) : k_swizzle<D>(lrow));
}

}  // namespace a2sf
