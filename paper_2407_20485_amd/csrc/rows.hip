// Row operators of a decoder layer: residual sum with root-mean-square norm, and conversion to 8-bit rows (of rows, of
// silu(gate) * rows, of weights).  All read and write each element once and are bound by memory.
#include <type_traits>

#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

__device__ __forceinline__ double wave_sum_f64(double v) {
  const auto halves = [](double x) { return __builtin_bit_cast(unsigned long long, x); };
  const auto whole = [](uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo); };
  const auto add = [&](auto move) {
    const unsigned long long x = halves(v);
    v += whole(move((uint32_t)x), move((uint32_t)(x >> 32)));
  };
  add([](uint32_t x) { return dpp_move_u32<0xB1>(x); });
  add([](uint32_t x) { return dpp_move_u32<0x4E>(x); });
  add([](uint32_t x) { return dpp_move_u32<0x141>(x); });
  add([](uint32_t x) { return dpp_move_u32<0x140>(x); });
  unsigned long long x = halves(v);
  u32x2_t lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  u32x2_t hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(x >> 32), false, false);
  v = whole(lo[0], hi[0]) + whole(lo[1], hi[1]);
  x = halves(v);
  lo = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  hi = __builtin_amdgcn_permlane32_swap((uint32_t)(x >> 32), (uint32_t)(x >> 32), false, false);
  return whole(lo[0], hi[0]) + whole(lo[1], hi[1]);
}

// ---- y = h / sqrt(mean(h^2) + eps) * w,  h = x + residual ----------------------------------------------------------------
// A row stays in registers between the sum of its squares and its scaling: V units of eight elements per lane, unit
// i * THREADS + t in lane t, so that 16 neighbouring lanes hold the 128 columns of a scale and the wave's accesses are
// contiguous.  h is formed and squared in fp32; only the stored sum is rounded to the rows' type (the norm is of the sum before that
// rounding, which costs nothing here and is nearer to the definition).  The squares of a unit are added in fp32, the units in 64 bits, and
// h is multiplied with what the roundings of its products cut off: then y is off by about one rounding to 32 bits, and
// next to none of its 8-bit values is another than the definition's.
// Rows whose squares leave the range of fp32 are summed once more in 64 bits (+0.4 us of 113 for the question).
// THREADS = 64: a wave per row, four rows per workgroup, no barrier.
// 16384 x 5120 in bf16 with a residual, its sum and 8-bit rows (588 MB): 113 us = 5.2 TB/s (a copy of 1 GiB: 5.2); 109 without the products' remainders,
// but then one 8-bit value in 1 500 000 goes the other way, now one in 12 000 000.
template <typename T, int THREADS, int V>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void rms_norm_kernel(NormArgs a) {
  constexpr int kRows = THREADS == 64 ? 4 : 1;
  const int t = threadIdx.x % THREADS;
  const long long row = (long long)blockIdx.x * kRows + threadIdx.x / THREADS;
  if (kRows > 1 && row >= a.rows) return;  // whole waves: nothing below waits for them
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* r = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
  float h[V][kUnit];
#pragma unroll
  for (int i = 0; i < V; ++i) load_unit(x + (i * THREADS + t) * kUnit, a.n - (i * THREADS + t) * kUnit, h[i]);
  if (r) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float g[kUnit];
      load_unit(r + (i * THREADS + t) * kUnit, a.n - (i * THREADS + t) * kUnit, g);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) h[i][j] += g[j];
    }
  }
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kUnit; ++j) s = fmaf(h[i][j], h[i][j], s);
    sum += s;
  }
  const auto row_sum = [&](double v, auto once_more) {
    v = wave_sum_f64(v);
    if constexpr (THREADS > 64) {
      __shared__ double part[THREADS / 64];
      if ((t & 63) == 0) part[t >> 6] = v;
      __syncthreads();
      v = 0.0;
      if constexpr (once_more) {
#pragma unroll 1
        for (int w = 0; w < THREADS / 64; ++w) v += part[w];
      } else {
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) v += part[w];
      }
    }
    return v;
  };
  double mean = row_sum(sum, std::false_type()) / a.n + a.eps;
  T* total = a.total ? (T*)a.total + row * a.total_stride : nullptr;
  double by = 1.0;  // what h was multiplied with
  if (!(mean < 0x1p128) || mean < 0x1p-100) {
    // Squares above the range of 32 bits, or so many under its normal numbers that their sum counts (the whole row sees the same mean): again in
    // 64 bits, and h by a power of two into the middle of the range, where the factor is a normal number too.  (The parts one by one: the
    // registers for all at once would cost every row a wave in eight: 7000 x 10000 bf16 107 us, so 99.)
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < kUnit; ++j) sum += (double)h[i][j] * h[i][j];
    if constexpr (THREADS > 64) __syncthreads();  // (the first sum's parts are read)
    mean = row_sum(sum, std::true_type()) / a.n + a.eps;
    by = mean < 1.0 ? 0x1p100 : 0x1p-64;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * THREADS + t) * kUnit;
      if (total && c < a.n) store_unit(total + c, a.n - c, h[i]);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) h[i][j] *= (float)by;
    }
    total = nullptr;
  }
  const double factor = 1.0 / sqrt(mean) / by;
  const float scale = (float)factor, rest = (float)(factor - scale);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * THREADS + t) * kUnit;
    const int have = a.n - c;
    // the 16 lanes of a block that ends inside it stay together: the exchange below reads all of them
    if ((c & ~(kBlock - 1)) >= a.n) break;
    if (total && have > 0) store_unit(total + c, have, h[i]);
    float w[kUnit];
    load_unit((const T*)a.weight + c, have, w);
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const float p = h[i][j] * scale, y = p * w[j];
      // (not a number where y is infinite: which it then stays)
      const float low = fmaxf(fmaf(fmaf(h[i][j], rest, fmaf(h[i][j], scale, -p)), w[j], fmaf(p, w[j], -y)), -3.402823466e38f);
      h[i][j] = y + low;
      w[j] = low - (h[i][j] - y);  // what this addition cut off
    }
    if (have < kUnit) {
      // columns past the end are 0 also where the row's scale is not a number
#pragma unroll
      for (int j = 0; j < kUnit; ++j) h[i][j] = j < have ? h[i][j] : 0.f;
    }
    if (sizeof(T) == 4 && a.out && have > 0) store_unit((T*)a.out + row * a.out_stride + c, have, h[i]);
    // What is rounded once more is cut off at 32 bits, and its last bit set if anything was: then it does not look like half-way between
    // two neighbours where it is not.
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const int bits = __float_as_int(h[i][j]);
      h[i][j] = fabsf(w[j]) > 0.f ? __int_as_float((bits + ((__float_as_int(w[j]) ^ bits) >> 31)) | 1) : h[i][j];
    }
    if (sizeof(T) == 2 && a.out && have > 0) store_unit((T*)a.out + row * a.out_stride + c, have, h[i]);
    if (a.q) {
      const uint32_t b = scale_byte(block_top(unit_top(h[i])));
      if (have > 0) store_eight_bits(a.q + row * a.q_stride + c, have, to_eight_bits(h[i], b));
      if ((t & 15) == 0) a.scales[row * a.scale_stride + c / kBlock] = (uint8_t)b;
    }
  }
}

template <typename T, int THREADS, int V>
bool norm(const NormArgs& a, hipStream_t st) {
  constexpr int kRows = THREADS == 64 ? 4 : 1, kLanes = THREADS == 64 ? 256 : THREADS;
  const uint32_t groups = ((uint32_t)a.rows + kRows - 1) / kRows;
  if (!grid_fits(groups, kLanes)) return false;
  rms_norm_kernel<T, THREADS, V><<<dim3(groups), dim3(kLanes), 0, st>>>(a);
  return true;
}
template <typename T, int THREADS>
bool norm_units(const NormArgs& a, hipStream_t st) {
  const int v = (a.n + THREADS * kUnit - 1) / (THREADS * kUnit);
  if (v <= 1) return norm<T, THREADS, 1>(a, st);
  if (v <= 2) return norm<T, THREADS, 2>(a, st);
  if constexpr (THREADS == 256 || THREADS == 512) {  // (no more units than three)
    return norm<T, THREADS, 3>(a, st);
  } else {
    if (v <= 3) return norm<T, THREADS, 3>(a, st);
    if (v <= 4 || THREADS == 64) return norm<T, THREADS, 4>(a, st);
    if constexpr (THREADS == 1024) return norm<T, THREADS, 8>(a, st);
  }
}
template <typename T>
bool norm_type(const NormArgs& a, hipStream_t st) {
  // A wave per row needs no barrier; of 16 bits also where it has four units (16384 x 1280: 31 us, by 256 lanes 40; fp32 47 and 44)
  if (a.n <= 2 * 64 * kUnit || (sizeof(T) == 2 && a.rows >= 4096 && a.n <= 4 * 64 * kUnit)) return norm_units<T, 64>(a, st);
  if (a.rows < 512 && a.n > 256 * kUnit) {
    // few rows: the time is a chain of round trips, the more lanes the shorter
    if (a.n <= 512 * kUnit) return norm<T, 512, 1>(a, st);
    return norm_units<T, 1024>(a, st);
  }
  // two or three units per lane (7000 x 10000: 98 us by 512 lanes, 120 by 256 with six units; 16384 x 4096: 88 by 256, 99 by 512 with one)
  if (a.n <= 3 * 256 * kUnit) return norm_units<T, 256>(a, st);
  if (a.n <= 3 * 512 * kUnit) return norm_units<T, 512>(a, st);
  return norm_units<T, 1024>(a, st);
}

// g / (1 + exp(-g)).  exp2 of the rounded product g log2(e) alone would be off by |g| units of rounding: what the product's rounding and the
// constant's have cut off comes back as a factor 1 + rest ln(2) (7001 x 11008 in bf16: 68.1 us without it, 68.5 with it).  With the last bits of
// v_exp_f32 and v_rcp_f32 the result is within 12 * 2^-24 of its size; below -87, where the reciprocal is no normal number any more, it is 0.
__device__ __forceinline__ float silu(float g) {
  constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147181f;
  const float a = fminf(g, 200.f);  // (so that the rest of infinity is a number; exp(-200) is 0)
  const float t = a * -kLog2e, rest = fmaf(a, -kLog2eRest, fmaf(a, -kLog2e, -t));
  const float e = __builtin_amdgcn_exp2f(t) * fmaf(rest, kLn2, 1.f);  // (infinity below -89: the factor is never 0)
  return g * __builtin_amdgcn_rcpf(1.f + e);
}

// ---- rows or silu(gate) * rows, to the rows' type and / or to 8 bits -------------------------------------------------------
// 16 lanes take a block of 128 columns.  7001 x 11008 in bf16 with a gate to 8-bit rows (386 MB): 68.5 us = 5.6 TB/s, 74 if the gate is fetched
// after x has arrived.
template <typename T, bool GATE>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a) {
  const uint32_t block = blockIdx.x * 16u + threadIdx.x / 16;
  const uint32_t row = block / (uint32_t)a.blocks_per_row;
  if (row >= (uint32_t)a.rows) return;  // all 16 lanes of a block
  const int c = (int)(block - row * (uint32_t)a.blocks_per_row) * kBlock + (threadIdx.x & 15) * kUnit;
  const int have = a.n - c;
  float f[kUnit], g[kUnit];
  const T* x = (const T*)a.x + (long long)row * a.x_stride + c;
  const T* gate = (const T*)a.gate + (long long)row * a.gate_stride + c;
  if (have >= kUnit) {  // (both on their way before the first is waited for)
    load_unit(x, f);
    if constexpr (GATE) load_unit(gate, g);
  } else {
    load_unit(x, have, f);
    if constexpr (GATE) load_unit(gate, have, g);
  }
  if constexpr (GATE) {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) f[j] = silu(g[j]) * f[j];
  }
  if (a.out && have > 0) store_unit((T*)a.out + (long long)row * a.out_stride + c, have, f);
  if (a.q) {
    const uint32_t b = scale_byte(block_top(unit_top(f)));
    if (have > 0) store_eight_bits(a.q + (long long)row * a.q_stride + c, have, to_eight_bits(f, b));
    if ((threadIdx.x & 15) == 0) a.scales[(long long)row * a.scale_stride + c / kBlock] = (uint8_t)b;
  }
}

// ---- weights: a scale per 128 x 128 ------------------------------------------------------------------------------------------
// A workgroup per tile, 16 rows of it per step; the tile stays in registers (64 values per lane) between its maximum and its conversion, so that
// it is read once.  Bound by memory: 12288 x 4096 bf16 (151 MB) 31 us = 4.8 TB/s, 32000 x 4096 77 = 5.1; fp32 43 and 113 = 5.8.
template <typename T>
__global__ __launch_bounds__(256) void quantize_weight_kernel(QuantArgs a) {
  const int r0 = (int)(blockIdx.x / (uint32_t)a.blocks_per_row) * kBlock;
  const int c = (int)(blockIdx.x % (uint32_t)a.blocks_per_row) * kBlock + (threadIdx.x & 15) * kUnit;
  const int have = a.n - c;
  float f[kBlock / 16][kUnit];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kBlock / 16; ++i) {
    const int row = r0 + i * 16 + threadIdx.x / 16;
    load_unit((const T*)a.x + (long long)row * a.x_stride + c, row < a.rows ? have : 0, f[i]);
    top = max(top, unit_top(f[i]));
  }
  top = block_top(top);
  __shared__ uint32_t part[16];
  if ((threadIdx.x & 15) == 0) part[threadIdx.x / 16] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, part[i]);
  const uint32_t b = scale_byte(top);
#pragma unroll
  for (int i = 0; i < kBlock / 16; ++i) {
    const int row = r0 + i * 16 + threadIdx.x / 16;
    if (row < a.rows && have > 0)
      store_eight_bits(a.q + (long long)row * a.q_stride + c, have, to_eight_bits(f[i], b));
  }
  if (threadIdx.x == 0) a.scales[(long long)(r0 / kBlock) * a.scale_stride + c / kBlock] = (uint8_t)b;
}

}  // namespace

bool launch_rms_norm(const NormArgs& a, int dtype, hipStream_t st) {
  return dtype == A2SF_F32 ? norm_type<float>(a, st) : norm_type<bf16_t>(a, st);
}

bool launch_quantize(const QuantArgs& a, int dtype, hipStream_t st) {
  const dim3 grid((uint32_t)(((long long)a.rows * a.blocks_per_row + 15) / 16));
  if (!grid_fits(grid.x, 256)) return false;
  if (dtype == A2SF_F32) {
    if (a.gate) quantize_kernel<float, true><<<grid, 256, 0, st>>>(a);
    else quantize_kernel<float, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (a.gate) quantize_kernel<bf16_t, true><<<grid, 256, 0, st>>>(a);
    else quantize_kernel<bf16_t, false><<<grid, 256, 0, st>>>(a);
  }
  return true;
}

bool launch_quantize_weight(const QuantArgs& a, int dtype, hipStream_t st) {
  const dim3 grid((uint32_t)((a.rows + kBlock - 1) / kBlock) * (uint32_t)a.blocks_per_row);
  if (!grid_fits(grid.x, 256)) return false;
  if (dtype == A2SF_F32) quantize_weight_kernel<float><<<grid, 256, 0, st>>>(a);
  else quantize_weight_kernel<bf16_t><<<grid, 256, 0, st>>>(a);
  return true;
}

}  // namespace a2sf
