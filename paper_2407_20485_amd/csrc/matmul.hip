// C[m, n] = A[m, k] B[n, k]^T of 8-bit floats with power-of-two scales per 128 of k (rows_dev.h): A's for each row, B's for each
// 128 rows.
//
// Two ways to form the sums; the caller chooses:
//  * A bf16 C, unless wider sums are asked for: the 8-bit instructions v_mfma_scale_f32_16x16x128_f8f6f4 (strips) and 32x32x64 (tiles) apply both
//    scales themselves, so the accumulators run through all of k and the vector unit has nothing to do for them (registers only: 4.3 PFLOP/s).
//    Inside them the products of eight neighbours of k are aligned to the largest of them and cut under 2^-13 of it, before they are added in
//    fp32: the sum is off by 8 * 2^-13 of the sum of magnitudes at most, for Gaussian data by 1.5e-5 of the result's size, a hundred times less than
//    the rounding to bf16 (2^-9 on the average).  The 8-bit values themselves are roundings of 2^-4, so what is cut is under 2^-8 of what the largest of
//    the eight products may be off; but for data that 8 bits hold exactly a sum that cancels keeps only 13 bits under its largest term.
//  * An fp32 C, where that cut would be the largest error by far, and a bf16 C with A2SF_WIDE_SUMS: the 8-bit values are made bf16 (which holds them
//    times their scale exactly for scale bytes of 10 to 246: from 2^-9 of the smallest scale, its last normal bit, to 448 of the largest) and multiplied by v_mfma_f32_16x16x32_bf16 or 32x32x16, whose sums are fp32's, at half the rate.
//
// In both the instruction's first operand is B, its second A: its result then has, per lane, four neighbouring columns of C of the
// row lane % 16.  An operand fragment is 16 rows x 128 bytes, 32 bytes per lane, of row lane % 16; which of the 128 they are is the same
// for both operands, and that is all that matters.
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kStep = 128;  // bytes of k per step: a scale block
constexpr int kComputeUnits = 256;
constexpr int kGroup = 4;   // steps whose scales are loaded together: four bytes

struct Scaled {  // the 8-bit instruction
  typedef i32x8_t Fragment;
  static __device__ __forceinline__ Fragment make(i32x8_t v, uint32_t) { return v; }
  static __device__ __forceinline__ f32x4_t mul(const Fragment& b, const Fragment& a, f32x4_t c, uint32_t b_scale, uint32_t a_scale) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, 0, (int)b_scale, 0, (int)a_scale);
  }
  static __device__ __forceinline__ f32x16_t mul(const Fragment& b, const Fragment& a, f32x16_t c, uint32_t b_scale, uint32_t a_scale, int block) {
    // (which byte of the scale operands is part of the instruction)
    switch (block) {
      case 0: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 0, (int)b_scale, 0, (int)a_scale);
      case 1: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 1, (int)b_scale, 1, (int)a_scale);
      case 2: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 2, (int)b_scale, 2, (int)a_scale);
      default: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, c, 0, 0, 3, (int)b_scale, 3, (int)a_scale);
    }
  }
};
struct Exact {  // by way of bf16, the scales applied on the way
  struct Fragment { bf16x8_t part[4]; };
  static __device__ __forceinline__ Fragment make(i32x8_t v, uint32_t scale) {
    const float s = __uint_as_float(scale << 23);  // (the instruction takes its exponent)
    Fragment f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x2_t p[4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        p[2 * j] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i + j], s, false);
        p[2 * j + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i + j], s, true);
      }
      f.part[i] = bf16x8_t{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
    }
    return f;
  }
  static __device__ __forceinline__ f32x4_t mul(const Fragment& b, const Fragment& a, f32x4_t c, uint32_t, uint32_t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.part[i], a.part[i], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x16_t mul(const Fragment& b, const Fragment& a, f32x16_t c, uint32_t, uint32_t, int) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.part[i], a.part[i], c, 0, 0, 0);
    return c;
  }
};
// S, the type that says how sums are formed: bf16_t by the 8-bit instruction, float in 32 bits
template <typename S> struct Way { typedef Scaled type; };
template <> struct Way<float> { typedef Exact type; };

__device__ __forceinline__ i32x8_t join(i32x4_t lo, i32x4_t hi) { return i32x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}; }

// 16 bytes of a row from column k0 on, zeros past column k (there may be anything in memory)
__device__ __forceinline__ i32x4_t load_chunk(const uint8_t* row, int k0, int k) {
  i32x4_t v = {0, 0, 0, 0};
  if (k0 < k) {
    v = *(const i32x4_t*)(row + k0);  // starts inside the row at a multiple of 16: never crosses a page
    const int have = k - k0;
    if (have < 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int bytes = have - 4 * i;
        v[i] = bytes >= 4 ? v[i] : bytes <= 0 ? 0 : v[i] & (int)((1u << (8 * bytes)) - 1u);
      }
    }
  }
  return v;
}

// four neighbouring columns, as far as there are
template <typename T>
__device__ __forceinline__ void store_columns(T* p, int have, f32x4_t v);
template <>
__device__ __forceinline__ void store_columns<bf16_t>(bf16_t* p, int have, f32x4_t v) {
  typedef uint32_t u32x2_at2_t __attribute__((ext_vector_type(2), aligned(2)));
  if (have >= 4) {
    *(u32x2_at2_t*)p = u32x2_at2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < have) store_one(p + i, v[i]);
}
template <>
__device__ __forceinline__ void store_columns<float>(float* p, int have, f32x4_t v) {
  typedef f32x4_t f32x4_at4_t __attribute__((aligned(4)));
  if (have >= 4) {
    *(f32x4_at4_t*)p = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < have) p[i] = v[i];
}

// sixteen bytes of neighbouring columns, as far as there are
template <typename T>
__device__ __forceinline__ void store_bytes(T* p, int have, u32x4_t v) {
  constexpr int kHere = 16 / (int)sizeof(T);
  if (have >= kHere) {
    *(u32x4_at2_t*)p = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < kHere; ++i)
    if (i < have) {
      if constexpr (sizeof(T) == 4) p[i] = __uint_as_float(v[i]);
      else p[i] = (T)(v[i / 2] >> (16 * (i & 1)));
    }
}

// ---- few rows of A: B is streamed once --------------------------------------------------------------------------------------
// A workgroup takes tiles of up to 64 rows (MT times 16) and 16 columns of C, one after the other; its waves share k and add their parts in LDS in a
// fixed order.  Each wave streams its part of k of B and A through a ring of its own in LDS, 128 bytes of each row to a slot, and
// the stream runs on from tile to tile: a wave waits for others at the sums only.
// Bound by the stream of B as long as A is short: a step takes 2 us from its fetch to its arrival, whatever its size, and A's rows
// take their share of the ring.  By way of LDS and not straight into registers, where an operand's lanes, each in another
// row, ask for 16 bytes at a time of 64 places: 48 x 4096 x 11008 33 us, so 12.5; 1 x 4096 x 11008 10.5, so 8.7.
// Where rows of B lie a multiple of 4096 bytes apart, workgroups that all began at the same place of k would all ask the same few of the
// caches' channels: each begins at another one (1 x 12288 x 4096 straight into registers 12.8 us, so 10.3).
// 1 x 12288 x 4096 9.2 us = 5.5 TB/s; 1 x 8192 x 8192 11.4 = 5.9; 32 x 12288 x 4096 10.2 = 4.9; 48 x 4096 x 11008 12.5 = 3.7 (weights that the last-level cache
// holds; from memory 1 x 12288 x 4096 11.2, 48 x 4096 x 11008 17.8).
template <int MT, int WAVES, int ROOM>
struct StripLds {
  static constexpr int kPart = WAVES * MT * 1024;
  static constexpr int kSlot = (1 + MT) * 2048 + 512;  // rows of B, of A; four scales of each of 64 rows of A, and of B
  static constexpr int kSlots = (ROOM - kPart) / WAVES / kSlot;
  static constexpr int kBytes = kPart + WAVES * kSlots * kSlot;
  static constexpr int kLoads = 2 + 2 * MT + 2;  // per step
  static_assert(kSlots >= 2 && (kSlots - 1) * kLoads < 64 && kBytes <= ROOM, "");
};

template <typename S, int MT, int WAVES, int ROOM, typename T>
__global__ __launch_bounds__(WAVES * 64) void matmul_strip_kernel(MatmulArgs g) {
  typedef typename Way<S>::type W;
  typedef StripLds<MT, WAVES, ROOM> L;
  static_assert(MT <= WAVES, "a lane stores one part of a tile at most");
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
  const int strips = (g.n + 15) / 16, tiles = strips * ((g.m + MT * 16 - 1) / (MT * 16)), steps = g.k / kStep;
  const int each = (steps + WAVES - 1) / WAVES, begin = min(wave * each, steps), end = min(begin + each, steps);
  const int mine = ((int)blockIdx.x < tiles ? (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0);
  int total = mine * (end - begin), issue_left = total;  // steps still to multiply, to fetch
  const uint32_t ring = L::kPart + wave * (L::kSlots * L::kSlot);

  // A load takes 8 rows' 128 bytes; chunk c of row r lies at c ^ (r / 2 % 8), so that 16 lanes that read the same chunk of 16 rows
  // meet all banks once.
  const int chunk = (lane & 7) ^ (lane >> 4);
  uint32_t a_off[2 * MT], b_off[2];
  uint32_t scale_off;
  const uint8_t *a_tile, *as_tile, *b_tile, *bs_tile;
  const int start = end > begin ? begin + (int)(blockIdx.x / 8) % (end - begin) : 0;
  int at_tile = blockIdx.x, at_step = start, at_slot = 0;  // of the next fetch
  const auto part_of = [&](int tile) { return tile < strips ? 0 : (int)((unsigned)tile / (unsigned)strips); };
  const auto aim = [&] {
    const int part = part_of(at_tile), strip = at_tile - part * strips, m0 = part * (MT * 16);
#pragma unroll
    for (int u = 0; u < 2; ++u)
      b_off[u] = (uint32_t)min(u * 8 + (lane >> 3), g.n - 1 - strip * 16) * (uint32_t)g.b_stride + (uint32_t)(chunk ^ u * 4) * 16;
#pragma unroll
    for (int u = 0; u < 2 * MT; ++u)
      a_off[u] = (uint32_t)min(u * 8 + (lane >> 3), g.m - 1 - m0) * (uint32_t)g.a_stride + (uint32_t)(chunk ^ (u & 1) * 4) * 16;
    scale_off = (uint32_t)min(lane, g.m - 1 - m0) * (uint32_t)g.a_scale_stride;
    a_tile = g.a + (long long)m0 * g.a_stride;
    as_tile = g.a_scales + (long long)m0 * g.a_scale_stride;
    b_tile = g.b + (long long)strip * 16 * g.b_stride;
    bs_tile = g.b_scales + (long long)(strip / 8) * g.b_scale_stride;
  };
  const auto fetch = [&] {
    const uint32_t to = ring + at_slot * L::kSlot;
    const uint8_t *b = b_tile + at_step * kStep, *a = a_tile + at_step * kStep;
    dma16(b, b_off[0], to);
    dma16(b, b_off[1], to + 1024);
#pragma unroll
    for (int u = 0; u < 2 * MT; ++u) dma16(a, a_off[u], to + 2048 + u * 1024);
    const int group = at_step & ~(kGroup - 1);
    dma4(as_tile + group, scale_off, to + (1 + MT) * 2048);
    dma4(bs_tile + group, 0, to + (1 + MT) * 2048 + 256);
    --issue_left;
    if (++at_slot == L::kSlots) at_slot = 0;
    if (++at_step == end) at_step = begin;
    if (at_step == start) {
      at_tile += gridDim.x;
      if (issue_left > 0) aim();
    }
  };
  const auto barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  if (issue_left > 0) aim();
#pragma unroll 1
  for (int i = 0; i < L::kSlots && issue_left > 0; ++i) fetch();

  const int row = lane & 15, swap = row >> 1 & 7;
  const uint32_t lo = row * 128 + ((lane >> 4) ^ swap) * 16, hi = row * 128 + (((lane >> 4) + 4) ^ swap) * 16;
  int slot = 0;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int part = part_of(tile), strip = tile - part * strips, m0 = part * (MT * 16);
    f32x4_t acc[MT] = {};
    int step = start;
#pragma unroll 1
    for (int i = begin; i < end; ++i) {
      if (total >= L::kSlots) wait_vm<(L::kSlots - 1) * L::kLoads>();
      else wait_vm<0>();
      --total;
      const uint8_t* s = lds + ring + slot * L::kSlot;
      if (++slot == L::kSlots) slot = 0;
      const i32x8_t bv = join(*(const i32x4_t*)(s + lo), *(const i32x4_t*)(s + hi));
      i32x8_t av[MT];
      uint32_t sa[MT];
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        const uint8_t* p = s + (1 + k) * 2048;
        av[k] = join(*(const i32x4_t*)(p + lo), *(const i32x4_t*)(p + hi));
        sa[k] = *(const uint32_t*)(s + (1 + MT) * 2048 + (k * 16 + row) * 4);
      }
      const int by = 8 * (step & (kGroup - 1));
      const uint32_t sb = *(const uint32_t*)(s + (1 + MT) * 2048 + 256) >> by & 255;
      if (++step == end) step = begin;
      wait_lds();
      if (issue_left > 0) fetch();
      const auto fb = W::make(bv, sb);
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        const uint32_t s1 = sa[k] >> by & 255;
        acc[k] = W::mul(fb, W::make(av[k], s1), acc[k], sb, s1);
      }
    }
    if (steps * kStep < g.k && wave == WAVES - 1) {  // the last, partial step: zeros behind the end of k
      const int kl = (lane >> 4) * 16, k0 = steps * kStep, by = 8 * (steps & (kGroup - 1)), group = steps & ~(kGroup - 1);
      const uint8_t* b = g.b + (long long)min(strip * 16 + row, g.n - 1) * g.b_stride + kl;
      const uint32_t sb = *(const uint32_t*)(g.b_scales + (long long)(strip / 8) * g.b_scale_stride + group) >> by & 255;
      const auto fb = W::make(join(load_chunk(b, k0, g.k - kl), load_chunk(b, k0 + 64, g.k - kl)), sb);
#pragma unroll
      for (int k = 0; k < MT; ++k) {
        const long long r = min(m0 + k * 16 + row, g.m - 1);
        const uint8_t* a = g.a + r * g.a_stride + kl;
        const uint32_t s1 = *(const uint32_t*)(g.a_scales + r * g.a_scale_stride + group) >> by & 255;
        acc[k] = W::mul(fb, W::make(join(load_chunk(a, k0, g.k - kl), load_chunk(a, k0 + 64, g.k - kl)), s1), acc[k], sb, s1);
      }
    }
    f32x4_t* left = (f32x4_t*)lds;
#pragma unroll
    for (int k = 0; k < MT; ++k) left[(wave * MT + k) * 64 + lane] = acc[k];
    barrier();
    if (wave < MT) {
      f32x4_t sum = left[t];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum += left[w * MT * 64 + t];
      const int r = m0 + wave * 16 + row, col = strip * 16 + (lane >> 4) * 4;
      if (r < g.m && col < g.n) store_columns((T*)g.c + (long long)r * g.c_stride + col, g.n - col, sum);
    }
    barrier();
  }
}

// ---- tiles of C ----------------------------------------------------------------------------------------------------------------
// BM x BN of C per workgroup of WM x WN waves, by the 32 x 32 instructions.  k goes by half blocks of 64 bytes: a ring of STAGES
// stages in LDS holds a half block of the tile's rows each, filled by loads that go from memory straight into LDS, STAGES - 1
// half blocks ahead.  Persistent: a workgroup goes from tile to tile and the stream of half blocks runs on across them.
//
// Eight waves: the two of a SIMD are half an iteration apart, with a barrier at each half: while one has the matrix pipe, the other
// reads the fragments of its next half block and fetches.  (8192 x 8192 x 8192: all waves in step 490 us, so 461; with a group's half blocks
// written out, which takes the questions about the end of the stream out of them, 440 = 2500 TFLOP/s.  8192 x 22016 x 4096 662 us: matrix pipe busy 54 %
// of the cycles, at 1.96 of 2.4 GHz, which its operands leave; on zeros 2.395 GHz and 599 us.)  Four waves: the next half block's
// fragments are read while this one's are multiplied, and workgroups share a compute unit.
//
// A row of a stage is 64 bytes, four chunks of 16; chunk c of row r lies at c ^ (r / 4 % 4): 16 lanes that read the same chunk of 16
// rows then meet all 64 banks once.  The scales of four blocks of the tile's rows come the same way, a group ahead.  Results go through
// LDS on their way out, so that they leave as 64 neighbouring bytes of a row (as a lane's own 8 bytes: 8192 x 22016 x 4096 707 us, so 675).
constexpr int kHalf = 64;

template <int BM, int BN, int STAGES>
struct TileLds {
  static constexpr int kStage = (BM + BN) * kHalf, kScales = (BM + 64) * 4;
  static constexpr int kRing = 2 * kScales;  // (not at 0: a load's LDS address is formed from one up to 448 bytes lower)
  static constexpr int kOut = kRing + STAGES * kStage;
  static constexpr int kBytes = kOut;  // and 2 KB per wave, through which results leave
};

struct TilePlan {
  int tiles_m, tiles_n;
  int group_m;  // tiles are taken in strips of so many rows of tiles, columns inside a strip first
  int splits;   // parts of k, each a tile of its own
  int groups;   // groups of four blocks per part
  float* partial;  // splits > 1: [splits][m][n]
};

template <int N, typename F, int... U>
__device__ __forceinline__ void with_each(F f, std::integer_sequence<int, U...>) { (f(std::integral_constant<int, U>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void with_each(F f) { with_each<N>(f, std::make_integer_sequence<int, N>()); }

template <typename S, int BM, int BN, int WM, int WN, int STAGES, typename T>
__global__ __launch_bounds__(WM* WN * 64, 2) void matmul_tile_kernel(MatmulArgs g, TilePlan plan) {
  typedef typename Way<S>::type W;
  typedef TileLds<BM, BN, STAGES> L;
  constexpr int kWavesHere = WM * WN, TM = BM / WM, TN = BN / WN, MT = TM / 32, NT = TN / 32;
  constexpr int kUnits = (BM + BN) / 16 / kWavesHere, kUnitsA = BM / 16 / kWavesHere;  // a unit: 16 rows, 1 KB, a load of a wave
  constexpr bool kApart = kWavesHere == 8;
  static_assert(BM % (16 * kWavesHere) == 0 && BN % (16 * kWavesHere) == 0 && BM % 64 == 0 && 128 % TN == 0 && (STAGES == 4 || STAGES == 8), "");
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
  const bool second = kApart && wave >= 4;

  // Workgroups go to the 8 dies in turn: a die works on a contiguous part of the order of tiles, so that what its 32 compute
  // units work on at a time is a block of C whose rows of A and B its L2 holds.
  const unsigned tiles = (unsigned)plan.tiles_m * plan.tiles_n * plan.splits;
  const unsigned dies = min(8u, gridDim.x), die = blockIdx.x % dies, slots = (gridDim.x - die + dies - 1) / dies;
  const unsigned tile_end = (die + 1) * (tiles / dies) + min(die + 1, tiles % dies);
  unsigned tile = die * (tiles / dies) + min(die, tiles % dies) + blockIdx.x / dies;
  if (tile >= tile_end) return;
  struct Place {
    int m0, n0, split, g0, g1, half, end;  // half blocks; end: rounded up to whole turns of the ring
  };
  const int groups = ((g.k + kStep - 1) / kStep + kGroup - 1) / kGroup;
  const auto place = [&](unsigned id) {
    Place p;
    p.split = (int)(id % plan.splits);
    id /= plan.splits;
    const unsigned strip = plan.group_m * plan.tiles_n, first_m = id / strip * plan.group_m;
    const unsigned here = min((unsigned)plan.group_m, plan.tiles_m - first_m);
    const unsigned in = id - id / strip * strip;
    p.m0 = (int)(first_m + in % here) * BM;
    p.n0 = (int)(in / here) * BN;
    p.g0 = p.split * plan.groups;
    p.g1 = min(groups, p.g0 + plan.groups);
    p.half = min((g.k + kHalf - 1) / kHalf - p.g0 * 2 * kGroup, (p.g1 - p.g0) * 2 * kGroup);
    p.end = (p.half + STAGES - 1) / STAGES * STAGES;
    return p;
  };

  // The stream of half blocks: this lane's part of each unit in bytes from the tile's first row, and where the next fetch is
  const uint32_t chunk = (uint32_t)(((lane & 3) ^ (lane >> 4)) * 16);
  uint32_t off[kUnits];
  const uint8_t *a0, *b0;
  Place next;
  unsigned next_tile = tile;
  int next_half = 0;
  bool drained = false;  // a fetch was not by loads into LDS: their count says nothing any more
  const auto aim = [&] {
    next = place(next_tile);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const bool of_a = i < kUnitsA;
      const int r = ((of_a ? i : i - kUnitsA) * kWavesHere + wave) * 16 + lane / 4;
      const int row = of_a ? min(r, g.m - 1 - next.m0) : min(r, g.n - 1 - next.n0);
      off[i] = (uint32_t)row * (uint32_t)(of_a ? g.a_stride : g.b_stride) + chunk;
    }
    a0 = g.a + (long long)next.m0 * g.a_stride + next.g0 * kGroup * kStep;
    b0 = g.b + (long long)next.n0 * g.b_stride + next.g0 * kGroup * kStep;
    next_half = 0;
  };
  const uint32_t lds_wave = (uint32_t)wave * 1024;
  // one more half block of the same tile, `ahead` half blocks from where the stream is
  const auto fetch_on = [&](int stage, auto ahead) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      dma16_ahead<decltype(ahead)::value * kHalf>(i < kUnitsA ? a0 : b0, off[i], lds_wave + L::kRing + stage * L::kStage + i * kWavesHere * 1024);
  };
  // the next half block, whatever it is
  const auto fetch = [&](int stage) {
    const uint32_t to = L::kRing + (uint32_t)stage * L::kStage + lds_wave;
    const int left = g.k - (next.g0 * kGroup * kStep + next_half * kHalf);  // bytes of k
    if (left > 0 && left < kHalf && next_half < next.half) {  // the last, partial one: zeros behind the end of k
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
        *(i32x4_t*)(lds + to + i * kWavesHere * 1024 + lane * 16) =
            load_chunk((i < kUnitsA ? a0 : b0) + (off[i] - chunk), (int)chunk, left);
      drained = true;
    } else if (next_half < next.half) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) dma16(i < kUnitsA ? a0 : b0, off[i], to + i * kWavesHere * 1024);
    } else {
      drained = true;  // (a half block that only fills up the turn of the ring)
    }
    a0 += kHalf;
    b0 += kHalf;
    if (++next_half == next.end) {
      // (past the last tile it is fetched again, for nobody)
      if (next_tile + slots < tile_end) next_tile += slots;
      aim();
    }
  };
  // Scales: the waves take 64 rows each, the one after them the tile's blocks of 128 columns
  int ring = 0;  // of the two places for a group's scales, the one that the next fetch goes to
  const auto fetch_scales = [&](const Place& p, int group) {
    const uint32_t to = ring * L::kScales;
    ring ^= 1;
#pragma unroll
    for (int u = 0; u < BM / 64 + 1; ++u) {
      if (u % kWavesHere != wave) continue;
      if (u < BM / 64) {
        const uint32_t row = (uint32_t)(min(p.m0 + u * 64 + lane, g.m - 1) - p.m0);
        dma4(g.a_scales + (long long)p.m0 * g.a_scale_stride + group * 4, row * (uint32_t)g.a_scale_stride, to + u * 256);
      } else {
        const uint32_t row = (uint32_t)(min(p.n0 / 128 + lane, (g.n - 1) / 128) - p.n0 / 128);
        dma4(g.b_scales + (long long)(p.n0 / 128) * g.b_scale_stride + group * 4, row * (uint32_t)g.b_scale_stride, to + u * 256);
      }
    }
  };

  const int wm = wave % WM * TM, wn = wave / WM * TN;
  // fragments: chunks lane / 32 and lane / 32 + 2 of row lane % 32
  const int lr = lane & 31, x = lr / 4 % 4;
  const uint32_t lo = (uint32_t)(lr * kHalf + ((lane >> 5) ^ x) * 16), hi = (uint32_t)(lr * kHalf + ((2 + (lane >> 5)) ^ x) * 16);
  i32x8_t a[kApart ? 1 : 2][MT], b[kApart ? 1 : 2][NT];
  const auto read = [&](int set, int stage) {
    const uint8_t* s = lds + L::kRing + stage * L::kStage;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const uint8_t* p = s + (BM + wn + j * 32) * kHalf;
      b[set][j] = join(*(const i32x4_t*)(p + lo), *(const i32x4_t*)(p + hi));
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint8_t* p = s + (wm + i * 32) * kHalf;
      a[set][i] = join(*(const i32x4_t*)(p + lo), *(const i32x4_t*)(p + hi));
    }
  };
  uint32_t as[MT], bs;
  f32x16_t acc[NT][MT];
  const auto multiply = [&](int set, int block) {
    typename W::Fragment fa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[i] = W::make(a[set][i], as[i] >> (8 * block) & 255);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const auto fb = W::make(b[set][j], bs >> (8 * block) & 255);
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[j][i] = W::mul(fb, fa[i], acc[j][i], bs, as[i], block);
    }
    // (here, and not past the barriers that follow, where the compiler would take them to the end of the group)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) asm volatile("" : "+v"(acc[j][i]));
  };
  int ready = 0;  // stages from here on that have landed already
  const auto landed = [&] {
    if (ready > 0) --ready;
    else if (drained) wait_vm<0>();
    else wait_vm<(STAGES - 2) * kUnits>();
  };
  const auto landed_on = [&](auto u) {  // the same in a group whose fetches are all alike
    if (decltype(u)::value >= STAGES - 1 || decltype(u)::value >= ready) wait_vm<(STAGES - 2) * kUnits>();
  };
  const auto barrier = [] { asm volatile("s_barrier" ::: "memory"); };

  aim();
  fetch_scales(next, next.g0);
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) fetch(i);
  wait_lds();  // (a first half block that k ends in went through registers: written before the barrier that its readers wait at)
  if constexpr (kApart) {
    if (second) {
      landed();
      barrier();
    }
  } else {
    landed();
    barrier();
    fetch(STAGES - 1);
    read(0, 0);
  }
  int taken = 0;  // of the two places for scales, the one with the present group's
  for (; tile < tile_end; tile += slots) {
    const Place p = place(tile);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[j][i][q] = 0.f;
    // One half block: h of the tile, `stage` of the ring, the `block`-th of a group's four blocks.  ON: so are the STAGES ones after it, in
    // the same tile, `ahead` of where the stream is noted to be, and nothing need be asked.
    const auto half_block = [&](int h, int stage, int set, int block, auto on, auto ahead) {
      constexpr bool ON = decltype(on)::value;
      // four waves: the next half block's stage has landed, for everybody, and everybody has read this one's;
      // eight: this one's has landed, everybody has read the one before
      if (!second) {
        if constexpr (ON) landed_on(ahead);
        else landed();
      }
      if constexpr (!kApart) wait_lds();
      barrier();
      const bool there = ON || h < p.half;
      if ((ON ? ahead == 0 : h % (2 * kGroup) == 0) && there) {
        const uint32_t* s = (const uint32_t*)(lds + taken * L::kScales);
        taken ^= 1;
#pragma unroll
        for (int i = 0; i < MT; ++i) as[i] = s[wm + i * 32 + lr];
        bs = s[BM + wn / 128];
        const int group = p.g0 + h / (2 * kGroup) + 1;
        if (ON || group < p.g1) {
          fetch_scales(p, group);
        } else if (tile + slots < tile_end) {
          const Place after = place(tile + slots);
          fetch_scales(after, after.g0);
        }
      } else if (!ON && h % 2 == 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i) as[i] >>= 8;
        bs >>= 8;
      }
      if constexpr (kApart) {
        if (there) read(0, stage);
        if constexpr (ON) fetch_on((stage + STAGES - 1) % STAGES, ahead);
        else fetch((stage + STAGES - 1) % STAGES);
        wait_lds();
        if (second) {
          if constexpr (ON) landed_on(ahead);
          else landed();
        }
        __builtin_amdgcn_sched_barrier(0);
        barrier();
        __builtin_amdgcn_s_setprio(1);
        if (there) multiply(0, block);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
      } else {
        read(set ^ 1, (stage + 1) % STAGES);
        if constexpr (ON) fetch_on(stage, ahead);
        else fetch(stage);
        if (there) multiply(set, block);
      }
    };
    int h = 0;
    const int whole = min(p.half, (g.k - p.g0 * kGroup * kStep) / kHalf);
#pragma unroll 1
    for (; h + 2 * kGroup + STAGES < whole; h += 2 * kGroup) {  // (the stream stays short of the tile's end)
      with_each<2 * kGroup>([&](auto u) {
        constexpr int U = decltype(u)::value;
        half_block(h + U, U % STAGES, U & 1, U / 2, std::true_type(), u);
      });
      ready = 0;
      a0 += 2 * kGroup * kHalf;
      b0 += 2 * kGroup * kHalf;
      next_half += 2 * kGroup;
    }
    const std::integral_constant<int, 0> none;
#pragma unroll 1
    for (; h < p.end; h += 2) {
      half_block(h, h % STAGES, 0, 0, std::false_type(), none);
      half_block(h + 1, (h + 1) % STAGES, 1, 0, std::false_type(), none);
    }
    // the next tile's first stages before the stores, which they would otherwise be waited for with
    wait_vm<0>();
    ready = second ? STAGES - 2 : STAGES - 1;  // (the second waves look one stage ahead)
    drained = false;
    const auto store = [&](auto* c, long long stride) {
      typedef typename std::remove_pointer<decltype(c)>::type U;
      constexpr int kPass = 64 / (int)sizeof(U);  // columns of C in 64 bytes
      uint8_t* own = lds + L::kOut + wave * 2048;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int e = 0; e < TN; e += kPass) {
          const f32x16_t& v = acc[e / 32][i];
          if constexpr (sizeof(U) == 2) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *(uint2*)(own + lr * 64 + ((q ^ x) * 16) + (lane >> 5) * 8) =
                  make_uint2(pack_bf16(v[4 * q], v[4 * q + 1]), pack_bf16(v[4 * q + 2], v[4 * q + 3]));
          } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const int r = (e % 32 / 8 + q) * 4;
              *(f32x4_t*)(own + lr * 64 + (((2 * q + (lane >> 5)) ^ x) * 16)) = f32x4_t{v[r], v[r + 1], v[r + 2], v[r + 3]};
            }
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int r = k * 16 + lane / 4, row = p.m0 + wm + i * 32 + r, col = p.n0 + wn + e + (lane & 3) * (kPass / 4);
            const u32x4_t out = *(const u32x4_t*)(own + r * 64 + (((lane & 3) ^ (r / 4 % 4)) * 16));
            if (row < g.m && col < g.n) store_bytes(c + row * stride + col, g.n - col, out);
          }
        }
      }
    };
    if (plan.splits > 1) store(plan.partial + (long long)p.split * g.m * g.n, (long long)g.n);
    else store((T*)g.c, g.c_stride);
  }
  if (kApart && !second) barrier();
  wait_vm<0>();
}

// The parts of a split product added in their order.
template <typename T>
__global__ __launch_bounds__(256) void matmul_add_kernel(MatmulArgs g, const float* partial, int splits) {
  const int per_row = (g.n + 3) / 4;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long row = at / per_row;
  if (row >= g.m) return;
  const int col = (int)(at - row * per_row) * 4;
  typedef f32x4_t f32x4_at4_t __attribute__((aligned(4)));
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const float* p = partial + ((long long)s * g.m + row) * g.n + col;
    if (col + 4 <= g.n) sum += *(const f32x4_at4_t*)p;
    else
      for (int i = 0; i < g.n - col; ++i) sum[i] += p[i];
  }
  store_columns((T*)g.c + row * g.c_stride + col, g.n - col, sum);
}

template <typename S, int MT, int PER_UNIT, int kWaves, typename T>
void strip_form(const MatmulArgs& g, hipStream_t st) {
  constexpr int kRoom = 163840 / PER_UNIT;
  typedef StripLds<MT, kWaves, kRoom> L;
  static const hipError_t raised =
      hipFuncSetAttribute((const void*)matmul_strip_kernel<S, MT, kWaves, kRoom, T>, hipFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  (void)raised;
  const int tiles = (g.n + 15) / 16 * ((g.m + MT * 16 - 1) / (MT * 16));
  matmul_strip_kernel<S, MT, kWaves, kRoom, T><<<std::min(tiles, kComputeUnits * PER_UNIT), kWaves * 64, L::kBytes, st>>>(g);
}

template <typename S, int BM, int BN, int WM, int WN, int ST, typename T>
void tile_form(const MatmulArgs& g, TilePlan plan, hipStream_t st) {
  plan.tiles_m = (g.m + BM - 1) / BM;
  plan.tiles_n = (g.n + BN - 1) / BN;
  plan.group_m = 4;
  static const hipError_t raised = hipFuncSetAttribute((const void*)matmul_tile_kernel<S, BM, BN, WM, WN, ST, T>,
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (TileLds<BM, BN, ST>::kBytes + WM * WN * 2048));
  (void)raised;
  matmul_tile_kernel<S, BM, BN, WM, WN, ST, T><<<std::min((unsigned)plan.tiles_m * plan.tiles_n * plan.splits, (unsigned)(kComputeUnits * (163840 / (TileLds<BM, BN, ST>::kBytes + WM * WN * 2048)))), WM * WN * 64, (TileLds<BM, BN, ST>::kBytes + WM * WN * 2048), st>>>(g, plan);
  if (plan.splits > 1) {
    const long long count = (long long)g.m * ((g.n + 3) / 4);
    matmul_add_kernel<T><<<(unsigned)((count + 255) / 256), 256, 0, st>>>(g, plan.partial, plan.splits);
  }
}

// ---- which form ------------------------------------------------------------------------------------------------------------------
// Up to 16 rows: strips.  Else the form that a model of its time says is the fastest.  A tile's time is its half blocks' times what an
// iteration takes, from measurements (k = 4096, us an iteration; few compute units at work / all / each of two or three workgroups on one):
//   256 x 256  0.57 / 0.84 (at a lower clock)   128 x 128  0.26 / 0.30 / 0.34   64 x 128  0.175 / 0.21 / 0.25   64 x 64  0.147 / 0.17 (rate of L2)
//   fp32: 128 x 128  0.30 / 0.44 / 0.44   64 x 128  0.26 / 0.30 / 0.30
// but no less than B takes from memory (5.2 TB/s).  A tile's start and end cost 1.6 to 3.4 us; parts of k cost a second launch and the traffic of the
// parts; strips take 0.36, 0.38 or 0.62 us for a step of each of a compute unit's four waves, with up to 32, 48 and 64 rows (more rows:
// several parts of as many), and a little more the longer the stream.
// 512 x 4096 x 4096: 64 x 128 17.4, 128 x 128 20.2; 512 x 12288 x 4096: 43.5, 36.5, 256 x 256 42.6; 512 x 22016 x 4096: 256 x 256 58, 128 x 128 67;
// 300 x 12288 x 4096 (fp32): 64 x 128 40.7, 128 x 128 48; 32 x 12288 x 4096: strips 10.4, 64 x 64 13.5; 64 x 12288 x 4096: 16.3 and 14.4;
// 48 x 4096 x 11008: 12.5 and 17.0; 512 x 512 x 2048 (fp32): 5.7 and 14.1; 1000 x 1000 x 256: 6.4 and 5.1.
enum Form { kStrip, kTile64, kTileWide, kTile128, kTile256 };  // wide: 64 x 128
struct Choice {
  Form form;
  int splits, groups;  // parts of k, groups of four blocks each
};
constexpr size_t kMostScratch = 32u << 20;
constexpr int kStripParts = 16;
// tiles of 16 rows of each of the parts of up to 64 rows that A is cut into
int strip_tiles(int m) {
  const int parts = (m + 63) / 64;
  return ((m + 15) / 16 + parts - 1) / parts;
}
Choice choose(int m, int n, int k, bool exact, size_t scratch) {
  const int groups = ((k + kStep - 1) / kStep + kGroup - 1) / kGroup;
  if (m <= 16) return {kStrip, 1, groups};
  Choice best = {kTile128, 1, groups};
  double least = 1e30;
  if (m <= 64 * kStripParts && n < 1 << 26) {
    const double a_step[] = {0.36, 0.36, exact ? 0.5 : 0.38, exact ? 0.74 : 0.62};
    const int parts = (m + 63) / 64, tiles16 = strip_tiles(m);
    const double rounds = ceil((n + 15) / 16 * parts / (double)kComputeUnits), steps = ceil(k / (double)(4 * kStep));
    least = 2.5 + fmax((double)n * k / 5.2e6, rounds * (steps * a_step[tiles16 - 1] * (1 + (tiles16 < 3 ? 0.02 : 0.05) * (rounds - 1)) + 0.25));
    best = {kStrip, 1, groups};
  }
  // few, all: an iteration with few workgroups and with one for each compute unit; more: for each, where `room` share a unit; pair: at least
  const struct { Form form; int rows, columns, room; double ends, few, all, more, pair; } forms[] = {
      {kTile64, 64, 64, 1, 1.6, exact ? 0.23 : 0.147, exact ? 0.36 : 0.17, 0, 0},
      {kTileWide, 64, 128, 3, 2.0, exact ? 0.26 : 0.175, exact ? 0.30 : 0.21, exact ? 0.30 : 0.25, exact ? 0.50 : 0.40},
      {kTile128, 128, 128, 2, 2.4, exact ? 0.30 : 0.26, exact ? 0.44 : 0.30, exact ? 0.44 : 0.34, exact ? 0.67 : 0.48},
      {kTile256, 256, 256, 1, 3.4, 0.57, 0.84, 0, 0}};
  for (const auto& f : forms) {
    if (exact && f.form == kTile256) continue;  // (its converted operands do not fit the registers)
    const double tiles = ceil(m / (double)f.rows) * ceil(n / (double)f.columns);
    for (int want = 1; want <= 8 && want <= groups; want *= 2) {
      const int per = (groups + want - 1) / want, splits = (groups + per - 1) / per;  // no empty parts
      const double parts = splits > 1 ? (double)splits * m * n * 4 : 0;
      if (parts > (double)scratch) break;
      const double units = tiles * splits / kComputeUnits, iterations = 2 * kGroup * (double)per;
      double us = units <= 1        ? f.ends + iterations * (f.few + (f.all - f.few) * units)
                  : units <= f.room ? f.ends + iterations * fmax(f.pair, f.more * units)
                                    : ceil(units) * (f.ends + iterations * fmax(f.all, f.more));
      us = 2.5 + fmax(us, (double)n * k / 5.2e6) + (splits > 1 ? 3.5 + 2 * parts / 4e6 : 0);
      if (us < least) {
        least = us;
        best = {f.form, splits, per};
      }
    }
  }
  return best;
}

template <typename S, typename T>
void matmul(const MatmulArgs& g, void* workspace, size_t workspace_bytes, hipStream_t st) {
  constexpr bool kExact = sizeof(S) == 4;
  Choice c = choose(g.m, g.n, g.k, kExact, kMostScratch);
  // (without room for its parts: none)
  if (c.splits > 1 && (!workspace || workspace_bytes < (size_t)c.splits * g.m * g.n * 4)) c = choose(g.m, g.n, g.k, kExact, 0);
  if (c.form == kStrip) {
    // Several workgroups to a compute unit where there are columns for them, eight waves else (1 x 5120 x 5120: three workgroups 6.4 us, two
    // 7.6, one 8.9; 1 x 4096 x 4096: eight waves 4.7, four 5.2; 32 x 12288 x 4096: two workgroups 10.4, one 12.0).
    const bool more = (long long)g.n * ((g.m + 63) / 64) > 16 * kComputeUnits;
    switch (strip_tiles(g.m)) {
      case 1: return more ? strip_form<S, 1, 3, 4, T>(g, st) : strip_form<S, 1, 2, 8, T>(g, st);
      case 2: return more ? strip_form<S, 2, 2, 4, T>(g, st) : strip_form<S, 2, 1, 8, T>(g, st);
      case 3: return more ? strip_form<S, 3, 2, 4, T>(g, st) : strip_form<S, 3, 1, 8, T>(g, st);
      default: return strip_form<S, 4, 1, 4, T>(g, st);
    }
  }
  TilePlan plan = {};
  plan.splits = c.splits;
  plan.groups = c.groups;
  plan.partial = (float*)workspace;
  if constexpr (!kExact) {
    if (c.form == kTile256) return tile_form<S, 256, 256, 2, 4, 4, T>(g, plan, st);
  }
  if (c.form == kTile64) return tile_form<S, 64, 64, 2, 2, 4, T>(g, plan, st);
  if (c.form == kTileWide) return tile_form<S, 64, 128, 2, 2, 4, T>(g, plan, st);
  tile_form<S, 128, 128, 2, 2, 4, T>(g, plan, st);
}

}  // namespace

size_t matmul_workspace(int m, int n, int k) {
  int splits = 1;  // the most of either way to form sums
  for (const bool exact : {false, true}) splits = std::max(splits, choose(m, n, k, exact, kMostScratch).splits);
  return splits > 1 ? (size_t)splits * m * n * 4 : 0;
}

void launch_matmul(const MatmulArgs& g, int dtype, bool wide_sums, void* workspace, size_t workspace_bytes, hipStream_t st) {
  if (dtype == A2SF_F32) matmul<float, float>(g, workspace, workspace_bytes, st);
  else if (wide_sums) matmul<float, bf16_t>(g, workspace, workspace_bytes, st);
  else matmul<bf16_t, bf16_t>(g, workspace, workspace_bytes, st);
}

}  // namespace a2sf
