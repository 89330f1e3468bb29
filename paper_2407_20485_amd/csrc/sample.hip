// A token from each row of logits: temperature, then the k most likely, then the shortest prefix of these with a share p of their
// mass, then those of at least min_p of the largest probability; of what is kept the token with the largest
// probability / random number, the numbers being exponential variates from the caller (the first of several
// independent exponential clocks to ring is each with the probability of its rate).
//
// Every filter keeps a prefix of the order "larger logit first, equal ones by index", so what they leave is described by its
// last token: a cut (logit, index).  It is found without sorting, in a list of candidates that is certain to hold it:
//  * top_k <= 512: the largest logit of each of 64, 256 or 512 groups of lanes is looked at; the smallest of these has so many
//    tokens at or above it, and only a few times as many on the average: these are the list;
//  * else: a histogram of the row's masses (32 bins per octave of probability) says in which bin the cut lies.  The list is all
//    that is not below this bin, or if that is too many what lies in it;
//  * min_p alone, or where it ends before this bin: what it keeps is the list, and no cut is needed.
// What is left in a list that holds all from the largest on also races from there.
// In the list a histogram finds the bin of the cut and the tokens of that bin are ranked against each other.  A list that
// overflows or misses the cut (rows of few different values) is replaced by the row itself, whose bins are split until one
// can be ranked, or holds one value only.
//
// Masses are whole numbers of 2^-41 of the largest token's weight, summed in 64 bits (2^22 tokens at most): their sums do not depend on the order
// in which the lanes add, so the same inputs give the same cut, whichever way it was found.  A mass has 21 bits or all of its weight's, down to
// weights of 2^-31, and what all tokens below 2^-42 lose is under 2^-20 of the largest one's.
//
// A workgroup of 1024 lanes takes a row.  Few rows are a chain of passes and barriers whose instructions are mostly fetched for the first
// time: what counts is little code, so passes are loops that read the row again (from the caches) instead of unrolled ones over
// registers (32 000 logits in fp32, all filters: 13.4 us, 24 with the row in registers; 256 rows of 50 272 in bf16, top-p and min-p: 23.3 us, 43 with
// a second pass for exact masses and a race over the whole row), and one function serves counts and masses.
#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBins = kSampleThreads;
constexpr int kRanked = kSampleThreads;  // tokens ranked against each other at once
constexpr int kListed = 512;             // tokens that a wave lists
constexpr float kBinsPerOctave = 32.f;
constexpr float kInf = __builtin_huge_valf();

struct SampleShared {
  unsigned long long mass[kBins];
  uint32_t count[kBins];
  float list[kSampleWaves][kListed];
  int list_index[kSampleWaves][kListed];
  float rank[kRanked];
  int rank_index[kRanked];
  unsigned long long rank_mass[kRanked];
  unsigned long long wave64[kSampleWaves], wave64b[kSampleWaves];
  uint32_t wave32[kSampleWaves], wave32b[kSampleWaves];
  float wavef[kSampleWaves], wavef2[kSampleWaves];
  // what the scan found
  unsigned long long before_mass, kept_mass;
  uint32_t before_count, in_bin, ranked;
  int bin, overflow;
  float cut;
  int cut_index;
};
constexpr int kSampleLds = (int)sizeof(SampleShared);

// Sums of this lane and all before it in the wave: shifts inside rows of 16, then the rows' totals.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ void scan_step(uint32_t& c, unsigned long long& m) {
  const uint32_t lo = dpp_or_zero<CTRL, ROWS>((uint32_t)m), hi = dpp_or_zero<CTRL, ROWS>((uint32_t)(m >> 32));
  c += dpp_or_zero<CTRL, ROWS>(c);
  m += ((unsigned long long)hi << 32) | lo;
}
__device__ __forceinline__ void wave_scan(uint32_t& c, unsigned long long& m) {
  scan_step<0x111, 0xF>(c, m);  // row_shr 1, 2, 4, 8
  scan_step<0x112, 0xF>(c, m);
  scan_step<0x114, 0xF>(c, m);
  scan_step<0x118, 0xF>(c, m);
  scan_step<0x142, 0xA>(c, m);  // the last lane of a row to the row after it
  scan_step<0x143, 0xC>(c, m);  // the last lane of the lower half to the upper
}

// Eight logits as they are in memory; -infinity past the end of the row.  A NaN comes as it is: maxima pass it over and it is
// not >= anything.
template <typename T> struct RawUnit;
template <> struct RawUnit<float> {
  float v[kUnit];
  __device__ __forceinline__ void load(const float* p, int have) {
    if (have >= kUnit) load_unit(p, v);
    else
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[j] = j < have ? p[j] : -kInf;
  }
  __device__ __forceinline__ float at(int j) const { return v[j]; }
};
template <> struct RawUnit<bf16_t> {
  u32x4_t v;
  __device__ __forceinline__ void load(const bf16_t* p, int have) {
    if (have >= kUnit) v = *(const u32x4_at2_t*)p;
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = 2 * j < have ? p[2 * j] : 0xFF80u, hi = 2 * j + 1 < have ? p[2 * j + 1] : 0xFF80u;
        v[j] = lo | hi << 16;
      }
  }
  __device__ __forceinline__ float at(int j) const {
    return __uint_as_float(j & 1 ? v[j / 2] & 0xFFFF0000u : v[j / 2] << 16);
  }
};
// A row of logits.  TOP_IS_INF: the largest is +infinity; then such tokens count as 0 and all others as -infinity.
template <typename T, bool TOP_IS_INF>
struct Row {
  const T* p;
  int n;
  static __device__ __forceinline__ float logit(float l) { return TOP_IS_INF ? (l == kInf ? 0.f : -kInf) : l; }
  // f(unit, index of its first element) for this lane's units, the next one on its way; whole waves go through the same ones
  template <typename F>
  __device__ __forceinline__ void each_unit(F f) const {
    int first = (int)threadIdx.x * kUnit;
    RawUnit<T> u;
    u.load(p + first, n - first);
    for (;;) {
      const int next = first + kSampleThreads * kUnit;
      const bool more = next - (int)(threadIdx.x & 63) * kUnit < n;
      RawUnit<T> v;
      if (more) v.load(p + next, n - next);
      f(u, first);
      if (!more) break;
      u = v;
      first = next;
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    each_unit([&](const RawUnit<T>& u, int first) {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) f(logit(u.at(j)), first + j);
    });
  }
};
// The candidates in a row's place: each wave goes through what it has listed itself.
struct List {
  SampleShared& s;
  int n;
  int count = 0;  // of this wave
  // Tokens are noted as bits, one of each lane's elements after the other, the newest lowest; 32 at a time they go to the list: one of each
  // lane per turn, their indices first.
  uint32_t bits = 0;
  int noted = 0, group = 0;  // units in `bits`, the first one's first element
  __device__ __forceinline__ void flush() {
    unsigned long long who;
    while ((who = __ballot(bits != 0)) != 0) {
      const int to = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
      const int top = 31 - __builtin_clz(bits | 1u), element = noted * kUnit - 1 - top;
      if (bits && to < kListed)
        s.list_index[threadIdx.x >> 6][to] = group + element / kUnit * (kSampleThreads * kUnit) + element % kUnit;
      bits &= ~(1u << top);
      count += __popcll(who);
    }
    noted = 0;
  }
  // after a unit's bits have gone in
  __device__ __forceinline__ void unit_done(int first) {
    if (noted == 0) group = first;
    if (++noted == 32 / kUnit) flush();
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    for (int i = threadIdx.x & 63; i < count; i += 64) f(s.list[threadIdx.x >> 6][i], s.list_index[threadIdx.x >> 6][i]);
  }
  // after the last unit: fetches the listed logits; whether all waves had room
  template <typename R>
  __device__ __forceinline__ bool complete(const R& row) {
    flush();
    if (count > kListed) s.overflow = 1;
    const int wave = threadIdx.x >> 6;
    for (int i = threadIdx.x & 63; i < min(count, kListed); i += 64) s.list[wave][i] = row.logit(load_one(row.p + s.list_index[wave][i]));
    __syncthreads();
    return !s.overflow;
  }
};

// Every wave has left a value: the sixteen of them in the sixteen lanes of a row, then across the row.
template <typename T, typename Op>
__device__ __forceinline__ T of_waves(const T* left, Op op) {
  T v = left[threadIdx.x & 15];
  const auto bits = [](T x) { return __builtin_bit_cast(uint32_t, x); };
  const auto back = [](uint32_t x) { return __builtin_bit_cast(T, x); };
  v = op(v, back(dpp_move_u32<0xB1>(bits(v))));
  v = op(v, back(dpp_move_u32<0x4E>(bits(v))));
  v = op(v, back(dpp_move_u32<0x141>(bits(v))));
  return op(v, back(dpp_move_u32<0x140>(bits(v))));
}
struct OpSumI { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a + b; } };
struct OpMaxI { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); } };
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, dpp_move_u32<0xB1>(v));
  v = max(v, dpp_move_u32<0x4E>(v));
  v = max(v, dpp_move_u32<0x141>(v));
  v = max(v, dpp_move_u32<0x140>(v));
  u32x2_t r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(r[0], r[1]);
}
// (their sums are whole numbers, or taken in one fixed order)
__device__ __forceinline__ uint32_t block_sum_u32(uint32_t v, uint32_t* left) {
  v = (uint32_t)wave_sum_i((int)v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) left[threadIdx.x >> 6] = v;
  __syncthreads();
  return of_waves(left, OpSumI());
}

// The distance below the largest logit in octaves of probability, its weight; its bin
struct Scale {
  float top, per;         // largest logit; octaves per unit of logit (log2(e) / temperature)
  float first, bins_per;  // the bins: from this logit down, so many per unit of logit
  __device__ __forceinline__ float below(float l) const { return (top - l) * per; }
  // (of finite numbers)
  __device__ __forceinline__ int bin(float l) const {
    return (int)fminf(fmaxf((first - l) * bins_per, 0.f), (float)(kBins - 1));
  }
  // bins over the whole row, by probability
  __device__ __forceinline__ Scale over_row() const { return {top, per, top, per * kBinsPerOctave}; }
  // ... over the logits from `high` to `low`
  __device__ __forceinline__ Scale over(float high, float low) const {
    high = fminf(high, top);
    const float range = high - low;
    return {top, per, high, range > 0.f && range < 1e30f ? fminf((float)(kBins - 1) / range, 1e30f) : per * kBinsPerOctave};
  }
};
// (of finite numbers)
__device__ __forceinline__ float next_above(float l) {
  const int bits = __float_as_int(l);
  return bits << 1 == 0 ? __int_as_float(1) : __int_as_float(bits + (bits < 0 ? -1 : 1));
}
__device__ __forceinline__ float weight(float below) { return __builtin_amdgcn_exp2f(-below); }
// Its mass: of the ten octaves below the largest a whole number of 2^-31, under them one of 2^-41; 32 bits either way
__device__ __forceinline__ unsigned long long mass_of(float below) {
  const bool near = below < 10.f;
  const uint32_t m = (uint32_t)fmaf(weight(below), near ? 0x1p31f : 0x1p41f, 0.5f);
  return near ? (unsigned long long)m << 10 : m;
}
constexpr float kMassUnit = 0x1p-41f;

// What is looked for: the token at which the count (by_mass: the mass) reaches a number
struct Target {
  bool by_mass;
  uint32_t tokens;
  unsigned long long mass;
};

// The mass with which a share p of `inside` is reached
__device__ __forceinline__ unsigned long long mass_for(float p, unsigned long long inside) {
  const unsigned long long mass = p > 0.f ? (unsigned long long)ceil((double)p * (double)inside) : 1ull;
  return mass < 1 ? 1 : mass > inside ? inside : mass;
}

__device__ __forceinline__ void clear_bins(SampleShared& s) {
  __syncthreads();
  s.mass[threadIdx.x] = 0;
  s.count[threadIdx.x] = 0;
  __syncthreads();
}

// The bin in which the target (share < 1: that share of the total mass) is reached and what lies before it; s.bin = -1 if there is none.
// Returns the total mass.  Four waves
// do it, a lane four bins: with all sixteen at it the vector units would be four times as long busy with the same few bins.
__device__ __forceinline__ unsigned long long scan_bins(SampleShared& s, Target to, uint32_t count0, unsigned long long mass0,
                                                        float share = 1.f) {
  __syncthreads();
  if (threadIdx.x == 0) s.bin = -1;  // (everybody has read the last scan's)
  const int t = threadIdx.x, wave = t >> 6;
  uint32_t c = 0, own_c[4];
  unsigned long long m = 0, own_m[4];
  if (t < kBins / 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      own_c[i] = s.count[4 * t + i];
      own_m[i] = s.mass[4 * t + i];
      c += own_c[i];
      m += own_m[i];
    }
    wave_scan(c, m);
    if ((t & 63) == 63) { s.wave32b[wave] = c; s.wave64[wave] = m; }
  }
  __syncthreads();
  unsigned long long total = mass0;
#pragma unroll
  for (int w = 0; w < 4; ++w) total += s.wave64[w];
  if (share < 1.f) to.mass = mass_for(share, total);
  if (t < kBins / 4) {
    c += count0;
    m += mass0;
#pragma unroll
    for (int w = 0; w < 3; ++w) {
      c += w < wave ? s.wave32b[w] : 0u;
      m += w < wave ? s.wave64[w] : 0ull;
    }
#pragma unroll
    for (int i = 3; i >= 0; --i) {  // back from the sum up to the lane's last bin
      const uint32_t c1 = c - own_c[i];
      const unsigned long long m1 = m - own_m[i];
      if (to.by_mass ? (m1 < to.mass && m >= to.mass) : (c1 < to.tokens && c >= to.tokens)) {
        s.bin = 4 * t + i;
        s.before_count = c1;
        s.before_mass = m1;
        s.in_bin = own_c[i];
      }
      c = c1;
      m = m1;
    }
  }
  __syncthreads();
  return total;
}

// Fills the bins of a row or of the list.
template <typename R>
__device__ __forceinline__ void fill_bins(const R& row, const Scale& sc, SampleShared& s) {
  clear_bins(s);
  // (the last bin, where most of a row may lie, in registers first)
  uint32_t far_count = 0;
  unsigned long long far_mass = 0;
  row.each([&](float l, int) {
    if (!(l > -kInf)) return;  // (a NaN, or -infinity at a temperature of infinity, would have some bin)
    const int bin = sc.bin(l);
    const unsigned long long m = mass_of(sc.below(l));
    if (bin < kBins - 1) {
      atomicAdd(&s.count[bin], 1u);
      atomicAdd(&s.mass[bin], m);
    } else {
      ++far_count;
      far_mass += m;
    }
  });
  if (far_count) {
    atomicAdd(&s.count[kBins - 1], far_count);
    atomicAdd(&s.mass[kBins - 1], far_mass);
  }
}

// The cut inside the bin that the scan found, left in s.cut / s.cut_index, with the mass up to and with it in s.kept_mass.  Returns
// whether the bins were overwritten.
template <typename R>
__device__ __forceinline__ bool cut_in_bin(const R& row, const Scale& sc, SampleShared& s, Target to) {
  const int t = threadIdx.x;
  const int bin = s.bin;
  uint32_t before_count = s.before_count, members = s.in_bin;
  unsigned long long before_mass = s.before_mass;
  uint32_t low = 1, high = 0;  // keys of the members; low > high: those of the bin
  bool split = false;
  if (members > kRanked) {
    // Too many: split the range of their keys, 10 bits at a time
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    row.each([&](float l, int) {
      if (l > -kInf && sc.bin(l) == bin) {
        const uint32_t key = ordered_key(l);
        lo = min(lo, key);
        hi = max(hi, key);
      }
    });
    hi = wave_max_u32(hi);
    lo = wave_max_u32(~lo);
    __syncthreads();
    if ((t & 63) == 0) { s.wave32[t >> 6] = hi; s.wave32b[t >> 6] = lo; }
    __syncthreads();
    high = of_waves(s.wave32, OpMaxI());
    low = ~of_waves(s.wave32b, OpMaxI());
    split = true;
    while (members > kRanked && low < high) {
      const int bits = 32 - __clz(high - low);
      const int shift = bits > 10 ? bits - 10 : 0;
      clear_bins(s);
      row.each([&](float l, int) {
        const uint32_t key = ordered_key(l);
        if (l > -kInf && key >= low && key <= high) {
          atomicAdd(&s.count[(high - key) >> shift], 1u);
          atomicAdd(&s.mass[(high - key) >> shift], mass_of(sc.below(l)));
        }
      });
      scan_bins(s, to, before_count, before_mass);
      before_count = s.before_count;
      before_mass = s.before_mass;
      members = s.in_bin;
      high -= (uint32_t)s.bin << shift;
      const uint32_t span = (1u << shift) - 1u;
      low = high - low > span ? high - span : low;
    }
    if (members > kRanked) {
      // all of one value: the cut is the r-th of them by index, found by halving the range of indices
      const float value = __uint_as_float((high & 0x80000000u) ? high ^ 0x80000000u : ~high);
      const unsigned long long each = mass_of(sc.below(value));
      uint32_t r = to.tokens - before_count;
      if (to.by_mass) r = each ? (uint32_t)((to.mass - before_mass + each - 1) / each) : members;
      int first = 0, last = row.n - 1;
      while (first < last) {
        const int mid = first + (last - first) / 2;
        int c = 0;
        row.each([&](float l, int at) { c += l == value && at <= mid; });
        if (block_sum_u32((uint32_t)c, s.wave32) >= r) last = mid;
        else first = mid + 1;
      }
      __syncthreads();
      if (t == 0) {
        s.cut = value;
        s.cut_index = first;
        s.kept_mass = before_mass + r * each;
      }
      __syncthreads();
      return split;
    }
  }
  if (t == 0) s.ranked = 0;
  __syncthreads();
  row.each([&](float l, int at) {
    const float below = sc.below(l);
    const uint32_t key = ordered_key(l);
    if (l > -kInf && (low > high ? sc.bin(l) == bin : key >= low && key <= high)) {
      const uint32_t slot = atomicAdd(&s.ranked, 1u);  // in any order: the ranks below do not depend on it
      s.rank[slot] = l;
      s.rank_index[slot] = at;
      s.rank_mass[slot] = mass_of(below);
    }
  });
  __syncthreads();
  // `share` lanes (of one wave) to a token, each comparing it with a part of the others
  int shift = 6;
  while (shift > 0 && ((int)members << shift) > kSampleThreads) --shift;
  const int share = 1 << shift, mine = t >> shift;
  uint32_t c = 0;
  unsigned long long m = 0;
  if (mine < (int)members) {
    const float l = s.rank[mine];
    const int at = s.rank_index[mine];
#pragma unroll 4
    for (int j = t & (share - 1); j < (int)members; j += share) {
      const float o = s.rank[j];
      const bool ahead = o > l || (o == l && s.rank_index[j] < at);
      c += ahead;
      m += ahead ? s.rank_mass[j] : 0ull;
    }
  }
  for (int by = 1; by < share; by *= 2) {
    c += __shfl_xor(c, by);
    const uint32_t lo = __shfl_xor((uint32_t)m, by), hi = __shfl_xor((uint32_t)(m >> 32), by);
    m += ((unsigned long long)hi << 32) | lo;
  }
  if (mine < (int)members && (t & (share - 1)) == 0) {
    c += before_count;
    m += before_mass;
    const unsigned long long own = s.rank_mass[mine];
    if (to.by_mass ? (m < to.mass && m + own >= to.mass) : c + 1 == to.tokens) {
      s.cut = s.rank[mine];
      s.cut_index = s.rank_index[mine];
      s.kept_mass = m + own;
    }
  }
  __syncthreads();
  return split;
}

struct Filters {
  int k;          // tokens, 0: all
  float p, min_p; // p >= 1: all
};

// Top-k and top-p on a row, or on a list of a row's first tokens.  inside: the mass that p is a share of where there is no k, 0: that
// of R.  Whether the cut lies in R: the tokens above -infinity may be fewer than k, and if R holds `all` of them they stay.
template <typename R>
__device__ __forceinline__ bool find_cut(const R& row, const Scale& sc, const Filters& f, unsigned long long inside, bool all, SampleShared& s) {
  Target to{false, f.k ? (uint32_t)f.k : 0xFFFFFFFFu, 0};
  if (inside) to = {true, 0, mass_for(f.p, inside)};
  bool filled = false;
#pragma unroll 1
  for (;;) {
    if (!filled) fill_bins(row, sc, s);
    filled = true;
    inside = scan_bins(s, to, 0, 0);
    if (s.bin >= 0) {
      filled = !cut_in_bin(row, sc, s, to);
      inside = s.kept_mass;
    } else if (!all) {
      return false;
    }
    if (to.by_mass || !(f.p < 1.f)) return true;
    to = {true, 0, mass_for(f.p, inside)};
  }
}

// The bin of a row in which the cut by mass (or by more tokens than groups of lanes give) lies.
struct Zone {
  int bin;                        // -1: none, or the last
  uint32_t above, in;             // tokens above the bin and in it; by mass: as many to twice as many
  unsigned long long above_mass;  // their mass
  unsigned long long all;         // the mass of the row
};

// inside: the mass that p is a share of, 0: the row's.
template <typename R>
__device__ __forceinline__ Zone find_zone(const R& row, const Scale& sc, const Filters& f, bool by_mass, unsigned long long inside,
                                          SampleShared& s) {
  clear_bins(s);
  // In the last bin lies what has next to no mass, and may be most of a row: in registers first (under 2^10 a token, 2^12 tokens a lane).
  uint32_t far = 0;
  row.each([&](float l, int) {
    const float below = sc.below(l);
    const unsigned long long m = mass_of(below);
    const uint32_t bin = (uint32_t)fminf(below * kBinsPerOctave, (float)(kBins - 1));
    far += bin < kBins - 1 ? 0u : (uint32_t)m;
    if (bin < kBins - 1) {
      atomicAdd(&s.mass[bin], m);
      if (!by_mass) atomicAdd(&s.count[bin], 1u);
    }
  });
  far = (uint32_t)wave_sum_i((int)far);  // (under 2^28; a thousand lanes at one address of LDS would take 2.5 us)
  if ((threadIdx.x & 63) == 0) atomicAdd(&s.mass[kBins - 1], (unsigned long long)far);
  __syncthreads();
  // (a token of octave o has between 2^(40 - o) and 2^(41 - o))
  if (by_mass) s.count[threadIdx.x] = (uint32_t)(s.mass[threadIdx.x] >> (40u - threadIdx.x / 32u));
  Zone zone;
  zone.all = scan_bins(s, Target{by_mass, (uint32_t)f.k, inside ? mass_for(f.p, inside) : 0}, 0, 0, by_mass && !inside ? f.p : 1.f);
  zone.bin = s.bin < kBins - 1 ? s.bin : -1;
  zone.above = s.before_count;
  zone.in = s.in_bin;
  zone.above_mass = s.before_mass;
  return zone;
}

// The cut in that bin, whose tokens are listed.  Returns false where they do not fit.
template <typename R>
__device__ __forceinline__ bool cut_in_zone(const R& row, const Scale& sc, const Filters& f, bool by_mass, unsigned long long inside,
                                            const Zone& zone, SampleShared& s) {
  if (zone.bin < 0) return false;
  __syncthreads();
  if (threadIdx.x == 0) s.overflow = 0;
  __syncthreads();
  List list{s, row.n};
  row.each_unit([&](const auto& u, int first) {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const float at = sc.below(u.at(j)) * kBinsPerOctave;
      list.bits = 2 * list.bits + (at >= (float)zone.bin && at < (float)(zone.bin + 1));
    }
    list.unit_done(first);
  });
  if (!list.complete(row)) return false;
  const float per = kBinsPerOctave * sc.per;
  const Scale bins = sc.over(sc.top - (float)zone.bin / per, sc.top - (float)(zone.bin + 1) / per);
  const Target to{by_mass, (uint32_t)f.k, by_mass ? mass_for(f.p, inside ? inside : zone.all) : 0};
  fill_bins(list, bins, s);
  scan_bins(s, to, zone.above, zone.above_mass);
  if (s.bin < 0) return false;
  cut_in_bin(list, bins, s, to);
  return true;
}

// What a token brings to the race.  Of equal ones the lowest index stays; a lane meets the tokens of a row by index, those of a list
// (ANY_ORDER) not.
struct Runner {
  float z = 0.f, best = -kInf;
  int at = -1;
  template <bool ANY_ORDER>
  __device__ __forceinline__ void enter(bool in, float below, float w, float log_noise, int index) {
    const float ring = in ? -below - log_noise : -kInf;  // (base 2; not a number: never taken)
    z += in ? w : 0.f;
    const bool ahead = ring > best || (ANY_ORDER && ring == best && index < at);
    best = ahead ? ring : best;
    at = ahead ? index : at;
  }
};

template <typename T, bool TOP_IS_INF>
__device__ __forceinline__ void sample_row(const SampleArgs& a, const Row<T, TOP_IS_INF>& row, float top, float low, Filters f, bool greedy,
                                           float temperature, SampleShared& s) {
  const int t = threadIdx.x;
  const long long r = blockIdx.x;
  Scale sc;
  sc.first = sc.bins_per = 0.f;
  sc.top = TOP_IS_INF ? 0.f : top;
  sc.per = greedy ? 1.f : fminf(1.44269504088896340736f / temperature, 1e30f);  // (0 times it stays 0)
  // A weight to the last bits: with what the roundings of log2(e) / temperature and of the product have cut off.
  const float per_rest = !greedy && sc.per > 1e-30f && sc.per < 1e30f ? (fmaf(-sc.per, temperature, 1.44269504f) + 1.92596299e-8f) * (0.69314718f * sc.per) : 0.f;
  const auto exact_weight = [&](float l) {
    const float d = sc.top - l, below = d * sc.per, w = weight(below);
    return below < 150.f ? fmaf(w, -0.69314718f * fmaf(d, per_rest, fmaf(d, sc.per, -below)), w) : w;
  };
  const float* noise = a.noise && !greedy ? a.noise + r * a.noise_stride : nullptr;
  const float min_p = f.min_p;
  const auto in_share = [&](float l, float below) { return weight(below) >= min_p || l == sc.top; };  // the first always stays
  const auto ring_of = [&](float l, float e) { return fmaf(l - sc.top, sc.per, -__builtin_amdgcn_logf(e)); };
  Runner run;
  int unit_cut = -1;  // not negative: run.at is the first of a unit of eight, and this the index of the cut
  // A list of all that is not below some logit, if the cut is certain to be there and it may be short enough; where min_p keeps less
  // than the other filters, of all that it keeps (a hundredth of an octave more, for the roundings).
  const bool cuts = f.k > 0 || f.p < 1.f, zoned = cuts && !(f.k > 0 && f.k <= 512) && !TOP_IS_INF;
  float least = fmaxf(low, -3.402823466e38f);  // (no -infinity)
  Zone zone;
  bool listed = !TOP_IS_INF && cuts, cut_there = listed;
  if (zoned) {
    zone = find_zone(row, sc, f, f.k == 0, 0, s);
    // (a bin more, so that edges need not be exact)
    least = fmaxf(sc.top - (float)(zone.bin + 2) / (kBinsPerOctave * sc.per), -3.402823466e38f);
    listed = zone.bin >= 0 && zone.above + zone.in <= kSampleWaves * kListed;
  }
  if (!TOP_IS_INF && min_p > 0.f && (zoned ? f.k == 0 || !(f.p < 1.f) : !cuts)) {
    // (no -infinity here either, where the distance is infinite: it would list what stands for logits behind the end of the row)
    const float share = fmaxf(fminf(sc.top, sc.top - (0.01f - __builtin_amdgcn_logf(min_p)) / sc.per), -3.402823466e38f);
    if (!cuts || (zone.bin > 1 && share > sc.top - (float)(zone.bin - 1) / (kBinsPerOctave * sc.per))) {
      least = share;
      listed = true;
      cut_there = false;
    }
  }
  List list{s, a.n};
  if (listed) {
    row.each_unit([&](const RawUnit<T>& u, int first) {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) list.bits = 2 * list.bits + (u.at(j) >= least);
      list.unit_done(first);
    });
    listed = list.complete(row);
    if (listed && cut_there) listed = find_cut(list, sc.over(kInf, least), f, f.k ? 0 : zone.all, !zoned, s);
  }
  if (listed) {
    const float cut = s.cut;
    const int cut_index = s.cut_index;
    list.each([&](float l, int at) {
      const float below = sc.below(l);
      const bool in = (l > cut || (l == cut && at <= cut_index)) && below < kInf && in_share(l, below);
      if (in) run.enter<true>(true, below, weight(below), noise ? __builtin_amdgcn_logf(noise[at]) : 0.f, at);
    });
  } else {
    // Where many tokens are left their random numbers are fetched for every unit, one unit ahead; else where one of the wave's
    // is still in.
    bool ahead = !(min_p > 0.f), known = false;
    if (cuts) {
      bool found = !TOP_IS_INF;
      unsigned long long inside = 0;
#pragma unroll 1
      for (int by_mass = f.k > 0 ? 0 : 1; found && by_mass < (f.p < 1.f ? 2 : 1); ++by_mass) {
        if (!zoned || inside) zone = find_zone(row, sc, f, by_mass, inside, s);
        found = cut_in_zone(row, sc, f, by_mass, inside, zone, s);
        inside = s.kept_mass;
      }
      if (!found) {
        __syncthreads();
        if (t == 0) s.cut = -kInf;
        find_cut(row, sc.over_row(), f, 0, true, s);
      }
      ahead = found && zone.above >= (uint32_t)a.n / 64 && !(min_p > 0.f);
      known = ahead && noise;
    }
    __syncthreads();
    const float cut = s.cut;
    const int cut_index = s.cut_index;
    ahead = ahead && noise;
    float next[kUnit];
    const auto fetch = [&](int first) {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) next[j] = 1.f;
      if (first + kUnit <= a.n) load_unit(noise + first, next);
      else if (first < a.n) load_unit(noise + first, a.n - first, next);
    };
    if (ahead) fetch(t * kUnit);
    // a token is in if it is not below `least`, from the one behind the cut on not below `behind`
    const float least = greedy ? sc.top : fmaxf(cut, -3.402823466e38f);
    const float behind = greedy ? sc.top : cut > -kInf ? next_above(cut) : least;
    if (known) {
      // Many tokens, and their mass is known: a unit's furthest runner only, the token is looked up at the end.
      row.each_unit([&](const RawUnit<T>& u, int first) {
        float ring[kUnit], most = -kInf;
        const int upto = cut_index - first;
        const float lowest = upto >= kUnit - 1 ? least : behind;
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
          const float l = row.logit(u.at(j));
          ring[j] = l >= lowest ? ring_of(l, next[j]) : -kInf;
        }
        if (upto >= 0 && upto < kUnit - 1) {  // the cut's own unit
#pragma unroll
          for (int j = 0; j < kUnit; ++j) {
            const float l = row.logit(u.at(j));
            ring[j] = l >= (j <= upto ? least : behind) ? ring_of(l, next[j]) : -kInf;
          }
        }
#pragma unroll
        for (int j = 0; j < kUnit; ++j) most = fmaxf(most, ring[j]);
        fetch(first + kSampleThreads * kUnit);
        run.at = most > run.best ? first : run.at;
        run.best = fmaxf(run.best, most);
      });
      if (t == 0) run.z = (float)s.kept_mass * kMassUnit;
      unit_cut = cut_index;
    } else {
      row.each_unit([&](const RawUnit<T>& u, int first) {
        float e[kUnit];
#pragma unroll
        for (int j = 0; j < kUnit; ++j) e[j] = ahead ? next[j] : 1.f;
        if (ahead) fetch(first + kSampleThreads * kUnit);
        float l[kUnit], most = -kInf;
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
          l[j] = row.logit(u.at(j));
          most = fmaxf(most, l[j]);
        }
        if (!__any(most >= least)) return;
        if (!ahead && noise && most >= least) load_unit(noise + first, a.n - first, e);
        const int upto = cut_index - first;
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
          const float below = sc.below(l[j]), w = weight(below);
          const bool in = l[j] >= (j <= upto ? least : behind) && (w >= min_p || l[j] == sc.top);
          run.enter<false>(in, below, w, __builtin_amdgcn_logf(e[j]), first + j);
        }
      });
    }
  }
  // the furthest runner; of equal ones the lowest index
  const float wave_z = wave_sum(run.z);
  const uint32_t ring = run.at < 0 ? 0u : ordered_key(run.best);
  const uint32_t wave_ring = wave_max_u32(ring);
  const uint32_t wave_at = wave_max_u32(ring == wave_ring ? ~(uint32_t)run.at : 0u);
  __syncthreads();
  if ((t & 63) == 0) {
    s.wavef[t >> 6] = wave_z;
    s.wave32[t >> 6] = wave_ring;
    s.wave32b[t >> 6] = wave_at;
  }
  if (t == 0) s.cut_index = a.n;
  __syncthreads();
  const float z = of_waves(s.wavef, OpAdd());
  const uint32_t best = of_waves(s.wave32, OpMaxI());
  const uint32_t own = s.wave32[t & 15] == best ? s.wave32b[t & 15] : 0u;
  uint32_t at = max(own, dpp_move_u32<0xB1>(own));
  at = max(at, dpp_move_u32<0x4E>(at));
  at = max(at, dpp_move_u32<0x141>(at));
  at = max(at, dpp_move_u32<0x140>(at));
  int token = (int)~at;
  if (unit_cut >= 0 && best != 0 && t < 64) {  // which of the unit
    bool here = false;
    if (t < kUnit && token + t < a.n) {
      const float l = row.logit(load_one(row.p + token + t));
      here = (l > s.cut || (l == s.cut && token + t <= unit_cut)) && ordered_key(ring_of(l, noise[token + t])) == best;
    }
    token += __builtin_ctzll(__ballot(here) | 1ull << 63);
  }
  if (best == 0) {  // no random number of the tokens that are left is one: the first token
    row.each([&](float l, int at) {
      if (l == sc.top) atomicMin(&s.cut_index, at);
    });
    __syncthreads();
    token = s.cut_index;
  }
  if (t == 0) {
    a.token[r] = token;
    if (a.prob) a.prob[r] = greedy ? 1.f : exact_weight(row.logit(load_one(row.p + token))) / z;
  }
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  SampleShared& s = *(SampleShared*)lds;
  const int t = threadIdx.x;
  const long long r = blockIdx.x;
  const Row<T, false> row{(const T*)a.logits + r * a.stride, a.n};
  const float temperature = a.temperature ? a.temperature[r] : 1.f;
  const bool greedy = !(temperature > 0.f);
  Filters f;
  f.k = a.top_k ? a.top_k[r] : 0;
  f.k = f.k > 0 && f.k < a.n ? f.k : 0;
  f.p = a.top_p ? a.top_p[r] : 1.f;
  f.min_p = a.min_p ? a.min_p[r] : 0.f;
  f.min_p = f.min_p > 0.f ? f.min_p : 0.f;  // (not a number: no filter)
  if (f.min_p > 1.f) f = {a.n > 1 ? 1 : 0, 1.f, 0.f};  // (nothing but the first, not even what equals it)
  if (greedy) f = {0, 1.f, 0.f};

  // The largest logit; and the smallest of the largest ones of `groups` groups of lanes: so many tokens at least are not below
  // it, and about groups * ln(groups) are.  Groups of 2, 4, 8, 16 lanes for up to 512, 256, 128, 64 tokens.
  float high = -kInf;
  row.each([&](float l, int) { high = fmaxf(high, l); });
  float low = fmaxf(high, dpp_move<0xB1>(high));
  if (f.k <= 256) low = fmaxf(low, dpp_move<0x4E>(low));
  if (f.k <= 128) low = fmaxf(low, dpp_move<0x141>(low));
  if (f.k <= 64) low = fmaxf(low, dpp_move<0x140>(low));
  high = wave_max(high);
  low = wave_max(-low);
  if ((t & 63) == 0) {
    s.wavef[t >> 6] = high;
    s.wavef2[t >> 6] = low;
  }
  if (t == 0) {
    s.overflow = 0;
    s.cut = -kInf;
    s.cut_index = 0x7FFFFFFF;
  }
  __syncthreads();
  high = of_waves(s.wavef, OpMax());
  low = -of_waves(s.wavef2, OpMax());
  if (high == -kInf) {
    if (t == 0) {
      a.token[r] = -1;
      if (a.prob) a.prob[r] = 0.f;
    }
  } else if (high < kInf) {
    sample_row(a, row, high, low, f, greedy, temperature, s);
  } else {
    sample_row(a, Row<T, true>{row.p, row.n}, high, low, f, greedy, temperature, s);
  }
}

template <typename T>
bool sample(const SampleArgs& a, hipStream_t st) {
  static const hipError_t raised =
      hipFuncSetAttribute((const void*)sample_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, kSampleLds);
  (void)raised;
  if (!grid_fits(a.rows, kSampleThreads)) return false;
  sample_kernel<T><<<a.rows, kSampleThreads, kSampleLds, st>>>(a);
  return true;
}

}  // namespace

bool launch_sample(const SampleArgs& a, int dtype, hipStream_t st) {
  return dtype == A2SF_F32 ? sample<float>(a, st) : sample<bf16_t>(a, st);
}

}  // namespace a2sf
