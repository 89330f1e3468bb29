// A token from each row of logits: temperature, then the k most likely, then the shortest prefix of these with a share p of their
// mass, then those of at least min_p of the largest probability; of what is kept the token with the largest
// probability / random number, the numbers being exponential variates from the caller (the first of several
// independent exponential clocks to ring is each with the probability of its rate).
//
// Every filter keeps a prefix of the order "larger logit first, equal ones by index", so what they leave is described by its
// last token: a cut (logit, index).  It is found without sorting: a histogram of how far the logits lie below the largest
// says in which bin the cut falls, and only that bin's tokens are ranked against each other.
//
// Masses are whole numbers of 2^-40 of the largest token's weight in 64 bits: their sums do not depend on the order in which
// the lanes add, so the same inputs give the same cut, and a bin's mass is exactly the sum of its tokens'.
#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBins = 2 * kSampleThreads;
constexpr int kList = kSampleThreads;  // tokens ranked against each other at once
constexpr float kBinsPerOctave = 64.f;
constexpr float kMassOne = 1099511627776.f;  // 2^40
constexpr float kInf = __builtin_huge_valf();

struct SampleShared {
  unsigned long long mass[kBins];
  uint32_t count[kBins];
  uint32_t list_key[kList];
  int list_index[kList];
  unsigned long long wave64[kSampleWaves];
  uint32_t wave32[kSampleWaves], wave32b[kSampleWaves];
  float wavef[kSampleWaves];
  // what the scan found
  unsigned long long before_mass, total_mass, kept_mass;
  uint32_t before_count, in_bin, listed;
  int bin;
  uint32_t cut_key;
  int cut_index;
};

__device__ __forceinline__ unsigned long long shfl_up64(unsigned long long v, int by) {
  const uint32_t lo = __shfl_up((uint32_t)v, by), hi = __shfl_up((uint32_t)(v >> 32), by);
  return ((unsigned long long)hi << 32) | lo;
}
__device__ __forceinline__ unsigned long long wave_max64(unsigned long long v) {
#pragma unroll
  for (int by = 1; by < 64; by *= 2) {
    const uint32_t lo = __shfl_xor((uint32_t)v, by), hi = __shfl_xor((uint32_t)(v >> 32), by);
    const unsigned long long o = ((unsigned long long)hi << 32) | lo;
    v = o > v ? o : v;
  }
  return v;
}

// One row of logits as a workgroup sees it: in registers (V units of eight per lane; unit i * threads + t), or read again for
// every pass where a row is longer than the registers are (V = 0).
template <typename T, int V>
struct Row {
  const T* p;
  int n;
  float at[V > 0 ? V : 1][kUnit];

  static __device__ __forceinline__ float clean(float l) { return l != l ? -kInf : l; }  // a NaN is never taken
  __device__ __forceinline__ void load() {
    if constexpr (V > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int first = (i * kSampleThreads + (int)threadIdx.x) * kUnit;
        load_unit(p + first, n - first, at[i]);
#pragma unroll
        for (int j = 0; j < kUnit; ++j) at[i][j] = first + j < n ? clean(at[i][j]) : -kInf;
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if constexpr (V > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < kUnit; ++j) f(at[i][j], (i * kSampleThreads + (int)threadIdx.x) * kUnit + j);
    } else {
      for (int first = (int)threadIdx.x * kUnit; first < n; first += kSampleThreads * kUnit) {
        float v[kUnit];
        load_unit(p + first, n - first, v);
#pragma unroll
        for (int j = 0; j < kUnit; ++j) f(first + j < n ? clean(v[j]) : -kInf, first + j);
      }
    }
  }
};

__device__ __forceinline__ float block_max(float v, SampleShared& s) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wavef[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s.wavef[0];
#pragma unroll
  for (int w = 1; w < kSampleWaves; ++w) v = fmaxf(v, s.wavef[w]);
  return v;
}
__device__ __forceinline__ float block_sum(float v, SampleShared& s) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wavef[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) v += s.wavef[w];
  return v;
}
__device__ __forceinline__ int block_sum_i(int v, SampleShared& s) {
  v = wave_sum_i(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wave32[threadIdx.x >> 6] = (uint32_t)v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kSampleWaves; ++w) v += (int)s.wave32[w];
  return v;
}

// The distance below the largest logit in octaves of probability, its weight, its bin
struct Scale {
  float top, per;  // largest logit; octaves per unit of logit (log2(e) / temperature)
  bool at_infinity;  // the largest is +inf: such tokens share the mass, nothing else has any
  __device__ __forceinline__ float below(float l) const {
    if (at_infinity) return l == kInf ? 0.f : kInf;
    return (top - l) * per;
  }
};
__device__ __forceinline__ float weight(float below) { return __builtin_amdgcn_exp2f(-below); }
__device__ __forceinline__ unsigned long long mass_of(float below) {
  // rintf: half a unit more than the product's own rounding; below 41 octaves nothing is left
  return below < 42.f ? (unsigned long long)rintf(weight(below) * kMassOne) : 0ull;
}
__device__ __forceinline__ int bin_of(float below) { return (int)fminf(below * kBinsPerOctave, (float)(kBins - 1)); }
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}

__device__ __forceinline__ void clear_bins(SampleShared& s) {
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s.mass[threadIdx.x + i * kSampleThreads] = 0;
    s.count[threadIdx.x + i * kSampleThreads] = 0;
  }
  __syncthreads();
}

// The bin in which the running count reaches `tokens` (MASS: the running mass reaches `mass`), and what lies before it.
template <bool MASS>
__device__ void scan_bins(SampleShared& s, uint32_t tokens, unsigned long long mass, uint32_t count0, unsigned long long mass0) {
  __syncthreads();
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const uint32_t c0 = s.count[2 * t], c1 = s.count[2 * t + 1];
  const unsigned long long m0 = s.mass[2 * t], m1 = s.mass[2 * t + 1];
  uint32_t c = c0 + c1;
  unsigned long long m = m0 + m1;
#pragma unroll
  for (int by = 1; by < 64; by *= 2) {
    const uint32_t pc = __shfl_up(c, by);
    const unsigned long long pm = shfl_up64(m, by);
    if (lane >= by) { c += pc; m += pm; }
  }
  if (lane == 63) { s.wave32b[wave] = c; s.wave64[wave] = m; }
  __syncthreads();
  c += count0;
  m += mass0;
  for (int w = 0; w < wave; ++w) { c += s.wave32b[w]; m += s.wave64[w]; }
  if (t == kSampleThreads - 1) s.total_mass = m;
  c -= c0 + c1;
  m -= m0 + m1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t ci = i ? c1 : c0;
    const unsigned long long mi = i ? m1 : m0;
    const bool here = MASS ? (m < mass && m + mi >= mass) : (c < tokens && c + ci >= tokens);
    if (here) {
      s.bin = 2 * t + i;
      s.before_count = c;
      s.before_mass = m;
      s.in_bin = ci;
    }
    c += ci;
    m += mi;
  }
  __syncthreads();
}

// Fills the bins of the whole row.
template <typename R>
__device__ void fill_bins(const R& row, const Scale& sc, SampleShared& s) {
  clear_bins(s);
  // the last bin takes the far tail, most of a row: summed in registers, not by everybody at one address
  uint32_t tail_count = 0;
  unsigned long long tail_mass = 0;
  row.each([&](float l, int) {
    const float below = sc.below(l);
    const int bin = bin_of(below);
    if (bin < kBins - 1) {
      atomicAdd(&s.count[bin], 1u);
      atomicAdd(&s.mass[bin], mass_of(below));
    } else {
      tail_count += l > -kInf;
      tail_mass += mass_of(below);
    }
  });
  if (tail_count) {
    atomicAdd(&s.count[kBins - 1], tail_count);
    atomicAdd(&s.mass[kBins - 1], tail_mass);
  }
}

// The cut inside the bin that the scan found: the token at which the count reaches `tokens` (the mass `mass`).  Leaves it in
// s.cut_key / s.cut_index and the mass up to and with it in s.kept_mass.  Returns whether the bins were overwritten.
template <bool MASS, typename R>
__device__ bool cut_in_bin(const R& row, const Scale& sc, SampleShared& s, uint32_t tokens, unsigned long long mass) {
  const int t = threadIdx.x;
  const int bin = s.bin;
  uint32_t before_count = s.before_count, members = s.in_bin;
  unsigned long long before_mass = s.before_mass;
  bool overwritten = false;
  uint32_t low = 1, high = 0;  // keys of the members; low > high: those of the bin
  if (members > kList) {
    // Too many: split the range of their keys again, 11 bits at a time
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    row.each([&](float l, int) {
      if (l > -kInf && bin_of(sc.below(l)) == bin) {
        const uint32_t key = ordered_key(l);
        lo = min(lo, key);
        hi = max(hi, key);
      }
    });
    const unsigned long long hi64 = wave_max64(hi), lo64 = wave_max64(~lo);
    __syncthreads();
    if ((t & 63) == 0) { s.wave32[t >> 6] = (uint32_t)hi64; s.wave32b[t >> 6] = (uint32_t)lo64; }
    __syncthreads();
    hi = lo = 0;
    for (int w = 0; w < kSampleWaves; ++w) { hi = max(hi, s.wave32[w]); lo = max(lo, s.wave32b[w]); }
    high = hi;
    low = ~lo;
    overwritten = true;
    while (members > kList && low < high) {
      const int bits = 32 - __clz(high - low);
      const int shift = bits > 11 ? bits - 11 : 0;
      clear_bins(s);
      row.each([&](float l, int) {
        const uint32_t key = ordered_key(l);
        if (l > -kInf && key >= low && key <= high) {
          atomicAdd(&s.count[(high - key) >> shift], 1u);
          atomicAdd(&s.mass[(high - key) >> shift], mass_of(sc.below(l)));
        }
      });
      scan_bins<MASS>(s, tokens, mass, before_count, before_mass);
      before_count = s.before_count;
      before_mass = s.before_mass;
      members = s.in_bin;
      high -= (uint32_t)s.bin << shift;
      const uint32_t span = (1u << shift) - 1u;
      low = high - low > span ? high - span : low;
    }
  }
  if (members > kList) {
    // all of one value: the cut is the r-th of them by index, found by halving the range of indices
    const unsigned long long each = mass_of(sc.below(logit_of(high)));
    uint32_t r = tokens - before_count;
    if (MASS) r = each ? (uint32_t)((mass - before_mass + each - 1) / each) : members;
    int lo = 0, hi = row.n - 1;
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      int c = 0;
      row.each([&](float l, int at) { c += l > -kInf && ordered_key(l) == high && at <= mid; });
      if ((uint32_t)block_sum_i(c, s) >= r) hi = mid;
      else lo = mid + 1;
    }
    __syncthreads();
    if (t == 0) {
      s.cut_key = high;
      s.cut_index = lo;
      s.kept_mass = before_mass + r * each;
    }
    __syncthreads();
    return overwritten;
  }
  __syncthreads();
  if (t == 0) s.listed = 0;
  __syncthreads();
  row.each([&](float l, int at) {
    if (!(l > -kInf)) return;
    const uint32_t key = ordered_key(l);
    if (low > high ? bin_of(sc.below(l)) == bin : (key >= low && key <= high)) {
      const uint32_t to = atomicAdd(&s.listed, 1u);  // in any order: the ranks below do not depend on it
      s.list_key[to] = key;
      s.list_index[to] = at;
    }
  });
  __syncthreads();
  if (t < (int)members) {
    const uint32_t key = s.list_key[t];
    const int at = s.list_index[t];
    uint32_t c = before_count;
    unsigned long long m = before_mass;
    for (int j = 0; j < (int)members; ++j) {
      const uint32_t k = s.list_key[j];
      if (k > key || (k == key && s.list_index[j] < at)) {
        ++c;
        m += mass_of(sc.below(logit_of(k)));
      }
    }
    const unsigned long long own = mass_of(sc.below(logit_of(key)));
    if (MASS ? (m < mass && m + own >= mass) : c + 1 == tokens) {
      s.cut_key = key;
      s.cut_index = at;
      s.kept_mass = m + own;
    }
  }
  __syncthreads();
  return overwritten;
}

template <typename T, int V>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared s;
  const int t = threadIdx.x;
  const long long r = blockIdx.x;
  Row<T, V> row;
  row.p = (const T*)a.logits + r * a.stride;
  row.n = a.n;
  row.load();
  const float temperature = a.temperature ? a.temperature[r] : 1.f;
  const int k = a.top_k ? a.top_k[r] : 0;
  const float p = a.top_p ? a.top_p[r] : 1.f;
  const float min_p = a.min_p ? a.min_p[r] : 0.f;

  Scale sc;
  float top = -kInf;
  row.each([&](float l, int) { top = fmaxf(top, l); });
  sc.top = block_max(top, s);
  if (sc.top == -kInf) {
    if (t == 0) {
      a.token[r] = -1;
      if (a.prob) a.prob[r] = 0.f;
    }
    return;
  }
  const bool greedy = !(temperature > 0.f);
  sc.at_infinity = sc.top == kInf;
  sc.per = greedy ? 1.f : fminf(1.44269504088896340736f / temperature, 1e30f);  // (0 times it stays 0)

  uint32_t cut_key = 0;  // below every key
  int cut_index = 0x7FFFFFFF;
  if (!greedy) {
    const bool by_count = k > 0 && k < a.n, by_mass = p < 1.f;
    if (by_count || by_mass) {
      bool filled = false;
      unsigned long long inside = 0;  // mass of the first k
      bool cut_by_count = false;
      fill_bins(row, sc, s);
      filled = true;
      if (t == 0) s.bin = -1;
      scan_bins<false>(s, by_count ? (uint32_t)k : 0xFFFFFFFFu, 0, 0, 0);
      inside = s.total_mass;
      cut_by_count = by_count && s.bin >= 0;  // fewer than k tokens have a logit above -inf: all of them stay
      if (cut_by_count) {
        filled = !cut_in_bin<false>(row, sc, s, (uint32_t)k, 0);
        cut_key = s.cut_key;
        cut_index = s.cut_index;
        inside = s.kept_mass;
      }
      if (by_mass) {
        const double share = p > 0.f ? ceil((double)p * (double)inside) : 1.0;
        unsigned long long mass = (unsigned long long)share;
        mass = mass < 1 ? 1 : mass > inside ? inside : mass;
        if (!filled) fill_bins(row, sc, s);
        scan_bins<true>(s, 0, mass, 0, 0);
        cut_in_bin<true>(row, sc, s, 0, mass);
        cut_key = s.cut_key;
        cut_index = s.cut_index;
      }
    }
  }

  // The race among what is left.  The first token of the order always takes part, whatever the filters say.
  float z = 0.f;
  unsigned long long best = 0;
  const float* noise = a.noise ? a.noise + r * a.noise_stride : nullptr;
  row.each([&](float l, int at) {
    const float below = sc.below(l);
    const float w = weight(below);
    const uint32_t key = ordered_key(l);
    bool kept = l > -kInf && below < kInf && (key > cut_key || (key == cut_key && at <= cut_index));
    kept = greedy ? l == sc.top : kept && (w >= min_p || l == sc.top);
    if (kept) {
      z += w;
      float ring = greedy || !noise ? -below : -below - __builtin_amdgcn_logf(noise[at]);  // (base 2)
      ring = ring == ring ? ring : -kInf;  // a number that is none loses
      const unsigned long long mine = ((unsigned long long)ordered_key(ring) << 32) | (uint32_t)~at;
      best = mine > best ? mine : best;
    }
  });
  z = block_sum(z, s);
  best = wave_max64(best);
  if ((t & 63) == 0) s.wave64[t >> 6] = best;
  __syncthreads();
  if (t == 0) {
    for (int w = 1; w < kSampleWaves; ++w) best = s.wave64[w] > best ? s.wave64[w] : best;
    const int token = (int)~(uint32_t)best;
    a.token[r] = token;
    if (a.prob) {
      const float l = Row<T, V>::clean(load_one(row.p + token));
      a.prob[r] = greedy ? 1.f : weight(sc.below(l)) / z;
    }
  }
}

template <typename T>
void sample(const SampleArgs& a, hipStream_t st) {
  const int units = (a.n + kSampleThreads * kUnit - 1) / (kSampleThreads * kUnit);
  if (units <= 1) sample_kernel<T, 1><<<a.rows, kSampleThreads, 0, st>>>(a);
  else if (units <= 2) sample_kernel<T, 2><<<a.rows, kSampleThreads, 0, st>>>(a);
  else if (units <= 4) sample_kernel<T, 4><<<a.rows, kSampleThreads, 0, st>>>(a);
  else if (units <= 8) sample_kernel<T, 8><<<a.rows, kSampleThreads, 0, st>>>(a);
  else sample_kernel<T, 0><<<a.rows, kSampleThreads, 0, st>>>(a);
}

}  // namespace

void launch_sample(const SampleArgs& a, int dtype, hipStream_t st) {
  if (dtype == A2SF_F32) sample<float>(a, st);
  else sample<bf16_t>(a, st);
}

}  // namespace a2sf
