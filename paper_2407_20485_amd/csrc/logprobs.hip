// Log probabilities of given tokens, the entropy, and the likeliest tokens of rows of logits.  Bound by memory: a row is read once.
//
// A workgroup takes a row, a lane eight neighbouring logits at a time.  A lane holds the largest logit m so far, z = sum exp(x - m) and
// zy = sum exp(x - m) (x - m); when m rises by s, zy becomes (zy - s z) e^-s and z becomes z e^-s; lanes join the same way.  The largest
// logit of the row has a term of exactly 1 and 0 in them, so a row with one likely token keeps its small entropy.
//
// The likeliest tokens: of the logits that all lanes ask for first (32 each in bf16, 16 in fp32) the largest in each of 256 groups of lanes
// are looked at; what k of these reach k logits reach, so what is below cannot be among the k.  What is not, in the row as it passes, goes
// to a list (somewhat more than k tokens for each time that the lanes take as many) whose tokens are ranked against each other.  A list
// that overflows (rows that rise, or of few values) is given up and the k found one by one.
//
// 2000 x 50272 in bf16 (201 MB): 42 us = 4.8 TB/s without alternatives, where the vector units are as busy as the memory (100 million
// exponentials), 52 with 20 of them; 1000 rows in fp32 36 us = 5.6 TB/s and 44.
#include <float.h>

#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

constexpr float kNan = __builtin_nanf(""), kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kGroups = 256, kListed = 1024;
constexpr float kFar = -200.f;  // exp(kFar) is 0 in fp32

// exp(y) for y <= 0, by exp2 of a rounded product: within |y| units of rounding of its value.  In a row's results that is about what 32-bit sums leave
// anyhow: 2000 rows of 50272 in bf16 are off by 2.2e-7 (root mean square; log probabilities, 32-bit exp 2.2e-7) and 4.3e-7 (entropies of 6 on the
// average, 3.3e-7).  With what the constant's rounding cuts off put back it is 2.3e-7 and 3.6e-7 for 4 % more time, with all of it 2.3e-7 and 3.7e-7 for 13 %.
__device__ __forceinline__ float exp_of(float y) { return __builtin_amdgcn_exp2f(y * kLog2e); }

struct Sums {
  float m, z, zy;
  __device__ __forceinline__ void rise(float to) {  // to >= m
    const float s = fmaxf(m - to, kFar), k = exp_of(s);  // (what is not a number is so in z already)
    zy = fmaf(z, s, zy) * k;
    z *= k;
    m = to;
  }
};

// larger logits first, equal ones by index; a NaN counts as -infinity
__device__ __forceinline__ unsigned long long token_key(float v, int index) {
  return (unsigned long long)ordered_key(v == v ? v : -kInf) << 32 | (uint32_t)~index;
}

__device__ __forceinline__ float of_key(unsigned long long key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}

// Eight logits as they are in memory; -infinity past the end of the row
template <typename T> struct Eight;
template <> struct Eight<float> {
  float v[kUnit];
  __device__ __forceinline__ void load(const float* x, int first, int n) {
    if (first + kUnit <= n) load_unit(x + first, v);
    else
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[j] = first + j < n ? x[first + j] : -kInf;
  }
  __device__ __forceinline__ float at(int j) const { return v[j]; }
};
template <> struct Eight<bf16_t> {
  u32x4_t v;
  __device__ __forceinline__ void load(const bf16_t* x, int first, int n) {
    if (first + kUnit <= n) v = *(const u32x4_at2_t*)(x + first);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = first + 2 * j < n ? x[first + 2 * j] : 0xFF80u, hi = first + 2 * j + 1 < n ? x[first + 2 * j + 1] : 0xFF80u;
        v[j] = lo | hi << 16;
      }
  }
  __device__ __forceinline__ float at(int j) const { return __uint_as_float(j & 1 ? v[j / 2] & 0xFFFF0000u : v[j / 2] << 16); }
};

// The largest logit, and a number that at least k of the groups' largest logits reach, and not many more: the range of their keys is cut in eight until it is found.
// For one wave, four groups to a lane.
__device__ __forceinline__ float floor_of(const float* group_top, int k, float& largest) {
  const float4 v = *(const float4*)(group_top + 4 * (threadIdx.x & 63));
  const uint32_t key[4] = {ordered_key(v.x), ordered_key(v.y), ordered_key(v.z), ordered_key(v.w)};
  const uint32_t least = min(min(key[0], key[1]), min(key[2], key[3])), most = max(max(key[0], key[1]), max(key[2], key[3]));
  uint32_t lo = ~((uint32_t)wave_max_i((int)(~least ^ 0x80000000u)) ^ 0x80000000u);   // all reach it
  uint32_t hi = ((uint32_t)wave_max_i((int)(most ^ 0x80000000u)) ^ 0x80000000u) + 1u;  // none does
  largest = of_key((unsigned long long)(hi - 1u) << 32);
  for (int round = 0; k > 0 && round < 11 && hi - lo > 1; ++round) {
    const uint32_t width = hi - lo, step = width / 8 + 1;
    int count = kGroups;
    uint32_t from = lo, to = hi;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      if (step * i >= width) break;
      const uint32_t cut = lo + step * i;
      int n = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) n += __popcll(__ballot(key[j] >= cut));
      if (n < k) {
        to = cut;
        break;
      }
      from = cut;
      count = n;
    }
    lo = from;
    hi = to;
    if (count <= k + k / 4 + 4) break;
  }
  return of_key((unsigned long long)lo << 32);
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, 8) void log_probs_kernel(LogProbsArgs a) {
  constexpr int WAVES = THREADS / 64, STEP = THREADS * kUnit, DEPTH = sizeof(T) == 2 ? 4 : 2;  // steps on their way
  __shared__ unsigned long long list[kListed], kept[A2SF_MAX_ALTERNATIVES];
  __shared__ __attribute__((aligned(16))) float group_top[kGroups];
  __shared__ float sm[WAVES], sz[WAVES], szy[WAVES];
  __shared__ unsigned long long best_of[WAVES];
  __shared__ int listed;
  __shared__ float shared_floor, shared_top;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long row = blockIdx.x;
  const T* x = (const T*)a.logits + row * a.stride;
  const int n = a.n, k = a.alternatives;
  Sums sums = {-FLT_MAX, 0.f, 0.f};
  Eight<T> f[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) f[i].load(x, i * STEP + tid * kUnit, n);  // (at most 3 STEP past 2^22)
  const auto top_of = [&](const Eight<T>& v) {
    float top = v.at(0);
#pragma unroll
    for (int j = 1; j < kUnit; ++j) top = fmaxf(top, v.at(j));
    return top;
  };
  const auto given_logit = [&](int i) {
    const int token = a.tokens[row * a.token_stride + i];
    return token >= 0 && token < n ? load_one(x + token) : kNan;
  };
  const float given = tid < a.given ? given_logit(tid) : 0.f;  // (asked for now: the end does not wait for it)
  // What is below cannot be one of the k (nor is what is infinitely far below).  All lanes begin with the largest logit of the first
  // ones of each: few rise later.
  float floor;
  {
    float top = top_of(f[0]);
#pragma unroll
    for (int i = 1; i < DEPTH; ++i) top = fmaxf(top, top_of(f[i]));
    if (THREADS >= 512) top = fmaxf(top, dpp_move<0xB1>(top));  // two or four lanes to a group
    if (THREADS == 1024) top = fmaxf(top, dpp_move<0x4E>(top));
    if (tid % (THREADS / kGroups) == 0) group_top[tid / (THREADS / kGroups)] = top == top ? top : -kInf;
    if (tid == 0) listed = 0;
    __syncthreads();
    if (wave == 0) {
      float most;
      const float bound = floor_of(group_top, k, most);
      if (lane == 0) {
        shared_floor = fmaxf(bound, -FLT_MAX);
        shared_top = fmaxf(most, -FLT_MAX);
      }
    }
    __syncthreads();
    floor = k > 0 ? shared_floor : kInf;
    sums.m = shared_top;
  }
  // the listed tokens ranked against each other: f(rank, token's key), eight lanes to a token, which share out the others
  const auto ranked = [&](int count, auto f) {
    for (int i0 = 0; i0 < count; i0 += THREADS / 8) {
      const int i = i0 + tid / 8;
      const unsigned long long mine = i < count ? list[i] : 0;
      uint32_t rank = 0;
#pragma unroll 4
      for (int j = tid % 8; j < count; j += 8) rank += list[j] > mine;
      rank += dpp_move_u32<0xB1>(rank);
      rank += dpp_move_u32<0x4E>(rank);
      rank += dpp_move_u32<0x141>(rank);
      if (tid % 8 == 0 && i < count && rank < (uint32_t)k) f((int)rank, mine);
    }
  };
  const int steps = (n + STEP - 1) / STEP;
  int look = 4;  // the list is looked at after 4, 8, 16 .. steps: the next ones as many add about k to a list of k
  for (int s0 = 0; s0 < steps; s0 += DEPTH) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      const int s = s0 + i;
      if (s >= steps) break;
      const int first = s * STEP + tid * kUnit;
      const float top = top_of(f[i]);
      if (top >= floor && k > 0) {
#pragma unroll
        for (int j = 0; j < kUnit; ++j)
          if (f[i].at(j) >= floor) {
            const int at = atomicAdd(&listed, 1);
            if (at < kListed) list[at] = token_key(f[i].at(j), first + j);
          }
      }
      if (__any(top > sums.m)) sums.rise(fmaxf(sums.m, top));
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const float y = f[i].at(j) - sums.m, w = exp_of(y);
        sums.z += w;
        sums.zy = fmaf(w, fmaxf(y, kFar), sums.zy);  // (-infinity has no weight)
      }
      if (s + DEPTH < steps) f[i].load(x, first + DEPTH * STEP, n);
      if (k > 0 && s + 1 == look && s + 1 < steps) {
        look *= 2;
        __syncthreads();
        const int count = listed;
        __syncthreads();
        if (count > kListed / 4 && count <= kListed) {
          ranked(count, [&](int rank, unsigned long long key) { kept[rank] = key; });
          __syncthreads();
          if (tid < k) list[tid] = kept[tid];
          if (tid == 0) listed = k;
          floor = of_key(kept[k - 1]);
          __syncthreads();
        }
      }
    }
  }
  sums.rise(wave_max(sums.m));
  sums.z = wave_sum(sums.z);
  sums.zy = wave_sum(sums.zy);
  if (lane == 0) {
    sm[wave] = sums.m;
    sz[wave] = sums.z;
    szy[wave] = sums.zy;
  }
  __syncthreads();
  {  // the waves' sums, one to a lane of a row of 16 (or four times each)
    const int w = lane % WAVES;
    sums = {sm[w], sz[w], szy[w]};
    sums.rise(wave_max(sums.m));
    sums.z = group_sum<16>(sums.z) * (WAVES / 16.f);
    sums.zy = group_sum<16>(sums.zy) * (WAVES / 16.f);
  }
  const float top = sums.m, lz = sums.z > 0.f ? logf(sums.z) : kNan;
  if (tid == 0 && a.entropy) a.entropy[row] = lz - sums.zy / sums.z;
  const auto logp_of = [&](float v) { return (v - top) - lz; };
  if (tid < a.given) a.logp[row * a.logp_stride + tid] = logp_of(given);
  for (int i = tid + THREADS; i < a.given; i += THREADS) a.logp[row * a.logp_stride + i] = logp_of(given_logit(i));
  if (k == 0) return;
  const auto put = [&](int rank, unsigned long long key, float v) {
    if (a.top) a.top[row * a.top_stride + rank] = logp_of(v);
    if (a.top_tokens) a.top_tokens[row * a.top_token_stride + rank] = (int)~(uint32_t)key;
  };
  const int count = listed;
  if (count <= kListed) {
    ranked(count, [&](int rank, unsigned long long key) { put(rank, key, of_key(key)); });
    if (count < k && wave == 0) {
      // fewer tokens than asked for have any probability: the first ones of the others follow, which are among the first k of the row
      const float v = lane < k ? load_one(x + lane) : 0.f;
      const unsigned long long others = __ballot(lane < k && !(v > -kInf));
      const int rank = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(others >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)others, 0));
      if ((others >> lane & 1) && rank < k) put(rank, ~(unsigned long long)lane, v);
    }
    return;
  }
  unsigned long long last = ~0ull;
  for (int i = 0; i < k; ++i) {
    unsigned long long best = 0;
    for (int j = tid; j < n; j += THREADS) {
      const unsigned long long key = token_key(load_one(x + j), j);
      if (key < last && key > best) best = key;
    }
    best = ~wave_min_u64(~best);
    __syncthreads();
    if (lane == 0) best_of[wave] = best;
    __syncthreads();
#pragma unroll 1
    for (int w = 0; w < WAVES; ++w) best = best_of[w] > best ? best_of[w] : best;
    last = best;
    if (tid == 0) put(i, best, of_key(best));
  }
}

template <typename T>
bool launch(const LogProbsArgs& a, hipStream_t st) {
  if (!grid_fits((unsigned long long)a.rows, 1024)) return false;
  // Half as many lanes to a row where there are more rows than the chip holds at once with 1024 to each: a row's barriers then wait beside
  // others' work (us with 512 / 1024 lanes, 50272 logits in bf16: 2000 rows with 20 alternatives 52 / 61, with 33 57 / 63, with 64, whose list grows
  // longer, 73 / 69; 513 rows 20 / 23, 300 rows 17.6 / 16.8).  Short rows take 256 (2000 rows of 8192 14.0, 17.5 with 512; 100 rows of 4096 in fp32 5.6, 6.8 with 1024,
  // of 16384 9.8 and 6.3).
  if (a.n <= 8192) log_probs_kernel<T, 256><<<(uint32_t)a.rows, 256, 0, st>>>(a);
  else if (a.rows > 512 && a.alternatives <= 32) log_probs_kernel<T, 512><<<(uint32_t)a.rows, 512, 0, st>>>(a);
  else log_probs_kernel<T, 1024><<<(uint32_t)a.rows, 1024, 0, st>>>(a);
  return true;
}

}  // namespace

bool launch_log_probs(const LogProbsArgs& a, int dtype, hipStream_t st) {
  return dtype == A2SF_F32 ? launch<float>(a, st) : launch<bf16_t>(a, st);
}

}  // namespace a2sf
