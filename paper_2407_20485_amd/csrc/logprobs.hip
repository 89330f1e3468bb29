// Log probabilities of given tokens, the entropy, and the likeliest tokens of rows of logits.  Bound by memory: the rows are read once
// from there.
#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

constexpr int kLogThreads = 1024, kLogWaves = kLogThreads / 64;
constexpr float kNan = __builtin_nanf("");

template <typename T>
__global__ __launch_bounds__(kLogThreads) void log_probs_kernel(LogProbsArgs a) {
  __shared__ float redf[kLogWaves], redg[kLogWaves];
  __shared__ unsigned long long red64[kLogWaves];
  const long long row = blockIdx.x;
  const T* x = (const T*)a.logits + row * a.stride;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < a.n; i += kLogThreads) top = fmaxf(top, load_one(x + i));
  top = wave_max(top);
  if (lane == 0) redf[wave] = top;
  __syncthreads();
  for (int w = 0; w < kLogWaves; ++w) top = fmaxf(top, redf[w]);
  __syncthreads();
  float z = 0.f, zy = 0.f;
  for (int i = threadIdx.x; i < a.n; i += kLogThreads) {
    const float y = load_one(x + i) - top, w = __expf(y);
    z += w;
    if (w != 0.f) zy += w * y;
  }
  z = wave_sum(z);
  zy = wave_sum(zy);
  if (lane == 0) { redf[wave] = z; redg[wave] = zy; }
  __syncthreads();
  z = zy = 0.f;
  for (int w = 0; w < kLogWaves; ++w) { z += redf[w]; zy += redg[w]; }
  const float lz = logf(z);
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = lz - zy / z;
  for (int i = threadIdx.x; i < a.given; i += kLogThreads) {
    const int token = a.tokens[row * a.token_stride + i];
    a.logp[row * a.logp_stride + i] = token >= 0 && token < a.n ? load_one(x + token) - top - lz : kNan;
  }
  // alternatives one by one: larger keys first, equal ones by index
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.alternatives; ++k) {
    unsigned long long best = 0;
    for (int i = threadIdx.x; i < a.n; i += kLogThreads) {
      const float v = load_one(x + i);
      const unsigned long long key = (unsigned long long)ordered_key(v != v ? -INFINITY : v) << 32 | (uint32_t)~i;
      if (key < last && key > best) best = key;
    }
    best = ~wave_min_u64(~best);
    __syncthreads();
    if (lane == 0) red64[wave] = best;
    __syncthreads();
    for (int w = 0; w < kLogWaves; ++w) best = red64[w] > best ? red64[w] : best;
    last = best;
    if (threadIdx.x == 0) {
      const int token = (int)~(uint32_t)best;
      if (a.top) a.top[row * a.top_stride + k] = load_one(x + token) - top - lz;
      if (a.top_tokens) a.top_tokens[row * a.top_token_stride + k] = token;
    }
  }
}

}  // namespace

bool launch_log_probs(const LogProbsArgs& a, int dtype, hipStream_t st) {
  if (!grid_fits((unsigned long long)a.rows, kLogThreads)) return false;
  if (dtype == A2SF_F32) log_probs_kernel<float><<<(uint32_t)a.rows, kLogThreads, 0, st>>>(a);
  else log_probs_kernel<bf16_t><<<(uint32_t)a.rows, kLogThreads, 0, st>>>(a);
  return true;
}

}  // namespace a2sf
