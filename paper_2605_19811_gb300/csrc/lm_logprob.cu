// Token log probabilities, entropy, top alternatives and their gradient
// (formulas at lm_token_logprob_args in lionmuon.h).  One block per row.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_train.h"

namespace lm {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float value(const __nv_bfloat16* p, int64_t i) { return __bfloat162float(p[i]); }
__device__ __forceinline__ float value(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ void put(__nv_bfloat16* p, int64_t i, float v) { p[i] = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, int64_t i, float v) { p[i] = v; }

// A float's place in the order of floats, as an integer.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

template <typename F>
__device__ __forceinline__ auto block_reduce(decltype(F::none()) v, F f) {
  __shared__ decltype(F::none()) part[kThreads / 32];
  for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < kThreads / 32; ++w) v = f(v, part[w]);
  return v;
}
struct Sum {
  static __device__ float none() { return 0.f; }
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {   // NaN where either is
  static __device__ float none() { return -INFINITY; }
  __device__ float operator()(float a, float b) const { return (a != a || a > b) ? a : b; }
};
struct MaxKey {
  static __device__ unsigned long long none() { return 0ull; }
  __device__ unsigned long long operator()(unsigned long long a, unsigned long long b) const { return a > b ? a : b; }
};

// Largest logit and log of the sum of exponentials above it: log p_j =
// (z_j - m) - log_s.  Kept apart, since beside a large m a sum m + log_s loses
// log_s (a row whose logits all are the type's lowest value).
struct RowStats {
  float m, s, t;   // t = sum e^(z - m) (z - m)
};
template <typename T>
__device__ RowStats row_stats(const T* z, int vocab) {
  float m = -INFINITY;
  for (int j = threadIdx.x; j < vocab; j += kThreads) m = Max()(m, value(z, j));
  m = block_reduce(m, Max());
  float s = 0.f, t = 0.f;
  for (int j = threadIdx.x; j < vocab; j += kThreads) {
    const float d = value(z, j) - m, e = expf(d);
    s += e;
    if (e > 0.f) t += e * d;
  }
  return RowStats{m, block_reduce(s, Sum()), block_reduce(t, Sum())};
}

template <typename T>
__device__ void gradient_row(const LogprobParams& p, int64_t row, const T* z, float lse, float m, float log_s, float entropy) {
  T* d = static_cast<T*>(p.dlogits) + row * p.ld_d;
  const int64_t y = p.targets != nullptr ? p.targets[row] : -1;
  float gl = (p.g_logp != nullptr && y >= 0) ? p.g_logp[row] : 0.f;
  if (y >= p.vocab) gl = __int_as_float(0x7FC00000);
  const float gh = p.g_entropy != nullptr ? p.g_entropy[row] : 0.f;
  const float gz = p.g_lse != nullptr ? p.g_lse[row] : 0.f;
  const bool bad = !(lse < INFINITY) || gl != gl;
  for (int j = threadIdx.x; j < p.vocab; j += kThreads) {
    const float lp = (value(z, j) - m) - log_s;
    const float e = expf(lp);
    float g = e > 0.f ? e * (gz - gl - gh * (lp + entropy)) : 0.f;
    if (lse == -INFINITY) g = 0.f;
    else if (j == y) g += gl;
    put(d, j, bad ? __int_as_float(0x7FC00000) : g);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const LogprobParams p) {
  const int64_t row = blockIdx.x;
  const T* z = static_cast<const T*>(p.logits) + row * p.ld;
  const RowStats r = row_stats(z, p.vocab);
  const float m = r.m, log_s = logf(r.s);
  const float nan = __int_as_float(0x7FC00000);
  float lse = m + log_s, entropy = log_s - r.t / r.s;
  if (m == -INFINITY) {
    lse = -INFINITY;
    entropy = 0.f;
  } else if (!(m < INFINITY)) {
    lse = entropy = nan;
  }
  if (threadIdx.x == 0) {
    if (p.lse != nullptr) p.lse[row] = lse;
    if (p.entropy != nullptr) p.entropy[row] = entropy;
    if (p.logp != nullptr) {
      const int64_t y = p.targets[row];
      float v = 0.f;
      if (lse != lse || y >= p.vocab) v = nan;
      else if (y >= 0) v = lse == -INFINITY ? -INFINITY : (value(z, y) - m) - log_s;
      p.logp[row] = v;
    }
  }
  // the largest keys (value, then lowest index) one after another
  unsigned long long last = ~0ull;
  for (int k = 0; k < p.top_k; ++k) {
    unsigned long long best = 0ull;
    for (int j = threadIdx.x; j < p.vocab; j += kThreads) {
      const float v = value(z, j);
      const unsigned long long key = ((unsigned long long)ordered(v) << 32) | (uint32_t)~j;
      if (v > -INFINITY && key < last && key > best) best = key;
    }
    best = block_reduce(best, MaxKey());
    if (threadIdx.x == 0) {
      const bool has = best != 0ull && lse == lse;
      const int j = (int)~(uint32_t)best;
      p.top_index[row * p.top_k + k] = has ? j : -1;
      p.top_logp[row * p.top_k + k] = lse != lse ? nan : has ? (value(z, j) - m) - log_s : -INFINITY;
    }
    last = best;
  }
  if (p.dlogits != nullptr) {
    __syncthreads();
    gradient_row(p, row, z, lse, m, log_s, entropy);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(const LogprobParams p) {
  const int64_t row = blockIdx.x;
  const T* z = static_cast<const T*>(p.logits) + row * p.ld;
  const float lse = p.lse[row], entropy = p.g_entropy != nullptr ? p.entropy[row] : 0.f;
  // lse alone gives p to 2^-24 |lse| relative; beyond 4096 the row's sums are formed anew
  float m = lse, log_s = 0.f;
  if (fabsf(lse) > 4096.f && fabsf(lse) < INFINITY) {
    const RowStats r = row_stats(z, p.vocab);
    m = r.m;
    log_s = logf(r.s);
    __syncthreads();
  }
  gradient_row(p, row, z, lse, m, log_s, entropy);
}

}  // namespace

cudaError_t launch_logprob(lm_dtype dt, const LogprobParams& p, cudaStream_t st) {
  count_launch();
  if (dt == LM_BF16) logprob_kernel<__nv_bfloat16><<<(unsigned)p.rows, kThreads, 0, st>>>(p);
  else logprob_kernel<float><<<(unsigned)p.rows, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}
cudaError_t launch_logprob_grad(lm_dtype dt, const LogprobParams& p, cudaStream_t st) {
  count_launch();
  if (dt == LM_BF16) logprob_grad_kernel<__nv_bfloat16><<<(unsigned)p.rows, kThreads, 0, st>>>(p);
  else logprob_grad_kernel<float><<<(unsigned)p.rows, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace lm
