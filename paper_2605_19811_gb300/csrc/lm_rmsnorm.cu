// RMS norm with the residual's addition and an 8-bit copy of its output, and
// its gradient (formulas at lm_rmsnorm and lm_rmsnorm_grad in lionmuon.h).
// One block per row; a warp takes a group of 128 channels, four to a lane.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_code8.cuh"
#include "lm_train.h"

namespace lm {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

template <typename T> __device__ __forceinline__ float at(const void* p, int64_t i);
template <> __device__ __forceinline__ float at<float>(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
template <> __device__ __forceinline__ float at<__nv_bfloat16>(const void* p, int64_t i) {
  return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ float at(int dt, const void* p, int64_t i) {
  return dt == LM_F32 ? at<float>(p, i) : at<__nv_bfloat16>(p, i);
}
__device__ __forceinline__ void put(int dt, void* p, int64_t i, float v) {
  if (dt == LM_F32) static_cast<float*>(p)[i] = v;
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ float block_sum(float v) {
  __shared__ float part[kWarps];
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < kWarps; ++w) v += part[w];
  return v;
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kThreads) rmsnorm_kernel(const NormParams p) {
  constexpr int dt = sizeof(T) == 4 ? LM_F32 : LM_BF16;
  const int64_t row = blockIdx.x;
  auto h_of = [&](int c) {
    const float x = at<T>(p.x.data, row * p.x.ld + c);
    return p.residual.data != nullptr ? x + at<T>(p.residual.data, row * p.residual.ld + c) : x;
  };
  float s = 0.f;
  for (int c = threadIdx.x; c < p.cols; c += kThreads) {
    const float h = h_of(c);
    s += h * h;
  }
  const float rstd = 1.f / sqrtf(block_sum(s) / (float)p.cols + p.eps);
  if (p.rstd != nullptr && threadIdx.x == 0) p.rstd[row] = rstd;
  const int lane = threadIdx.x & 31;
  for (int c0 = (threadIdx.x >> 5) * LM_CODE_GROUP; c0 < p.cols; c0 += kWarps * LM_CODE_GROUP) {
    float y[4];
    uint32_t most = 0;
    for (int k = 0; k < 4; ++k) {
      const int c = c0 + 4 * lane + k;
      y[k] = 0.f;
      if (c >= p.cols) continue;
      const float h = h_of(c);
      y[k] = h * rstd * (p.weight != nullptr ? at(p.wdt, p.weight, c) : 1.f);
      if (p.y.data != nullptr) put(dt, p.y.data, row * p.y.ld + c, y[k]);
      if (p.h.data != nullptr) put(dt, p.h.data, row * p.h.ld + c, h);   // may be x or residual: read above
      most = max(most, code8::magnitude(y[k]));
    }
    if (kFormat >= 0) {
      most = __reduce_max_sync(0xFFFFFFFFu, most);
      const float scale = code8::group_scale<kFormat>(most), inv = code8::inverse_scale(scale);
      if (lane == 0) p.kept.scales[(c0 / LM_CODE_GROUP) * p.kept.ld_scales + row] = scale;
      const uint32_t four = code8::encode2<kFormat>(y[0], y[1], inv) | (code8::encode2<kFormat>(y[2], y[3], inv) << 16);
      if (c0 + 4 * lane < p.cols)   // the pitch is a multiple of 16: the last word is inside the row
        *reinterpret_cast<uint32_t*>(p.kept.data + row * p.kept.ld + c0 + 4 * lane) = four;
    }
  }
}

// kFormat < 0: h is a matrix.
template <typename T, int kFormat>
__global__ void __launch_bounds__(kThreads) rmsnorm_grad_kernel(const NormGradParams p) {
  constexpr int dt = sizeof(T) == 4 ? LM_F32 : LM_BF16;
  float* part = p.parts + (int64_t)blockIdx.x * p.cols;
  if (p.dweight != nullptr)
    for (int c = threadIdx.x; c < p.cols; c += kThreads) part[c] = 0.f;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const float rstd = p.rstd[row];
    auto xh_of = [&](int c) {
      float h;
      if (kFormat < 0) h = at(p.hdt, p.h.data, row * p.h.ld + c);
      else h = code8::decode2<kFormat>(p.h8.data[row * p.h8.ld + c]).x * p.h8.scales[(c / LM_CODE_GROUP) * p.h8.ld_scales + row];
      return h * rstd;
    };
    auto w_of = [&](int c) { return p.weight != nullptr ? at(p.wdt, p.weight, c) : 1.f; };
    float s = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kThreads) s += w_of(c) * at<T>(p.dy.data, row * p.dy.ld + c) * xh_of(c);
    const float mean = block_sum(s) / (float)p.cols;
    for (int c = threadIdx.x; c < p.cols; c += kThreads) {
      const float dy = at<T>(p.dy.data, row * p.dy.ld + c), xh = xh_of(c);
      float dx = rstd * (w_of(c) * dy - xh * mean);
      if (p.dh.data != nullptr) dx += at<T>(p.dh.data, row * p.dh.ld + c);
      if (p.dx.data != nullptr) put(dt, p.dx.data, row * p.dx.ld + c, dx);
      if (p.dweight != nullptr) part[c] += dy * xh;
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kThreads) norm_dweight_kernel(const float* parts, int nparts, int cols, void* dweight,
                                                                int dwdt) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= cols) return;
  float s = 0.f;
  for (int k = 0; k < nparts; ++k) s += parts[(int64_t)k * cols + c];
  put(dwdt, dweight, c, s);
}

template <typename T>
void launch_fwd(const NormParams& p, cudaStream_t st) {
  const unsigned grid = (unsigned)p.rows;
  if (p.kept.data == nullptr) rmsnorm_kernel<T, -1><<<grid, kThreads, 0, st>>>(p);
  else if (p.kept.format == LM_CODE_I8) rmsnorm_kernel<T, LM_CODE_I8><<<grid, kThreads, 0, st>>>(p);
  else rmsnorm_kernel<T, LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(p);
}
template <typename T>
void launch_bwd(const NormGradParams& p, unsigned grid, cudaStream_t st) {
  if (p.h8.data == nullptr) rmsnorm_grad_kernel<T, -1><<<grid, kThreads, 0, st>>>(p);
  else if (p.h8.format == LM_CODE_I8) rmsnorm_grad_kernel<T, LM_CODE_I8><<<grid, kThreads, 0, st>>>(p);
  else rmsnorm_grad_kernel<T, LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(p);
}

}  // namespace

cudaError_t launch_rmsnorm(lm_dtype dt, const NormParams& p, cudaStream_t st) {
  count_launch();
  if (dt == LM_BF16) launch_fwd<__nv_bfloat16>(p, st);
  else launch_fwd<float>(p, st);
  return cudaGetLastError();
}

cudaError_t launch_rmsnorm_grad(lm_dtype dt, const NormGradParams& p, cudaStream_t st) {
  const int blocks = (int)(p.rows < kNormGradBlocks ? p.rows : kNormGradBlocks);
  if (blocks > 0) {
    count_launch();
    if (dt == LM_BF16) launch_bwd<__nv_bfloat16>(p, blocks, st);
    else launch_bwd<float>(p, blocks, st);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (p.dweight != nullptr) {
    count_launch();
    norm_dweight_kernel<<<(p.cols + kThreads - 1) / kThreads, kThreads, 0, st>>>(p.parts, blocks, p.cols, p.dweight, p.dwdt);
  }
  return cudaGetLastError();
}

}  // namespace lm
