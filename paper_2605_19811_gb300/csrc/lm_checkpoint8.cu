// Packing a matrix into 8-bit codes with a power-of-two scale for each group
// of 128 channels (the format is stated at lm_checkpoint8 in lionmuon.h), and
// back.  A warp takes one group, four channels to a lane.
#include <cuda_bf16.h>

#include "lm_code8.cuh"
#include "lm_train.h"

namespace lm {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float get(const float* p) { return *p; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

template <typename T, int kFormat>
__global__ void __launch_bounds__(kThreads) pack8_kernel(Mat x, int64_t rows, int64_t cols, Codes c) {
  const int64_t groups = (cols + LM_CODE_GROUP - 1) / LM_CODE_GROUP;
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); w < rows * groups; w += nwarps) {
    const int64_t row = w / groups, group = w % groups, c0 = group * LM_CODE_GROUP + 4 * lane;
    const T* src = static_cast<const T*>(x.data) + row * x.ld + c0;
    float v[4];
    uint32_t most = 0;
    for (int k = 0; k < 4; ++k) {
      v[k] = c0 + k < cols ? get(src + k) : 0.f;
      most = max(most, code8::magnitude(v[k]));
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    const float scale = code8::group_scale<kFormat>(most), inv = code8::inverse_scale(scale);
    if (lane == 0) c.scales[group * c.ld_scales + row] = scale;
    const uint32_t four = code8::encode2<kFormat>(v[0], v[1], inv) | (code8::encode2<kFormat>(v[2], v[3], inv) << 16);
    if (c0 < cols) *reinterpret_cast<uint32_t*>(c.data + row * c.ld + c0) = four;
  }
}

template <typename T, int kFormat>
__global__ void __launch_bounds__(kThreads) unpack8_kernel(Codes c, int64_t rows, int64_t cols, Mat x) {
  const int64_t groups = (cols + LM_CODE_GROUP - 1) / LM_CODE_GROUP;
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); w < rows * groups; w += nwarps) {
    const int64_t row = w / groups, group = w % groups, c0 = group * LM_CODE_GROUP + 4 * lane;
    if (c0 >= cols) continue;
    const float scale = c.scales[group * c.ld_scales + row];
    const uint32_t four = *reinterpret_cast<const uint32_t*>(c.data + row * c.ld + c0);
    const float2 lo = code8::decode2<kFormat>(four), hi = code8::decode2<kFormat>(four >> 16);
    const float v[4] = {lo.x * scale, lo.y * scale, hi.x * scale, hi.y * scale};
    T* dst = static_cast<T*>(x.data) + row * x.ld + c0;
    for (int k = 0; k < 4; ++k)
      if (c0 + k < cols) put(dst + k, v[k]);
  }
}

unsigned grid_for(int64_t rows, int64_t cols) {
  const int64_t warps = rows * ((cols + LM_CODE_GROUP - 1) / LM_CODE_GROUP);
  const int64_t blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  return (unsigned)(blocks < 152 * 16 ? blocks : 152 * 16);
}

}  // namespace

cudaError_t launch_pack8(lm_dtype dt, const Mat& x, int64_t rows, int64_t cols, const Codes& c, cudaStream_t st) {
  const unsigned grid = grid_for(rows, cols);
  count_launch();
  if (dt == LM_BF16 && c.format == LM_CODE_I8) pack8_kernel<__nv_bfloat16, LM_CODE_I8><<<grid, kThreads, 0, st>>>(x, rows, cols, c);
  else if (dt == LM_BF16) pack8_kernel<__nv_bfloat16, LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(x, rows, cols, c);
  else if (c.format == LM_CODE_I8) pack8_kernel<float, LM_CODE_I8><<<grid, kThreads, 0, st>>>(x, rows, cols, c);
  else pack8_kernel<float, LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(x, rows, cols, c);
  return cudaGetLastError();
}

cudaError_t launch_unpack8(lm_dtype dt, const Codes& c, int64_t rows, int64_t cols, const Mat& x, cudaStream_t st) {
  const unsigned grid = grid_for(rows, cols);
  count_launch();
  if (dt == LM_BF16 && c.format == LM_CODE_I8) unpack8_kernel<__nv_bfloat16, LM_CODE_I8><<<grid, kThreads, 0, st>>>(c, rows, cols, x);
  else if (dt == LM_BF16) unpack8_kernel<__nv_bfloat16, LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(c, rows, cols, x);
  else if (c.format == LM_CODE_I8) unpack8_kernel<float, LM_CODE_I8><<<grid, kThreads, 0, st>>>(c, rows, cols, x);
  else unpack8_kernel<float, LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(c, rows, cols, x);
  return cudaGetLastError();
}

}  // namespace lm
