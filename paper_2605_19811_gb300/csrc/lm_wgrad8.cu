// Weight gradient of a linear layer whose input was kept in 8 bits:
// dW (+)= dY^T X, X = code * scale (lm_linear_wgrad8 in lionmuon.h).  A block
// computes a 64 x 64 tile of dW with fp32 multiply-adds, 16 tokens at a time.
#include <cuda_bf16.h>

#include "lm_code8.cuh"
#include "lm_train.h"

namespace lm {
namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

template <int kFormat>
__global__ void __launch_bounds__(kThreads) wgrad8_kernel(const WgradParams p) {
  __shared__ float dy[kStep][kTile + 4], x[kStep][kTile + 4];
  const int o0 = blockIdx.y * kTile, i0 = blockIdx.x * kTile;
  const int to = (threadIdx.x >> 4) * 4, ti = (threadIdx.x & 15) * 4;
  float acc[4][4] = {};
  for (int64_t t0 = 0; t0 < p.tokens; t0 += kStep) {
    for (int e = threadIdx.x; e < kStep * kTile; e += kThreads) {
      const int64_t t = t0 + e / kTile;
      const int o = o0 + e % kTile, i = i0 + e % kTile;
      float a = 0.f, b = 0.f;
      if (t < p.tokens && o < p.out)
        a = p.dydt == LM_F32 ? static_cast<const float*>(p.dy.data)[t * p.dy.ld + o]
                             : __bfloat162float(static_cast<const __nv_bfloat16*>(p.dy.data)[t * p.dy.ld + o]);
      if (t < p.tokens && i < p.in)
        b = code8::decode2<kFormat>(p.x.data[t * p.x.ld + i]).x * p.x.scales[(i / LM_CODE_GROUP) * p.x.ld_scales + t];
      dy[e / kTile][e % kTile] = a;
      x[e / kTile][e % kTile] = b;
    }
    __syncthreads();
    for (int k = 0; k < kStep; ++k)
      for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) acc[a][b] += dy[k][to + a] * x[k][ti + b];
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a)
    for (int b = 0; b < 4; ++b) {
      const int o = o0 + to + a, i = i0 + ti + b;
      if (o >= p.out || i >= p.in) continue;
      const int64_t at = o * p.dw.ld + i;
      if (p.dwdt == LM_F32) {
        float* d = static_cast<float*>(p.dw.data) + at;
        *d = p.accumulate ? *d + acc[a][b] : acc[a][b];
      } else {
        __nv_bfloat16* d = static_cast<__nv_bfloat16*>(p.dw.data) + at;
        *d = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*d) + acc[a][b] : acc[a][b]);
      }
    }
}

}  // namespace

size_t wgrad8_workspace(int64_t, int64_t, int64_t) { return 0; }

cudaError_t launch_wgrad8(const WgradParams& p, cudaStream_t st) {
  const dim3 grid((p.in + kTile - 1) / kTile, (p.out + kTile - 1) / kTile);
  count_launch();
  if (p.x.format == LM_CODE_I8) wgrad8_kernel<LM_CODE_I8><<<grid, kThreads, 0, st>>>(p);
  else wgrad8_kernel<LM_CODE_E4M3><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace lm
