// Queries and keys: the norm of each head, its gain, and the rotation by
// position, in one pass, and the gradient (formulas at lm_qk_rotary_args in
// lionmuon.h).
//
// A warp takes a head of a token.  For the gradient the head's rstd is computed
// again: the head is read anyway.  dweight: each warp keeps sums over its heads in
// shared memory, a block's are joined, and a second kernel adds the blocks', all
// in a fixed order.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_train.h"
#include "lm_gemm_tc.cuh"

namespace lm {
namespace {

using gemm::launch_after;
using tc::griddep_launch_dependents;
using tc::griddep_wait;

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kMostBlocks = 152 * 4;
constexpr uint32_t kAll = 0xFFFFFFFFu;

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float gain(const void* w, int dt, int c) {
  if (w == nullptr) return 1.f;
  return dt == LM_F32 ? static_cast<const float*>(w)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c]);
}
template <typename T>
__device__ __forceinline__ T* head_of(const Heads& h, int64_t token, int head) {
  return static_cast<T*>(h.data) + token * h.ld_token + head * h.ld_head;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// The i-th of a head's turned / 2 pairs and, after them, of its other channels:
// one or two channels.
struct Channels {
  int a, b;     // b < 0: a channel that does not turn
};
__device__ __forceinline__ Channels channels(int i, int turned, bool interleaved) {
  const int half = turned >> 1;
  if (i >= half) return {turned + (i - half), -1};
  return interleaved ? Channels{2 * i, 2 * i + 1} : Channels{i, i + half};
}
__device__ __forceinline__ float2 turn_of(const RotaryParams& p, int64_t token, int i) {
  const int64_t at = p.positions[token];
  if (at < 0 || at >= p.table_rows) return make_float2(__int_as_float(0x7FC00000), __int_as_float(0x7FC00000));
  const float* t = p.table + (at * (p.turned >> 1) + i) * 2;
  return make_float2(t[0], t[1]);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, heads = p.part[0].heads + p.part[1].heads;
  const int items = (p.turned >> 1) + (p.dim - p.turned);
  const int64_t all = p.tokens * heads;
  for (int64_t i = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); i < all; i += (int64_t)gridDim.x * kWarps) {
    const int64_t token = i / heads;
    int head = (int)(i - token * heads);
    const RotaryPart& part = p.part[head >= p.part[0].heads ? 1 : 0];
    if (head >= p.part[0].heads) head -= p.part[0].heads;
    const T* x = head_of<const T>(part.x, token, head);
    T* y = head_of<T>(part.y, token, head);
    float rstd = 1.f;
    if (p.norm) {
      float s = 0.f;
      for (int c = lane; c < p.dim; c += 32) {
        const float v = value(x + c);
        s += v * v;
      }
      rstd = 1.f / sqrtf(warp_sum(s) / (float)p.dim + p.eps);
    }
    for (int k = lane; k < items; k += 32) {
      const Channels c = channels(k, p.turned, p.interleaved);
      const float a = value(x + c.a) * rstd * gain(part.weight, part.wdt, c.a);
      if (c.b < 0) {
        put(y + c.a, a);
        continue;
      }
      const float b = value(x + c.b) * rstd * gain(part.weight, part.wdt, c.b);
      const float2 t = turn_of(p, token, k);
      put(y + c.a, a * t.x - b * t.y);
      put(y + c.b, b * t.x + a * t.y);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rotary_grad_kernel(const __grid_constant__ RotaryParams p) {
  extern __shared__ float sums[];     // warps x dim
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const RotaryPart& part = p.part[blockIdx.y];
  const int items = (p.turned >> 1) + (p.dim - p.turned);
  const bool dw = part.dweight != nullptr;
  float* mine = sums + warp * p.dim;
  if (dw)
    for (int c = lane; c < p.dim; c += 32) mine[c] = 0.f;
  __syncwarp();
  const int64_t all = p.tokens * part.heads;
  for (int64_t i = (int64_t)blockIdx.x * kWarps + warp; i < all; i += (int64_t)gridDim.x * kWarps) {
    const int64_t token = i / part.heads;
    const int head = (int)(i - token * part.heads);
    const T* dy = head_of<const T>(part.dy, token, head);
    const T* x = head_of<const T>(part.x, token, head);
    T* dx = head_of<T>(part.dx, token, head);
    float rstd = 1.f, mean = 0.f;
    auto back = [&](int k, const Channels& c, float& a, float& b) {
      a = value(dy + c.a);
      b = 0.f;
      if (c.b < 0) return;
      b = value(dy + c.b);
      const float2 t = turn_of(p, token, k);
      const float u = a * t.x + b * t.y;
      b = b * t.x - a * t.y;
      a = u;
    };
    if (p.norm) {
      float s = 0.f, q = 0.f;
      for (int k = lane; k < items; k += 32) {
        const Channels c = channels(k, p.turned, p.interleaved);
        float a, b;
        back(k, c, a, b);
        const float xa = value(x + c.a);
        s += xa * xa;
        q += a * gain(part.weight, part.wdt, c.a) * xa;
        if (c.b < 0) continue;
        const float xb = value(x + c.b);
        s += xb * xb;
        q += b * gain(part.weight, part.wdt, c.b) * xb;
      }
      rstd = 1.f / sqrtf(warp_sum(s) / (float)p.dim + p.eps);
      mean = warp_sum(q) * rstd / (float)p.dim;
    }
    for (int k = lane; k < items; k += 32) {
      const Channels c = channels(k, p.turned, p.interleaved);
      float d[2];
      back(k, c, d[0], d[1]);
      const int at[2] = {c.a, c.b};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (at[j] < 0) continue;
        float g = d[j];
        if (p.norm) {
          const float xh = value(x + at[j]) * rstd;
          if (dw) mine[at[j]] += g * xh;
          g = rstd * (g * gain(part.weight, part.wdt, at[j]) - xh * mean);
        }
        put(dx + at[j], g);
      }
    }
  }
  if (!dw) return;
  __syncthreads();
  for (int c = threadIdx.x; c < p.dim; c += kThreads) {
    float s = 0.f;
    for (int k = 0; k < kWarps; ++k) s += sums[k * p.dim + c];
    p.sums[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * p.dim + c] = s;
  }
}

// dweight of each part: the blocks' sums added, a warp a channel.
__global__ void __launch_bounds__(kThreads) rotary_join_kernel(const __grid_constant__ RotaryParams p, int blocks) {
  griddep_wait();
  griddep_launch_dependents();
  const int c = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const RotaryPart& part = p.part[blockIdx.y];
  if (c >= p.dim || part.dweight == nullptr) return;
  const float* from = p.sums + (int64_t)blockIdx.y * blocks * p.dim + c;
  float s = 0.f;
  for (int k = threadIdx.x & 31; k < blocks; k += 32) s += from[(int64_t)k * p.dim];
  s = warp_sum(s);
  if ((threadIdx.x & 31) != 0) return;
  if (part.dwdt == LM_F32) static_cast<float*>(part.dweight)[c] = s;
  else static_cast<__nv_bfloat16*>(part.dweight)[c] = __float2bfloat16_rn(s);
}

int grad_blocks(int64_t tokens, int64_t heads) {
  const int64_t b = (tokens * heads + kWarps - 1) / kWarps;
  return (int)std::min<int64_t>(b, kMostBlocks);
}

}  // namespace

size_t rotary_grad_workspace(int64_t tokens, int64_t heads, int32_t dim) {
  return tokens <= 0 || heads <= 0 ? 0 : (size_t)grad_blocks(tokens, heads) * 2 * dim * sizeof(float);
}

cudaError_t launch_rotary(lm_dtype dt, const RotaryParams& p, cudaStream_t st) {
  const int64_t rows = p.tokens * (p.part[0].heads + p.part[1].heads);
  const dim3 grid((unsigned)std::min<int64_t>((rows + kWarps - 1) / kWarps, 152 * 16));
  return launch_after(dt == LM_F32 ? rotary_kernel<float> : rotary_kernel<__nv_bfloat16>, grid, kThreads, 0, st, p);
}

cudaError_t launch_rotary_grad(lm_dtype dt, const RotaryParams& p, cudaStream_t st) {
  const int blocks = grad_blocks(p.tokens, std::max(p.part[0].heads, p.part[1].heads));
  const bool dw = p.part[0].dweight != nullptr || p.part[1].dweight != nullptr;
  if (blocks > 0) {
    const cudaError_t e = launch_after(dt == LM_F32 ? rotary_grad_kernel<float> : rotary_grad_kernel<__nv_bfloat16>, dim3((unsigned)blocks, p.part[1].heads > 0 ? 2 : 1),
                                       kThreads, dw ? (size_t)kWarps * p.dim * sizeof(float) : 0, st, p);
    if (e != cudaSuccess) return e;
  }
  if (!dw) return cudaSuccess;
  return launch_after(rotary_join_kernel, dim3((unsigned)((p.dim + kWarps - 1) / kWarps), 2), kThreads, 0, st, p, blocks);
}

}  // namespace lm
