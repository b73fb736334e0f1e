// What the RMS norm's kernels (lm_rmsnorm.cu, lm_rmsnorm_grad.cu) share: eight
// channels of a row as they are read, sums over a row, shapes by channels.
#pragma once

#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "lm_code8.cuh"
#include "lm_train.h"

namespace lm {
namespace rows {
namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;

// Eight channels as they are read, `left` of them inside the row (zeros
// beyond).  kVec: eights lie on 16-byte boundaries; else one by one.
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void zero() { u = make_uint4(0u, 0u, 0u, 0u); }
  template <bool kVec>
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int left) {
    if (kVec && left >= 8) {
      u = __ldcs(reinterpret_cast<const uint4*>(p));
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
      uint32_t e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = k < left ? q[k] : 0u;
      u = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  }
};
template <> struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  template <bool kVec>
  __device__ __forceinline__ void load(const float* p, int left) {
    if (kVec && left >= 8) {
      a = __ldcs(reinterpret_cast<const float4*>(p));
      b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    } else {
      float e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = k < left ? p[k] : 0.f;
      a = make_float4(e[0], e[1], e[2], e[3]);
      b = make_float4(e[4], e[5], e[6], e[7]);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
// Eight channels of an 8-bit checkpoint: their codes and scale.
template <int kFormat>
struct RawCodes {
  uint2 q;
  float scale;
  __device__ __forceinline__ void zero() {
    q = make_uint2(0u, 0u);
    scale = 0.f;
  }
  __device__ __forceinline__ void load(const Codes& k, int64_t row, int c) {
    q = __ldcs(reinterpret_cast<const uint2*>(k.data + row * k.ld + c));
    scale = k.scales[(int64_t)(c / LM_CODE_GROUP) * k.ld_scales + row];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t two[4] = {q.x, q.x >> 16, q.y, q.y >> 16};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 d = code8::decode2<kFormat>(two[k]);
      v[2 * k] = d.x * scale;
      v[2 * k + 1] = d.y * scale;
    }
  }
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool kVec>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int left, const float (&v)[8]) {
  if (kVec && left >= 8) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = __float2bfloat16_rn(v[k]);
  }
}
template <bool kVec>
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
  if (kVec && left >= 8) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = v[k];
  }
}
// Eight channels of the gain (ones where there is none).
__device__ __forceinline__ void weight8(const void* w, int dt, int c, int left, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = 1.f;
    if (w != nullptr && k < left) v[k] = dt == LM_F32 ? static_cast<const float*>(w)[c + k] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c + k]);
  }
}

// Sum over the kThreads threads of a row; rows of a block are told apart by
// `slot`, `turn` alternates so that one barrier a sum is enough.
template <int kThreads, int kRows>
__device__ __forceinline__ float row_sum(float s, float (*part)[kRows][kThreads < 32 ? 1 : kThreads / 32], int slot, int turn) {
#pragma unroll
  for (int o = (kThreads < 32 ? kThreads : 32) / 2; o; o >>= 1) s += __shfl_xor_sync(kAll, s, o);
  if constexpr (kThreads > 32) {
    constexpr int kWarps = kThreads / 32;
    const int t = (int)threadIdx.x % kThreads;
    if ((t & 31) == 0) part[turn][slot][t >> 5] = s;
    __syncthreads();
    s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += part[turn][slot][w];
  }
  return s;
}

// The 8-bit copy of eight channels: the scale of the 16 lanes' 128 channels,
// the codes, eight bytes a lane (the row pitch is a multiple of 16, so eight
// are inside the row wherever one is).
template <int kFormat>
__device__ __forceinline__ void keep8(const Codes& k, int64_t row, int c, int cols, const float (&y)[8]) {
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = max(most, code8::magnitude(y[e]));
#pragma unroll
  for (int o = 8; o; o >>= 1) most = max(most, __shfl_xor_sync(kAll, most, o));
  if (c >= cols) return;
  const float scale = code8::group_scale<kFormat>(most), inv = code8::inverse_scale(scale);
  if ((c & (LM_CODE_GROUP - 1)) == 0) k.scales[(int64_t)(c / LM_CODE_GROUP) * k.ld_scales + row] = scale;
  const uint32_t lo = code8::encode2<kFormat>(y[0], y[1], inv) | (code8::encode2<kFormat>(y[2], y[3], inv) << 16);
  const uint32_t hi = code8::encode2<kFormat>(y[4], y[5], inv) | (code8::encode2<kFormat>(y[6], y[7], inv) << 16);
  __stcs(reinterpret_cast<uint2*>(k.data + row * k.ld + c), make_uint2(lo, hi));
}

template <typename T>
__device__ __forceinline__ T* row_of(const Mat& m, int64_t row) {
  return static_cast<T*>(m.data) + row * m.ld;
}

// Of a block's shape: threads a row, rows at a time, eights a thread.
template <int kThreads_, int kRows_, int kVecs_>
struct Shape {
  static constexpr int kThreads = kThreads_, kRows = kRows_, kVecs = kVecs_;
  static constexpr int kBlock = kThreads * kRows, kSpan = 8 * kThreads;
  static constexpr int kWarps = kThreads < 32 ? 1 : kThreads / 32;
};

bool aligned(const Mat& m, int size, int64_t rows) {
  return m.data == nullptr || (reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (rows == 1 || m.ld * size % 16 == 0));
}

// Shape by channels: registers hold a row of up to 8192 (fp32) or 16384 (bf16)
// channels; what is longer is read twice.  An eight of fp32 takes the registers
// of two of bf16.
template <typename T, typename F>
void by_shape(int cols, F f) {
  constexpr int v = sizeof(T) == 4 ? 1 : 2, m = 3 - v;   // fp32: twice the threads
  if (cols <= 256) f(Shape<32, 8, 1>());
  else if (cols <= 512) f(Shape<32 * m, 8 / m, v>());
  else if (cols <= 1024) f(Shape<64 * m, 4 / m, v>());
  else if (cols <= 2048) f(Shape<128 * m, 2 / m, v>());
  else if (cols <= 4096) f(Shape<256 * m, 1, v>());
  else f(Shape<512 * m, 1, v>());
}

}  // namespace
}  // namespace rows
}  // namespace lm
