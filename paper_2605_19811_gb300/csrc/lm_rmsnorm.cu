// RMS norm with the residual's addition and an 8-bit copy of its output, and
// its gradient (formulas at lm_rmsnorm and lm_rmsnorm_grad in lionmuon.h).
//
// Both are bound by memory: 8 bytes an element and 1 for the 8-bit copy
// forward (x, r, h, y in bf16), 8 in the gradient (dy, h, dh, dx).  A row is
// read once and stays in registers: kThreads threads take it, kVecs groups of
// 8 consecutive channels each, channel 8 (t + v kThreads) first, so a scale's
// 128 channels are 16 neighbouring lanes.  Rows beyond what registers hold
// (kThreads x kVecs x 8 channels) are read twice, from L2 the second time.
// Blocks of small rows take several rows at a time (kRows), and every block
// goes on to further rows with the next row's loads ahead of this one's sums.
//
// dweight is summed over each block's rows in registers, then over the
// blocks, in order, by a second kernel.
#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "lm_code8.cuh"
#include "lm_train.h"

namespace lm {
namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int kForwardBlocks = 152 * 16;   // most blocks that share the rows

// ---- eight channels ----
__device__ __forceinline__ void unpack_bf16(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(w[k] << 16);
    v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// kVec: the eight lie on a 16-byte boundary and inside the row; else one by
// one, `left` of them inside (zeros beyond).
template <bool kVec>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int left, float (&v)[8]) {
  if (kVec) {
    unpack_bf16(__ldcs(reinterpret_cast<const uint4*>(p)), v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < left ? __bfloat162float(p[k]) : 0.f;
  }
}
template <bool kVec>
__device__ __forceinline__ void load8(const float* p, int left, float (&v)[8]) {
  if (kVec) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < left ? p[k] : 0.f;
  }
}
template <bool kVec>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int left, const float (&v)[8]) {
  if (kVec) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = __float2bfloat16_rn(v[k]);
  }
}
template <bool kVec>
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
  if (kVec) {
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

// kThreads threads a row, kRows rows a block, kVecs eights a thread in
// registers; kVec: rows are 16-byte aligned and whole eights.  kFormat < 0: no
// 8-bit copy.
template <typename T, int kFormat, int kThreads, int kRows, int kVecs, bool kVec>
__global__ void __launch_bounds__(kThreads * kRows) rmsnorm_kernel(const NormParams p) {
  __shared__ float part[2][kRows][kThreads < 32 ? 1 : kThreads / 32];
  constexpr int kSpan = 8 * kThreads;
  const int t = (int)threadIdx.x % kThreads, slot = (int)threadIdx.x / kThreads;
  const bool whole = p.cols <= kVecs * kSpan;     // the row fits the registers
  float gain[kVecs][8];                           // of the thread's channels, for every row
#pragma unroll
  for (int v = 0; v < kVecs; ++v) weight8(p.weight, p.wdt, 8 * t + v * kSpan, whole ? p.cols - 8 * t - v * kSpan : 0, gain[v]);
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < p.rows; row0 += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool live = row < p.rows;
    auto h_of = [&](int c, float (&h)[8]) {
      const int left = live ? p.cols - c : 0;
      if (left <= 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = 0.f;
        return;
      }
      load8<kVec>(row_of<const T>(p.x, row) + c, left, h);
      if (p.residual.data != nullptr) {
        float r[8];
        load8<kVec>(row_of<const T>(p.residual, row) + c, left, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += r[e];
      }
    };
    float h[kVecs][8], s = 0.f;
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        h_of(8 * t + v * kSpan, h[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += h[v][e] * h[v][e];
      }
    } else {
      for (int c = 8 * t; c < p.cols; c += kSpan) {
        h_of(c, h[0]);
        float q = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) q += h[0][e] * h[0][e];
        s += q;
      }
    }
    s = row_sum<kThreads, kRows>(s, part, slot, turn);
    const float rstd = 1.f / sqrtf(s / (float)p.cols + p.eps);
    if (live && t == 0 && p.rstd != nullptr) p.rstd[row] = rstd;
    auto put = [&](int c, const float (&hh)[8], const float (&w)[8]) {
      const int left = live ? p.cols - c : 0;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = hh[e] * rstd * w[e];
      if (left > 0) {
        if (p.h.data != nullptr) store8<kVec>(row_of<T>(p.h, row) + c, left, hh);
        if (p.y.data != nullptr) store8<kVec>(row_of<T>(p.y, row) + c, left, y);
      }
      if constexpr (kFormat >= 0) {
        if (left < 8) {   // nothing beyond the row counts for the scale
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e >= left) y[e] = 0.f;
        }
        keep8<kFormat>(p.kept, row, left > 0 ? c : p.cols, p.cols, y);
      }
    };
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
        if (v * kSpan < p.cols) put(8 * t + v * kSpan, h[v], gain[v]);
    } else {
      for (int c = 8 * t; c < (p.cols + kSpan - 1) / kSpan * kSpan; c += kSpan) {
        h_of(c, h[0]);   // an h written over x or residual: this thread reads its eight before it writes them
        weight8(p.weight, p.wdt, c, p.cols - c, gain[0]);
        put(c, h[0], gain[0]);
      }
    }
  }
}

// kFormat < 0: h is a matrix of kH.
template <typename T, typename kH, int kFormat, int kThreads, int kRows, int kVecs, bool kVec>
__global__ void __launch_bounds__(kThreads * kRows) rmsnorm_grad_kernel(const NormGradParams p) {
  __shared__ float part[2][kRows][kThreads < 32 ? 1 : kThreads / 32];
  constexpr int kSpan = 8 * kThreads;
  const int t = (int)threadIdx.x % kThreads, slot = (int)threadIdx.x / kThreads;
  const bool whole = p.cols <= kVecs * kSpan;
  const bool want = p.dweight != nullptr;
  float* sums = want ? p.parts + ((int64_t)blockIdx.x * kRows + slot) * p.cols : nullptr;   // of this slot's rows
  float acc[kVecs][8];
#pragma unroll
  for (int v = 0; v < kVecs; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[v][e] = 0.f;
  float gain[kVecs][8];                           // of the thread's channels, for every row
#pragma unroll
  for (int v = 0; v < kVecs; ++v) weight8(p.weight, p.wdt, 8 * t + v * kSpan, whole ? p.cols - 8 * t - v * kSpan : 0, gain[v]);
  if (want && !whole)
    for (int c = 8 * t; c < p.cols; c += kSpan)
      for (int e = 0; e < 8 && c + e < p.cols; ++e) sums[c + e] = 0.f;
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < p.rows; row0 += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool live = row < p.rows;
    const float rstd = live ? p.rstd[row] : 0.f;
    // dy and xh = h rstd of eight channels
    auto load = [&](int c, float (&dy)[8], float (&xh)[8]) {
      const int left = live ? p.cols - c : 0;
      if (left <= 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dy[e] = xh[e] = 0.f;
        return;
      }
      load8<kVec>(row_of<const T>(p.dy, row) + c, left, dy);
      if constexpr (kFormat < 0) {
        load8<kVec>(row_of<const kH>(p.h, row) + c, left, xh);
#pragma unroll
        for (int e = 0; e < 8; ++e) xh[e] *= rstd;
      } else {
        const uint2 q = __ldcs(reinterpret_cast<const uint2*>(p.h8.data + row * p.h8.ld + c));
        const float scale = p.h8.scales[(int64_t)(c / LM_CODE_GROUP) * p.h8.ld_scales + row];
        const uint32_t two[4] = {q.x, q.x >> 16, q.y, q.y >> 16};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 d = code8::decode2<kFormat>(two[k]);
          xh[2 * k] = 2 * k < left ? d.x * scale * rstd : 0.f;
          xh[2 * k + 1] = 2 * k + 1 < left ? d.y * scale * rstd : 0.f;
        }
      }
    };
    float dy[kVecs][8], xh[kVecs][8], s = 0.f;
    auto dot = [&](const float (&w)[8], const float (&g)[8], const float (&x)[8]) {
      float q = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) q += w[e] * g[e] * x[e];
      return q;
    };
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) load(8 * t + v * kSpan, dy[v], xh[v]);
#pragma unroll
      for (int v = 0; v < kVecs; ++v)
        if (8 * t + v * kSpan < p.cols) s += dot(gain[v], dy[v], xh[v]);
    } else {
      for (int c = 8 * t; c < p.cols; c += kSpan) {
        load(c, dy[0], xh[0]);
        weight8(p.weight, p.wdt, c, p.cols - c, gain[0]);
        s += dot(gain[0], dy[0], xh[0]);
      }
    }
    s = row_sum<kThreads, kRows>(s, part, slot, turn);
    const float mean = s / (float)p.cols;
    auto put = [&](int c, const float (&w)[8], const float (&g)[8], const float (&x)[8], float (&a)[8]) {
      const int left = live ? p.cols - c : 0;
      if (left <= 0) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] += g[e] * x[e];
      if (p.dx.data == nullptr) return;
      float dx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) dx[e] = rstd * (w[e] * g[e] - x[e] * mean);
      if (p.dh.data != nullptr) {
        float d[8];
        load8<kVec>(row_of<const T>(p.dh, row) + c, left, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[e] += d[e];
      }
      store8<kVec>(row_of<T>(p.dx, row) + c, left, dx);
    };
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) put(8 * t + v * kSpan, gain[v], dy[v], xh[v], acc[v]);
    } else {
      for (int c = 8 * t; c < p.cols; c += kSpan) {
        float a[8] = {};
        load(c, dy[0], xh[0]);
        weight8(p.weight, p.wdt, c, p.cols - c, gain[0]);
        put(c, gain[0], dy[0], xh[0], a);
        if (want && live)
          for (int e = 0; e < 8 && c + e < p.cols; ++e) sums[c + e] += a[e];
      }
    }
  }
  if (want && whole) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int c = 8 * t + v * kSpan;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < p.cols) sums[c + e] = acc[v][e];
    }
  }
}

// dweight from the parts: 32 columns a block, 32 runs of parts each, both in order.
__global__ void __launch_bounds__(1024) norm_dweight_kernel(const float* parts, int nparts, int cols, void* dweight, int dwdt) {
  __shared__ float run[32][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), k = threadIdx.x >> 5;
  const int each = (nparts + 31) / 32, p0 = min(nparts, k * each), p1 = min(nparts, p0 + each);
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int i = p0; i < p1; ++i) s += parts[(int64_t)i * cols + c];
  }
  run[k][threadIdx.x & 31] = s;
  __syncthreads();
  if (k != 0 || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += run[i][threadIdx.x];
  if (dwdt == LM_F32) static_cast<float*>(dweight)[c] = s;
  else static_cast<__nv_bfloat16*>(dweight)[c] = __float2bfloat16_rn(s);
}

bool aligned(const Mat& m, int size, int64_t rows) {
  return m.data == nullptr || (reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (rows == 1 || m.ld * size % 16 == 0));
}

// Threads a row by its channels: two eights a thread keep a row in registers up
// to 16384 channels, and what is longer is read twice.
template <typename F>
void by_shape(int cols, F f) {
  using std::integral_constant;
  if (cols <= 256) f(integral_constant<int, 32>(), integral_constant<int, 8>(), integral_constant<int, 1>());
  else if (cols <= 512) f(integral_constant<int, 32>(), integral_constant<int, 8>(), integral_constant<int, 2>());
  else if (cols <= 1024) f(integral_constant<int, 64>(), integral_constant<int, 4>(), integral_constant<int, 2>());
  else if (cols <= 2048) f(integral_constant<int, 128>(), integral_constant<int, 2>(), integral_constant<int, 2>());
  else if (cols <= 4096) f(integral_constant<int, 256>(), integral_constant<int, 1>(), integral_constant<int, 2>());
  else if (cols <= 8192) f(integral_constant<int, 512>(), integral_constant<int, 1>(), integral_constant<int, 2>());
  else f(integral_constant<int, 1024>(), integral_constant<int, 1>(), integral_constant<int, 2>());
}

template <typename T, int kFormat>
void forward(const NormParams& p, bool vec, cudaStream_t st) {
  by_shape(p.cols, [&](auto threads, auto rows, auto vecs) {
    constexpr int kT = decltype(threads)::value, kR = decltype(rows)::value, kV = decltype(vecs)::value;
    const int64_t blocks = (p.rows + kR - 1) / kR;
    const unsigned grid = (unsigned)(blocks < kForwardBlocks ? blocks : kForwardBlocks);
    if (vec) rmsnorm_kernel<T, kFormat, kT, kR, kV, true><<<grid, kT * kR, 0, st>>>(p);
    else rmsnorm_kernel<T, kFormat, kT, kR, kV, false><<<grid, kT * kR, 0, st>>>(p);
  });
}
template <typename T, typename kH, int kFormat>
int backward(const NormGradParams& p, bool vec, cudaStream_t st) {
  int parts = 0;
  by_shape(p.cols, [&](auto threads, auto rows, auto vecs) {
    constexpr int kT = decltype(threads)::value, kR = decltype(rows)::value, kV = decltype(vecs)::value;
    const int64_t blocks = (p.rows + kR - 1) / kR;
    constexpr int kMost = kNormGradParts / kR;
    const unsigned grid = (unsigned)(blocks < kMost ? blocks : kMost);
    parts = (int)grid * kR;
    if (vec) rmsnorm_grad_kernel<T, kH, kFormat, kT, kR, kV, true><<<grid, kT * kR, 0, st>>>(p);
    else rmsnorm_grad_kernel<T, kH, kFormat, kT, kR, kV, false><<<grid, kT * kR, 0, st>>>(p);
  });
  return parts;
}
template <typename T>
int backward(const NormGradParams& p, bool vec, cudaStream_t st) {
  if (p.h8.data != nullptr) return p.h8.format == LM_CODE_I8 ? backward<T, T, LM_CODE_I8>(p, vec, st) : backward<T, T, LM_CODE_E4M3>(p, vec, st);
  return p.hdt == LM_F32 ? backward<T, float, -1>(p, vec, st) : backward<T, __nv_bfloat16, -1>(p, vec, st);
}

}  // namespace

cudaError_t launch_rmsnorm(lm_dtype dt, const NormParams& p, cudaStream_t st) {
  const int size = dt == LM_F32 ? 4 : 2;
  const bool vec = p.cols % 8 == 0 && aligned(p.x, size, p.rows) && aligned(p.residual, size, p.rows) && aligned(p.h, size, p.rows) && aligned(p.y, size, p.rows);
  count_launch();
  const int format = p.kept.data == nullptr ? -1 : p.kept.format;
  if (dt == LM_BF16) {
    if (format < 0) forward<__nv_bfloat16, -1>(p, vec, st);
    else if (format == LM_CODE_I8) forward<__nv_bfloat16, LM_CODE_I8>(p, vec, st);
    else forward<__nv_bfloat16, LM_CODE_E4M3>(p, vec, st);
  } else {
    if (format < 0) forward<float, -1>(p, vec, st);
    else if (format == LM_CODE_I8) forward<float, LM_CODE_I8>(p, vec, st);
    else forward<float, LM_CODE_E4M3>(p, vec, st);
  }
  return cudaGetLastError();
}

cudaError_t launch_rmsnorm_grad(lm_dtype dt, const NormGradParams& p, cudaStream_t st) {
  int parts = 0;
  if (p.rows > 0) {
    const int size = dt == LM_F32 ? 4 : 2;
    const bool vec = p.cols % 8 == 0 && aligned(p.dy, size, p.rows) && aligned(p.h, p.hdt == LM_F32 ? 4 : 2, p.rows) &&
                     aligned(p.dh, size, p.rows) && aligned(p.dx, size, p.rows);
    count_launch();
    parts = dt == LM_BF16 ? backward<__nv_bfloat16>(p, vec, st) : backward<float>(p, vec, st);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (p.dweight != nullptr) {
    count_launch();
    norm_dweight_kernel<<<(p.cols + 31) / 32, 1024, 0, st>>>(p.parts, parts, p.cols, p.dweight, p.dwdt);
  }
  return cudaGetLastError();
}

}  // namespace lm
