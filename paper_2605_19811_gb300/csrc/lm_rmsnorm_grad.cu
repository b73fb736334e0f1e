// Gradient of the RMS norm, from the stored h or its 8-bit checkpoint (formulas
// at lm_rmsnorm_grad in lionmuon.h).
//
// Bound by memory: 8 bytes an element (dy, h, dh, dx in bf16).  Rows are taken
// as in the forward kernel: once, in registers, the next row's loads ahead.
// dweight is summed over each share's rows in registers, then over the shares,
// in order, by a second kernel.
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace rows;

// kFormat < 0: h is a matrix.  kPast: dh is added.
template <typename T, int kFormat, bool kPast, typename S, bool kVec>
__global__ void __launch_bounds__(S::kBlock, S::kBlock <= 256 ? 512 / S::kBlock : 1) rmsnorm_grad_kernel(const NormGradParams p) {
  constexpr int kThreads = S::kThreads, kRows = S::kRows, kVecs = S::kVecs, kSpan = S::kSpan;
  __shared__ float part[2][kRows][S::kWarps];
  const int t = (int)threadIdx.x % kThreads, slot = (int)threadIdx.x / kThreads;
  const bool whole = p.cols <= kVecs * kSpan;
  const bool want = p.dweight != nullptr;
  float* sums = want ? p.parts + ((int64_t)blockIdx.x * kRows + slot) * p.cols : nullptr;   // of this share's rows
  float acc[kVecs][8], gain[kVecs][8];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[v][e] = 0.f;
    weight8(p.weight, p.wdt, 8 * t + v * kSpan, whole ? p.cols - 8 * t - v * kSpan : 0, gain[v]);
  }
  if (want && !whole)
    for (int c = 8 * t; c < p.cols; c += kSpan)
      for (int e = 0; e < 8 && c + e < p.cols; ++e) sums[c + e] = 0.f;
  struct Eight {
    Raw<T> dy, dh;
    std::conditional_t<(kFormat < 0), Raw<T>, RawCodes<(kFormat < 0 ? 0 : kFormat)>> h;
    __device__ __forceinline__ void load(const NormGradParams& p, int64_t row, int c) {
      const int left = row < p.rows ? p.cols - c : 0;
      if (left <= 0) {
        dy.zero();
        h.zero();
        if (kPast) dh.zero();
        return;
      }
      dy.template load<kVec>(row_of<const T>(p.dy, row) + c, left);
      if constexpr (kFormat < 0) h.template load<kVec>(row_of<const T>(p.h, row) + c, left);
      else h.load(p.h8, row, c);
      if (kPast) dh.template load<kVec>(row_of<const T>(p.dh, row) + c, left);
    }
    // dy and xh = h rstd; codes beyond the row are no numbers
    __device__ __forceinline__ void get(float rstd, int left, float (&g)[8], float (&x)[8]) const {
      dy.get(g);
      h.get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (kFormat < 0 || e < left) ? x[e] * rstd : 0.f;
    }
  };
  auto dot = [](const Eight& e8, float rstd, int left, const float (&w)[8]) {
    float g[8], x[8], q = 0.f;
    e8.get(rstd, left, g, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) q += w[e] * g[e] * x[e];
    return q;
  };
  Eight now[kVecs];
  float rstd = 0.f;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row0 = (int64_t)blockIdx.x * kRows;
  if (row0 + slot < p.rows) rstd = p.rstd[row0 + slot];
  if (whole) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) now[v].load(p, row0 + slot, 8 * t + v * kSpan);
  }
  for (int turn = 0; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool live = row < p.rows;
    Eight next[kVecs];
    const float rstd_next = row + step < p.rows ? p.rstd[row + step] : 0.f;
    float s = 0.f;
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) next[v].load(p, row0 + step + slot, 8 * t + v * kSpan);
#pragma unroll
      for (int v = 0; v < kVecs; ++v) s += dot(now[v], rstd, live ? p.cols - 8 * t - v * kSpan : 0, gain[v]);
    } else {
      for (int c = 8 * t; c < p.cols; c += kSpan) {
        now[0].load(p, row, c);
        weight8(p.weight, p.wdt, c, p.cols - c, gain[0]);
        s += dot(now[0], rstd, live ? p.cols - c : 0, gain[0]);
      }
    }
    s = row_sum<kThreads, kRows>(s, part, slot, turn);
    const float mean = s / (float)p.cols;
    auto put = [&](int c, const Eight& e8, const float (&w)[8], float (&a)[8]) {
      const int left = live ? p.cols - c : 0;
      if (left <= 0) return;
      float g[8], x[8], dx[8];
      e8.get(rstd, left, g, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] += g[e] * x[e];
      if (p.dx.data == nullptr) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) dx[e] = rstd * (w[e] * g[e] - x[e] * mean);
      if (kPast) {
        float d[8];
        e8.dh.get(d);
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[e] += d[e];
      }
      store8<kVec>(row_of<T>(p.dx, row) + c, left, dx);
    };
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        put(8 * t + v * kSpan, now[v], gain[v], acc[v]);
        now[v] = next[v];
      }
    } else {
      for (int c = 8 * t; c < p.cols; c += kSpan) {
        float a[8] = {};
        now[0].load(p, row, c);
        weight8(p.weight, p.wdt, c, p.cols - c, gain[0]);
        put(c, now[0], gain[0], a);
        if (want && live)
          for (int e = 0; e < 8 && c + e < p.cols; ++e) sums[c + e] += a[e];
      }
    }
    rstd = rstd_next;
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

template <typename T, int kFormat, bool kPast>
int backward(const NormGradParams& p, bool vec, cudaStream_t st) {
  int parts = 0;
  by_shape<T>(p.cols, [&](auto shape) {
    using S = decltype(shape);
    const int64_t blocks = (p.rows + S::kRows - 1) / S::kRows;
    constexpr int kFit = 152 * (S::kBlock <= 512 ? 512 / S::kBlock : 1), kMost = kFit * S::kRows < kNormGradParts ? kFit : kNormGradParts / S::kRows;
    const unsigned grid = (unsigned)(blocks < kMost ? blocks : kMost);
    parts = (int)grid * S::kRows;
    if (vec) rmsnorm_grad_kernel<T, kFormat, kPast, S, true><<<grid, S::kBlock, 0, st>>>(p);
    else rmsnorm_grad_kernel<T, kFormat, kPast, S, false><<<grid, S::kBlock, 0, st>>>(p);
  });
  return parts;
}
template <typename T, int kFormat>
int backward(const NormGradParams& p, bool vec, cudaStream_t st) {
  return p.dh.data != nullptr ? backward<T, kFormat, true>(p, vec, st) : backward<T, kFormat, false>(p, vec, st);
}
template <typename T>
int backward(const NormGradParams& p, bool vec, cudaStream_t st) {
  if (p.h8.data != nullptr) return p.h8.format == LM_CODE_I8 ? backward<T, LM_CODE_I8>(p, vec, st) : backward<T, LM_CODE_E4M3>(p, vec, st);
  return backward<T, -1>(p, vec, st);
}

}  // namespace

cudaError_t launch_rmsnorm_grad(lm_dtype dt, const NormGradParams& p, cudaStream_t st) {
  int parts = 0;
  if (p.rows > 0) {
    const int size = dt == LM_F32 ? 4 : 2;
    const bool vec = aligned(p.dy, size, p.rows) && aligned(p.h, size, p.rows) &&
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
