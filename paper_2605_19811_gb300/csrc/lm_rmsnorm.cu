// RMS norm with the residual's addition and an 8-bit copy of its output
// (formulas at lm_rmsnorm in lionmuon.h).
//
// Bound by memory: 8 bytes an element (x, r, h, y in bf16) and 1 for the 8-bit
// copy.  A row is read once and stays in registers as it was read: kThreads threads take it,
// kVecs groups of 8 consecutive channels each, channel 8 (t + v kThreads)
// first, so a scale's 128 channels are 16 neighbouring lanes.  A block goes
// from row to row (several at a time where rows are short) with the next
// row's loads ahead of this row's sums.  Rows beyond what registers hold
// (kThreads kVecs 8 channels) are read twice, from L2 the second time.
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace rows;

// kVec: rows are 16-byte aligned.  kFormat < 0: no 8-bit copy.
// kResidual: x + residual is normed.
template <typename T, int kFormat, bool kResidual, typename S, bool kVec>
__global__ void __launch_bounds__(S::kBlock, S::kBlock <= 256 ? 768 / S::kBlock : 1) rmsnorm_kernel(const NormParams p) {
  constexpr int kThreads = S::kThreads, kRows = S::kRows, kVecs = S::kVecs, kSpan = S::kSpan;
  __shared__ float part[2][kRows][S::kWarps];
  const int t = (int)threadIdx.x % kThreads, slot = (int)threadIdx.x / kThreads;
  const bool whole = p.cols <= kVecs * kSpan;     // the row fits the registers
  float gain[kVecs][8];                           // of the thread's channels, for every row
#pragma unroll
  for (int v = 0; v < kVecs; ++v) weight8(p.weight, p.wdt, 8 * t + v * kSpan, whole ? p.cols - 8 * t - v * kSpan : 0, gain[v]);
  struct Eight {
    Raw<T> x, r;
    __device__ __forceinline__ void load(const NormParams& p, int64_t row, int c) {
      const int left = row < p.rows ? p.cols - c : 0;
      if (left <= 0) {
        x.zero();
        if (kResidual) r.zero();
        return;
      }
      x.template load<kVec>(row_of<const T>(p.x, row) + c, left);
      if (kResidual) r.template load<kVec>(row_of<const T>(p.residual, row) + c, left);
    }
    __device__ __forceinline__ void get(float (&h)[8]) const {
      x.get(h);
      if (kResidual) {
        float a[8];
        r.get(a);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += a[e];
      }
    }
  };
  auto squares = [](const Eight& e8) {
    float h[8], q = 0.f;
    e8.get(h);
#pragma unroll
    for (int e = 0; e < 8; ++e) q += h[e] * h[e];
    return q;
  };
  Eight now[kVecs];
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row0 = (int64_t)blockIdx.x * kRows;
  if (whole) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) now[v].load(p, row0 + slot, 8 * t + v * kSpan);
  }
  for (int turn = 0; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool live = row < p.rows;
    Eight next[kVecs];
    float s = 0.f;
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) next[v].load(p, row0 + step + slot, 8 * t + v * kSpan);
#pragma unroll
      for (int v = 0; v < kVecs; ++v) s += squares(now[v]);
    } else {
      for (int c = 8 * t; c < p.cols; c += kSpan) {
        now[0].load(p, row, c);
        s += squares(now[0]);
      }
    }
    s = row_sum<kThreads, kRows>(s, part, slot, turn);
    const float rstd = 1.f / sqrtf(s / (float)p.cols + p.eps);
    if (live && t == 0 && p.rstd != nullptr) p.rstd[row] = rstd;
    auto put = [&](int c, const Eight& e8, const float (&w)[8]) {
      const int left = live ? p.cols - c : 0;
      float h[8], y[8];
      e8.get(h);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[e] * rstd * w[e];
      if (left > 0) {
        if (p.h.data != nullptr) store8<kVec>(row_of<T>(p.h, row) + c, left, h);
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
      for (int v = 0; v < kVecs; ++v) {
        if (v * kSpan < p.cols) put(8 * t + v * kSpan, now[v], gain[v]);
        now[v] = next[v];
      }
    } else {
      for (int c = 8 * t; c < (p.cols + kSpan - 1) / kSpan * kSpan; c += kSpan) {
        now[0].load(p, row, c);   // an h written over x or residual: this thread reads its eight before it writes them
        weight8(p.weight, p.wdt, c, p.cols - c, gain[0]);
        put(c, now[0], gain[0]);
      }
    }
  }
}

template <typename T, int kFormat, bool kResidual>
void forward(const NormParams& p, bool vec, cudaStream_t st) {
  by_shape<T>(p.cols, [&](auto shape) {
    using S = decltype(shape);
    const int64_t blocks = (p.rows + S::kRows - 1) / S::kRows;
    constexpr int kMost = 152 * (S::kBlock <= 256 ? 768 / S::kBlock : 1);   // what the SMs hold at once
    const unsigned grid = (unsigned)(blocks < kMost ? blocks : kMost);
    if (vec) rmsnorm_kernel<T, kFormat, kResidual, S, true><<<grid, S::kBlock, 0, st>>>(p);
    else rmsnorm_kernel<T, kFormat, kResidual, S, false><<<grid, S::kBlock, 0, st>>>(p);
  });
}
template <typename T, int kFormat>
void forward(const NormParams& p, bool vec, cudaStream_t st) {
  if (p.residual.data != nullptr) forward<T, kFormat, true>(p, vec, st);
  else forward<T, kFormat, false>(p, vec, st);
}
}  // namespace

cudaError_t launch_rmsnorm(lm_dtype dt, const NormParams& p, cudaStream_t st) {
  const int size = dt == LM_F32 ? 4 : 2;
  const bool vec = aligned(p.x, size, p.rows) && aligned(p.residual, size, p.rows) && aligned(p.h, size, p.rows) && aligned(p.y, size, p.rows);
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

}  // namespace lm
