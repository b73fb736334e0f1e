// RMS norm with the residual's addition and an 8-bit copy of its output
// (formulas at lm_rmsnorm in lionmuon.h).
//
// Bound by memory: 8 bytes an element (x, r, h, y in bf16) and 1 for the 8-bit
// copy.  A row is read once and stays in registers as it was read.  A warp
// takes a row of up to 1536 channels (bf16), several warps a longer one, with
// as many eights a lane as registers allow: what a row needs once (its sum, its
// root, its addresses) is then shared by many channels.  16384 x 1280 with
// residual and 8-bit copy: 44 us with a warp and five eights a lane, 50 us with
// 128 threads and two eights each.  A lane has 8 consecutive channels of every
// 256, so a scale's 128 channels are half a warp.  rstd is rsqrtf's, within two
// units of the last place.
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace rows;

// kVec: rows are 16-byte aligned.  kFormat < 0: no 8-bit copy.
template <typename T, int kFormat, int kVecs, bool kVec>
__global__ void __launch_bounds__(512) rmsnorm_kernel(const NormParams p, int threads) {
  __shared__ float part[2][32];
  const Team team(threads);
  const int t = team.t, slot = team.slot, nrows = team.rows, span = team.span;
  const bool whole = p.cols <= kVecs * span;     // the row fits the registers
  const bool wvec = (reinterpret_cast<uintptr_t>(p.weight) & 15u) == 0;
  const bool residual = p.residual.data != nullptr;
  const float inv_cols = 1.f / (float)p.cols;
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * nrows; row0 < p.rows; row0 += (int64_t)gridDim.x * nrows, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool live = row < p.rows;
    const int64_t at = live ? row : 0;
    const Row<const T> x(p.x, at, p.rows), r(p.residual, at, p.rows);
    auto left_of = [&](int c) { return live ? p.cols - c : kNoRow; };
    auto h_of = [&](const Raw<T>& a, const Raw<T>& b, float (&h)[8]) {
      a.get(h);
      if (residual) {
        float q[8];
        b.get(q);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += q[e];
      }
    };
    auto squares = [&](const Raw<T>& a, const Raw<T>& b) {
      float h[8], q = 0.f;
      h_of(a, b, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) q += h[e] * h[e];
      return q;
    };
    Raw<T> xr[kVecs], rr[kVecs];
    auto fetch = [&](int c) {
      xr[0].template load<kVec>(x, c, left_of(c));
      xr[0].template settle<kVec>(x, c, left_of(c));
      if (!residual) return;
      rr[0].template load<kVec>(r, c, left_of(c));
      rr[0].template settle<kVec>(r, c, left_of(c));
    };
    float s = 0.f;
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        const int c = 8 * t + v * span;
        xr[v].template load<kVec>(x, c, left_of(c));
        rr[v].zero();
        if (residual) rr[v].template load<kVec>(r, c, left_of(c));
      }
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        const int c = 8 * t + v * span;
        xr[v].template settle<kVec>(x, c, left_of(c));
        if (residual) rr[v].template settle<kVec>(r, c, left_of(c));
        s += squares(xr[v], rr[v]);
      }
    } else {
      rr[0].zero();
      for (int c = 8 * t; c - 8 * t < p.cols; c += span) {
        fetch(c);
        s += squares(xr[0], rr[0]);
      }
    }
    s = team.sum(s, part, turn);
    const float rstd = rsqrtf(fmaf(s, inv_cols, p.eps));
    if (live && t == 0 && p.rstd != nullptr) p.rstd[row] = rstd;
    T* hp = row_of<T>(p.h, at);
    T* yp = row_of<T>(p.y, at);
    auto put = [&](int c, const Raw<T>& a, const Raw<T>& b) {
      const int left = left_of(c);
      float h[8], y[8];
      h_of(a, b, h);
      weight8(p.weight, p.wdt, c, left, wvec, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= h[e] * rstd;
      Raw<T> out;
      if (p.h.data != nullptr) {
        out.set(h);
        out.template store<kVec>(hp + c, left);
      }
      if (p.y.data != nullptr) {
        out.set(y);
        out.template store<kVec>(yp + c, left);
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
        if (v * span < p.cols) put(8 * t + v * span, xr[v], rr[v]);
    } else {
      for (int c = 8 * t; c - 8 * t < p.cols; c += span) {
        // an h written over x or residual: this warp reads its 256 channels before it writes them
        fetch(c);
        put(c, xr[0], rr[0]);
      }
    }
  }
}

template <typename T, int kFormat, int kVecs, bool kVec>
void forward(const NormParams& p, cudaStream_t st) {
  const int threads = row_threads(p.cols, kVecs, 512), nrows = block_rows(threads), block = threads * nrows;
  const int64_t blocks = (p.rows + nrows - 1) / nrows, most = 152 * (2048 / block);
  rmsnorm_kernel<T, kFormat, kVecs, kVec><<<(unsigned)(blocks < most ? blocks : most), block, 0, st>>>(p, threads);
}
// Eights a thread by the channels: one warp a row while that takes at most six
// (three of fp32, whose eights take twice the registers); four and two beyond,
// and two where rows are not aligned, whose loads take more of them.
template <typename T, int kFormat, bool kVec>
void forward(const NormParams& p, cudaStream_t st) {
  const int n = (p.cols + 255) / 256;
  if constexpr (!kVec) {
    n <= 32 ? forward<T, kFormat, 2, kVec>(p, st) : forward<T, kFormat, 4, kVec>(p, st);
  } else if constexpr (sizeof(T) == 4) {
    n == 3 || n == 5 || n == 6 ? forward<T, kFormat, 3, kVec>(p, st) : n <= 32 ? forward<T, kFormat, 2, kVec>(p, st) : forward<T, kFormat, 4, kVec>(p, st);
  } else {
    if (n <= 2) forward<T, kFormat, 2, kVec>(p, st);
    else if (n == 3) forward<T, kFormat, 3, kVec>(p, st);
    else if (n == 5) forward<T, kFormat, 5, kVec>(p, st);
    else if (n == 6) forward<T, kFormat, 6, kVec>(p, st);
    else forward<T, kFormat, 4, kVec>(p, st);
  }
}
template <typename T>
cudaError_t forward(const NormParams& p, cudaStream_t st) {
  constexpr int size = sizeof(T);
  const bool vec = aligned(p.x, size, p.rows) && aligned(p.residual, size, p.rows) && aligned(p.h, size, p.rows) && aligned(p.y, size, p.rows);
  const int format = p.kept.data == nullptr ? -1 : p.kept.format;
  count_launch();
  if (format < 0) vec ? forward<T, -1, true>(p, st) : forward<T, -1, false>(p, st);
  else if (format == LM_CODE_I8) vec ? forward<T, LM_CODE_I8, true>(p, st) : forward<T, LM_CODE_I8, false>(p, st);
  else vec ? forward<T, LM_CODE_E4M3, true>(p, st) : forward<T, LM_CODE_E4M3, false>(p, st);
  return cudaGetLastError();
}

// rstd of rows without channels, whose mean square is 0.
__global__ void __launch_bounds__(256) rstd_of_nothing_kernel(float* rstd, int64_t rows, float value) {
  for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < rows; r += (int64_t)gridDim.x * 256) rstd[r] = value;
}

}  // namespace

cudaError_t launch_rmsnorm(lm_dtype dt, const NormParams& p, cudaStream_t st) {
  if (p.cols == 0) {
    const int64_t blocks = (p.rows + 255) / 256;
    count_launch();
    rstd_of_nothing_kernel<<<(unsigned)(blocks < 152 * 8 ? blocks : 152 * 8), 256, 0, st>>>(p.rstd, p.rows, 1.f / sqrtf(p.eps));
    return cudaGetLastError();
  }
  return dt == LM_BF16 ? forward<__nv_bfloat16>(p, st) : forward<float>(p, st);
}

}  // namespace lm
