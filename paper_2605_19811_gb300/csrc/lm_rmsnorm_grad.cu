// Gradient of the RMS norm, from the stored h or its 8-bit checkpoint (formulas
// at lm_rmsnorm_grad in lionmuon.h).
//
// Bound by memory: 8 bytes an element (dy, h, dh, dx in bf16).  A row is read
// once and stays in registers, one or two eights a thread, and the next row's
// loads go out before this row's sums: 16384 x 1280 takes 50 us so, and 64 us
// with a warp a row, five eights a lane and nothing ahead.  dweight is summed over a slot's
// rows in registers, over the slots of a block in shared memory, and over the
// blocks by a second kernel, each in a fixed order.
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace rows;

// kFormat < 0: h is a matrix.
// kMost: threads a block has at most.
template <typename T, int kFormat, int kVecs, bool kVec, int kMost>
__global__ void __launch_bounds__(kMost, kMost == 256 ? 2 : 1) rmsnorm_grad_kernel(const NormGradParams p, int threads) {
  constexpr bool kMatrix = kFormat < 0, kAhead = kMost < 1024;   // the next row's loads before this row's sums
  __shared__ float part[2][32];
  __shared__ float joined[64 * 8 * kVecs];        // where rows share a block they have at most 64 threads
  const Team team(threads);
  const int t = team.t, slot = team.slot, nrows = team.rows, span = team.span;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const bool whole = p.cols <= kVecs * span;
  const bool want = p.dweight != nullptr, past = p.dh.data != nullptr;
  const bool wvec = (reinterpret_cast<uintptr_t>(p.weight) & 15u) == 0;
  const float inv_cols = 1.f / (float)p.cols;
  float* sums = want ? p.parts + (int64_t)blockIdx.x * p.cols : nullptr;   // of this block's rows
  float acc[kVecs][8];
#pragma unroll
  for (int v = 0; v < kVecs; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[v][e] = 0.f;
  if (want && !whole)   // (such rows have a block of their own)
    for (int c = 8 * t; c < p.cols; c += span)
      for (int e = 0; e < 8 && c + e < p.cols; ++e) sums[c + e] = 0.f;
  // fp32 rows off 16-byte boundaries are read one by one here: 8191 x 1283 49 us
  // so, 70 us in pieces; 4095 x 4095 64 and 92.  Beyond 4096 channels, where the
  // next row is not loaded ahead, pieces would be ahead by a little (2047 x 8191
  // 102 and 98, 2047 x 12001 332 and 297).
  struct Eight {
    Raw<T, sizeof(T) == 4> dy, dh;
    std::conditional_t<kMatrix, Raw<T, sizeof(T) == 4>, RawCodes<kMatrix ? 0 : kFormat>> h;
  };
  auto load = [&](int64_t row, int c, Eight& e8) {
    const bool live = row < p.rows;
    const int64_t at = live ? row : 0;
    const int left = live ? p.cols - c : kNoRow;
    e8.dy.template load<kVec>(Row<const T>(p.dy, at, p.rows), c, left);
    if constexpr (kMatrix) e8.h.template load<kVec>(Row<const T>(p.h, at, p.rows), c, left);
    else e8.h.load(p.h8, at, c, left > 0);
    e8.dh.zero();
    if (past) e8.dh.template load<kVec>(Row<const T>(p.dh, at, p.rows), c, left);
  };
  auto settle = [&](int64_t row, int c, Eight& e8) {
    const int64_t at = row < p.rows ? row : 0;
    const int left = row < p.rows ? p.cols - c : kNoRow;
    e8.dy.template settle<kVec>(Row<const T>(p.dy, at, p.rows), c, left);
    if constexpr (kMatrix) e8.h.template settle<kVec>(Row<const T>(p.h, at, p.rows), c, left);
    if (past) e8.dh.template settle<kVec>(Row<const T>(p.dh, at, p.rows), c, left);
  };
  // The gain of the thread's channels, for every row.
  float gain[kVecs][8];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) weight8(p.weight, p.wdt, 8 * t + v * span, whole ? p.cols - 8 * t - v * span : 0, wvec, gain[v]);
  const int64_t step = (int64_t)gridDim.x * nrows;
  int64_t row0 = (int64_t)blockIdx.x * nrows;
  Eight now[kVecs];
  float rstd = row0 + slot < p.rows ? p.rstd[row0 + slot] : 0.f;
  if (kAhead && whole) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) load(row0 + slot, 8 * t + v * span, now[v]);
  }
  for (int turn = 0; row0 < p.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool live = row < p.rows;
    auto left_of = [&](int c) { return live ? p.cols - c : kNoRow; };
    // dy and xh = h rstd; codes beyond the row are no numbers
    auto get = [&](const Eight& e8, int left, float (&g)[8], float (&x)[8]) {
      e8.dy.get(g);
      e8.h.get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (kMatrix || e < left) ? x[e] * rstd : 0.f;
    };
    auto dot = [&](int c, const Eight& e8, const float (&w)[8]) {
      float g[8], x[8], q = 0.f;
      get(e8, left_of(c), g, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) q += w[e] * g[e] * x[e];
      return q;
    };
    Eight next[kVecs];
    const float rstd_next = row + step < p.rows ? p.rstd[row + step] : 0.f;
    float s = 0.f;
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) load(kAhead ? row + step : row, 8 * t + v * span, kAhead ? next[v] : now[v]);
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        settle(row, 8 * t + v * span, now[v]);
        s += dot(8 * t + v * span, now[v], gain[v]);
      }
    } else {
      for (int c = 8 * t; c - 8 * t < p.cols; c += span) {
        load(row, c, now[0]);
        settle(row, c, now[0]);
        weight8(p.weight, p.wdt, c, left_of(c), wvec, gain[0]);
        s += dot(c, now[0], gain[0]);
      }
    }
    s = team.sum(s, part, turn);
    const float mean = s * inv_cols;
    T* dxp = row_of<T>(p.dx, live ? row : 0);
    auto put = [&](int c, const Eight& q, const float (&w)[8], float (&a)[8]) {
      const int left = left_of(c);
      float g[8], x[8], d[8];
      get(q, left, g, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] += g[e] * x[e];
      if (p.dx.data == nullptr) return;
      q.dh.get(d);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] += rstd * (w[e] * g[e] - x[e] * mean);
      Raw<T> out;
      out.set(d);
      out.template store<kVec>(dxp + c, left);
    };
    if (whole) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        if (v * span < p.cols) put(8 * t + v * span, now[v], gain[v], acc[v]);
        if (kAhead) now[v] = next[v];
      }
    } else {
      for (int c = 8 * t; c - 8 * t < p.cols; c += span) {
        float a[8] = {};
        load(row, c, now[0]);
        settle(row, c, now[0]);
        weight8(p.weight, p.wdt, c, left_of(c), wvec, gain[0]);
        put(c, now[0], gain[0], a);
        if (want)
          for (int e = 0; e < 8 && c + e < p.cols; ++e) sums[c + e] += a[e];
      }
    }
    rstd = rstd_next;
  }
  if (!want || !whole) return;
  if (nrows > 1) {
    for (int k = 0; k < nrows; ++k) {   // slot by slot
      if (slot == k) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int i = 8 * t + v * span + e;
            if (k > 0) acc[v][e] += joined[i];
            joined[i] = acc[v][e];
          }
      }
      __syncthreads();
    }
    if (slot != nrows - 1) return;
  }
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    const int c = 8 * t + v * span;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < p.cols) sums[c + e] = acc[v][e];
  }
}

template <typename T, int kFormat, int kVecs, bool kVec, int kMost>
int backward(const NormGradParams& p, cudaStream_t st) {
  const int threads = row_threads(p.cols, kVecs, 1024), nrows = block_rows(threads), block = threads * nrows;
  const int64_t blocks = (p.rows + nrows - 1) / nrows;
  const int fit = block <= 512 ? 152 * (512 / block) : 152, most = fit < kNormGradParts ? fit : kNormGradParts;
  const int grid = (int)(blocks < most ? blocks : most);
  rmsnorm_grad_kernel<T, kFormat, kVecs, kVec, kMost><<<(unsigned)grid, block, 0, st>>>(p, threads);
  return grid;
}
// One eight a thread up to 4096 channels; beyond, two of bf16 (16384 x 1280:
// one 50 us, two 68 us; 2048 x 8192: 89 and 56 us).
// 1024 threads (fp32 beyond 4096 channels, bf16 beyond 8192) have 64 registers
// each, too few for the next row's loads too: 2048 x 8192 fp32 158 us with
// them, 70 without (two eights and 512 threads: 88); 2048 x 16384 bf16 225 and
// 123; 2047 x 12001 bf16 352 and 132.
template <typename T, int kFormat, bool kVec>
int backward(const NormGradParams& p, cudaStream_t st) {
  if (p.cols <= 2048) return backward<T, kFormat, 1, kVec, 256>(p, st);
  if (p.cols <= 4096) return backward<T, kFormat, 1, kVec, 512>(p, st);
  if constexpr (sizeof(T) == 4) return backward<T, kFormat, 1, kVec, 1024>(p, st);
  else return p.cols <= 8192 ? backward<T, kFormat, 2, kVec, 512>(p, st) : backward<T, kFormat, 2, kVec, 1024>(p, st);
}
// Returns the number of blocks, each of which leaves a part of dweight.
template <typename T>
int backward(const NormGradParams& p, cudaStream_t st) {
  constexpr int size = sizeof(T);
  const bool vec = aligned(p.dy, size, p.rows) && aligned(p.h, size, p.rows) && aligned(p.dh, size, p.rows) && aligned(p.dx, size, p.rows);
  count_launch();
  if (p.h8.data == nullptr) return vec ? backward<T, -1, true>(p, st) : backward<T, -1, false>(p, st);
  if (p.h8.format == LM_CODE_I8) return vec ? backward<T, LM_CODE_I8, true>(p, st) : backward<T, LM_CODE_I8, false>(p, st);
  return vec ? backward<T, LM_CODE_E4M3, true>(p, st) : backward<T, LM_CODE_E4M3, false>(p, st);
}

// dweight from the blocks' parts: 8 columns a block, 32 runs of parts each, both
// in order.  Its set-up overlaps the gradient kernel's end.
__global__ void __launch_bounds__(256) norm_dweight_kernel(const float* parts, int nparts, int cols, void* dweight, int dwdt) {
  __shared__ float run[32][9];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int c = blockIdx.x * 8 + (threadIdx.x & 7), k = threadIdx.x >> 3;
  const int each = (nparts + 31) / 32, p0 = min(nparts, k * each), p1 = min(nparts, p0 + each);
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int i = p0; i < p1; ++i) s += parts[(int64_t)i * cols + c];
  }
  run[k][threadIdx.x & 7] = s;
  __syncthreads();
  if (k != 0 || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += run[i][threadIdx.x];
  if (dwdt == LM_F32) static_cast<float*>(dweight)[c] = s;
  else static_cast<__nv_bfloat16*>(dweight)[c] = __float2bfloat16_rn(s);
}

}  // namespace

cudaError_t launch_rmsnorm_grad(lm_dtype dt, const NormGradParams& p, cudaStream_t st) {
  int parts = 0;
  if (p.rows > 0) {
    parts = dt == LM_BF16 ? backward<__nv_bfloat16>(p, st) : backward<float>(p, st);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (p.dweight != nullptr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.cols + 7) / 8), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 0 ? 1 : 0;
    count_launch();
    return cudaLaunchKernelEx(&cfg, norm_dweight_kernel, (const float*)p.parts, parts, (int)p.cols, p.dweight, (int)p.dwdt);
  }
  return cudaGetLastError();
}

}  // namespace lm
