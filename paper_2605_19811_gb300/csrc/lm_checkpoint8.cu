// Packing a matrix into 8-bit codes with a power-of-two scale for each group
// of 128 channels (the format is stated at lm_checkpoint8 in lionmuon.h), and
// back.  Bound by memory: 3 bytes an element in bf16.  A warp takes 256
// channels of a row, eight a lane, so that a group is half a warp; four such
// pieces are loaded before the first is worked on.
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace rows;

constexpr int kThreads = 256, kPiece = 256, kAhead = 4;

// Piece i of the matrix: 256 channels of a row, this lane's first.
struct Place {
  int64_t row;
  int c;
  __device__ __forceinline__ Place(int64_t i, int64_t per_row) {
    row = i / per_row;
    c = (int)(i - row * per_row) * kPiece + 8 * (int)(threadIdx.x & 31);
  }
};

template <typename T, int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads) pack8_kernel(Mat x, int64_t nrows, int cols, Codes out) {
  const int64_t per = (cols + kPiece - 1) / kPiece, all = nrows * per, step = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t i0 = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i0 < all; i0 += kAhead * step) {
    Raw<T> raw[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const Place at(i0 + k * step, per);
      const int left = i0 + k * step < all ? cols - at.c : 0;
      if (left > 0) raw[k].template load<kVec>(row_of<const T>(x, at.row) + at.c, left);
      else raw[k].zero();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + k * step >= all) break;
      const Place at(i0 + k * step, per);
      float v[8];
      raw[k].get(v);
      keep8<kFormat>(out, at.row, at.c, cols, v);
    }
  }
}

template <typename T, int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads) unpack8_kernel(Codes in, int64_t nrows, int cols, Mat x) {
  const int64_t per = (cols + kPiece - 1) / kPiece, all = nrows * per, step = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t i0 = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i0 < all; i0 += kAhead * step) {
    RawCodes<kFormat> raw[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const Place at(i0 + k * step, per);
      if (i0 + k * step < all && at.c < cols) raw[k].load(in, at.row, at.c);
      else raw[k].zero();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const Place at(i0 + k * step, per);
      if (i0 + k * step >= all || at.c >= cols) continue;
      float v[8];
      raw[k].get(v);
      store8<kVec>(row_of<T>(x, at.row) + at.c, cols - at.c, v);
    }
  }
}

unsigned grid_for(int64_t nrows, int64_t cols) {
  const int64_t pieces = nrows * ((cols + kPiece - 1) / kPiece), blocks = (pieces + kThreads / 32 - 1) / (kThreads / 32);
  return (unsigned)(blocks < 152 * 8 ? blocks : 152 * 8);
}

template <typename T, int kFormat>
void pack(const Mat& x, int64_t nrows, int cols, const Codes& c, cudaStream_t st) {
  if (aligned(x, sizeof(T), nrows)) pack8_kernel<T, kFormat, true><<<grid_for(nrows, cols), kThreads, 0, st>>>(x, nrows, cols, c);
  else pack8_kernel<T, kFormat, false><<<grid_for(nrows, cols), kThreads, 0, st>>>(x, nrows, cols, c);
}
template <typename T, int kFormat>
void unpack(const Codes& c, int64_t nrows, int cols, const Mat& x, cudaStream_t st) {
  if (aligned(x, sizeof(T), nrows)) unpack8_kernel<T, kFormat, true><<<grid_for(nrows, cols), kThreads, 0, st>>>(c, nrows, cols, x);
  else unpack8_kernel<T, kFormat, false><<<grid_for(nrows, cols), kThreads, 0, st>>>(c, nrows, cols, x);
}

}  // namespace

cudaError_t launch_pack8(lm_dtype dt, const Mat& x, int64_t nrows, int64_t cols, const Codes& c, cudaStream_t st) {
  count_launch();
  const int n = (int)cols;
  if (dt == LM_BF16) c.format == LM_CODE_I8 ? pack<__nv_bfloat16, LM_CODE_I8>(x, nrows, n, c, st) : pack<__nv_bfloat16, LM_CODE_E4M3>(x, nrows, n, c, st);
  else c.format == LM_CODE_I8 ? pack<float, LM_CODE_I8>(x, nrows, n, c, st) : pack<float, LM_CODE_E4M3>(x, nrows, n, c, st);
  return cudaGetLastError();
}

cudaError_t launch_unpack8(lm_dtype dt, const Codes& c, int64_t nrows, int64_t cols, const Mat& x, cudaStream_t st) {
  count_launch();
  const int n = (int)cols;
  if (dt == LM_BF16) c.format == LM_CODE_I8 ? unpack<__nv_bfloat16, LM_CODE_I8>(c, nrows, n, x, st) : unpack<__nv_bfloat16, LM_CODE_E4M3>(c, nrows, n, x, st);
  else c.format == LM_CODE_I8 ? unpack<float, LM_CODE_I8>(c, nrows, n, x, st) : unpack<float, LM_CODE_E4M3>(c, nrows, n, x, st);
  return cudaGetLastError();
}

}  // namespace lm
