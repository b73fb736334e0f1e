// Packing a matrix into 8-bit codes with a power-of-two scale for each group
// of 128 channels (the format is stated at lm_checkpoint8 in lionmuon.h), and
// back.  Bound by memory: 3 bytes an element in bf16.  A warp takes 256
// channels of a row, eight a lane, so that a group is half a warp; several
// such pieces are loaded before the first is worked on.  32768 x 5120 bf16 to
// int8: 119 us (4.3 TB/s), back 91 us (5.6 TB/s).
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace rows;

constexpr int kThreads = 256, kPiece = 256;
constexpr int kPackAhead = 2, kUnpackAhead = 4;   // pieces loaded at once: packing has more to do for each

// A warp's way over the pieces (256 channels of a row each), `warps` apart.
struct Way {
  int64_t row, drow;
  int k, dk, per;
  __device__ __forceinline__ explicit Way(int cols) {
    per = (cols + kPiece - 1) / kPiece;
    const int64_t first = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = (int64_t)gridDim.x * (kThreads / 32);
    row = first / per;
    k = (int)(first - row * per);
    drow = warps / per;
    dk = (int)(warps - drow * per);
  }
  __device__ __forceinline__ int column() const { return k * kPiece + 8 * (int)(threadIdx.x & 31); }
  __device__ __forceinline__ void advance() {
    row += drow;
    k += dk;
    if (k >= per) {
      k -= per;
      ++row;
    }
  }
};

template <typename T, int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads) pack8_kernel(Mat x, int64_t nrows, int cols, Codes out) {
  Way at(cols);
  while (at.row < nrows) {
    Raw<T> raw[kPackAhead];
    int64_t row[kPackAhead];
    int c[kPackAhead];
#pragma unroll
    for (int k = 0; k < kPackAhead; ++k, at.advance()) {
      row[k] = at.row;
      c[k] = at.column();
      const int left = at.row < nrows ? cols - c[k] : kNoRow;
      raw[k].template load<kVec>(Row<const T>(x, at.row < nrows ? at.row : 0, nrows), c[k], left);
    }
#pragma unroll
    for (int k = 0; k < kPackAhead; ++k) {
      if (row[k] >= nrows) break;
      float v[8];
      raw[k].template settle<kVec>(Row<const T>(x, row[k], nrows), c[k], cols - c[k]);
      raw[k].get(v);
      keep8<kFormat>(out, row[k], c[k], cols, v);
    }
  }
}

template <typename T, int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads) unpack8_kernel(Codes in, int64_t nrows, int cols, Mat x) {
  Way at(cols);
  while (at.row < nrows) {
    RawCodes<kFormat> raw[kUnpackAhead];
    int64_t row[kUnpackAhead];
    int c[kUnpackAhead];
#pragma unroll
    for (int k = 0; k < kUnpackAhead; ++k, at.advance()) {
      row[k] = at.row;
      c[k] = at.column();
      raw[k].load(in, at.row, c[k], at.row < nrows && c[k] < cols);
    }
#pragma unroll
    for (int k = 0; k < kUnpackAhead; ++k) {
      if (row[k] >= nrows) break;
      float v[8];
      raw[k].get(v);
      Raw<T> out;
      out.set(v);
      out.template store<kVec>(row_of<T>(x, row[k]) + c[k], cols - c[k]);
    }
  }
}

unsigned grid_for(int64_t nrows, int64_t cols) {
  const int64_t pieces = nrows * ((cols + kPiece - 1) / kPiece), blocks = (pieces + kThreads / 32 - 1) / (kThreads / 32);
  return (unsigned)(blocks < 152 * 16 ? blocks : 152 * 16);
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
