// Linear layers in 8 bits (lm_weight8, lm_linear8 and lm_linear8_grad in
// lionmuon.h):
//   y = x W^T (tokens x out),  dx = dy W (tokens x in)
// with activations of one scale for each token's 128 channels and weights of one
// scale for each block of 128 x 128.
//
// A code times its power-of-two scale is a bf16 number: both operands are laid
// out as bf16 in the workspace without a rounding, and the product of bf16
// matrices follows.
#include <cuda_bf16.h>

#include "lm_code8.cuh"
#include "lm_gemm_tc.cuh"
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace gemm;

constexpr int kBlock = LM_CODE_GROUP;

// Weights packed, a 128 x 128 block a CTA: a warp takes 16 rows, two at a time,
// eight columns a lane.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) weight8_pack_kernel(Mat w, int64_t rows, int64_t cols, Blocks out) {
  __shared__ uint32_t part[8];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * kBlock + 8 * (lane & 15);
  const int left = (int)min((int64_t)8, cols - c);
  for (int64_t block = blockIdx.y; block * kBlock < rows; block += gridDim.y) {
    const int64_t r0 = block * kBlock + warp * 16 + (lane >> 4);
    rows::Raw<T> raw[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t r = r0 + 2 * k;
      raw[k].zero();
      if (r >= rows || left <= 0) continue;
      const T* p = static_cast<const T*>(w.data) + r * w.ld + c;
      if (kVec && left == 8) {
#pragma unroll
        for (int i = 0; i < rows::Raw<T>::kPieces; ++i) rows::load16(raw[k].w + 4 * i, reinterpret_cast<const uint4*>(p) + i, true);
      } else {
        raw[k].single(p, left);
      }
    }
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float v[8];
      raw[k].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, code8::magnitude(v[e]));
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    __syncthreads();     // the last block's maxima have been read
    if (lane == 0) part[warp] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) most = max(most, part[k]);
    const float scale = code8::group_scale<LM_CODE_E4M3>(most), inv = code8::inverse_scale(scale);
    if (threadIdx.x == 0) out.scales[block * out.ld_scales + blockIdx.x] = scale;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t r = r0 + 2 * k;
      if (r >= rows || left <= 0) continue;
      float v[8];
      raw[k].get(v);
      uint32_t q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = code8::encode2<LM_CODE_E4M3>(v[2 * i], v[2 * i + 1], inv);
      // the pitch is a multiple of 16: eight codes are inside the row wherever one is
      *reinterpret_cast<uint2*>(out.data + r * out.ld + c) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
    }
  }
}

// Codes back to values, eight a thread: of weights, or (kRows) of activations.
template <typename T, bool kRows>
__global__ void __launch_bounds__(256) values_kernel(const uint8_t* codes, int64_t ld, const float* scales, int64_t ld_scales, int64_t nrows, int64_t cols, T* to,
                                                     int64_t ld_to, int vec) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t per = (cols + 7) / 8, all = nrows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per, c = 8 * (i - r * per);
    const uint2 q = *reinterpret_cast<const uint2*>(codes + r * ld + c);
    const float s = kRows ? scales[c / kBlock * ld_scales + r] : scales[r / kBlock * ld_scales + c / kBlock];
    const uint32_t two[4] = {q.x, q.x >> 16, q.y, q.y >> 16};
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 d = code8::decode2<LM_CODE_E4M3>(two[k]);
      v[2 * k] = d.x * s;
      v[2 * k + 1] = d.y * s;
    }
    rows::Raw<T> o;
    o.set(v);
    T* p = to + r * ld_to + c;
    if (vec && cols - c >= 8) {
#pragma unroll
      for (int k = 0; k < rows::Raw<T>::kPieces; ++k) reinterpret_cast<uint4*>(p)[k] = make_uint4(o.w[4 * k], o.w[4 * k + 1], o.w[4 * k + 2], o.w[4 * k + 3]);
    } else {
      o.put_single(p, 0, (int)min((int64_t)8, cols - c));
    }
  }
}
unsigned blocks_for(int64_t nrows, int64_t cols) {
  const int64_t b = (nrows * ((cols + 7) / 8) + 255) / 256;
  return (unsigned)std::min<int64_t>(b, 152 * 16);
}

struct Layout {
  int64_t ldx, ldw, k, n;
  size_t x, w, parts, total;
};
Layout make_layout(const Linear8Params& q) {
  Layout l{};
  l.k = q.grad ? q.out : q.in;
  l.n = q.grad ? q.in : q.out;
  l.ldx = (l.k + 7) / 8 * 8;
  l.ldw = ((int64_t)q.in + 7) / 8 * 8;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  l.w = up((size_t)q.tokens * l.ldx * 2);
  l.parts = l.w + up((size_t)q.out * l.ldw * 2);
  l.total = l.parts + parts_bytes(split_schedule(q.tokens, l.n, l.k));
  return l;
}

}  // namespace

cudaError_t launch_weight8_pack(lm_dtype dt, const Mat& w, int64_t nrows, int64_t cols, const Blocks& c, cudaStream_t st) {
  const dim3 grid((unsigned)((cols + kBlock - 1) / kBlock), (unsigned)std::min<int64_t>((nrows + kBlock - 1) / kBlock, 65535));
  const bool vec = rows::aligned(w, dt == LM_F32 ? 4 : 2, nrows);
  if (dt == LM_F32) return launch_after(vec ? weight8_pack_kernel<float, true> : weight8_pack_kernel<float, false>, grid, 256, 0, st, w, nrows, cols, c);
  return launch_after(vec ? weight8_pack_kernel<__nv_bfloat16, true> : weight8_pack_kernel<__nv_bfloat16, false>, grid, 256, 0, st, w, nrows, cols, c);
}

cudaError_t launch_weight8_unpack(lm_dtype dt, const Blocks& c, int64_t nrows, int64_t cols, const Mat& w, cudaStream_t st) {
  const int vec = rows::aligned(w, dt == LM_F32 ? 4 : 2, nrows);
  const dim3 grid(blocks_for(nrows, cols));
  if (dt == LM_F32)
    return launch_after(values_kernel<float, false>, grid, 256, 0, st, (const uint8_t*)c.data, c.ld, (const float*)c.scales, c.ld_scales, nrows, cols,
                        static_cast<float*>(w.data), w.ld, vec);
  return launch_after(values_kernel<__nv_bfloat16, false>, grid, 256, 0, st, (const uint8_t*)c.data, c.ld, (const float*)c.scales, c.ld_scales, nrows, cols,
                      static_cast<__nv_bfloat16*>(w.data), w.ld, vec);
}

size_t linear8_workspace(const Linear8Params& q) { return q.tokens <= 0 ? 0 : make_layout(q).total; }

cudaError_t launch_linear8(const Linear8Params& q, cudaStream_t st) {
  if ((q.grad ? q.out : q.in) == 0) return start_zero(q.y, q.ydt, q.tokens, q.grad ? q.in : q.out, st);
  const Layout l = make_layout(q);
  uint8_t* ws = static_cast<uint8_t*>(q.workspace);
  __nv_bfloat16 *x = reinterpret_cast<__nv_bfloat16*>(ws), *w = reinterpret_cast<__nv_bfloat16*>(ws + l.w);
  cudaError_t e = launch_after(values_kernel<__nv_bfloat16, true>, dim3(blocks_for(q.tokens, l.k)), 256, 0, st, (const uint8_t*)q.x.data, q.x.ld,
                               (const float*)q.x.scales, q.x.ld_scales, q.tokens, l.k, x, l.ldx, 1);
  if (e != cudaSuccess) return e;
  e = launch_after(values_kernel<__nv_bfloat16, false>, dim3(blocks_for(q.out, q.in)), 256, 0, st, (const uint8_t*)q.w.data, q.w.ld,
                   (const float*)q.w.scales, q.w.ld_scales, (int64_t)q.out, (int64_t)q.in, w, l.ldw, 1);
  if (e != cudaSuccess) return e;
  Params<StoreEpi> s{};
  s.sch = split_schedule(q.tokens, l.n, l.k);
  s.m = (int32_t)q.tokens;
  s.n = (int32_t)l.n;
  s.wait_ns = env_wait_limit_ns();
  s.parts = reinterpret_cast<float*>(ws + l.parts);
  const Mat y{q.y.data, q.y.ld};
  s.epi.out = make_store(y, q.ydt, q.tokens, false);
  if ((e = encode_operand(&s.a, x, l.k, q.tokens, l.ldx, false)) != cudaSuccess) return e;
  if ((e = encode_operand(&s.b, w, q.in, q.out, l.ldw, q.grad)) != cudaSuccess) return e;
  return q.grad ? start_store<kRowsK, kRowsMn>(s, st) : start_store<kRowsK, kRowsK>(s, st);
}

}  // namespace lm
