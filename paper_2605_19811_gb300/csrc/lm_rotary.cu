// Queries and keys: the norm of each head, its gain, and the rotation by
// position, in one pass, and the gradient (formulas at lm_qk_rotary_args in
// lionmuon.h).
//
// Eight channels, four pairs, to a lane: two pieces of four channels, (j .., j +
// turned / 2 ..) of the halves or eight neighbours (interleaved), so that a pair
// is always in one lane; what does not turn goes along in two halves with cos = 1.
// dim / 8 lanes, made a power of two, take a head, four heads at once, for one
// token, whose cosines and sines stay in registers.  For the gradient the head's
// rstd is computed again: the head is read anyway.  dweight: each lane keeps sums
// over its heads, a block's are joined in shared memory, and a second kernel adds
// the blocks', all in a fixed order.
// Heads of other sizes or alignments take a warp each, a pair or a channel a lane.
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
constexpr int kMostBlocks = 152 * 6;
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

// dweight of each part: its blocks' sums added, eight warps to 32 channels.
__global__ void __launch_bounds__(kThreads) rotary_join_kernel(const __grid_constant__ RotaryParams p, int first1, int blocks0, int blocks1) {
  __shared__ float sums[kWarps][32];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const RotaryPart& part = p.part[blockIdx.y];
  if (part.dweight == nullptr) return;
  const int blocks = blockIdx.y ? blocks1 : blocks0;
  const float* from = p.sums + (int64_t)(blockIdx.y ? first1 : 0) * p.dim + c;
  float s = 0.f;
  if (c < p.dim) {
#pragma unroll 8
    for (int k = warp; k < blocks; k += kWarps) s += from[(int64_t)k * p.dim];
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= p.dim) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < kWarps; ++k) s += sums[k][lane];
  if (part.dwdt == LM_F32) static_cast<float*>(part.dweight)[c] = s;
  else static_cast<__nv_bfloat16*>(part.dweight)[c] = __float2bfloat16_rn(s);
}

// --- four pairs a lane ---

// How a part's heads fall to groups of lanes: `lanes` (a power of two) to a
// head, `chunk` heads of a token one after another.
struct Deal {
  int32_t lanes, active;      // active: lanes that hold channels
  int32_t chunk, chunks[2];   // heads of an item; items a token of each part
};
constexpr int kAhead = 4;     // heads loaded at once

__device__ __forceinline__ void load4(const float* p, float (&v)[8], int at) {
  const float4 x = __ldcs(reinterpret_cast<const float4*>(p));
  v[at] = x.x; v[at + 1] = x.y; v[at + 2] = x.z; v[at + 3] = x.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&v)[8], int at) {
  const uint2 x = __ldcs(reinterpret_cast<const uint2*>(p));
  v[at] = __uint_as_float(x.x << 16);
  v[at + 1] = __uint_as_float(x.x & 0xFFFF0000u);
  v[at + 2] = __uint_as_float(x.y << 16);
  v[at + 3] = __uint_as_float(x.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[8], int at) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[at], v[at + 1], v[at + 2], v[at + 3]));
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&v)[8], int at) {
  __stcs(reinterpret_cast<uint2*>(p), make_uint2(tc::pack_bf2(v[at], v[at + 1]), tc::pack_bf2(v[at + 2], v[at + 3])));
}

// A lane's channels: pieces of four from a and b.  Pair k is (v[k], v[4 + k]) of
// the halves, (v[2 k], v[2 k + 1]) interleaved.
template <bool kInterleaved>
struct Lane {
  int a, b, pair;       // pair: the first of its four; -1 where they do not turn
  bool in;
  __device__ __forceinline__ Lane(const RotaryParams& p, int i) : in(8 * i < p.dim) {
    const int half = p.turned >> 1;
    if (kInterleaved) {
      a = 8 * i;
      b = a + 4;
      pair = a < p.turned ? 4 * i : -1;
    } else if (4 * i < half) {
      a = 4 * i;
      b = half + a;
      pair = a;
    } else {
      a = p.turned + 4 * i - half;
      b = a + (p.dim - p.turned) / 2;
      pair = -1;
    }
  }
  // cosines and sines of its pairs at the token's position
  __device__ __forceinline__ void turns(const RotaryParams& p, int64_t token, float (&c)[4], float (&s)[4]) const {
    if (pair < 0 || !in) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        c[k] = 1.f;
        s[k] = 0.f;
      }
      return;
    }
    const int64_t at = p.positions[token];
    if (at < 0 || at >= p.table_rows) {
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] = s[k] = __int_as_float(0x7FC00000);
      return;
    }
    const float* t = p.table + (at * (p.turned >> 1) + pair) * 2;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[k] = __ldg(t + 2 * k);
      s[k] = __ldg(t + 2 * k + 1);
    }
  }
  __device__ __forceinline__ void gains(const void* w, int dt, float (&v)[8]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = in ? gain(w, dt, a + k) : 1.f;
      v[4 + k] = in ? gain(w, dt, b + k) : 1.f;
    }
  }
  static __device__ __forceinline__ void turn(float (&v)[8], const float (&c)[4], const float (&s)[4], bool back) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float &x = v[kInterleaved ? 2 * k : k], &y = v[kInterleaved ? 2 * k + 1 : 4 + k];
      const float sn = back ? -s[k] : s[k];
      const float u = x * c[k] - y * sn;
      y = y * c[k] + x * sn;
      x = u;
    }
  }
};
template <typename T, bool kInterleaved>
__device__ __forceinline__ void load8(const Heads& h, int64_t token, int head, const Lane<kInterleaved>& l, bool in, float (&v)[8]) {
  if (in) {
    const T* p = head_of<const T>(h, token, head);
    load4(p + l.a, v, 0);
    load4(p + l.b, v, 4);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.f;
  }
}
__device__ __forceinline__ float group_sum(float v, int lanes) {
  for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rotary8_kernel(const __grid_constant__ RotaryParams p, const __grid_constant__ Deal d) {
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x % d.lanes, groups = kThreads / d.lanes, per = d.chunks[0] + d.chunks[1];
  const Lane<kInterleaved> l(p, lane);
  const int64_t items = p.tokens * per;
  // whole warps go round together: an item beyond the last has no heads
  for (int64_t first = (int64_t)blockIdx.x * groups; first < items; first += (int64_t)gridDim.x * groups) {
    const int64_t item = first + threadIdx.x / d.lanes;
    const int64_t token = item / per;
    const int sub = (int)(item - token * per), which = sub >= d.chunks[0] ? 1 : 0;
    const RotaryPart& part = p.part[which];
    int head = (sub - (which ? d.chunks[0] : 0)) * d.chunk;
    const int end = item < items ? min(head + d.chunk, part.heads) : head;
    float c[4], s[4], w[8];
    if (head < end) {
      l.turns(p, token, c, s);
      if (p.norm) l.gains(part.weight, part.wdt, w);
    }
    for (int at = 0; at < d.chunk; at += kAhead) {      // the same number of rounds for every group
      float v[kAhead][8];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) load8<T>(part.x, token, head + at + k, l, l.in && head + at + k < end, v[k]);
      if (p.norm) {
        float q[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          q[k] = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) q[k] = fmaf(v[k][e], v[k][e], q[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float rstd = rsqrtf(group_sum(q[k], d.lanes) / (float)p.dim + p.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[k][e] *= rstd * w[e];
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (!l.in || head + at + k >= end) continue;
        l.turn(v[k], c, s, false);
        T* y = head_of<T>(part.y, token, head + at + k);
        store4(y + l.a, v[k], 0);
        store4(y + l.b, v[k], 4);
      }
    }
  }
}

// Blocks below q_blocks take the queries' items, the others the keys'.
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) rotary8_grad_kernel(const __grid_constant__ RotaryParams p, const __grid_constant__ Deal d, int q_blocks) {
  extern __shared__ float sums[];     // groups x dim
  griddep_wait();
  griddep_launch_dependents();
  constexpr int kTogether = 2;        // heads loaded at once: dy and x of each
  const int lane = threadIdx.x % d.lanes, group = threadIdx.x / d.lanes, groups = kThreads / d.lanes;
  const int which = (int)blockIdx.x >= q_blocks ? 1 : 0;
  const RotaryPart& part = p.part[which];
  const int per = d.chunks[which], block = which ? blockIdx.x - q_blocks : blockIdx.x, blocks = which ? gridDim.x - q_blocks : q_blocks;
  const Lane<kInterleaved> l(p, lane);
  const int64_t items = p.tokens * per;
  float w[8], dw[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[e] = 0.f;
  if (p.norm) l.gains(part.weight, part.wdt, w);
  for (int64_t first = (int64_t)block * groups; first < items; first += (int64_t)blocks * groups) {
    const int64_t item = first + group, token = item / per;
    const int head = (int)(item - token * per) * d.chunk;
    const int end = item < items ? min(head + d.chunk, part.heads) : head;
    float c[4], s[4];
    if (head < end) l.turns(p, token, c, s);
    for (int at = 0; at < d.chunk; at += kTogether) {
      float v[kTogether][8], x[kTogether][8];
      bool in[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        in[k] = l.in && head + at + k < end;
        load8<T>(part.dy, token, head + at + k, l, in[k], v[k]);
        if (p.norm) load8<T>(part.x, token, head + at + k, l, in[k], x[k]);
      }
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        if (in[k]) l.turn(v[k], c, s, true);
        if (p.norm) {
          float q = 0.f, r = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            q = fmaf(x[k][e], x[k][e], q);
            r = fmaf(v[k][e] * w[e], x[k][e], r);
          }
          const float rstd = rsqrtf(group_sum(q, d.lanes) / (float)p.dim + p.eps);
          const float mean = group_sum(r, d.lanes) * rstd / (float)p.dim;
          if (in[k]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float xh = x[k][e] * rstd;
              dw[e] = fmaf(v[k][e], xh, dw[e]);
              v[k][e] = rstd * (v[k][e] * w[e] - xh * mean);
            }
          }
        }
        if (in[k]) {
          T* dx = head_of<T>(part.dx, token, head + at + k);
          store4(dx + l.a, v[k], 0);
          store4(dx + l.b, v[k], 4);
        }
      }
    }
  }
  if (part.dweight == nullptr) return;
  if (l.in) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sums[group * p.dim + l.a + k] = dw[k];
      sums[group * p.dim + l.b + k] = dw[4 + k];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < p.dim; c += kThreads) {
    float t = 0.f;
    for (int k = 0; k < groups; ++k) t += sums[k * p.dim + c];
    p.sums[(int64_t)blockIdx.x * p.dim + c] = t;
  }
}

bool pieces_of_four(const Heads& h, int size) {
  return reinterpret_cast<uintptr_t>(h.data) % (4 * size) == 0 && h.ld_token % 4 == 0 && h.ld_head % 4 == 0;
}
// Whether eight channels go to a lane, and how.
bool deal(const RotaryParams& p, lm_dtype dt, bool grad, Deal* d) {
  const int size = dt == LM_F32 ? 4 : 2;
  if (p.dim % 8 != 0 || p.dim > 256 || p.turned % 8 != 0) return false;
  for (const RotaryPart& r : p.part) {
    if (r.heads == 0) continue;
    if ((!grad || p.norm) && !pieces_of_four(r.x, size)) return false;
    if (!pieces_of_four(grad ? r.dy : r.y, size)) return false;
    if (grad && !pieces_of_four(r.dx, size)) return false;
  }
  d->active = p.dim / 8;
  d->lanes = 1;
  while (d->lanes < d->active) d->lanes *= 2;
  // as many heads to an item as leave every SM 32 warps of items
  const int64_t groups = (int64_t)152 * 32 * (32 / d->lanes), heads = p.part[0].heads + p.part[1].heads;
  const int64_t each = p.tokens * heads / groups;
  d->chunk = (int)std::min<int64_t>(std::max<int64_t>(1, each), 16);
  if (d->chunk > kAhead) d->chunk = d->chunk / kAhead * kAhead;
  for (int i = 0; i < 2; ++i) d->chunks[i] = (p.part[i].heads + d->chunk - 1) / d->chunk;
  return true;
}

int grad_blocks(int64_t tokens, int64_t heads) {
  const int64_t b = (tokens * heads + kWarps - 1) / kWarps;
  return (int)std::min<int64_t>(b, kMostBlocks);
}

}  // namespace

size_t rotary_grad_workspace(int64_t tokens, int64_t heads, int32_t dim) {
  // the most blocks of either form: as many for each part, or kMostBlocks and one for each
  return tokens <= 0 || heads <= 0 ? 0 : (size_t)std::max(2 * grad_blocks(tokens, heads), kMostBlocks + 2) * dim * sizeof(float);
}

cudaError_t launch_rotary(lm_dtype dt, const RotaryParams& p, cudaStream_t st) {
  Deal d{};
  if (deal(p, dt, false, &d)) {
    const int64_t items = p.tokens * (d.chunks[0] + d.chunks[1]), groups = kThreads / d.lanes;
    const dim3 grid((unsigned)std::min<int64_t>((items + groups - 1) / groups, 152 * 32));
    using Kernel = void (*)(RotaryParams, Deal);
    const Kernel kernels[2][2] = {{rotary8_kernel<float, false>, rotary8_kernel<float, true>},
                                  {rotary8_kernel<__nv_bfloat16, false>, rotary8_kernel<__nv_bfloat16, true>}};
    return launch_after(kernels[dt == LM_F32 ? 0 : 1][p.interleaved ? 1 : 0], grid, kThreads, 0, st, p, d);
  }
  const int64_t rows = p.tokens * (p.part[0].heads + p.part[1].heads);
  const dim3 grid((unsigned)std::min<int64_t>((rows + kWarps - 1) / kWarps, 152 * 16));
  return launch_after(dt == LM_F32 ? rotary_kernel<float> : rotary_kernel<__nv_bfloat16>, grid, kThreads, 0, st, p);
}

cudaError_t launch_rotary_grad(lm_dtype dt, const RotaryParams& p, cudaStream_t st) {
  const bool dw = p.part[0].dweight != nullptr || p.part[1].dweight != nullptr;
  int first1 = 0, blocks[2] = {0, 0};
  Deal d{};
  if (p.tokens > 0 && p.part[0].heads + p.part[1].heads > 0) {
    cudaError_t e;
    if (deal(p, dt, true, &d)) {
      const int64_t groups = kThreads / d.lanes, most = kMostBlocks;
      const int64_t heads = p.part[0].heads + p.part[1].heads;
      for (int i = 0; i < 2; ++i) {
        const int64_t want = (p.tokens * d.chunks[i] + groups - 1) / groups, share = std::max<int64_t>(1, most * p.part[i].heads / heads);
        blocks[i] = (int)std::min(want, share);
      }
      first1 = blocks[0];
      using Kernel = void (*)(RotaryParams, Deal, int);
      const Kernel kernels[2][2] = {{rotary8_grad_kernel<float, false>, rotary8_grad_kernel<float, true>},
                                    {rotary8_grad_kernel<__nv_bfloat16, false>, rotary8_grad_kernel<__nv_bfloat16, true>}};
      e = launch_after(kernels[dt == LM_F32 ? 0 : 1][p.interleaved ? 1 : 0], dim3((unsigned)(blocks[0] + blocks[1])), kThreads,
                       dw ? (size_t)groups * p.dim * sizeof(float) : 0, st, p, d, blocks[0]);
    } else {
      blocks[0] = blocks[1] = first1 = grad_blocks(p.tokens, std::max(p.part[0].heads, p.part[1].heads));
      e = launch_after(dt == LM_F32 ? rotary_grad_kernel<float> : rotary_grad_kernel<__nv_bfloat16>, dim3((unsigned)first1, p.part[1].heads > 0 ? 2 : 1),
                       kThreads, dw ? (size_t)kWarps * p.dim * sizeof(float) : 0, st, p);
    }
    if (e != cudaSuccess) return e;
  }
  if (!dw) return cudaSuccess;
  return launch_after(rotary_join_kernel, dim3((unsigned)((p.dim + 31) / 32), 2), kThreads, 0, st, p, first1, blocks[0], blocks[1]);
}

}  // namespace lm
