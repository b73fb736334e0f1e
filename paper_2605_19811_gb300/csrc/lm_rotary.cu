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
// Bound by memory: 16384 tokens of 32 + 8 heads of 128, bf16, views of a QKV product:
// 61 us (5.6 TB/s), the gradient 104 us (4.9 TB/s), fp32 gradient of 4097 tokens of 20 +
// 20 heads of 80 34 us (4.7 TB/s).  What that took, at the first of these (245 us with a
// warp a head): no shuffles for the pairs and a token's angles in registers (134 us);
// the next heads' loads under way while these are worked on, packed fp32, and one wave
// of blocks shared between queries and keys by the steps that they take (61 us).  One
// token: 3 us, a call 20 us: host time.
// Heads of other sizes or alignments take a warp each, a pair or a channel a lane.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_train.h"
#include "lm_gemm_tc.cuh"

namespace lm {
namespace {

using gemm::add2;
using gemm::fma2;
using gemm::launch_after;
using gemm::mul2;
using tc::griddep_launch_dependents;
using tc::griddep_wait;

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kMostBlocks = 152 * 2;
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

// How heads fall to groups of lanes: `lanes` (a power of two) to a head, a part's
// `chunk` heads of a token to an item, one after another; blocks below q_blocks
// take the queries' items, the others the keys'.
struct Deal {
  int32_t lanes;
  int32_t chunk[2], chunks[2];   // heads of an item; items a token
  int32_t q_blocks;
};

// Four channels as they are read.
template <typename T> struct Piece;
template <> struct Piece<float> {
  float4 w;
  __device__ __forceinline__ void zero() { w = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) { w = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void get(float2& a, float2& b) const {
    a = make_float2(w.x, w.y);
    b = make_float2(w.z, w.w);
  }
  static __device__ __forceinline__ void store(float* p, float2 a, float2 b) { __stcs(reinterpret_cast<float4*>(p), make_float4(a.x, a.y, b.x, b.y)); }
};
template <> struct Piece<__nv_bfloat16> {
  uint2 w;
  __device__ __forceinline__ void zero() { w = make_uint2(0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void get(float2& a, float2& b) const {
    a = make_float2(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u));
    b = make_float2(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float2 a, float2 b) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(tc::pack_bf2(a.x, a.y), tc::pack_bf2(b.x, b.y)));
  }
};

// A lane's channels: pieces of four from a and b, as v[0], v[1] and v[2], v[3].
// Its four pairs are (v[0], v[2]) and (v[1], v[3]) element by element (halves),
// or the two elements of each v (interleaved).
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
    if (!in) pair = -1;
  }
  __device__ __forceinline__ void gains(const void* w, int dt, float2 (&v)[4]) const {
    const int at[4] = {a, a + 2, b, b + 2};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = in ? make_float2(gain(w, dt, at[k]), gain(w, dt, at[k] + 1)) : make_float2(1.f, 1.f);
  }
};
// Cosines and sines of a lane's four pairs.
template <bool kInterleaved>
struct Turns {
  float2 c[2], s[2];    // pairs 0, 1 and 2, 3
  __device__ __forceinline__ void load(const RotaryParams& p, const Lane<kInterleaved>& l, int64_t at) {
    c[0] = c[1] = make_float2(1.f, 1.f);
    s[0] = s[1] = make_float2(0.f, 0.f);
    if (l.pair < 0) return;
    const bool in = at >= 0 && at < p.table_rows;
    const float2* t = reinterpret_cast<const float2*>(p.table) + (in ? at : 0) * (p.turned >> 1) + l.pair;
    const float2 none = make_float2(__int_as_float(0x7FC00000), __int_as_float(0x7FC00000));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 v = in ? __ldg(t + k) : none;
      (k & 1 ? c[k >> 1].y : c[k >> 1].x) = v.x;
      (k & 1 ? s[k >> 1].y : s[k >> 1].x) = v.y;
    }
  }
  template <bool kBack>
  __device__ __forceinline__ void turn(float2 (&v)[4]) const {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (kInterleaved) {
        const float c0[2] = {c[k].x, c[k].y}, s0[2] = {kBack ? -s[k].x : s[k].x, kBack ? -s[k].y : s[k].y};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float2& x = v[2 * k + h];
          x = fma2(x, make_float2(c0[h], c0[h]), mul2(make_float2(x.y, x.x), make_float2(-s0[h], s0[h])));
        }
      } else {
        const float2 s0 = kBack ? make_float2(-s[k].x, -s[k].y) : s[k], s1 = make_float2(-s0.x, -s0.y), x = v[k], y = v[2 + k];
        v[k] = fma2(x, c[k], mul2(y, s1));
        v[2 + k] = fma2(y, c[k], mul2(x, s0));
      }
    }
  }
};
template <int kN>
__device__ __forceinline__ void group_sums(float (&v)[kN], int lanes) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    if (lanes <= o) continue;       // the same for all
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] += __shfl_xor_sync(kAll, v[k], o);
  }
}

// A group's way through its part's items, kAhead heads a step; the groups of a
// block take the same number of steps (those without heads among them).
template <int kAhead>
struct Walk {
  int64_t item, items, stride, token;
  int head, end, per, chunk, heads;
  __device__ __forceinline__ Walk(const RotaryParams& p, const Deal& d, int which, int block, int blocks) {
    const int groups = kThreads / d.lanes;
    per = d.chunks[which];
    chunk = d.chunk[which];
    heads = p.part[which].heads;
    items = p.tokens * per;
    stride = (int64_t)blocks * groups;
    item = (int64_t)block * groups + threadIdx.x / d.lanes;
    place();
  }
  __device__ __forceinline__ void place() {
    const int64_t i = min(item, items);
    token = items <= 0xFFFFFFFFll ? (int64_t)((uint32_t)i / (uint32_t)per) : i / per;
    head = (int)(i - token * per) * chunk;
    end = item < items ? min(head + chunk, heads) : head;
  }
};
// Steps of every group of a block.
__device__ __forceinline__ int64_t steps_of(int64_t items, int64_t stride, int block, int groups, int rounds) {
  const int64_t first = (int64_t)block * groups;
  return first < items ? (items - first + stride - 1) / stride * rounds : 0;
}

template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, 2) rotary8_kernel(const __grid_constant__ RotaryParams p, const __grid_constant__ Deal d) {
  constexpr int kAhead = 4;
  griddep_wait();
  griddep_launch_dependents();
  const int which = (int)blockIdx.x >= d.q_blocks ? 1 : 0;
  const RotaryPart& part = p.part[which];
  const int block = which ? blockIdx.x - d.q_blocks : blockIdx.x, blocks = which ? gridDim.x - d.q_blocks : d.q_blocks;
  const Lane<kInterleaved> l(p, threadIdx.x % d.lanes);
  Walk<kAhead> at(p, d, which, block, blocks);
  const int rounds = (at.chunk + kAhead - 1) / kAhead;
  const int64_t steps = steps_of(at.items, at.stride, block, kThreads / d.lanes, rounds);
  const float inv = 1.f / (float)p.dim;
  const int64_t ldx = part.x.ld_head, ldy = part.y.ld_head;
  const int gap = l.b - l.a;
  float2 w[4];
  if (p.norm) l.gains(part.weight, part.wdt, w);
  Turns<kInterleaved> t;
  Piece<T> raw[kAhead][2];
  int64_t position = 0;
  auto load = [&]() {
    const T* x = head_of<const T>(part.x, at.token, at.head) + l.a;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      raw[k][0].zero();
      raw[k][1].zero();
      if (l.in && at.head + k < at.end) {
        raw[k][0].load(x);
        raw[k][1].load(x + gap);
      }
      x += ldx;
    }
  };
  if (steps > 0) {
    load();
    if (l.pair >= 0 && at.head < at.end) position = p.positions[at.token];
  }
  int round = 0;
  for (int64_t n = 0; n < steps; ++n) {
    if (round == 0) t.load(p, l, position);
    float2 v[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      raw[k][0].get(v[k][0], v[k][1]);
      raw[k][1].get(v[k][2], v[k][3]);
    }
    T* y = head_of<T>(part.y, at.token, at.head) + l.a;
    const int left = l.in ? at.end - at.head : 0;
    // the next step's heads, before this one's are worked on
    at.head += kAhead;
    if (++round == rounds) {
      round = 0;
      at.item += at.stride;
      at.place();
      if (l.pair >= 0 && at.head < at.end) position = p.positions[at.token];
    }
    load();
    if (p.norm) {
      float q[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        float2 a = mul2(v[k][0], v[k][0]);
#pragma unroll
        for (int e = 1; e < 4; ++e) a = fma2(v[k][e], v[k][e], a);
        q[k] = a.x + a.y;
      }
      group_sums(q, d.lanes);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float rstd = rsqrtf(fmaf(q[k], inv, p.eps));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = mul2(mul2(v[k][e], make_float2(rstd, rstd)), w[e]);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      t.template turn<false>(v[k]);
      if (k < left) {
        Piece<T>::store(y, v[k][0], v[k][1]);
        Piece<T>::store(y + gap, v[k][2], v[k][3]);
      }
      y += ldy;
    }
  }
}

// Heads of a step, dy and x of each, and resident blocks: fp32 heads hold twice
// the registers of bf16 ones (4097 tokens, 40 heads of 80, fp32: 33 us with four
// and one block, 47 with two and two, which spill; bf16 16384 tokens, 40 heads of
// 128: 100 us with two and two, 108 with four and one).
template <typename T> constexpr int kGradAhead = sizeof(T) == 4 ? 4 : 2;
template <typename T> constexpr int kGradBlocks = sizeof(T) == 4 ? 1 : 2;
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, kGradBlocks<T>) rotary8_grad_kernel(const __grid_constant__ RotaryParams p, const __grid_constant__ Deal d) {
  extern __shared__ float sums[];     // groups x dim
  constexpr int kAhead = kGradAhead<T>;
  griddep_wait();
  griddep_launch_dependents();
  const int which = (int)blockIdx.x >= d.q_blocks ? 1 : 0, groups = kThreads / d.lanes;
  const RotaryPart& part = p.part[which];
  const int block = which ? blockIdx.x - d.q_blocks : blockIdx.x, blocks = which ? gridDim.x - d.q_blocks : d.q_blocks;
  const Lane<kInterleaved> l(p, threadIdx.x % d.lanes);
  Walk<kAhead> at(p, d, which, block, blocks);
  const int rounds = (at.chunk + kAhead - 1) / kAhead;
  const int64_t steps = steps_of(at.items, at.stride, block, groups, rounds);
  const float inv = 1.f / (float)p.dim;
  const int64_t ldx = part.x.ld_head, ldd = part.dy.ld_head, ldo = part.dx.ld_head;
  const int gap = l.b - l.a;
  float2 w[4], dw[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) dw[e] = make_float2(0.f, 0.f);
  if (p.norm) l.gains(part.weight, part.wdt, w);
  Turns<kInterleaved> t;
  Piece<T> rawd[kAhead][2], rawx[kAhead][2];
  int64_t position = 0;
  auto load = [&]() {
    const T* dy = head_of<const T>(part.dy, at.token, at.head) + l.a;
    const T* x = head_of<const T>(part.x, at.token, at.head) + l.a;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        rawd[k][h].zero();
        rawx[k][h].zero();
        if (l.in && at.head + k < at.end) {
          rawd[k][h].load(dy + h * gap);
          if (p.norm) rawx[k][h].load(x + h * gap);
        }
      }
      dy += ldd;
      x += ldx;
    }
  };
  if (steps > 0) {
    load();
    if (l.pair >= 0 && at.head < at.end) position = p.positions[at.token];
  }
  int round = 0;
  for (int64_t n = 0; n < steps; ++n) {
    if (round == 0) t.load(p, l, position);
    float2 v[kAhead][4], x[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      rawd[k][0].get(v[k][0], v[k][1]);
      rawd[k][1].get(v[k][2], v[k][3]);
      rawx[k][0].get(x[k][0], x[k][1]);
      rawx[k][1].get(x[k][2], x[k][3]);
    }
    T* dx = head_of<T>(part.dx, at.token, at.head) + l.a;
    const int left = l.in ? at.end - at.head : 0;
    at.head += kAhead;
    const bool turned_on = ++round == rounds;
    if (turned_on) {
      round = 0;
      at.item += at.stride;
      at.place();
      if (l.pair >= 0 && at.head < at.end) position = p.positions[at.token];
    }
    load();
#pragma unroll
    for (int k = 0; k < kAhead; ++k) t.template turn<true>(v[k]);
    if (p.norm) {
      float q[2 * kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        float2 a = make_float2(0.f, 0.f), b = a;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a = fma2(x[k][e], x[k][e], a);
          b = fma2(mul2(v[k][e], w[e]), x[k][e], b);
        }
        q[2 * k] = a.x + a.y;
        q[2 * k + 1] = b.x + b.y;
      }
      group_sums(q, d.lanes);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float rstd = rsqrtf(fmaf(q[2 * k], inv, p.eps)), mean = -q[2 * k + 1] * rstd * inv;
        const float2 r = make_float2(rstd, rstd), m = make_float2(mean, mean);
        // a head beyond the item's has v = 0, and x = 0 times a finite rstd unless eps is 0
        if (k >= left) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 xh = mul2(x[k][e], r);
          dw[e] = fma2(v[k][e], xh, dw[e]);
          v[k][e] = mul2(r, fma2(xh, m, mul2(v[k][e], w[e])));
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k < left) {
        Piece<T>::store(dx, v[k][0], v[k][1]);
        Piece<T>::store(dx + gap, v[k][2], v[k][3]);
      }
      dx += ldo;
    }
  }
  if (part.dweight == nullptr) return;
  if (l.in) {
    float* mine = sums + (threadIdx.x / d.lanes) * p.dim;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      mine[l.a + 2 * k] = dw[k].x;
      mine[l.a + 2 * k + 1] = dw[k].y;
      mine[l.b + 2 * k] = dw[2 + k].x;
      mine[l.b + 2 * k + 1] = dw[2 + k].y;
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < p.dim; c += kThreads) {
    float s = 0.f;
    for (int k = 0; k < groups; ++k) s += sums[k * p.dim + c];
    p.sums[(int64_t)blockIdx.x * p.dim + c] = s;
  }
}

bool pieces_of_four(const Heads& h, int size) {
  return reinterpret_cast<uintptr_t>(h.data) % (4 * size) == 0 && h.ld_token % 4 == 0 && h.ld_head % 4 == 0;
}
// Whether eight channels go to a lane, and how.
bool deal(const RotaryParams& p, lm_dtype dt, bool grad, Deal* d, int* k_blocks) {
  const int64_t most = grad && dt == LM_F32 ? kMostBlocks / 2 : kMostBlocks;     // one wave of blocks
  const int size = dt == LM_F32 ? 4 : 2;
  if (p.dim % 8 != 0 || p.dim > 256 || p.turned % 8 != 0 || reinterpret_cast<uintptr_t>(p.table) % 8 != 0) return false;
  for (const RotaryPart& r : p.part) {
    if (r.heads == 0) continue;
    if ((!grad || p.norm) && !pieces_of_four(r.x, size)) return false;
    if (!pieces_of_four(grad ? r.dy : r.y, size)) return false;
    if (grad && !pieces_of_four(r.dx, size)) return false;
  }
  d->lanes = 1;
  while (8 * d->lanes < p.dim) d->lanes *= 2;
  // as many heads to an item as leave every SM 32 warps of items, 16 at most,
  // and blocks to each part by the steps of four heads that its items take
  const int64_t all = (int64_t)152 * 32 * (32 / d->lanes), heads = p.part[0].heads + p.part[1].heads, groups = kThreads / d->lanes;
  const int64_t chunk = std::min<int64_t>(std::max<int64_t>(1, p.tokens * heads / all), 16);
  int64_t steps[2] = {0, 0};
  for (int i = 0; i < 2; ++i) {
    const int64_t n = p.part[i].heads, items = (n + chunk - 1) / chunk;
    if (n == 0) continue;
    d->chunk[i] = (int)((n + items - 1) / items);
    if (d->chunk[i] > 4) d->chunk[i] = (d->chunk[i] + 3) / 4 * 4;
    d->chunks[i] = (int)((n + d->chunk[i] - 1) / d->chunk[i]);
    steps[i] = (int64_t)d->chunks[i] * ((d->chunk[i] + 3) / 4);
  }
  int blocks[2];
  for (int i = 0; i < 2; ++i) {
    const int64_t want = (p.tokens * d->chunks[i] + groups - 1) / groups, share = std::max<int64_t>(1, most * steps[i] / (steps[0] + steps[1]));
    blocks[i] = (int)std::min(want, share);
  }
  d->q_blocks = blocks[0];
  *k_blocks = blocks[1];
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
  int k_blocks = 0;
  if (deal(p, dt, false, &d, &k_blocks)) {
    using Kernel = void (*)(RotaryParams, Deal);
    const Kernel kernels[2][2] = {{rotary8_kernel<float, false>, rotary8_kernel<float, true>},
                                  {rotary8_kernel<__nv_bfloat16, false>, rotary8_kernel<__nv_bfloat16, true>}};
    return launch_after(kernels[dt == LM_F32 ? 0 : 1][p.interleaved ? 1 : 0], dim3((unsigned)(d.q_blocks + k_blocks)), kThreads, 0, st, p, d);
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
    if (deal(p, dt, true, &d, &blocks[1])) {
      blocks[0] = first1 = d.q_blocks;
      using Kernel = void (*)(RotaryParams, Deal);
      const Kernel kernels[2][2] = {{rotary8_grad_kernel<float, false>, rotary8_grad_kernel<float, true>},
                                    {rotary8_grad_kernel<__nv_bfloat16, false>, rotary8_grad_kernel<__nv_bfloat16, true>}};
      e = launch_after(kernels[dt == LM_F32 ? 0 : 1][p.interleaved ? 1 : 0], dim3((unsigned)(blocks[0] + blocks[1])), kThreads,
                       dw ? (size_t)(kThreads / d.lanes) * p.dim * sizeof(float) : 0, st, p, d);
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
