// Token log probabilities, entropy, top alternatives and their gradient
// (formulas at lm_token_logprob_args in lionmuon.h).
//
// A row is read once, 16 bytes a load; each thread keeps a running maximum m
// with s = sum 2^d and t = sum 2^d d, d = (z - m) log2 e, and scales s and t
// when m grows:  s <- 2^a s,  t <- 2^a (t + a s),  a = (m_old - m) log2 e <= 0.
// d is one multiply-add z log2 e - c with c = m log2 e rounded once: c, not m,
// is the reference, so its rounding cancels (log p: 2.5e-6 off at most for logits
// around 0 and around 20000 alike).  With the row's M, C, S, T:
//   lse = M + ln2 (log2 S - (M log2 e - C)),  log p_j = ln2 (d_j - log2 S),  H = ln2 (log2 S - T / S)
// (M log2 e - C is exact, so lse is rounded once at its own size: for logits of
// 1000 to 1250 6.1e-5 off, half a unit, where ln2 (C + log2 S) was 1.1e-4 off.)
//   dz_j = 2^d_j (a0 + a1 d_j) (+ g_logp at the target),
//   a1 = -g_H ln2 / S,  a0 = (g_lse - g_logp - g_H (H - ln2 log2 S)) / S
// 2^d is the exponential unit's (2^-22 relative), and 0 below 2^-126: a token that
// much less likely than the most likely one has p = 0 (and its own log p).
// The gradient in the same call reads the row again, from L2, which its first
// reading asks to keep it and its second to give it up: 2432 x 50304 bf16 (245
// MB) then reads 270 MB from memory; an earlier form without the hints, 403 MB.
// Bound by memory: 16384 x 50304 bf16, forward 262 us (6.3 TB/s), with the
// gradient 552 us (6.0 TB/s read and written once), gradient alone 483 us (6.8
// TB/s).  Issue slots are 59% and the exponential unit 31% busy.  fp32 forward
// 2049 x 50257: 80 us (5.1 TB/s), with five alternatives 100 us.
//
// Values below -2^21 (masks: -inf, the type's lowest, -1e9 ..) are raised to it,
// which changes nothing in a row whose maximum is within +-1e6: p = 0 for both.
// A reference is then never large: at z = m, d is c's rounding error, which
// would itself be 100 and more for masks beyond 1e9 and overflow s and t of a
// thread that has met nothing else.  Rows beyond that take a plain loop with the
// differences z - m (it also sorts out rows of -inf, +inf and NaN).
//
// Few rows: a cluster of up to eight blocks takes a row and joins its parts
// through distributed shared memory, in order.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_train.h"
#include "lm_tc_ptx.cuh"

namespace lm {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -2097152.f;               // -2^21, a bf16 number: what smaller values are raised to
constexpr float kFar = 1e6f;                        // 2^((kLowest + kFar) log2 e) is 0
constexpr float kGone = -1e5f;                      // 2^kGone is 0
constexpr int kMaxCluster = 8;
constexpr int kCandidates = 1024;                   // of a block's alternatives

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// 16 bytes of a row: kWidth values raised to `low` (Low: what that compares
// with), and the largest of several as it is.
template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
  static constexpr int kWidth = 8;
  using Low = __nv_bfloat162;
  float2 v[4];
  static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  __device__ __forceinline__ Vec(uint4 u, Low low) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 h = __hmax2_nan(pair(w[k]), low);
      const uint32_t b = *reinterpret_cast<const uint32_t*>(&h);
      v[k] = make_float2(tc::bf_lo(b), tc::bf_hi(b));
    }
  }
  template <int kN>
  static __device__ __forceinline__ float most(const uint4 (&u)[kN]) {
    __nv_bfloat162 m = pair(u[0].x);
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      if (k > 0) m = __hmax2(m, pair(u[k].x));
      m = __hmax2(__hmax2(m, pair(u[k].y)), __hmax2(pair(u[k].z), pair(u[k].w)));
    }
    const uint32_t b = *reinterpret_cast<const uint32_t*>(&m);
    return fmaxf(tc::bf_lo(b), tc::bf_hi(b));
  }
  static __device__ __forceinline__ Low floor_of(float low) { return __bfloat162bfloat162(__float2bfloat16_rd(low)); }
};
template <> struct Vec<float> {
  static constexpr int kWidth = 4;
  using Low = float;
  float2 v[2];
  __device__ __forceinline__ Vec(uint4 u, Low low) {
    v[0] = make_float2(max_nan(__uint_as_float(u.x), low), max_nan(__uint_as_float(u.y), low));
    v[1] = make_float2(max_nan(__uint_as_float(u.z), low), max_nan(__uint_as_float(u.w), low));
  }
  template <int kN>
  static __device__ __forceinline__ float most(const uint4 (&u)[kN]) {
    float m = __uint_as_float(u[0].x);
#pragma unroll
    for (int k = 0; k < kN; ++k)
      m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(u[k].x)), fmaxf(__uint_as_float(u[k].y), __uint_as_float(u[k].z))), __uint_as_float(u[k].w));
    return m;
  }
  static __device__ __forceinline__ Low floor_of(float low) { return low; }
};

__device__ __forceinline__ float value(const __nv_bfloat16* p, int64_t i) { return __bfloat162float(p[i]); }
__device__ __forceinline__ float value(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ void put(__nv_bfloat16* p, int64_t i, float v) { p[i] = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, int64_t i, float v) { p[i] = v; }

// A value's place among the alternatives: the value's order above, the lower
// index first among equals (-0 counts as 0); 0 for a masked value.
__device__ __forceinline__ unsigned long long key_of(float x, int j) {
  if (!(x > -INFINITY)) return 0ull;
  const uint32_t u = __float_as_uint(x + 0.f);
  return ((unsigned long long)(u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u)) << 32) | (uint32_t)~j;
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)~(uint32_t)k; }

// How a row of `vocab` elements at z splits: `head` elements up to a 16-byte
// boundary, nvec whole vectors, a tail.  Elements of head and tail are single.
template <typename T>
struct RowSplit {
  int head, nvec, tail_at;
  __device__ __forceinline__ RowSplit(const T* z, int vocab) {
    constexpr int kW = 16 / (int)sizeof(T);
    head = min(vocab, (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(z) & 15u)) & 15u) / sizeof(T)));
    nvec = (vocab - head) / kW;
    tail_at = head + nvec * kW;
  }
};
// The part of a row that one block of its cluster takes.
template <typename T>
struct Part {
  int v0, v1;       // vectors
  bool single;      // this block also takes head and tail
  __device__ __forceinline__ Part(const RowSplit<T>& r, int rank, int blocks) {
    const int each = (r.nvec + blocks - 1) / blocks;
    v0 = min(r.nvec, rank * each);
    v1 = min(r.nvec, v0 + each);
    single = rank == 0;
  }
};

// Vectors a thread loads ahead, by what measured best with the gradient: bf16
// 16384 x 50304 four 557 us, six 564, eight 621; fp32 2049 x 50257 four 188 us,
// eight 162.  Two for 128 threads: 16384 x 2000 54 us, four 59 us.
template <typename T>
constexpr int ahead_of(int threads) { return threads == 128 ? 2 : sizeof(T) == 4 ? 8 : 4; }

struct Stats {
  float c, s;
  float t;
};
// The rounded product that is a reference; never fused into what is done with it.
__device__ __forceinline__ float reference(float m) { return __fmul_rn(m, kLog2e); }

// Sums of a thread: reference m with c = m log2 e.
struct Running {
  float m, c;
  float2 s, t;
  __device__ __forceinline__ void start() {
    m = kLowest;
    c = reference(kLowest);
    s = t = make_float2(0.f, 0.f);
  }
  __device__ __forceinline__ void raise(float to) {
    const float c2 = reference(to), a = fmaxf(c - c2, kGone), f = ex2(a);   // a s stays finite where 2^a is 0
    t = make_float2(f * (t.x + a * s.x), f * (t.y + a * s.y));
    s = make_float2(f * s.x, f * s.y);
    m = to;
    c = c2;
  }
  __device__ __forceinline__ void add(float2 x) {
    const float2 d = fma2(x, make_float2(kLog2e, kLog2e), make_float2(-c, -c));
    const float2 e = make_float2(ex2(d.x), ex2(d.y));
    s = add2(s, e);
    t = fma2(e, d, t);
  }
  __device__ __forceinline__ void add1(float x) {
    x = max_nan(x, kLowest);
    if (x > m) raise(x);
    const float d = fmaf(x, kLog2e, -c), e = ex2(d);
    s.x += e;
    t.x += e * d;
  }
};

template <int kThreads, bool kTop>
struct Shared {
  float join[3][kThreads / 32], red[2][kThreads / 32];
  Stats part[kMaxCluster];                    // of every block of the cluster
  float m_part[kMaxCluster];
};
template <int kThreads>
struct Shared<kThreads, true> : Shared<kThreads, false> {
  float group[kThreads / 4];                  // the largest value of every four threads
  float bound;
  int count;
  unsigned long long warp_best[kThreads / 32];
  unsigned long long cand[kCandidates];
  unsigned long long best[kMaxCluster * 32];  // block r's alternatives at 32 r (block 0 of the cluster)
};

template <int kThreads, typename F>
__device__ __forceinline__ float block_reduce(float v, float* part, F f) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) v = f(v, part[w]);
  return v;
}
struct Add {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// What a row's outputs are made of.  Far rows hold natural-log statistics with
// the maximum itself as reference (c = m, ls = log s, h = entropy).
struct Row {
  bool far, empty, bad;
  float c, ls, h, lse;
  Row() = default;
  __device__ __forceinline__ Row(float m, float c_, float s, float t) : far(false), empty(false), bad(false), c(c_) {
    ls = log2f(s);
    lse = fmaf(kLn2, ls - fmaf(m, kLog2e, -c), m);
    h = kLn2 * (ls - t / s);
  }
  __device__ __forceinline__ float logp(float z) const {
    if (bad) return __int_as_float(0x7FC00000);
    if (empty || z == -INFINITY) return -INFINITY;
    if (far) return (z - c) - ls;
    return fabsf(z) < kFar ? kLn2 * (fmaf(z, kLog2e, -c) - ls) : z - lse;
  }
};

// The plain form of a far row's statistics, by every block of its cluster.
template <typename T, int kThreads>
__device__ __noinline__ void far_row(const T* z, int vocab, float (*red)[kThreads / 32], Row& row) {
  float m = -INFINITY, bad = 0.f;
  for (int j = threadIdx.x; j < vocab; j += kThreads) {
    const float x = value(z, j);
    m = fmaxf(m, x);
    if (!(x < INFINITY)) bad = 1.f;   // NaN or +inf
  }
  __syncthreads();
  m = block_reduce<kThreads>(m, red[0], Max());
  bad = block_reduce<kThreads>(bad, red[1], Max());
  __syncthreads();
  row.far = true;
  row.bad = bad != 0.f;
  row.empty = !row.bad && m == -INFINITY;
  float s = 0.f, t = 0.f;
  if (!row.bad && !row.empty)
    for (int j = threadIdx.x; j < vocab; j += kThreads) {
      const float d = value(z, j) - m, e = expf(d);
      s += e;
      if (e > 0.f) t += e * d;
    }
  s = block_reduce<kThreads>(s, red[0], Add());
  t = block_reduce<kThreads>(t, red[1], Add());
  __syncthreads();
  const float nan = __int_as_float(0x7FC00000);
  row.c = m;
  row.ls = logf(s);
  row.h = row.bad ? nan : row.empty ? 0.f : row.ls - t / s;
  row.lse = row.bad ? nan : row.empty ? -INFINITY : m + row.ls;
}

// 16 bytes past L1, and how L2 is to treat them: kept in preference to what
// streams through it (they are read again soon), given up first, or neither.
enum L2Use { kKeep, kGiveUp, kNeither };
template <L2Use kUse>
__device__ __forceinline__ uint64_t l2_policy() {
  uint64_t p;
  if (kUse == kKeep) asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  else if (kUse == kGiveUp) asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  else asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint4 load_with(const uint4* at, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(at), "l"(policy));
  return v;
}

// Every kThreads-th vector of [0, n), a batch of kBatch loaded ahead of the one
// at work.  f takes an array of vectors, kThreads apart, and the first one's
// place: kBatch of them, or one where the batch passes the end.
template <int kThreads, int kBatch, typename F>
__device__ __forceinline__ void walk(const uint4* src, int n, uint64_t policy, F f) {
  uint4 ahead[kBatch];
  int v = (int)threadIdx.x;
#pragma unroll
  for (int k = 0; k < kBatch; ++k)
    if (v + k * kThreads < n) ahead[k] = load_with(src + v + k * kThreads, policy);
  for (; v < n; v += kBatch * kThreads) {
    uint4 now[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      now[k] = ahead[k];
      if (v + (kBatch + k) * kThreads < n) ahead[k] = load_with(src + v + (kBatch + k) * kThreads, policy);
    }
    if (v + (kBatch - 1) * kThreads < n) {
      f(now, v);
    } else {
#pragma unroll
      for (int k = 0; k < kBatch - 1; ++k)
        if (v + k * kThreads < n) {
          const uint4 one[1] = {now[k]};
          f(one, v + k * kThreads);
        }
    }
  }
}

// What a row's end needs, asked for at its start: its target and the loss's weights.
struct RowArgs {
  int64_t y;
  float gl, gh, gz;
  bool weighed;           // log p is in the loss
  __device__ __forceinline__ RowArgs(const LogprobParams& p, int64_t row_i, bool grad) : gl(0.f), gh(0.f), gz(0.f), weighed(p.g_logp != nullptr) {
    y = p.targets != nullptr ? p.targets[row_i] : -1;
    if (!grad) return;
    if (p.g_logp != nullptr) gl = p.g_logp[row_i];
    if (p.g_entropy != nullptr) gh = p.g_entropy[row_i];
    if (p.g_lse != nullptr) gz = p.g_lse[row_i];
  }
  // the weight of log p_y: 0 without a target or weights, NaN for a target beyond the vocabulary
  __device__ __forceinline__ float weight(int vocab) const { return y < 0 || !weighed ? 0.f : y >= vocab ? __int_as_float(0x7FC00000) : gl; }
};

// A row's gradient, value by value: p_j (a + b lp) with p_j = 2^(d - ls), and
// g_logp more at the target.
template <typename T>
struct Slope {
  static constexpr int kW = Vec<T>::kWidth;
  float c, a0, a1, gl, floor;
  int y, vy, ey;                                  // the target, its vector and its place there (-1: none)
  typename Vec<T>::Low low;
  __device__ __forceinline__ Slope(const Row& row, float h, float gl_, float gh, float gz, int64_t target, const RowSplit<T>& split) {
    const float is = ex2(-row.ls);
    c = row.c;
    a1 = -gh * kLn2 * is;
    a0 = (gz - gl_ - gh * (h - kLn2 * row.ls)) * is;
    gl = gl_;
    // values with p = 0 are raised to where p is still 0 and a1 d no infinity
    floor = (c - 2000.f) * kLn2;
    low = Vec<T>::floor_of(floor);
    y = (int)target;
    const bool in = target >= split.head && target < split.tail_at;
    vy = in ? (y - split.head) / kW : -1;
    ey = in ? (y - split.head) % kW : -1;
  }
  __device__ __forceinline__ float single(float z, int j) const {
    const float d = fmaf(fmaxf(z, floor), kLog2e, -c);
    return ex2(d) * fmaf(a1, d, a0) + (j == y ? gl : 0.f);
  }
  __device__ __forceinline__ void vector(uint4 raw, int v, T* dst, bool together) const {
    Vec<T> x(raw, low);
#pragma unroll
    for (int e = 0; e < kW / 2; ++e) {
      const float2 d = fma2(x.v[e], make_float2(kLog2e, kLog2e), make_float2(-c, -c));
      x.v[e] = mul2(make_float2(ex2(d.x), ex2(d.y)), fma2(make_float2(a1, a1), d, make_float2(a0, a0)));
    }
    if (v == vy) {
#pragma unroll
      for (int e = 0; e < kW / 2; ++e) {
        if (ey == 2 * e) x.v[e].x += gl;
        if (ey == 2 * e + 1) x.v[e].y += gl;
      }
    }
    uint4 out;
    if constexpr (sizeof(T) == 2)
      out = make_uint4(tc::pack_bf2(x.v[0].x, x.v[0].y), tc::pack_bf2(x.v[1].x, x.v[1].y), tc::pack_bf2(x.v[2].x, x.v[2].y), tc::pack_bf2(x.v[3].x, x.v[3].y));
    else
      out = make_uint4(__float_as_uint(x.v[0].x), __float_as_uint(x.v[0].y), __float_as_uint(x.v[1].x), __float_as_uint(x.v[1].y));
    if (together) {
      __stcs(reinterpret_cast<uint4*>(dst) + v, out);
    } else {
      const T* o = reinterpret_cast<const T*>(&out);
#pragma unroll
      for (int e = 0; e < kW; ++e) dst[(int64_t)v * kW + e] = o[e];
    }
  }
};

// Gradient of the part of a row that this block takes.
template <typename T, int kThreads, L2Use kUse>
__device__ __forceinline__ void gradient(const LogprobParams& p, int64_t row_i, const T* z, const RowSplit<T>& split, const Part<T>& part,
                                         const Row& row, float h, const RowArgs& args) {
  constexpr int kW = Vec<T>::kWidth;
  T* d = static_cast<T*>(p.dlogits) + row_i * p.ld_d;
  const int64_t y = args.y;
  const float gl = args.weight(p.vocab), gh = args.gh, gz = args.gz;
  const bool together = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;   // d's vectors lie as z's
  if (row.bad || row.empty || row.far || gl != gl) {
    const float fill = row.empty && gl == gl ? 0.f : __int_as_float(0x7FC00000);
    const int j0 = part.single ? 0 : split.head + part.v0 * kW;
    auto one = [&](int j) {
      float g = fill;
      if (row.far && !row.bad && !row.empty && gl == gl) {
        const float lp = (value(z, j) - row.c) - row.ls, e = expf(lp);
        g = (e > 0.f ? e * (gz - gl - gh * (lp + h)) : 0.f) + (j == y ? gl : 0.f);
      }
      put(d, j, g);
    };
    for (int j = j0 + threadIdx.x; j < split.head + part.v1 * kW; j += kThreads) one(j);
    if (part.single)
      for (int j = split.tail_at + threadIdx.x; j < p.vocab; j += kThreads) one(j);
    return;
  }
  const Slope<T> g(row, h, gl, gh, gz, y, split);
  auto single = [&](int j) { put(d, j, g.single(value(z, j), j)); };
  if (part.single) {
    for (int j = threadIdx.x; j < split.head; j += kThreads) single(j);
    for (int j = split.tail_at + threadIdx.x; j < p.vocab; j += kThreads) single(j);
  }
  T* dst = d + split.head;
  walk<kThreads, ahead_of<T>(kThreads)>(reinterpret_cast<const uint4*>(z + split.head) + part.v0, part.v1 - part.v0, l2_policy<kUse>(), [&](const auto& raw, int i) {
    constexpr int kN = sizeof(raw) / sizeof(raw[0]);
#pragma unroll
    for (int k = 0; k < kN; ++k) g.vector(raw[k], part.v0 + i + k * kThreads, dst, together);
  });
}

// This block's top_k alternatives, best first, into out (shared memory; 0 for
// none).  best: the largest of this thread's elements (whole: not known).  The
// top_k-th largest of the maxima of groups of four threads bounds the answer
// from below; only threads whose own maximum reaches the bound can hold more
// of it, and their warps look through their elements again, a vector a lane.
template <typename T, int kThreads>
__device__ void block_top(Shared<kThreads, true>& sh, const T* z, int vocab, int top_k, const RowSplit<T>& split, const Part<T>& part,
                          float best, bool whole, unsigned long long* out) {
  constexpr int kW = Vec<T>::kWidth, kGroups = kThreads / 4;
  float g = best;
  g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, 1));
  g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, 2));
  if ((threadIdx.x & 3) == 0) sh.group[threadIdx.x >> 2] = g;
  if (threadIdx.x == 0) {
    sh.bound = -INFINITY;   // fewer than top_k groups hold anything: every element counts
    sh.count = 0;
  }
  if (threadIdx.x < 32) out[threadIdx.x] = 0ull;
  __syncthreads();
  if (threadIdx.x < kGroups) {
    const float own = sh.group[threadIdx.x];
    int above = 0;
#pragma unroll 8
    for (int i = 0; i < kGroups; ++i) {
      const float o = sh.group[i];
      above += (o > own || (o == own && i < (int)threadIdx.x)) ? 1 : 0;
    }
    if (above == top_k - 1) sh.bound = own;
  }
  __syncthreads();
  const float bound = sh.bound;
  auto look = [&](float x, int j) {
    if (x >= bound && x > -INFINITY) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kCandidates) sh.cand[at] = key_of(x, j);
    }
  };
  const bool hot = !whole && best >= bound && best > -INFINITY;
  if (hot && part.single) {
    for (int j = threadIdx.x; j < split.head; j += kThreads) look(value(z, j), j);
    for (int j = split.tail_at + threadIdx.x; j < vocab; j += kThreads) look(value(z, j), j);
  }
  const uint4* src = reinterpret_cast<const uint4*>(z + split.head);
  for (unsigned todo = __ballot_sync(0xFFFFFFFFu, hot); todo != 0u; todo &= todo - 1u) {
    const int thread = (int)(threadIdx.x & ~31u) + __ffs(todo) - 1;
    for (int v = part.v0 + thread + (int)(threadIdx.x & 31) * kThreads; v < part.v1; v += 32 * kThreads) {
      const uint4 raw[1] = {src[v]};
      if (!(Vec<T>::most(raw) >= bound)) continue;
      const T* e = reinterpret_cast<const T*>(raw);
#pragma unroll
      for (int k = 0; k < kW; ++k) look(value(e, k), split.head + v * kW + k);
    }
  }
  __syncthreads();
  const int n = sh.count;
  if (n <= kCandidates && !whole) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const unsigned long long own = sh.cand[i];
      int above = 0;
      for (int k = 0; k < n && above < top_k; ++k) above += sh.cand[k] > own ? 1 : 0;
      if (above < top_k) out[above] = own;   // keys differ: one each place
    }
    __syncthreads();
    return;
  }
  // Too many elements above the bound (all in a few threads): one after another.
  unsigned long long last = ~0ull;
  for (int k = 0; k < top_k; ++k) {
    unsigned long long best = 0ull;
    auto look = [&](int j) {
      const unsigned long long x = key_of(value(z, j), j);
      if (x < last && x > best) best = x;
    };
    for (int j = split.head + part.v0 * kW + threadIdx.x; j < split.head + part.v1 * kW; j += kThreads) look(j);
    if (part.single) {
      for (int j = threadIdx.x; j < split.head; j += kThreads) look(j);
      for (int j = split.tail_at + threadIdx.x; j < vocab; j += kThreads) look(j);
    }
    for (int o = 16; o; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xFFFFFFFFu, best, o);
      best = best > other ? best : other;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.warp_best[threadIdx.x >> 5] = best;
    __syncthreads();
    best = 0ull;
    for (int w = 0; w < kThreads / 32; ++w) best = sh.warp_best[w] > best ? sh.warp_best[w] : best;
    if (threadIdx.x == 0) out[k] = best;
    last = best;
  }
  __syncthreads();
}

__device__ __forceinline__ void put_stats(const LogprobParams& p, int64_t row_i, int64_t y, float zy, const Row& row) {
  if (p.lse != nullptr) p.lse[row_i] = row.lse;
  if (p.entropy != nullptr) p.entropy[row_i] = row.h;
  if (p.logp != nullptr) p.logp[row_i] = (row.bad || y >= p.vocab) ? __int_as_float(0x7FC00000) : y < 0 ? 0.f : row.logp(zy);
}
__device__ __forceinline__ void put_top(const LogprobParams& p, int64_t row_i, int k, unsigned long long key, const Row& row) {
  const bool has = key != 0ull && !row.bad;
  p.top_index[row_i * p.top_k + k] = has ? key_index(key) : -1;
  p.top_logp[row_i * p.top_k + k] = row.bad ? __int_as_float(0x7FC00000) : has ? row.logp(key_value(key)) : -INFINITY;
}

// Stores into the shared memory of block `rank` of the cluster.
__device__ __forceinline__ uint32_t of_block(const void* p, int rank) { return tc::peer_addr(p, (uint32_t)rank); }
__device__ __forceinline__ void store_block(float* p, int rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(of_block(p, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void store_block(unsigned long long* p, int rank, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(of_block(p, rank)), "l"(v) : "memory");
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// kTop: with alternatives.  kCluster: several blocks a row.
template <typename T, int kThreads, bool kTop, bool kCluster>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const LogprobParams p) {
  constexpr int kW = Vec<T>::kWidth;
  __shared__ Shared<kThreads, kTop> sh;
  const int blocks = kCluster ? p.cluster : 1;
  const int rank = kCluster ? (int)tc::cluster_rank() : 0;
  const int64_t row_i = kCluster ? blockIdx.x / p.cluster : blockIdx.x;
  if (kCluster) cluster_arrive();   // waited for before another block's memory is written: it has started then
  const T* z = static_cast<const T*>(p.logits) + row_i * p.ld;
  const RowSplit<T> split(z, p.vocab);
  const Part<T> part(split, rank, blocks);
  const int n = part.v1 - part.v0;
  const uint4* src = reinterpret_cast<const uint4*>(z + split.head) + part.v0;
  const RowArgs args(p, row_i, p.dlogits != nullptr);
  const int64_t y = args.y;

  Running r;
  r.start();
  const auto low = Vec<T>::floor_of(kLowest);
  float best = -INFINITY;   // the thread's largest value
  if (part.single) {
    for (int j = threadIdx.x; j < split.head; j += kThreads) {
      const float x = value(z, j);
      r.add1(x);
      if (kTop) best = fmaxf(best, x);
    }
  }
  walk<kThreads, ahead_of<T>(kThreads)>(src, n, p.dlogits != nullptr ? l2_policy<kKeep>() : l2_policy<kGiveUp>(), [&](const auto& raw, int i) {
    constexpr int kN = sizeof(raw) / sizeof(raw[0]);
    const float most = Vec<T>::most(raw);
    if (most > r.m) r.raise(most);
    if (kTop) best = fmaxf(best, most);
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const Vec<T> x(raw[k], low);
#pragma unroll
      for (int e = 0; e < kW / 2; ++e) r.add(x.v[e]);
    }
  });
  if (part.single) {
    for (int j = split.tail_at + threadIdx.x; j < p.vocab; j += kThreads) {
      const float x = value(z, j);
      r.add1(x);
      if (kTop) best = fmaxf(best, x);
    }
  }
  // the target's logit, before a gradient may be written over it
  const float zy = (threadIdx.x == 0 && y >= 0 && y < p.vocab) ? value(z, y) : 0.f;
  // Joined over the warp, the block (every warp joins the warps' sums for itself)
  // and the cluster; s is NaN where a NaN or +inf was.
  constexpr int kWarps = kThreads / 32;
  float m = r.m;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  r.raise(m);
  float s = r.s.x + r.s.y, t = r.t.x + r.t.y;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
  }
  if ((threadIdx.x & 31) == 0) {
    sh.join[0][threadIdx.x >> 5] = m;
    sh.join[1][threadIdx.x >> 5] = s;
    sh.join[2][threadIdx.x >> 5] = t;
  }
  __syncthreads();
  m = sh.join[0][threadIdx.x & (kWarps - 1)];
  s = sh.join[1][threadIdx.x & (kWarps - 1)];
  t = sh.join[2][threadIdx.x & (kWarps - 1)];
  float mm = m;
#pragma unroll
  for (int o = kWarps / 2; o; o >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xFFFFFFFFu, mm, o));
  float c = reference(mm);
  {
    const float a = fmaxf(reference(m) - c, kGone), f = ex2(a);
    t = f * (t + a * s);
    s = f * s;
  }
#pragma unroll
  for (int o = kWarps / 2; o; o >>= 1) {
    s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
  }
  if (kCluster) {
    cluster_wait();
    if (threadIdx.x < blocks) {
      store_block(&sh.m_part[rank], threadIdx.x, mm);
      store_block(&sh.part[rank].c, threadIdx.x, c);
      store_block(&sh.part[rank].s, threadIdx.x, s);
      store_block(&sh.part[rank].t, threadIdx.x, t);
    }
    tc::cluster_sync();
    for (int b = 0; b < blocks; ++b) mm = fmaxf(mm, sh.m_part[b]);
    c = reference(mm);
    s = t = 0.f;
    for (int b = 0; b < blocks; ++b) {
      const float a = fmaxf(sh.part[b].c - c, kGone), f = ex2(a);
      t += f * (sh.part[b].t + a * sh.part[b].s);
      s += f * sh.part[b].s;
    }
  }
  Row row(mm, c, s, t);
  if (!(s < INFINITY) || !(fabsf(mm) < kFar)) far_row<T, kThreads>(z, p.vocab, sh.red, row);

  if (rank == 0 && threadIdx.x == 0) put_stats(p, row_i, y, zy, row);
  if constexpr (kTop) {
    unsigned long long* out = sh.best + 32 * rank;
    block_top<T, kThreads>(sh, z, p.vocab, p.top_k, split, part, best, row.far, out);
    if (kCluster) {
      if (rank != 0 && threadIdx.x < 32) store_block(&sh.best[32 * rank + threadIdx.x], 0, out[threadIdx.x]);
      tc::cluster_sync();
      if (rank == 0) {
        for (int i = threadIdx.x; i < 32 * blocks; i += kThreads) {
          const unsigned long long own = sh.best[i];
          int above = 0;
          for (int k = 0; k < 32 * blocks; ++k) above += sh.best[k] > own ? 1 : 0;
          if (own != 0ull && above < p.top_k) sh.cand[above] = own;
        }
        __syncthreads();
        out = sh.cand;
      }
    }
    if (rank == 0) {
      // how many places are filled: all, unless the row holds fewer values
      int filled = p.top_k;
      if (kCluster) {
        filled = 0;
        for (int i = 0; i < 32 * blocks; ++i) filled += sh.best[i] != 0ull ? 1 : 0;
      }
      for (int k = threadIdx.x; k < p.top_k; k += kThreads) put_top(p, row_i, k, k < filled ? out[k] : 0ull, row);
    }
  }
  if (p.dlogits != nullptr) {
    if (kCluster && row.far) tc::cluster_sync();   // every block has read the whole row; it may be written over now
    if (!kCluster) __syncthreads();
    gradient<T, kThreads, kGiveUp>(p, row_i, z, split, part, row, row.h, args);
  }
  if (kCluster) tc::cluster_sync();   // no block leaves while another may write into it
}

template <typename T, int kThreads, bool kCluster>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(const LogprobParams p) {
  __shared__ float red[2][kThreads / 32];
  const int rank = kCluster ? (int)(blockIdx.x % p.cluster) : 0;
  const int64_t row_i = kCluster ? blockIdx.x / p.cluster : blockIdx.x;
  const T* z = static_cast<const T*>(p.logits) + row_i * p.ld;
  const RowSplit<T> split(z, p.vocab);
  const Part<T> part(split, rank, kCluster ? p.cluster : 1);
  const RowArgs args(p, row_i, true);
  const float lse = p.lse[row_i], h = p.g_entropy != nullptr ? p.entropy[row_i] : 0.f;
  Row row;
  row.bad = !(lse < INFINITY);
  row.empty = lse == -INFINITY;
  row.far = false;
  row.c = lse * kLog2e;
  row.ls = 0.f;
  // lse alone gives p to 2^-24 |lse| relative; beyond 4096 the row's sums are
  // formed anew (the launch then gives such rows to one block)
  if (!row.bad && !row.empty && fabsf(lse) > 4096.f) far_row<T, kThreads>(z, p.vocab, red, row);
  gradient<T, kThreads, kNeither>(p, row_i, z, split, part, row, h, args);
}

// Vectors of a row up to which 128 threads take it, else 256: 16384 x 2000 bf16
// with the gradient 54 us with 128 threads, 99 with 256; 16384 x 5000 bf16
// gradient alone 61 and 82; 16384 x 50304 with the gradient 757 and 717 us
// (both before the later steps).
constexpr int kShort = 2500;

// Blocks a row: as many, up to eight, as give every SM a block and leave each
// thread a vector.  V 50304 bf16, forward: 1 row 8 us with a cluster, 10 without;
// 200 rows 17 us with clusters up to three blocks an SM, 12 without; gradient of
// 64 rows 8 us with, 12 without.
int cluster_for(int64_t rows, int64_t vectors, int threads) {
  int c = 1;
  while (c < kMaxCluster && rows * c < 152 && vectors / (2 * c) >= threads) c *= 2;
  return c;
}

template <typename Kernel>
cudaError_t start(Kernel kernel, int threads, const LogprobParams& p, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.rows * p.cluster), 1, 1);
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster > 1 ? 1 : 0;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T, int kThreads>
cudaError_t forward(const LogprobParams& p, cudaStream_t st) {
  if (p.cluster > 1)
    return p.top_k > 0 ? start(logprob_kernel<T, kThreads, true, true>, kThreads, p, st) : start(logprob_kernel<T, kThreads, false, true>, kThreads, p, st);
  return p.top_k > 0 ? start(logprob_kernel<T, kThreads, true, false>, kThreads, p, st) : start(logprob_kernel<T, kThreads, false, false>, kThreads, p, st);
}
template <typename T>
cudaError_t launch(LogprobParams p, bool gradient_only, cudaStream_t st) {
  const int64_t vectors = p.vocab / Vec<T>::kWidth;
  const int threads = vectors <= kShort ? 128 : 256;
  if (gradient_only) {
    p.cluster = p.dlogits == p.logits ? 1 : cluster_for(p.rows, vectors, threads);   // a far row is read whole by each of its blocks, before any writes
    if (threads == 128)
      return p.cluster > 1 ? start(logprob_grad_kernel<T, 128, true>, 128, p, st) : start(logprob_grad_kernel<T, 128, false>, 128, p, st);
    return p.cluster > 1 ? start(logprob_grad_kernel<T, 256, true>, 256, p, st) : start(logprob_grad_kernel<T, 256, false>, 256, p, st);
  }
  p.cluster = cluster_for(p.rows, vectors, threads);
  return threads == 128 ? forward<T, 128>(p, st) : forward<T, 256>(p, st);
}

}  // namespace

cudaError_t launch_logprob(lm_dtype dt, const LogprobParams& p, cudaStream_t st) {
  return dt == LM_BF16 ? launch<__nv_bfloat16>(p, false, st) : launch<float>(p, false, st);
}
cudaError_t launch_logprob_grad(lm_dtype dt, const LogprobParams& p, cudaStream_t st) {
  return dt == LM_BF16 ? launch<__nv_bfloat16>(p, true, st) : launch<float>(p, true, st);
}

}  // namespace lm
