// Log probabilities of given tokens from the last hidden states and the head's
// matrix, and the gradients of a loss over them, without the logits (formulas at
// lm_linear_logprob_args in lionmuon.h).
//
// Forward: the product z = h W^T tile by tile; a tile's epilogue keeps, for its
// rows, the maximum m, s = sum e^(z - m) and t = sum e^(z - m) (z - m), from tile to
// tile of a strip, and the target's z where the tile holds it.  A second kernel
// joins a row's parts:
//   lse = M + log S,  logp = (z_y - M) - log S,  H = log S - T / S.
// The tensor cores sum 256 products of a logit at a time (128 for few rows), half as
// many as elsewhere: the epilogue has the time, and log p is then as exact as plain
// fp32's (rows of 4096: 9e-8 off, 1.8e-7 with 512; one token of 768, whose target's
// products have one sign: 7e-8 in the median of 40, 6e-7 at most, and 2e-6).
//
// Gradients, for a piece of the tokens at a time.  In the forward call the
// product's epilogue also leaves every logit in the workspace in 16 bits, as
// its distance below the row's running maximum r in steps of 2^-10,
//   q = rint((r - z) 2^10),  65535 and more (64 below): p = 0
// (p is then off by 2^-11 of itself at most, a quarter of the bf16 rounding that
// follows).  Once M and S are known, a kernel makes of q, in its place,
//   d = p (a - g_H (log p + H)) (+ g_logp at the target),  a = g_lse - g_logp
// as bf16 (the rounding that the tensor cores ask for; times a scale, see put_scale),
// and two products of it follow, dh = d W and dW = d^T h.  Where lse comes from an earlier call the
// logits' product writes d itself.  Over several pieces dW is summed in fp32, each
// piece's tiles added by the TMA.
//
// q and d lie in blocks of 64 columns, so that a box of either product is one
// piece of memory.
//
// Why 16-bit logits and not the logits' product a second time: 2 bytes written, 2
// read and 2 written again take 0.9 ns a thousand logits, the product 1.2 ns a
// thousand logits for each thousand of the width; and why pieces of tokens and not
// of the vocabulary: dh needs no sums of its own and dW's are added once a piece.
// (16384 x 768 x 50304: 5554 us with the product twice and d written element by
// element, 4035 us so.)
//
// Measured: 16384 x 768 x 50304 with both gradients 3.42 ms (each product of 0.32
// TFLOP a piece: logits 233 us, dh 205, dW 205; d 145 us at 5.7 TB/s), 4096 x 4096 x
// 50257 3.47 ms (logits 941 us, 1.79 PFLOP/s; dh 968, dW 974, 1.74), the latter under
// the power limit (by itself 3.05).  The products are bound by what the SMs take from
// L2 (64 bytes a cycle for each: 512 cycles of MMAs for 64 of the sum take 640); the
// logits' at a width of 768 also by their epilogue and the 16-bit logits' way out
// (181 us without either).  One token, 768 x 50304: 20 us of kernels (77 MB), 27
// to 29 us a call: host time.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_gemm_tc.cuh"
#include "lm_rows.cuh"

namespace lm {
namespace {

using namespace gemm;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGone = -1e4f;      // e^kGone is 0
constexpr float kOutside = -INFINITY;
constexpr int kForwardUnits = 16 * kPairs, kLeastStrips = 8;   // of the forward product (forward_strip)
constexpr int64_t kPieceBytes = (int64_t)512 << 20;   // of the gradient's bf16 values in the workspace
constexpr int64_t kLeastPiece = 1024;                 // tokens
constexpr float kSteps = 1024.f;                      // of q

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the reference of a maximum: -inf (nothing there) counts from 0
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// 2^23 + q holds q in its low bits
constexpr float kWhole = 8388608.f;
__device__ __forceinline__ uint32_t two_q(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410); }

// The warp's two boxes (64 columns each) to their blocks.
template <typename P>
__device__ __forceinline__ void store_boxes(const P& p, const Place& at) {
  box_ready();
  if (at.lane != 0 || at.row >= p.m) return;
  if (at.col < p.n) box_store(&p.out, at.box, 0, at.row, at.col / 64);
  if (at.col + 64 < p.n) box_store(&p.out, at.box + kBoxBytes, 0, at.row, at.col / 64 + 1);
  bulk_commit();
}

// What a row's gradient takes: lse, a = g_lse - g_logp, g_H, H.  In the call that computes
// them, M in the place of lse, and log S beside it: log p = (z - M) - log S then lacks
// lse's rounding at its own size, which is all that is left of the dz of a target with p
// near 1 (1 - p = 2e-5 with lse = 52: such a token's dh 6% off, 0.6% so).
struct RowTerms {
  float4* terms;
  float* log_s;       // NULL: terms hold lse
  float* g_logp;      // 0 in a row without a target
  int32_t* target;    // -1 in a row without one
  float* scale;       // d = scale[0] dz is rounded, and scale[1] = 1 / scale[0] times the products
};

// The rounding of d to bf16 costs 2^-8 of values just above a power of two, half of
// that just below the next one.  Where the tokens count alike, the targets' dz, which
// carry most of the gradient, are g_logp times what is left to 1, and lie together:
// the scale puts the largest g_logp of the piece's first 32 tokens (`g`: one a lane of
// `lanes`) on 127/64 of a power of two.  Weights of -1 / tokens, 1000 tokens: both
// gradients are 1.17 times as far off as by their own rounding alone instead of 1.33
// (100 tokens: 1.17 instead of 1.46).  It takes nothing of the logits, so that one
// token's never change another's gradient.
__device__ __forceinline__ void put_scale(float* scale, unsigned lanes, float g) {
  const uint32_t most = __reduce_max_sync(lanes, __float_as_uint(fabsf(g)));
  if ((threadIdx.x & 31) != 0) return;
  float s = 1.f;
  if (most >= 0x00800000u && most < 0x7F800000u) s = (127.f / 64.f) / __uint_as_float((most & 0x007FFFFFu) | 0x3F800000u);
  scale[0] = s;
  scale[1] = 1.f / s;
}

// kKeep: the logits are kept in 16 bits for the gradient.  kFew: at most kFewRows
// rows, without it; W's bytes are then all that counts, and more of them are under
// way.
constexpr int kFewRows = 32;
template <bool kKeep, bool kFew>
struct ForwardEpi {
  static constexpr int kStages = kKeep ? 5 : kFew ? 10 : 6, kBoxes = kKeep ? 2 : 0, kRowsA = kFew ? kFewRows : kHalf;
  static constexpr int kFewRegs = 120;             // (fewest spills)
  static constexpr int kChunk = kFew ? 2 : 4;      // blocks of a logit's sum in one accumulator: 128 products, or 256
  float* from;          // kKeep: r of each half tile's rows, (2 tiles_n) x rows
  const int64_t* targets;
  float *m, *s, *t;     // (2 strips) x rows
  float* z_target;
  int64_t rows;
  template <typename P>
  struct Warp {
    float m, s, t;
    int tm, y;      // y: the row's target, -1 for none inside the vocabulary
    __device__ __forceinline__ Warp(const P&, const Place&) : m(-INFINITY), s(0.f), t(0.f), tm(-1), y(-1) {}
    __device__ __forceinline__ void tile(const P& p, const Item& it, const Place& at, float (&acc)[4][32]) {
      const int row = at.row + at.lane;
      const bool in = row < p.m;
      if (tm != at.tm) {
        tm = at.tm;
        const int64_t target = in && p.epi.targets != nullptr ? p.epi.targets[row] : -1;
        y = target < p.n ? (int)target : -1;
        if (target < 0) y = -1;
      }
      const int left = p.n - at.col;      // columns of the vocabulary from this warp's first
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if ((unsigned)(y - at.col - 32 * b) < 32u && y >= 0) {
          float z = 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) z = y - at.col == 32 * b + e ? acc[b][e] : z;
          p.epi.z_target[row] = z;
        }
      if (left < 128) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = 32 * b + e < left ? acc[b][e] : kOutside;
      }
      float most = m;
      {
        float mb[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          mb[b] = acc[b][0];
#pragma unroll
          for (int e = 1; e < 31; e += 2) mb[b] = fmaxf(mb[b], fmaxf(acc[b][e], acc[b][e + 1]));
          mb[b] = fmaxf(mb[b], acc[b][31]);
        }
        most = fmaxf(most, fmaxf(fmaxf(mb[0], mb[1]), fmaxf(mb[2], mb[3])));
      }
      const float from = reference(most);
      {
        const float d = fmaxf(reference(m) - from, kGone), k = m == -INFINITY ? 0.f : ex2(d * kLog2e);
        t = k * (t + d * s);
        s = k * s;
      }
      if (kKeep) {
        if (in) p.epi.from[(int64_t)(2 * at.tn + at.half) * p.epi.rows + row] = from;
        box_free(at.lane);
      }
      float2 s2[2] = {{0.f, 0.f}, {0.f, 0.f}}, t2[2] = {{0.f, 0.f}, {0.f, 0.f}};
      const float2 minus = make_float2(-from, -from), log2e = make_float2(kLog2e, kLog2e);
      const float2 steps = make_float2(-kSteps, -kSteps), whole = make_float2(kWhole, kWhole);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int o = 0; o < 32; o += 8) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float2 d = add2(make_float2(acc[b][o + e], acc[b][o + e + 1]), minus);
            const float2 a = mul2(d, log2e);
            const float2 x = make_float2(ex2(a.x), ex2(a.y));      // NaN for a NaN, and for infinity
            const int k = e >> 1 & 1;
            s2[k] = add2(s2[k], x);
            t2[k] = fma2(x, d, t2[k]);                              // NaN for -inf too
            if (kKeep) {
              const float2 q = fma2(d, steps, whole);
              w[e >> 1] = two_q(fminf(q.x, kWhole + 65535.f), fminf(q.y, kWhole + 65535.f));
            }
          }
          if (kKeep) box_put(at.box + (b >> 1) * kBoxBytes, at.lane, (b & 1) * 4 + o / 8, w[0], w[1], w[2], w[3]);
        }
      }
      s2[0] = add2(s2[0], s2[1]);
      t2[0] = add2(t2[0], t2[1]);
      const float sn = s2[0].x + s2[0].y;
      float tn = t2[0].x + t2[0].y;
      if (tn != tn && sn == sn) {      // logits of -inf: nothing is added for them
        tn = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float d = fmaxf(acc[b][e] - from, kGone);
            tn += ex2(d * kLog2e) * d;
          }
      }
      s += sn;
      t += tn;
      m = most;
      if (kKeep) store_boxes(p, at);
      if (it.strip >= 0) {
        if (in) {
          const int64_t o = (int64_t)(2 * it.strip + at.half) * p.epi.rows + row;
          p.epi.m[o] = m;
          p.epi.s[o] = s;
          p.epi.t[o] = t;
        }
        m = -INFINITY;
        s = t = 0.f;
      }
    }
  };
};

__device__ __forceinline__ float gradient(float lp, const float4& w) {
  return ex2(lp * kLog2e) * (w.y - w.z * (fmaxf(lp, kGone) + w.w));
}

struct GradEpi {
  static constexpr int kStages = 5, kBoxes = 2, kRowsA = kHalf, kChunk = 8, kFewRegs = 120;
  RowTerms rows;
  template <typename P>
  struct Warp {
    __device__ __forceinline__ Warp(const P&, const Place&) {}
    __device__ __forceinline__ void tile(const P& p, const Item&, const Place& at, float (&acc)[4][32]) {
      const int row = at.row + at.lane;
      const bool in = row < p.m;
      float4 w = in ? p.epi.rows.terms[row] : make_float4(0.f, 0.f, 0.f, 0.f);
      const float scale = p.epi.rows.scale[0];
      w.y *= scale;
      w.z *= scale;
      const int y = in ? p.epi.rows.target[row] - at.col : -1;
      // The blocks go on to a multiple of 64 columns, and dh's product takes them whole
      // (times rows of 0 beyond W): a logit of 0 there, as the product leaves it, would
      // count e^(0 - lse), which is infinite below lse = -88.7.
      if (p.n - at.col < 128) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = 32 * b + e < p.n - at.col ? acc[b][e] : kOutside;
      }
      box_free(at.lane);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int e = 0; e < 32; ++e) acc[b][e] = gradient(acc[b][e] - w.x, w);
        if ((unsigned)(y - 32 * b) < 32u) {
          const float gl = p.epi.rows.g_logp[row] * scale;
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] += y == 32 * b + e ? gl : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float* v = &acc[b][8 * e];
          box_put(at.box + (b >> 1) * kBoxBytes, at.lane, (b & 1) * 4 + e, pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7]));
        }
      }
      store_boxes(p, at);
    }
  };
};

// from: what log p counts from, lse, or M with log_s.
__device__ __forceinline__ void put_terms(const RowTerms& o, int64_t row, float from, float log_s, bool empty, float h, int64_t y, int64_t vocab,
                                          const float* g_logp, const float* g_entropy, const float* g_lse) {
  const bool has = y >= 0 && g_logp != nullptr;
  float gl = has ? g_logp[row] : 0.f;
  float a = (g_lse != nullptr ? g_lse[row] : 0.f) - gl;
  const float gh = g_entropy != nullptr ? g_entropy[row] : 0.f;
  if (has && y >= vocab) a = __int_as_float(0x7FC00000);
  if (empty) {       // every logit -inf: no gradient
    from = log_s = INFINITY;
    gl = 0.f;
  }
  o.terms[row] = make_float4(from, a, gh, h);
  if (o.log_s != nullptr) o.log_s[row] = log_s;
  o.g_logp[row] = gl;
  o.target[row] = has && y < vocab ? (int32_t)y : -1;
}

// Rows' parts joined: 32 rows a block, 16 parts of a row at a time.
constexpr int kJoinParts = 16;
struct JoinParams {
  const float *m, *s, *t, *z_target;
  int32_t parts;
  int64_t rows, vocab;
  const int64_t* targets;
  float *logp, *entropy, *lse;
  const float *g_logp, *g_entropy, *g_lse;
  RowTerms out;         // terms NULL: no gradient follows
};
__global__ void __launch_bounds__(32 * kJoinParts) linlogp_join_kernel(const JoinParams p) {
  __shared__ float sm[kJoinParts][32], ss[kJoinParts][32], st[kJoinParts][32];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * 32 + lane;
  const bool in = row < p.rows;
  // the row's maximum first, so that the sums that follow do not wait for one another
  float m = -INFINITY, s = 0.f, t = 0.f;
  if (in) {
#pragma unroll 8
    for (int i = k; i < p.parts; i += kJoinParts) m = fmaxf(m, p.m[i * p.rows + row]);
  }
  sm[k][lane] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kJoinParts; ++i) m = fmaxf(m, sm[i][lane]);
  const float from = reference(m);
  if (in) {
#pragma unroll 4
    for (int i = k; i < p.parts; i += kJoinParts) {
      const float mi = p.m[i * p.rows + row], si = p.s[i * p.rows + row], ti = p.t[i * p.rows + row];
      const float d = fmaxf(reference(mi) - from, kGone), f = mi == -INFINITY ? 0.f : ex2(d * kLog2e);
      // a part that holds NaN or infinity has s NaN, whatever its maximum
      s = fmaf(f, si, s);
      t = fmaf(f, fmaf(d, si, ti), t);
    }
  }
  ss[k][lane] = s;
  st[k][lane] = t;
  __syncthreads();
  const unsigned lanes = __ballot_sync(0xFFFFFFFFu, in);
  if (k != 0 || !in) return;
  s = t = 0.f;
#pragma unroll
  for (int i = 0; i < kJoinParts; ++i) {
    s += ss[i][lane];
    t += st[i][lane];
  }
  const int64_t y = p.targets != nullptr ? p.targets[row] : -1;
  float lse, h, logp, log_s = 0.f;
  const bool empty = m == -INFINITY && s == 0.f;
  if (empty) {
    lse = -INFINITY;
    h = 0.f;
    logp = y < 0 ? 0.f : -INFINITY;
  } else {
    log_s = logf(s);      // NaN where the row holds NaN or infinity
    lse = m + log_s;
    h = log_s - t / s;
    logp = y >= 0 && y < p.vocab ? (p.z_target[row] - m) - log_s : 0.f;
    if (!(s == s)) logp = s;
  }
  if (y >= p.vocab) logp = __int_as_float(0x7FC00000);
  if (p.logp != nullptr) p.logp[row] = logp;
  if (p.entropy != nullptr) p.entropy[row] = h;
  if (p.lse != nullptr) p.lse[row] = lse;
  if (p.out.terms == nullptr) return;
  put_terms(p.out, row, from, log_s, empty, h, y, p.vocab, p.g_logp, p.g_entropy, p.g_lse);
  if (row < 32) put_scale(p.out.scale, lanes, p.g_logp != nullptr ? p.g_logp[row] : 0.f);
}

// The gradient's terms from lse and entropy of an earlier call.
__global__ void __launch_bounds__(256) linlogp_terms_kernel(const JoinParams p) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const unsigned lanes = __ballot_sync(0xFFFFFFFFu, row < p.rows);
  if (row >= p.rows) return;
  put_terms(p.out, row, p.lse[row], 0.f, p.lse[row] == -INFINITY, p.entropy != nullptr && p.g_entropy != nullptr ? p.entropy[row] : 0.f,
            p.targets != nullptr ? p.targets[row] : -1, p.vocab, p.g_logp, p.g_entropy, p.g_lse);
  if (row < 32) put_scale(p.out.scale, lanes, p.g_logp != nullptr ? p.g_logp[row] : 0.f);
}

// d in the place of q: eight lanes to a row of a block (64 columns), a block of
// threads 32 rows of kDzBlocks column blocks one after another.
constexpr int kDzBlocks = 16;
__global__ void __launch_bounds__(256) linlogp_dz_kernel(uint4* q, const float* from, RowTerms t, int64_t rows, int blocks) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
  if (row >= rows) return;
  const int part = threadIdx.x & 7;
  float4 w = t.terms[row];
  const float scale = t.scale[0], log_s = t.log_s[row];
  w.y *= scale;
  w.z *= scale;
  const int y = t.target[row];
  for (int b0 = (int)blockIdx.y * kDzBlocks; b0 < blocks; b0 += (int)gridDim.y * kDzBlocks) {
#pragma unroll 4
    for (int b = b0; b < min(b0 + kDzBlocks, blocks); ++b) {
      uint4* at = q + ((int64_t)b * rows + row) * 8 + part;
      const uint4 v = __ldcs(at);
      const float ref = (from[(int64_t)(b >> 1) * rows + row] - w.x) - log_s;
      const uint32_t u[4] = {v.x, v.y, v.z, v.w};
      float2 d[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // 2^23 + q from q's two bytes; 65535: the logit is 64 below or more, or -inf
        const float2 whole = add2(make_float2(__uint_as_float(__byte_perm(u[k], 0x4B000000u, 0x7610)), __uint_as_float(__byte_perm(u[k], 0x4B000000u, 0x7632))),
                                  make_float2(-kWhole, -kWhole));
        float2 lp = fma2(whole, make_float2(-1.f / kSteps, -1.f / kSteps), make_float2(ref, ref));
        lp.x = whole.x == 65535.f ? -INFINITY : lp.x;
        lp.y = whole.y == 65535.f ? -INFINITY : lp.y;
        const float2 a = mul2(lp, make_float2(kLog2e, kLog2e));
        const float2 h = add2(make_float2(fmaxf(lp.x, kGone), fmaxf(lp.y, kGone)), make_float2(w.w, w.w));
        d[k] = mul2(make_float2(ex2(a.x), ex2(a.y)), fma2(make_float2(-w.z, -w.z), h, make_float2(w.y, w.y)));
      }
      const int c = y - 64 * b - 8 * part;
      if ((unsigned)c < 8u) {
        const float gl = t.g_logp[row] * scale;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          d[k].x += c == 2 * k ? gl : 0.f;
          d[k].y += c == 2 * k + 1 ? gl : 0.f;
        }
      }
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = pack_bf2(d[k].x, d[k].y);
      *at = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// The fp32 sums of dW to its own type.
__global__ void __launch_bounds__(256) linlogp_round_kernel(const float* sum, int64_t ld, Store out, int64_t rows, int cols) {
  griddep_wait();
  griddep_launch_dependents();
  const int per = (cols + 3) / 4;
  const int64_t all = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per;
    const int c = 4 * (int)(i - r * per);
    out.put(r, c, *reinterpret_cast<const float4*>(sum + r * ld + c), cols - c);
  }
}

// A matrix laid out anew with rows that the TMA takes: a warp takes 256 columns of
// a row, eight a lane, four such pieces at once (50257 x 1285 of 1280: element by
// element 125 us).
__global__ void __launch_bounds__(256) linlogp_copy_kernel(Mat from, int64_t nrows, int cols, __nv_bfloat16* to, int64_t ld) {
  constexpr int kAhead = 4;
  griddep_wait();
  griddep_launch_dependents();
  const int per = (cols + 255) / 256, lane = threadIdx.x & 31;
  // a warp's way over the pieces, `step` apart
  const int64_t first = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), step = (int64_t)gridDim.x * 8, drow = step / per;
  int64_t row = first / per;
  int piece = (int)(first - row * per);
  const int dpiece = (int)(step - drow * per);
  while (row < nrows) {
    rows::Raw<__nv_bfloat16> raw[kAhead];
    int64_t r[kAhead];
    int c[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      r[k] = row;
      c[k] = piece * 256 + 8 * lane;
      raw[k].load<false>(rows::Row<const __nv_bfloat16>(from, row < nrows ? row : 0, nrows), c[k], row < nrows ? cols - c[k] : rows::kNoRow);
      row += drow;
      piece += dpiece;
      if (piece >= per) {
        piece -= per;
        ++row;
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (r[k] >= nrows) break;
      raw[k].settle<false>(rows::Row<const __nv_bfloat16>(from, r[k], nrows), c[k], cols - c[k]);
      // (ld is a multiple of eight: eight are inside the row wherever one is)
      if (c[k] < cols) *reinterpret_cast<uint4*>(to + r[k] * ld + c[k]) = make_uint4(raw[k].w[0], raw[k].w[1], raw[k].w[2], raw[k].w[3]);
    }
  }
}

// Tiles of the forward product whose statistics one part holds: as many as leave
// each pair 16 units (an uneven end then costs 6% at most), so that the parts
// stay few.
int forward_strip(int64_t rows, int64_t vocab) {
  const int64_t tiles_m = (rows + kTileM - 1) / kTileM, tiles_n = (vocab + kTileN - 1) / kTileN;
  const int64_t strips = std::min(tiles_n, std::max<int64_t>(kLeastStrips, (kForwardUnits + tiles_m - 1) / tiles_m));
  return (int)((tiles_n + strips - 1) / strips);
}

struct Layout {
  bool copy_h, copy_w;
  int64_t ld;                        // of the copies
  int64_t piece;                     // tokens of a piece
  int32_t pieces;
  int32_t blocks;                    // column blocks of q and d
  int32_t strip;                     // of the forward product
  int32_t parts;                     // of a row's statistics
  // offsets in the workspace
  size_t h, w, z, terms, log_s, gl, target, scale, stats, from, d, dw, partial, total;
};
bool dw_is_sum(const LinLogpParams& q) { return q.dwdt == LM_F32; }   // several pieces are summed in dW itself
Layout make_layout(const LinLogpParams& q) {
  Layout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  const bool grad = q.dh.data != nullptr || q.dw.data != nullptr;
  l.ld = ((int64_t)q.width + 7) / 8 * 8;
  l.copy_h = !tma_rows(q.h, q.rows, q.width);
  l.copy_w = !tma_rows(q.w, q.vocab, q.width);
  l.h = take(l.copy_h ? (size_t)q.rows * l.ld * 2 : 0);
  l.w = take(l.copy_w ? (size_t)q.vocab * l.ld * 2 : 0);
  l.blocks = (q.vocab + 63) / 64;
  l.piece = q.rows;
  if (grad) {
    const int64_t most = std::max<int64_t>(kLeastPiece, kPieceBytes / 128 / l.blocks / kTileM * kTileM);
    const int64_t pieces = (q.rows + most - 1) / most;
    l.piece = std::min<int64_t>(((q.rows + pieces - 1) / pieces + kTileM - 1) / kTileM * kTileM, q.rows);
  }
  l.pieces = (int32_t)((q.rows + l.piece - 1) / l.piece);
  const size_t n = (size_t)l.piece;
  l.strip = forward_strip(l.piece, q.vocab);
  l.parts = 2 * plain_schedule(l.piece, q.vocab, q.width, l.strip).strips;
  l.z = take(n * 4);
  l.stats = take(q.gradient_only ? 0 : n * l.parts * 12);
  if (grad) {
    l.terms = take(n * 16);
    l.log_s = take(q.gradient_only ? 0 : n * 4);
    l.gl = take(n * 4);
    l.target = take(n * 4);
    l.scale = take(8);
    l.from = take(q.gradient_only ? 0 : n * (2 * (((size_t)q.vocab + kTileN - 1) / kTileN)) * 4);
    l.d = take(n * l.blocks * 128);
    if (q.dw.data != nullptr && l.pieces > 1 && !dw_is_sum(q)) l.dw = take((size_t)q.vocab * l.ld * 4);
    size_t parts = 0;
    for (int i = 0; i < 2; ++i) {      // the last piece may be smaller
      const int64_t rows = i == 0 ? l.piece : q.rows - (l.pieces - 1) * l.piece;
      if (q.dh.data != nullptr) parts = std::max(parts, parts_bytes(split_schedule(rows, q.width, q.vocab)));
      if (q.dw.data != nullptr) parts = std::max(parts, parts_bytes(split_schedule(q.vocab, q.width, rows)));
    }
    l.partial = take(parts);
  }
  l.total = at;
  return l;
}

#define LM_RUN(call)                          \
  do {                                        \
    const cudaError_t e_ = (call);            \
    if (e_ != cudaSuccess) return e_;         \
  } while (0)

template <typename T>
T* from_row(T* p, int64_t first) {
  return p != nullptr ? p + first : nullptr;
}

// Tokens first .. first + rows - 1; h begins at the first of them.
cudaError_t piece(const LinLogpParams& q, const Layout& l, const Mat& h, const Mat& w, int64_t first, int64_t rows, bool last, bool grad, cudaStream_t st) {
  const uint64_t wait_ns = env_wait_limit_ns();
  uint8_t* ws = static_cast<uint8_t*>(q.workspace);
  JoinParams j{};
  j.rows = rows;
  j.vocab = q.vocab;
  j.targets = from_row(q.targets, first);
  j.logp = from_row(q.logp, first);
  j.entropy = from_row(q.entropy, first);
  j.lse = from_row(q.lse, first);
  j.g_logp = from_row(q.g_logp, first);
  j.g_entropy = from_row(q.g_entropy, first);
  j.g_lse = from_row(q.g_lse, first);
  if (grad)
    j.out = RowTerms{reinterpret_cast<float4*>(ws + l.terms), q.gradient_only ? nullptr : reinterpret_cast<float*>(ws + l.log_s),
                     reinterpret_cast<float*>(ws + l.gl), reinterpret_cast<int32_t*>(ws + l.target), reinterpret_cast<float*>(ws + l.scale)};
  const bool few = !grad && rows <= kFewRows;
  // the operands of the logits' product, and the blocks that its epilogue fills
  auto logits = [&](auto& p) {
    p.m = (int32_t)rows;
    p.n = q.vocab;
    p.wait_ns = wait_ns;
    cudaError_t e = encode_operand(&p.a, h.data, q.width, rows, h.ld, false, few ? kFewRows : kHalf);
    if (e == cudaSuccess) e = encode_operand(&p.b, w.data, q.width, q.vocab, w.ld, false);
    if (e == cudaSuccess && grad) e = encode_blocks(&p.out, ws + l.d, q.vocab, rows, 32);
    return e;
  };
  if (q.gradient_only) {
    LM_RUN(launch_after(linlogp_terms_kernel, dim3((unsigned)((rows + 255) / 256)), 256, 0, st, j));
    Params<GradEpi> g{};
    g.sch = plain_schedule(rows, q.vocab, q.width, 1);
    g.epi.rows = j.out;
    LM_RUN(logits(g));
    LM_RUN((start<kRowsK, kRowsK, GradEpi>(g, st)));
  } else {
    auto forward = [&](auto& f) {
      f.sch = plain_schedule(rows, q.vocab, q.width, l.strip);
      const size_t each = (size_t)2 * f.sch.strips * rows;
      f.epi.targets = j.targets;
      f.epi.m = reinterpret_cast<float*>(ws + l.stats);
      f.epi.s = f.epi.m + each;
      f.epi.t = f.epi.s + each;
      f.epi.z_target = reinterpret_cast<float*>(ws + l.z);
      f.epi.from = reinterpret_cast<float*>(ws + l.from);
      f.epi.rows = rows;
      j.m = f.epi.m;
      j.s = f.epi.s;
      j.t = f.epi.t;
      j.z_target = f.epi.z_target;
      j.parts = 2 * f.sch.strips;
      return logits(f);
    };
    if (grad) {
      Params<ForwardEpi<true, false>> f{};
      LM_RUN(forward(f));
      LM_RUN((start<kRowsK, kRowsK, ForwardEpi<true, false>>(f, st)));
    } else if (few) {
      Params<ForwardEpi<false, true>> f{};
      LM_RUN(forward(f));
      LM_RUN((start<kRowsK, kRowsK, ForwardEpi<false, true>>(f, st)));
    } else {
      Params<ForwardEpi<false, false>> f{};
      LM_RUN(forward(f));
      LM_RUN((start<kRowsK, kRowsK, ForwardEpi<false, false>>(f, st)));
    }
    LM_RUN(launch_after(linlogp_join_kernel, dim3((unsigned)((rows + 31) / 32)), 32 * kJoinParts, 0, st, j));
    if (grad)
      LM_RUN(launch_after(linlogp_dz_kernel, dim3((unsigned)((rows + 31) / 32), (unsigned)std::min((l.blocks + kDzBlocks - 1) / kDzBlocks, 65535)), 256, 0, st,
                          reinterpret_cast<uint4*>(ws + l.d), (const float*)(ws + l.from), j.out, rows, (int)l.blocks));
  }
  if (q.dh.data != nullptr) {
    Params<StoreEpi> s{};
    s.sch = split_schedule(rows, q.width, q.vocab);
    s.m = (int32_t)rows;
    s.n = q.width;
    s.wait_ns = wait_ns;
    s.parts = reinterpret_cast<float*>(ws + l.partial);
    s.epi.factor = j.out.scale + 1;
    s.epi.out = make_store(Mat{static_cast<__nv_bfloat16*>(q.dh.data) + first * q.dh.ld, q.dh.ld}, LM_BF16, rows, false);
    LM_RUN(encode_blocks(&s.a, ws + l.d, q.vocab, rows, 128));
    LM_RUN(encode_operand(&s.b, w.data, q.width, q.vocab, w.ld, true));
    LM_RUN((start_store<kBlocksK, kRowsMn>(s, st)));
  }
  if (q.dw.data != nullptr) {
    Params<StoreEpi> s{};
    s.sch = split_schedule(q.vocab, q.width, rows);
    s.m = q.vocab;
    s.n = q.width;
    s.wait_ns = wait_ns;
    s.parts = reinterpret_cast<float*>(ws + l.partial);
    s.epi.factor = j.out.scale + 1;
    const bool own_sum = !dw_is_sum(q) && l.pieces > 1;
    const Mat sum{ws + l.dw, l.ld};
    if (own_sum) s.epi.out = make_store(sum, LM_F32, q.vocab, first > 0);
    else s.epi.out = make_store(q.dw, q.dwdt, q.vocab, q.accumulate != 0 || first > 0);
    LM_RUN(encode_blocks(&s.a, ws + l.d, q.vocab, rows, 64));
    LM_RUN(encode_operand(&s.b, h.data, q.width, rows, h.ld, true));
    LM_RUN((start_store<kBlocksMn, kRowsMn>(s, st)));
    if (own_sum && last)
      LM_RUN(launch_after(linlogp_round_kernel, dim3((unsigned)std::min<int64_t>(q.vocab, 152 * 16)), 256, 0, st, (const float*)sum.data, l.ld,
                          make_store(q.dw, q.dwdt, q.vocab, q.accumulate != 0), (int64_t)q.vocab, q.width));
  }
  return cudaSuccess;
}

cudaError_t copy_rows(const Mat& from, int64_t rows, int cols, void* to, int64_t ld, cudaStream_t st) {
  const int64_t blocks = (rows * ((cols + 255) / 256) + 31) / 32;
  return launch_after(linlogp_copy_kernel, dim3((unsigned)std::min<int64_t>(blocks, 152 * 8)), 256, 0, st, from, rows, cols,
                      static_cast<__nv_bfloat16*>(to), ld);
}

}  // namespace

size_t linlogp_workspace(const LinLogpParams& q) { return q.rows <= 0 ? 0 : make_layout(q).total; }

cudaError_t launch_linlogp(const LinLogpParams& q, cudaStream_t st) {
  if (q.rows == 0) return start_zero(q.dw, q.dwdt, q.vocab, q.width, st);   // dW of no tokens
  const Layout l = make_layout(q);
  uint8_t* ws = static_cast<uint8_t*>(q.workspace);
  Mat h = q.h, w = q.w;
  if (l.copy_h) {
    LM_RUN(copy_rows(q.h, q.rows, q.width, ws + l.h, l.ld, st));
    h = Mat{ws + l.h, l.ld};
  }
  if (l.copy_w) {
    LM_RUN(copy_rows(q.w, q.vocab, q.width, ws + l.w, l.ld, st));
    w = Mat{ws + l.w, l.ld};
  }
  const bool grad = q.dh.data != nullptr || q.dw.data != nullptr;
  for (int32_t i = 0; i < l.pieces; ++i) {
    const int64_t first = i * l.piece, rows = std::min<int64_t>(l.piece, q.rows - first);
    LM_RUN(piece(q, l, Mat{static_cast<__nv_bfloat16*>(h.data) + first * h.ld, h.ld}, w, first, rows, i + 1 == l.pieces, grad, st));
  }
  return cudaSuccess;
}

}  // namespace lm
