// Log probabilities of given tokens from the last hidden states and the head's
// matrix, and the gradients of a loss over them, without the logits (formulas at
// lm_linear_logprob_args in lionmuon.h).
//
// Forward: the product z = h W^T tile by tile; a tile's epilogue keeps, for its
// rows, the maximum m, s = sum e^(z - m) and t = sum e^(z - m) (z - m), and the
// target's z where the tile holds it.  A second kernel joins a row's parts:
//   lse = M + log S,  logp = (z_y - M) - log S,  H = log S - T / S.
//
// Gradients, for a piece of the vocabulary at a time: the piece's logits are
// computed once more, and the epilogue writes
//   d = p (a - g_H (log p + H)) (+ g_logp at the target),  a = g_lse - g_logp
// as bf16 (its one rounding below 32 bits: the tensor cores take it so) into the
// workspace; two products of it follow, dh += d W and dW = d^T h.  Where there
// are several pieces dh is summed in fp32 in the workspace.
#include <cuda_bf16.h>
#include <math.h>

#include "lm_gemm_tc.cuh"

namespace lm {
namespace {

using namespace gemm;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGone = -1e4f;      // e^kGone is 0
constexpr int kForwardUnits = 16 * kPairs, kLeastStrips = 8;   // of the forward product (forward_strip)
constexpr int64_t kPieceBytes = (int64_t)512 << 20;   // of the gradient's bf16 values in the workspace
constexpr int64_t kLeastPiece = 2048;                 // columns

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the reference of a maximum: -inf (nothing there) counts from 0
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// What a row's gradient takes: lse, a = g_lse - g_logp, g_H, H.
struct RowTerms {
  float4* terms;
  float* g_logp;      // 0 in a row without a target
  int32_t* target;    // -1 in a row without one
};

struct ForwardEpi {
  const int64_t* targets;
  float *m, *s, *t;     // (2 strips) x rows
  float* z_target;
  int64_t rows;
  template <typename P>
  struct Warp {
    float m, s, t;
    __device__ __forceinline__ Warp(const P&, const Place&) : m(-INFINITY), s(0.f), t(0.f) {}
    __device__ __forceinline__ void tile(const P& p, const Item& it, const Place& at, float (&acc)[4][32]) {
      const int row = at.row + at.lane;
      const bool in = row < p.m;
      const int64_t y = in && p.epi.targets != nullptr ? p.epi.targets[row] : -1;
      const int left = p.n - at.col;      // columns of the vocabulary from this warp's first
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if ((uint64_t)(y - at.col - 32 * b) < 32u && y < p.n) {
          float z = 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) z = (int)(y - at.col) == 32 * b + e ? acc[b][e] : z;
          p.epi.z_target[row] = z;
        }
      if (left < 128) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = 32 * b + e < left ? acc[b][e] : -INFINITY;
      }
      float most = m;
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 32; ++e) most = fmaxf(most, acc[b][e]);
      const float from = reference(most);
      {
        const float d = fmaxf(reference(m) - from, kGone), k = m == -INFINITY ? 0.f : ex2(d * kLog2e);
        t = k * (t + d * s);
        s = k * s;
      }
      float s4[4], t4[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        s4[b] = t4[b] = 0.f;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const float d = acc[b][e] - from;
          const float x = ex2(d * kLog2e);      // NaN for a NaN, and for infinity
          s4[b] += x;
          t4[b] += x * fmaxf(d, kGone);
        }
      }
      s += (s4[0] + s4[1]) + (s4[2] + s4[3]);
      t += (t4[0] + t4[1]) + (t4[2] + t4[3]);
      m = most;
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

struct GradEpi {
  RowTerms rows;
  int32_t first;        // the piece's first token of the vocabulary
  Store out;
  template <typename P>
  struct Warp {
    __device__ __forceinline__ Warp(const P&, const Place&) {}
    __device__ __forceinline__ void tile(const P& p, const Item&, const Place& at, float (&acc)[4][32]) {
      const int row = at.row + at.lane, rows = min(32, p.m - at.row);
      if (rows <= 0) return;
      const bool in = row < p.m;
      const float4 w = in ? p.epi.rows.terms[row] : make_float4(0.f, 0.f, 0.f, 0.f);
      const float gl = in ? p.epi.rows.g_logp[row] : 0.f;
      const int y = in ? p.epi.rows.target[row] : -1;
      const int yc = y >= 0 ? y - p.epi.first - at.col : -1;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = at.col + 32 * b;
        if (c >= p.n) continue;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const float lp = acc[b][e] - w.x;
          const float d = ex2(lp * kLog2e) * (w.y - w.z * (fmaxf(lp, kGone) + w.w));
          acc[b][e] = yc == 32 * b + e ? d + gl : d;
        }
        put_block(acc[b], at, rows, c, [&](int r, int col, float4 v) {
          if (col < p.n) p.epi.out.put(at.row + r, col, v, p.n - col);
        });
      }
    }
  };
};

__device__ __forceinline__ void put_terms(const RowTerms& o, int64_t row, float lse, float h, int64_t y, int64_t vocab, const float* g_logp,
                                          const float* g_entropy, const float* g_lse) {
  const bool has = y >= 0 && g_logp != nullptr;
  float gl = has ? g_logp[row] : 0.f;
  float a = (g_lse != nullptr ? g_lse[row] : 0.f) - gl;
  const float gh = g_entropy != nullptr ? g_entropy[row] : 0.f;
  if (has && y >= vocab) a = __int_as_float(0x7FC00000);
  if (lse == -INFINITY) {       // every logit -inf: no gradient
    lse = INFINITY;
    gl = 0.f;
  }
  o.terms[row] = make_float4(lse, a, gh, h);
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
  float m = -INFINITY, s = 0.f, t = 0.f;
  auto add = [&](float m2, float s2, float t2) {
    const float most = fmaxf(m, m2), from = reference(most);
    const float d1 = fmaxf(reference(m) - from, kGone), d2 = fmaxf(reference(m2) - from, kGone);
    const float k1 = m == -INFINITY ? 0.f : ex2(d1 * kLog2e), k2 = m2 == -INFINITY ? 0.f : ex2(d2 * kLog2e);
    // a part that holds NaN or infinity has s NaN, whatever its maximum
    t = k1 * (t + d1 * s) + k2 * (t2 + d2 * s2);
    s = k1 * s + k2 * s2;
    m = most;
  };
  if (in) {
#pragma unroll 4
    for (int i = k; i < p.parts; i += kJoinParts) add(p.m[i * p.rows + row], p.s[i * p.rows + row], p.t[i * p.rows + row]);
  }
  sm[k][lane] = m;
  ss[k][lane] = s;
  st[k][lane] = t;
  __syncthreads();
  if (k != 0 || !in) return;
  for (int i = 1; i < kJoinParts; ++i) add(sm[i][lane], ss[i][lane], st[i][lane]);
  const int64_t y = p.targets != nullptr ? p.targets[row] : -1;
  float lse, h, logp;
  if (m == -INFINITY && s == 0.f) {
    lse = -INFINITY;
    h = 0.f;
    logp = y < 0 ? 0.f : -INFINITY;
  } else {
    const float log_s = logf(s);      // NaN where the row holds NaN or infinity
    lse = m + log_s;
    h = log_s - t / s;
    logp = y >= 0 && y < p.vocab ? (p.z_target[row] - m) - log_s : 0.f;
    if (!(s == s)) logp = s;
  }
  if (y >= p.vocab) logp = __int_as_float(0x7FC00000);
  if (p.logp != nullptr) p.logp[row] = logp;
  if (p.entropy != nullptr) p.entropy[row] = h;
  if (p.lse != nullptr) p.lse[row] = lse;
  if (p.out.terms != nullptr) put_terms(p.out, row, lse, h, y, p.vocab, p.g_logp, p.g_entropy, p.g_lse);
}

// The gradient's terms from lse and entropy of an earlier call.
__global__ void __launch_bounds__(256) linlogp_terms_kernel(const JoinParams p) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row >= p.rows) return;
  put_terms(p.out, row, p.lse[row], p.entropy != nullptr && p.g_entropy != nullptr ? p.entropy[row] : 0.f,
            p.targets != nullptr ? p.targets[row] : -1, p.vocab, p.g_logp, p.g_entropy, p.g_lse);
}

// A matrix laid out anew with rows that the TMA takes.
__global__ void __launch_bounds__(256) linlogp_copy_kernel(Mat from, int64_t rows, int cols, __nv_bfloat16* to, int64_t ld) {
  griddep_wait();
  griddep_launch_dependents();
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(from.data) + r * from.ld;
    for (int c = threadIdx.x; c < cols; c += 256) to[r * ld + c] = src[c];
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
  int32_t pieces;
  int64_t piece;                     // columns of a piece
  Schedule forward;
  // offsets in the workspace
  size_t h, w, z, terms, gl, target, stats, d, dh, parts, total;
};
Layout make_layout(const LinLogpParams& q) {
  Layout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  const size_t n = (size_t)q.rows;
  const bool grad = q.dh.data != nullptr || q.dw.data != nullptr;
  l.ld = ((int64_t)q.width + 7) / 8 * 8;
  l.copy_h = !tma_rows(q.h, q.rows, q.width);
  l.copy_w = !tma_rows(q.w, q.vocab, q.width);
  l.h = take(l.copy_h ? n * l.ld * 2 : 0);
  l.w = take(l.copy_w ? (size_t)q.vocab * l.ld * 2 : 0);
  l.forward = plain_schedule(q.rows, q.vocab, q.width, forward_strip(q.rows, q.vocab));
  l.z = take(n * 4);
  l.terms = take(grad ? n * 16 : 0);
  l.gl = take(grad ? n * 4 : 0);
  l.target = take(grad ? n * 4 : 0);
  // the forward pass's parts and the gradient's values are not wanted at once
  const size_t stats = q.gradient_only ? 0 : (size_t)l.forward.strips * 2 * n * 4 * 3;
  size_t d = 0;
  if (grad) {
    const int64_t most = std::max<int64_t>(kLeastPiece, kPieceBytes / 2 / q.rows);
    l.pieces = (int32_t)((q.vocab + most - 1) / most);
    l.piece = ((q.vocab + l.pieces - 1) / l.pieces + kTileN - 1) / kTileN * kTileN;
    l.pieces = (int32_t)((q.vocab + l.piece - 1) / l.piece);
    d = n * (size_t)l.piece * 2;
  }
  l.stats = l.d = take(std::max(stats, d));
  if (q.dh.data != nullptr && l.pieces > 1) l.dh = take(n * (size_t)l.ld * 4);
  size_t parts = 0;
  for (int i = 0; grad && i < 2; ++i) {      // the last piece may be smaller
    const int64_t cols = i == 0 ? l.piece : q.vocab - (l.pieces - 1) * l.piece;
    if (q.dh.data != nullptr) parts = std::max(parts, parts_bytes(split_schedule(q.rows, q.width, cols)));
    if (q.dw.data != nullptr) parts = std::max(parts, parts_bytes(split_schedule(cols, q.width, q.rows)));
  }
  l.parts = take(parts);
  l.total = at;
  return l;
}

#define LM_RUN(call)                          \
  do {                                        \
    const cudaError_t e_ = (call);            \
    if (e_ != cudaSuccess) return e_;         \
  } while (0)

cudaError_t copy_rows(const Mat& from, int64_t rows, int cols, void* to, int64_t ld, cudaStream_t st) {
  return launch_after(linlogp_copy_kernel, dim3((unsigned)std::min<int64_t>(rows, 152 * 8)), 256, 0, st, from, rows, cols,
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
  const uint64_t wait_ns = env_wait_limit_ns();
  const bool grad = q.dh.data != nullptr || q.dw.data != nullptr;
  JoinParams j{};
  j.rows = q.rows;
  j.vocab = q.vocab;
  j.targets = q.targets;
  j.logp = q.logp;
  j.entropy = q.entropy;
  j.lse = q.lse;
  j.g_logp = q.g_logp;
  j.g_entropy = q.g_entropy;
  j.g_lse = q.g_lse;
  if (grad) j.out = RowTerms{reinterpret_cast<float4*>(ws + l.terms), reinterpret_cast<float*>(ws + l.gl), reinterpret_cast<int32_t*>(ws + l.target)};
  if (q.gradient_only) {
    LM_RUN(launch_after(linlogp_terms_kernel, dim3((unsigned)((q.rows + 255) / 256)), 256, 0, st, j));
  } else {
    Params<ForwardEpi> f{};
    f.sch = l.forward;
    f.m = (int32_t)q.rows;
    f.n = q.vocab;
    f.wait_ns = wait_ns;
    const size_t each = (size_t)l.forward.strips * 2 * q.rows;
    f.epi.targets = q.targets;
    f.epi.m = reinterpret_cast<float*>(ws + l.stats);
    f.epi.s = f.epi.m + each;
    f.epi.t = f.epi.s + each;
    f.epi.z_target = reinterpret_cast<float*>(ws + l.z);
    f.epi.rows = q.rows;
    LM_RUN(encode_operand(&f.a, h.data, q.width, q.rows, h.ld, false));
    LM_RUN(encode_operand(&f.b, w.data, q.width, q.vocab, w.ld, false));
    LM_RUN((start<false, false, ForwardEpi>(f, st)));
    j.m = f.epi.m;
    j.s = f.epi.s;
    j.t = f.epi.t;
    j.z_target = f.epi.z_target;
    j.parts = 2 * l.forward.strips;
    LM_RUN(launch_after(linlogp_join_kernel, dim3((unsigned)((q.rows + 31) / 32)), 32 * kJoinParts, 0, st, j));
  }
  for (int32_t i = 0; grad && i < l.pieces; ++i) {
    const int64_t first = i * l.piece, cols = std::min<int64_t>(l.piece, q.vocab - first);
    const __nv_bfloat16* wp = static_cast<const __nv_bfloat16*>(w.data) + first * w.ld;
    const Mat d{ws + l.d, l.piece};
    Params<GradEpi> g{};
    g.sch = plain_schedule(q.rows, cols, q.width, 1);
    g.m = (int32_t)q.rows;
    g.n = (int32_t)cols;
    g.wait_ns = wait_ns;
    g.epi.rows = j.out;
    g.epi.first = (int32_t)first;
    g.epi.out = make_store(d, LM_BF16, q.rows, false);
    LM_RUN(encode_operand(&g.a, h.data, q.width, q.rows, h.ld, false));
    LM_RUN(encode_operand(&g.b, wp, q.width, cols, w.ld, false));
    LM_RUN((start<false, false, GradEpi>(g, st)));
    if (q.dh.data != nullptr) {
      Params<StoreEpi> s{};
      s.sch = split_schedule(q.rows, q.width, cols);
      s.m = (int32_t)q.rows;
      s.n = q.width;
      s.wait_ns = wait_ns;
      s.parts = reinterpret_cast<float*>(ws + l.parts);
      const Mat sum{ws + l.dh, l.ld};
      s.epi.out = i + 1 < l.pieces ? make_store(sum, LM_F32, q.rows, false) : make_store(q.dh, LM_BF16, q.rows, false);
      if (i > 0) {
        s.epi.out.add = static_cast<const float*>(sum.data);
        s.epi.out.ld_add = l.ld;
      }
      LM_RUN(encode_operand(&s.a, d.data, cols, q.rows, d.ld, false));
      LM_RUN(encode_operand(&s.b, wp, q.width, cols, w.ld, true));
      LM_RUN((start_store<false, true>(s, st)));
    }
    if (q.dw.data != nullptr) {
      Params<StoreEpi> s{};
      s.sch = split_schedule(cols, q.width, q.rows);
      s.m = (int32_t)cols;
      s.n = q.width;
      s.wait_ns = wait_ns;
      s.parts = reinterpret_cast<float*>(ws + l.parts);
      const int64_t size = q.dwdt == LM_F32 ? 4 : 2;
      s.epi.out = make_store(Mat{static_cast<uint8_t*>(q.dw.data) + first * q.dw.ld * size, q.dw.ld}, q.dwdt, cols, q.accumulate != 0);
      LM_RUN(encode_operand(&s.a, d.data, cols, q.rows, d.ld, true));
      LM_RUN(encode_operand(&s.b, h.data, q.width, q.rows, h.ld, true));
      LM_RUN((start_store<true, true>(s, st)));
    }
  }
  return cudaSuccess;
}

}  // namespace lm
