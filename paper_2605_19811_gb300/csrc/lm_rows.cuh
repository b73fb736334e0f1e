// What the row kernels (lm_rmsnorm.cu, lm_rmsnorm_grad.cu, lm_checkpoint8.cu)
// share: eight channels of a row to a lane, 256 consecutive ones to a warp,
// whatever the row's alignment; sums over a row; shapes by channel count.
#pragma once

#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "lm_code8.cuh"
#include "lm_train.h"

namespace lm {
namespace rows {
namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int kNoRow = -(1 << 30);

// A row of a matrix for loads in 16-byte pieces: `edge` where such a piece,
// begun in the row, could reach beyond the matrix's first or last element (its
// first and last rows, and all where a row is shorter than a piece).
template <typename T>
struct Row {
  T* p;
  bool edge;
  __device__ __forceinline__ Row(const Mat& m, int64_t row, int64_t nrows)
      : p(static_cast<T*>(m.data) + row * m.ld), edge(row == 0 || row == nrows - 1 || m.ld * (int64_t)sizeof(T) < 16) {}
};

// 16 bytes into registers of their own, zero without `in`: one piece of code, so
// that nothing waits for the load before its values are used.
__device__ __forceinline__ void load16(uint32_t* w, const void* p, bool in) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "mov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
      "@q ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=&r"(w[0]), "=&r"(w[1]), "=&r"(w[2]), "=&r"(w[3])
      : "l"(p), "r"((int)in));
}

// Eight channels of a row as they are read; `left`: channels from the first of
// them to the row's end (kNoRow where there is no row), zeros beyond.  All 32
// lanes of a warp take part, each with the eight after its neighbour's.  load
// sends the loads out, settle (with the same arguments) makes the eight of them.
//   kVec: eights lie on 16-byte boundaries, one or two 16-byte loads.
//   else: the warp's 256 channels begin `shift` bytes after such a boundary; the
//   lanes load the 16-byte pieces from there on, lane 31 one more, and each puts
//   its eight together from its own pieces and its neighbour's (8191 x 1283:
//   bf16 norm 48 us, 72 us with elements one by one; fp32 unpacking 16 and 37 us).
//   kSingly: where not kVec, elements are loaded one by one.
template <typename T, bool kSingly = false>
struct Raw {
  static constexpr int kPieces = 8 * (int)sizeof(T) / 16, kWords = 4 * kPieces;
  uint32_t w[kWords + 4];     // the last four: lane 31's further piece, until settle
  // Bytes to the row's end, from `least` elements up; no more of them than the
  // pieces of load and store reach (in a long row they would pass 31 bits).
  static __device__ __forceinline__ int bytes_left(int left, int least) { return min(max(left, least), 16) * (int)sizeof(T); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < kWords + 4; ++k) w[k] = 0u;
  }
  template <bool kVec>
  __device__ __forceinline__ void load(const Row<const T>& row, int c, int left) {
    const T* p = row.p + c;
    if (kVec) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k) load16(w + 4 * k, reinterpret_cast<const uint4*>(p) + k, left >= 8);
      if (left > 0 && left < 8) single(p, left);
      return;
    }
    if constexpr (kSingly) {
      single(p, left);
      return;
    }
    const int shift = (int)(reinterpret_cast<uintptr_t>(p) & 15u), bytes = bytes_left(left, -8);
    const uint8_t* first = reinterpret_cast<const uint8_t*>(p) - shift;
    const int mine = (threadIdx.x & 31) == 31 ? kPieces + 1 : kPieces;
#pragma unroll
    for (int k = 0; k <= kPieces; ++k) load16(w + 4 * k, first + 16 * k, !row.edge && left != kNoRow && k < mine && 16 * k - shift < bytes);
  }
  template <bool kVec>
  __device__ __forceinline__ void settle(const Row<const T>& row, int c, int left) {
    if (kVec || kSingly) return;
    const T* p = row.p + c;
    if (row.edge) {
      single(p, left);
      return;
    }
    const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u);   // the same in every lane: eights are 16 or 32 bytes apart
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t next = __shfl_down_sync(kAll, w[k], 1);
      if ((threadIdx.x & 31) != 31) w[kWords + k] = next;
    }
    // by two words, one word, and half a word
#pragma unroll
    for (int k = 0; k < kWords + 2; ++k) w[k] = (shift & 8u) ? w[k + 2] : w[k];
#pragma unroll
    for (int k = 0; k < kWords + 1; ++k) w[k] = (shift & 4u) ? w[k + 1] : w[k];
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = sizeof(T) == 2 ? __funnelshift_r(w[k], w[k + 1], (shift & 2u) * 8u) : w[k];
    if (left < 8) {
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        if (sizeof(T) == 4) w[k] = k < left ? w[k] : 0u;
        else w[k] = 2 * k + 1 < left ? w[k] : 2 * k < left ? w[k] & 0xFFFFu : 0u;
      }
    }
  }
  __device__ __forceinline__ void single(const T* p, int left) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = k < left ? reinterpret_cast<const uint32_t*>(p)[k] : 0u;
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = (2 * k < left ? (uint32_t)q[2 * k] : 0u) | (2 * k + 1 < left ? (uint32_t)q[2 * k + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(v[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
        w[k] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
  }
  // The counterpart of load: all 32 lanes.  Pieces that a warp's 256 channels
  // fill are stored 16 bytes at a time, the others one element at a time.
  template <bool kVec>
  __device__ __forceinline__ void store(T* p, int left) const {
    if (kVec) {
      if (left >= 8) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) __stcs(reinterpret_cast<uint4*>(p) + k, make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]));
      } else {
        put_single(p, 0, left);
      }
      return;
    }
    const int lane = (int)threadIdx.x & 31;
    const int shift = (int)(reinterpret_cast<uintptr_t>(p) & 15u), bytes = bytes_left(left, 0);
    // c: the neighbour's last words, then this lane's; taken back by `shift` bytes
    uint32_t c[kWords + 4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = __shfl_up_sync(kAll, w[kWords - 4 + k], 1);
#pragma unroll
    for (int k = 0; k < kWords; ++k) c[4 + k] = w[k];
    // words from 4 - shift / 4 on: first the whole words, then half a word
#pragma unroll
    for (int k = kWords + 3; k >= 2; --k) c[k] = (shift & 8) ? c[k - 2] : c[k];
#pragma unroll
    for (int k = kWords + 3; k >= 3; --k) c[k] = (shift & 4) ? c[k - 1] : c[k];
    uint32_t o[kWords];
#pragma unroll
    for (int k = 0; k < kWords; ++k) o[k] = sizeof(T) == 2 ? ((shift & 2) ? __funnelshift_l(c[k + 3], c[k + 4], 16u) : c[k + 4]) : c[k + 4];
    uint8_t* first = reinterpret_cast<uint8_t*>(p) - shift;
    // Piece k is stored whole where it begins among the warp's channels and ends
    // inside the row; the last, the neighbour's first, by the neighbour.
    bool whole[kPieces + 1];
#pragma unroll
    for (int k = 0; k <= kPieces; ++k) whole[k] = 16 * k + 16 - shift <= bytes && (k > 0 || lane != 0 || shift == 0) && (k < kPieces || lane != 31);
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      if (whole[k]) __stcs(reinterpret_cast<uint4*>(first) + k, make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]));
    // the elements that no whole piece took
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int b = e * (int)sizeof(T);   // pieces b / 16 (shift below 16 - b % 16) or the next
      const bool taken = shift + b % 16 < 16 ? whole[b / 16] : whole[b / 16 + 1];
      if (e < left && !taken) put_one(p, e);
    }
  }
  __device__ __forceinline__ void put_one(T* p, int e) const {
    if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p)[e] = w[e];
    else reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
  }
  __device__ __forceinline__ void put_single(T* p, int from, int left) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= from && e < left) put_one(p, e);
  }
};
// Eight channels of an 8-bit checkpoint: their codes and scale.
template <int kFormat>
struct RawCodes {
  uint2 q;
  float scale;
  __device__ __forceinline__ void zero() {
    q = make_uint2(0u, 0u);
    scale = 0.f;
  }
  __device__ __forceinline__ void load(const Codes& k, int64_t row, int c, bool in) {
    const uint8_t* q_at = k.data + row * k.ld + c;
    const float* s_at = k.scales + (int64_t)(c / LM_CODE_GROUP) * k.ld_scales + row;
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.f32 %2, 0f00000000;\n\t"
        "@q ld.global.cs.v2.u32 {%0, %1}, [%3];\n\t@q ld.global.f32 %2, [%4];\n\t}"
        : "=&r"(q.x), "=&r"(q.y), "=&f"(scale)
        : "l"(q_at), "l"(s_at), "r"((int)in));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t two[4] = {q.x, q.x >> 16, q.y, q.y >> 16};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 d = code8::decode2<kFormat>(two[k]);
      v[2 * k] = d.x * scale;
      v[2 * k + 1] = d.y * scale;
    }
  }
};

// Eight channels of the gain (ones where there is none); from L1 after a
// block's first row.
__device__ __forceinline__ void weight8(const void* w, int dt, int c, int left, bool vec, float (&v)[8]) {
  if (w == nullptr) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 1.f;
  } else if (vec && left >= 8) {
    if (dt == LM_F32) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + c)), b = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + c) + 1);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + c));
      const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = __uint_as_float(x[k] << 16);
        v[2 * k + 1] = __uint_as_float(x[k] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = k < left ? (dt == LM_F32 ? static_cast<const float*>(w)[c + k] : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[c + k])) : 1.f;
  }
}

// How a block takes rows: `threads` (whole warps) to a row, `rows` of them side
// by side, a thread kVecs eights, `span` channels apart.
struct Team {
  int threads, rows, span, t, slot;
  __device__ __forceinline__ explicit Team(int per_row)
      : threads(per_row), rows((int)blockDim.x / per_row), span(8 * per_row), t((int)threadIdx.x % per_row), slot((int)threadIdx.x / per_row) {}
  // Sum over a row's threads; `turn` alternates so that one barrier a sum is
  // enough (every thread of the block calls it).
  __device__ __forceinline__ float sum(float s, float (*part)[32], int turn) const {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kAll, s, o);
    if (threads == 32) return s;
    const int warps = threads >> 5;
    if ((t & 31) == 0) part[turn][slot * warps + (t >> 5)] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < warps; ++w) s += part[turn][slot * warps + w];
    return s;
  }
};
// Threads for rows of cols channels, kVecs eights each, at most `most`; and how
// many rows make a block of about 128 threads.
int row_threads(int cols, int vecs, int most) {
  const int t = (cols + 256 * vecs - 1) / (256 * vecs) * 32;
  return t < most ? t : most;
}
int block_rows(int threads) { return threads < 128 ? 128 / threads : 1; }

// The 8-bit copy of eight channels: the scale of the 16 lanes' 128 channels,
// the codes, eight bytes a lane (the row pitch is a multiple of 16, so eight
// are inside the row wherever one is).
template <int kFormat>
__device__ __forceinline__ void keep8(const Codes& k, int64_t row, int c, int cols, const float (&y)[8]) {
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = max(most, code8::magnitude(y[e]));
#pragma unroll
  for (int o = 8; o; o >>= 1) most = max(most, __shfl_xor_sync(kAll, most, o));
  if (c >= cols) return;
  const float scale = code8::group_scale<kFormat>(most), inv = code8::inverse_scale(scale);
  if ((c & (LM_CODE_GROUP - 1)) == 0) k.scales[(int64_t)(c / LM_CODE_GROUP) * k.ld_scales + row] = scale;
  const uint32_t lo = code8::encode2<kFormat>(y[0], y[1], inv) | (code8::encode2<kFormat>(y[2], y[3], inv) << 16);
  const uint32_t hi = code8::encode2<kFormat>(y[4], y[5], inv) | (code8::encode2<kFormat>(y[6], y[7], inv) << 16);
  __stcs(reinterpret_cast<uint2*>(k.data + row * k.ld + c), make_uint2(lo, hi));
}

template <typename T>
__device__ __forceinline__ T* row_of(const Mat& m, int64_t row) {
  return static_cast<T*>(m.data) + row * m.ld;
}

bool aligned(const Mat& m, int size, int64_t nrows) {
  return m.data == nullptr || (reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (nrows == 1 || m.ld * size % 16 == 0));
}

}  // namespace
}  // namespace rows
}  // namespace lm
