// Matrix product on the tensor cores, D = A B^T with bf16 operands: CTA pairs
// (tcgen05.mma, cta_group::2), one 256 x 256 tile of D a pair, 64 of the summed
// dimension at a time, operands by TMA, what happens to a finished tile in an
// epilogue that the caller supplies.
//
// Either operand lies K-major (rows of the summed dimension: one box of 64 x
// 128 rows a CTA) or MN-major (rows of D's dimension, one row an element of the
// sum: two boxes of 64 x 64), as a matrix or in blocks of 64 columns.  CTA r of the pair holds rows 128 r .. of the
// tile (A) and columns 128 r .. (B).
//
// CTA roles (12 warps, one CTA per SM):
//   warp 0      TMA producer (one lane); both CTAs' copies signal CTA 0
//   warp 1      TMEM allocation; MMA issuer (CTA 0, one lane)
//   warps 4-11  epilogue: one TMEM lane quadrant and half of the columns each
//
// Accumulation: the tensor cores drop up to a unit of the last place of the
// accumulator at each addition (16 of the sum), always towards zero, so a sum of
// more than Epi::kChunk blocks (64 each) is cut: the epilogue adds the accumulator, in
// fp32, to sums that it holds in registers while the MMA fills the other one.
//
// Schedule: units of `strip` tiles of one tile row, dealt to the pairs in turn.
// With split sums, as many tiles as fill whole waves go one to a pair; the tiles
// left over are shared, each cut into equal ranges of its sum where that leaves few
// pairs out, else as one line of (tile, block) work cut into equal ranges.  A tile
// that falls to several pairs is summed from their fp32 parts, in order, by a second
// kernel.  Where D has few tile columns, as many pairs walk a tile row together, one
// a column, and what is dealt and cut is tile rows: they read the same blocks of A
// at the same time, from L2 (each column for itself, A came from memory once for
// each: 4096 x 768 over 50304, 284 us).
//
// The whole issuing warp goes through the MMAs' loop, so that what they take is
// uniform, and asks for the next block before this one's: their queue is short, and
// what lies between two blocks' MMAs is not hidden (4096 x 4096 x 50257: 1010 -> 930
// us).  Registers go from the first warpgroup to the epilogue's (setmaxnreg).
//
// Every wait is bounded (LM_WAIT_LIMIT_NS); a tile whose wait gave up, and what
// its CTA had yet to do, reach the epilogue as NaN.
#pragma once

#include <cuda_bf16.h>
#include <cudaTypedefs.h>

#include <algorithm>

#include "lm_ns_tc_shared.cuh"
#include "lm_train.h"

namespace lm {
namespace gemm {
namespace {

using namespace tc;
using tcs::ProducerLog;
using tcs::pair_finish;
using tcs::kCleanupWaitNs;

constexpr int kTileM = 256, kTileN = 256, kBlockK = 64;
constexpr int kHalf = 128;
constexpr int kFirstEpi = 4, kEpiWarps = 8;            // whole warpgroups: a warp reads the TMEM lanes of its number mod 4
constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
constexpr int kLeast = 16;                             // blocks of a split sum's part: the parts and their join cost as much
constexpr int kPairs = 76;                             // CTA pairs of the GPU (152 SMs)
constexpr int kTmemCols = 512;
constexpr int kBoxBytes = 32 * 128;                    // an epilogue warp's 32 rows of 128 bytes (128-byte swizzle), as the TMA stores them
// Shared memory of a CTA: stages, the epilogue warps' boxes, barriers.
// Epi::kRowsA rows of A are loaded and have room: kHalf, or fewer where D has no
// more rows.  The MMA then reads kHalf rows from A's place all the same; the others
// are bytes of B, and the rows of D that they reach are left alone.
template <typename Epi>
struct Smem {
  static constexpr int kA = Epi::kRowsA * kBlockK * 2, kB = kHalf * kBlockK * 2, kStage = kA + kB;
  static_assert(kStage >= kHalf * kBlockK * 2, "what the MMA reads as A is inside the stage");
  static constexpr size_t kBoxes = (size_t)Epi::kStages * kStage;
  static constexpr size_t kBars = kBoxes + (size_t)kEpiWarps * Epi::kBoxes * kBoxBytes;
  static constexpr size_t kBytes = 1024 + kBars + 512;
  static_assert(kBytes <= 232448, "shared memory of one SM");
};
constexpr int kMostSharers = kPairs;

// How the work falls to the pairs.
struct Schedule {
  int32_t tiles_m, tiles_n;
  int32_t nkb;          // blocks of the sum
  int32_t team;         // pairs that take a unit together, one a tile column; 1: each for itself
  int32_t strip;        // tiles of one row taken in turn by one pair
  int32_t strips;       // of a tile row
  int32_t units;        // units dealt to the teams in turn (tile row, strip)
  int32_t rest;         // units left over, shared by range (strip 1)
  int32_t sharers;      // teams that share them; 0: none left over
  int32_t cuts;         // as many to each unit, over equal ranges of its sum; 0: equal ranges of the line
  int64_t begin[kMostSharers + 1];   // sharer k's first (tile, block) in the line of left-over work
};
template <typename Epi>
struct Params {
  CUtensorMap a, b, out;
  Schedule sch;
  int32_t m, n;
  float* parts;
  uint64_t wait_ns;
  Epi epi;
};

// Units run over groups of 8 tile rows, strip by strip, so that the units of a
// wave cover a compact block of D and share its operands in L2.
__device__ __forceinline__ void unit_place(const Schedule& s, int unit, int& tm, int& strip) {
  constexpr int kGroup = 8;
  if (s.team > 1) {     // a unit is a tile row
    tm = unit;
    strip = 0;
    return;
  }
  const int per = kGroup * s.strips, g = unit / per, r = unit - g * per;
  const int rows = min(kGroup, s.tiles_m - g * kGroup);
  strip = r / rows;
  tm = g * kGroup + r - strip * rows;
}
// A pair's work items in order: a tile, its blocks, and where the sum goes.
struct Item {
  int tm, tn, kb0, kb1;
  int slot;             // -1: the whole sum; else part slot of the workspace
  int strip;            // the tile's strip, where the item ends it; else -1 (units dealt in turn)
};
struct Items {
  int pair, column;     // column: this pair's of its team
  int team, unit, tn, tn_end, tm, strip;
  int64_t at, end;      // left-over (unit, block) yet to do
  bool first;
  __device__ __forceinline__ Items(const Schedule& s, int p) : pair(p), column(0), team(p), unit(p), tn(0), tn_end(0), tm(0), strip(0), at(0), end(0), first(true) {
    if (s.team > 1) {
      unit = team = p / s.team;
      column = p - team * s.team;
    }
    if (s.sharers > 0 && team < s.sharers) {
      at = s.begin[team];
      end = s.begin[team + 1];
    }
  }
  __device__ __forceinline__ bool next(const Schedule& s, Item& it) {
    if (tn >= tn_end && unit < s.units) {
      unit_place(s, unit, tm, strip);
      tn = strip * s.strip + column;
      tn_end = min(tn + s.strip, s.tiles_n);
      unit += kPairs / s.team;
    }
    if (tn < tn_end) {
      it = Item{tm, tn, 0, s.nkb, -1, tn + 1 == tn_end ? strip : -1};
      ++tn;
      return true;
    }
    if (at >= end) return false;
    const int t = (int)(at / s.nkb), kb0 = (int)(at - (int64_t)t * s.nkb);
    const int kb1 = (int)min((int64_t)s.nkb, kb0 + (end - at));
    unit_place(s, s.units + t, it.tm, it.tn);
    it.tn += column;
    it.kb0 = kb0;
    it.kb1 = kb1;
    it.slot = (kb0 == 0 && kb1 == s.nkb) ? -1 : 2 * pair + (first ? 0 : 1);
    it.strip = -1;
    at += kb1 - kb0;
    first = false;
    return true;
  }
};

// Bounded wait; false where it gave up.  Without a call: a call would spill the
// sums that the epilogue holds in registers.
__device__ __forceinline__ bool await(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t limit_ns) {
  // the clock is read every 256 probes (each may already sleep a while), at
  // every probe under a limit below a millisecond
  const uint32_t every = limit_ns < 1000000ull ? 0u : 255u;
  uint64_t t0 = 0;
  for (uint32_t i = 0; !mbar_try_wait(bar, parity); ++i) {
    if ((i & every) != every) continue;
    if (*abort_flag) return false;
    const uint64_t now = globaltimer();
    if (t0 == 0) t0 = now;
    else if (now - t0 > limit_ns) return false;
  }
  return true;
}

// 32 columns of the warp's lanes; the values are there after tmem_wait, which
// takes them as its own results so that no use of them moves before it.
__device__ __forceinline__ void tmem_load(uint32_t taddr, float (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32"
      " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15,"
      " %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]),
        "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]),
        "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait(float (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]),
                 "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]), "+f"(r[17]),
                 "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]), "+f"(r[25]), "+f"(r[26]),
                 "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])
               :
               : "memory");
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
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// The issuing warp comes to these as a whole, so that what they take is the same in
// every lane; its leader acts.
__device__ __forceinline__ void umma_by(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t leader, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(smem_u32(bar)),
      "h"((uint16_t)0x3), "r"(leader)
      : "memory");
}
// Whether the phase is over, at once.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

// Arrive on a barrier of CTA 0.  What the arrival announces is TMEM columns of the
// arriving CTA read to the end (tcgen05.wait::ld, fence before_thread_sync).
// Nothing in global memory hangs on it, so the arrival needs no fence of cluster
// scope.
__device__ __forceinline__ void arrive_cta0(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(bar, 0)) : "memory");
}

// 384 threads have 168 registers each at launch; the first warpgroup leaves some
// to the epilogue's two.
template <int kFew>
__device__ __forceinline__ void few_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFew));
}
template <int kFew>
__device__ __forceinline__ void many_registers() {
  constexpr int kMany = (168 * 3 - kFew) / 2 / 8 * 8;
  static_assert(kFew % 8 == 0 && kFew + 2 * kMany <= 168 * 3, "registers of the launch");
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMany));
}

// Where an epilogue warp stands: lane l holds row `row + l` of D, columns
// `col` .. `col` + 127 (of them < n inside).
struct Place {
  int tm, tn;
  int row, col;
  int lane, half;       // half: which 128 columns of the tile
  uint32_t box;         // the warp's boxes (shared address)
};

// Where 16 bytes of a box lie (chunk 0 .. 7 of a row's 128 bytes).
__device__ __forceinline__ uint32_t box_at(uint32_t box, int row, int chunk) { return box + row * 128 + ((chunk ^ (row & 7)) << 4); }
__device__ __forceinline__ void box_put(uint32_t box, int row, int chunk, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box_at(box, row, chunk)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void box_put(uint32_t box, int row, int chunk, const float* v) {
  box_put(box, row, chunk, __float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ float4 box_get(uint32_t box, int row, int chunk) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(box_at(box, row, chunk)) : "memory");
  return v;
}
__device__ __forceinline__ void box_store(const CUtensorMap* map, uint32_t box, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(box),
               "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
// fp32 values added to what is there (one addition an element).
__device__ __forceinline__ void box_add(const CUtensorMap* map, uint32_t box, int c0, int c1, int c2) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(box),
               "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
// The TMA has read the warp's boxes: they may be written again.
__device__ __forceinline__ void box_free(int lane) {
  if (lane == 0) bulk_wait_read();
  __syncwarp();
}
// What the warp wrote into its boxes is there for the TMA (then lane 0 stores and commits).
__device__ __forceinline__ void box_ready() {
  fence_proxy_async_smem();
  __syncwarp();
}

// Four elements of a row, `left` of them inside.
struct Store {
  Mat d;
  int32_t dt;
  int32_t accumulate;   // adds to d
  int32_t vec;          // d takes four elements at a time
  int32_t tma;          // whole tiles go to d by the TMA (a map of it; fp32 may be added)
  __device__ __forceinline__ void put(int64_t row, int col, float4 v, int left) const {
    float e[4] = {v.x, v.y, v.z, v.w};
    const int64_t at = row * d.ld + col;
    if (dt == LM_F32) {
      float* o = static_cast<float*>(d.data) + at;
      if (vec && left >= 4) {
        if (accumulate) {
          const float4 q = *reinterpret_cast<const float4*>(o);
          e[0] += q.x;
          e[1] += q.y;
          e[2] += q.z;
          e[3] += q.w;
        }
        *reinterpret_cast<float4*>(o) = make_float4(e[0], e[1], e[2], e[3]);
        return;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) o[k] = accumulate ? o[k] + e[k] : e[k];
    } else {
      __nv_bfloat16* o = static_cast<__nv_bfloat16*>(d.data) + at;
      if (vec && left >= 4) {
        if (accumulate) {
          const uint2 q = *reinterpret_cast<const uint2*>(o);
          e[0] += bf_lo(q.x);
          e[1] += bf_hi(q.x);
          e[2] += bf_lo(q.y);
          e[3] += bf_hi(q.y);
        }
        *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf2(e[0], e[1]), pack_bf2(e[2], e[3]));
        return;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) o[k] = __float2bfloat16_rn(accumulate ? __bfloat162float(o[k]) + e[k] : e[k]);
    }
  }
};
inline Store make_store(const Mat& d, int dt, int64_t rows, bool accumulate) {
  Store s{};
  s.d = d;
  s.dt = dt;
  s.accumulate = accumulate ? 1 : 0;
  const uintptr_t four = dt == LM_F32 ? 16 : 8;   // bytes of four elements
  s.vec = reinterpret_cast<uintptr_t>(d.data) % four == 0 && (rows == 1 || d.ld % 4 == 0);
  return s;
}

// 32 rows (one a lane) x 32 columns from column c: through a box, then four
// rows a step, four columns a lane.
template <typename Put>
__device__ __forceinline__ void put_block(const float (&v)[32], const Place& at, int rows, int c, const Put& put) {
  const int q = at.lane & 7, r4 = at.lane >> 3;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    box_put(at.box, at.lane, e, v + 4 * e);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = r4 + 4 * k;
    if (r < rows) put(r, c + 4 * q, box_get(at.box, r, q));
  }
  __syncwarp();
}

// 32 rows (one a lane) x 32 columns from column c, stored and not added: four
// columns a lane where D's rows take them, else a row a step and a column a lane,
// so that a row's elements still go out side by side.  One way through the rows,
// without a question an element (dW of 150000 x 2500 over 700 tokens, rows of 5000
// bytes: 909 us with Store::put).
__device__ __forceinline__ void put_plain4(float* o, float4 v) { *reinterpret_cast<float4*>(o) = v; }
__device__ __forceinline__ void put_plain4(__nv_bfloat16* o, float4 v) { *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf2(v.x, v.y), pack_bf2(v.z, v.w)); }
__device__ __forceinline__ void put_plain(float* o, float v) { *o = v; }
__device__ __forceinline__ void put_plain(__nv_bfloat16* o, float v) { *o = __float2bfloat16_rn(v); }
template <typename T>
__device__ __forceinline__ void put_plain_block(const float (&v)[32], const Place& at, int rows, int c, int n, const Store& out) {
#pragma unroll
  for (int e = 0; e < 8; ++e) box_put(at.box, at.lane, e, v + 4 * e);
  __syncwarp();
  T* o = static_cast<T*>(out.d.data) + (int64_t)at.row * out.d.ld + c;
  if (out.vec && c + 32 <= n) {
    const int q = at.lane & 7, r4 = at.lane >> 3;
    o += r4 * out.d.ld + 4 * q;
    const int64_t step = 4 * out.d.ld;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (r4 + 4 * k < rows) put_plain4(o, box_get(at.box, r4 + 4 * k, q));
      o += step;
    }
  } else {
    o += at.lane;
    const bool in = c + at.lane < n;
#pragma unroll 8
    for (int r = 0; r < rows; ++r) {
      float x;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(box_at(at.box, r, at.lane >> 2) + 4 * (at.lane & 3)) : "memory");
      if (in) put_plain(o, x);
      o += out.d.ld;
    }
  }
  __syncwarp();
}

// Epilogue that stores D.
struct StoreEpi {
  static constexpr int kStages = 6, kBoxes = 1, kRowsA = kHalf, kChunk = 8;
  // registers a thread of the first warpgroup: with 136 (and 184) ptxas spills none,
  // with 96 (and 200) 212 bytes (dh of 4096 x 4096 over 50257: 1006 us, 968 so)
  static constexpr int kFewRegs = 136;
  Store out;
  const float* factor;        // of the product, in device memory
  template <typename P>
  struct Warp {
    __device__ __forceinline__ Warp(const P&, const Place&) {}
    __device__ __forceinline__ void tile(const P& p, const Item& it, const Place& at, float (&acc)[4][32]) {
      const int rows = min(32, p.m - at.row);
      const float f = *p.epi.factor;
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 v = mul2(make_float2(acc[b][e], acc[b][e + 1]), make_float2(f, f));
          acc[b][e] = v.x;
          acc[b][e + 1] = v.y;
        }
      if (it.slot < 0 && p.epi.out.tma) {
        if (rows <= 0) return;
        if (p.epi.out.dt == LM_F32) {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int c = at.col + 32 * b;
            if (c >= p.n) continue;
            box_free(at.lane);
#pragma unroll
            for (int e = 0; e < 8; ++e) box_put(at.box, at.lane, e, &acc[b][4 * e]);
            box_ready();
            if (at.lane == 0) {
              if (p.epi.out.accumulate) box_add(&p.out, at.box, c, at.row, 0);
              else box_store(&p.out, at.box, c, at.row, 0);
              bulk_commit();
            }
          }
        } else {
#pragma unroll
          for (int b = 0; b < 4; b += 2) {
            const int c = at.col + 32 * b;
            if (c >= p.n) continue;
            box_free(at.lane);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float* v = &acc[b + e / 4][8 * (e % 4)];
              box_put(at.box, at.lane, e, pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7]));
            }
            box_ready();
            if (at.lane == 0) {
              box_store(&p.out, at.box, c, at.row, 0);
              bulk_commit();
            }
          }
        }
        return;
      }
      box_free(at.lane);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = at.col + 32 * b;
        if (c >= p.n || rows <= 0) continue;
        if (it.slot >= 0) {
          float* part = p.parts + (size_t)it.slot * (kTileM * kTileN);
          const int r0 = at.row - at.tm * kTileM, c0 = at.tn * kTileN;
          put_block(acc[b], at, rows, c, [&](int r, int col, float4 v) {
            *reinterpret_cast<float4*>(part + (size_t)(r0 + r) * kTileN + (col - c0)) = v;
          });
        } else if (!p.epi.out.accumulate) {
          if (p.epi.out.dt == LM_F32) put_plain_block<float>(acc[b], at, rows, c, p.n, p.epi.out);
          else put_plain_block<__nv_bfloat16>(acc[b], at, rows, c, p.n, p.epi.out);
        } else {
          put_block(acc[b], at, rows, c, [&](int r, int col, float4 v) {
            if (col < p.n) p.epi.out.put(at.row + r, col, v, p.n - col);
          });
        }
      }
    }
  };
};

// How an operand lies: K-major, MN-major, or MN-major's or K-major's elements in
// column blocks of 64 (block, row, 64: each TMA box is one piece of memory).
enum Lie { kRowsK = 0, kRowsMn = 1, kBlocksK = 2, kBlocksMn = 3 };
__host__ __device__ constexpr bool is_mn(int lie) { return (lie & 1) != 0; }
__host__ __device__ constexpr bool is_blocks(int lie) { return lie >= 2; }

// 3-D tiled TMA load, signalled like tma_load_3d, with an L2 policy.
__device__ __forceinline__ void load_box(void* dst, const CUtensorMap* map, uint32_t bar_cluster, int c0, int c1, int c2, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster), "r"(c0), "r"(c1), "r"(c2), "l"(policy)
      : "memory");
}
// What is read once goes from L2 first, what every pair reads last.
__device__ __forceinline__ uint64_t once_policy() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t often_policy() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}

// One K block (kb) of an operand's half tile from row or column `mn` on.
template <int kLie>
__device__ __forceinline__ void load_operand(uint8_t* dst, const CUtensorMap* map, uint32_t bar, int mn, int kb, uint64_t policy) {
  constexpr int kBytes = kHalf * kBlockK * 2;
  if (kLie == kRowsK) load_box(dst, map, bar, kb * kBlockK, mn, 0, policy);
  if (kLie == kBlocksK) load_box(dst, map, bar, 0, mn, kb, policy);
  if (kLie == kRowsMn) {
    load_box(dst, map, bar, mn, kb * kBlockK, 0, policy);
    load_box(dst + kBytes / 2, map, bar, mn + 64, kb * kBlockK, 0, policy);
  }
  if (kLie == kBlocksMn) {
    load_box(dst, map, bar, 0, kb * kBlockK, mn / 64, policy);
    load_box(dst + kBytes / 2, map, bar, 0, kb * kBlockK, mn / 64 + 1, policy);
  }
}

template <int kALie, int kBLie, typename Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) gemm_kernel(const __grid_constant__ Params<Epi> p) {
  constexpr int kChunk = Epi::kChunk;
  constexpr int kStages = Epi::kStages, kABytes = Smem<Epi>::kA, kBBytes = Smem<Epi>::kB, kStageBytes = Smem<Epi>::kStage;
  static_assert(Epi::kRowsA == kHalf || kALie == kRowsK, "fewer rows are rows of a box");
  constexpr bool kAMn = is_mn(kALie), kBMn = is_mn(kBLie);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + Smem<Epi>::kBars);
  uint64_t* empty = full + kStages;
  uint64_t* accfull = empty + kStages;
  uint64_t* accempty = accfull + 2;
  uint64_t* done = accempty + 2;
  ProducerLog<kStages>* log = reinterpret_cast<ProducerLog<kStages>*>(done + 1);
  int* armed = reinterpret_cast<int*>(log + 1);       // last phase CTA 0 armed on each stage, or -1 (producer lane)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(armed + kStages);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1;
  const Schedule& sch = p.sch;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
      armed[s] = -1;
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&accfull[b], 1);
      mbar_init(&accempty[b], 2 * kEpiWarps);
    }
    mbar_init(done, 1);
    log->n = 0;
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  cluster_sync();   // barriers of both CTAs initialised
  tc_fence_after();
  griddep_wait();   // the operands are there
  griddep_launch_dependents();
  const uint32_t tmem_base = *tmem_slot;
  const uint64_t wait_ns = p.wait_ns;

  if (warp == 0) {
    // -------------------------------- producer ---------------------------------
    few_registers<Epi::kFewRegs>();
    if (lane == 0) {
      int stage = 0;
      uint32_t ph = 0;
      bool ok = true;
      // A in blocks is a passing value (the gradient's d), larger than L2
      const uint64_t often = often_policy(), a_policy = is_blocks(kALie) ? once_policy() : often;
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        const int row = it.tm * kTileM + (int)rank * kHalf, col = it.tn * kTileN + (int)rank * kHalf;
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
          if (!await(&empty[stage], ph ^ 1u, abort_flag, wait_ns)) {
            ok = false;
            break;
          }
          uint8_t* sa = smem + (size_t)stage * kStageBytes;
          uint8_t* sb = sa + kABytes;
          const uint32_t fb = peer_addr(&full[stage], 0);
          if (rank == 0) {
            mbar_arrive_expect_tx(&full[stage], 2u * kStageBytes);
            armed[stage] = (int)ph;
          }
          log->bytes[stage] = kStageBytes;
          log->n += 1u;
          load_operand<kALie>(sa, &p.a, fb, row, kb, a_policy);
          load_operand<kBLie>(sb, &p.b, fb, col, kb, often);
          if (++stage == kStages) {
            stage = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok) *abort_flag = 1;
    }
  } else if (warp == 1) {
    // -------------------------------- MMA issuer -------------------------------
    few_registers<Epi::kFewRegs>();
    if (rank == 0) {
      constexpr uint32_t idesc = make_idesc(kTileM, kTileN, kAMn, kBMn);
      // 16 of the sum: 16 rows of 128 bytes (MN-major), 32 bytes of a row (K-major)
      constexpr uint64_t a_step = (kAMn ? 2048 : 32) >> 4, b_step = (kBMn ? 2048 : 32) >> 4;
      const uint32_t leader = lane == 0 ? 1u : 0u, smem0 = smem_u32(smem), tmem0 = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
      int stage = 0, ab = 0;
      uint32_t ph = 0, aph = 0;
      bool ok = true, ready = false;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (!__all_sync(0xFFFFFFFFu, await(bar, parity, abort_flag, wait_ns))) ok = false;
        return ok;
      };
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        for (int kc = it.kb0; ok && kc < it.kb1;) {
          const int ke = min(kc + kChunk, it.kb1);
          if (!wait(&accempty[ab], aph ^ 1u)) break;
          tc_fence_after();
          const uint32_t d = tmem0 + (uint32_t)(ab * kTileN);
          for (int kb = kc; kb < ke; ++kb) {
            if (!ready && !wait(&full[stage], ph)) break;
            tc_fence_after();
            const uint32_t sa = smem0 + (uint32_t)(stage * kStageBytes);
            const uint64_t a0 = sw128_desc(sa, kAMn ? kABytes / 2 : 16, 1024), b0 = sw128_desc(sa + kABytes, kBMn ? kBBytes / 2 : 16, 1024);
            uint64_t* const free = &empty[stage];
            // Whether the next block is there is asked now and known after this
            // block's MMAs: the answer comes late, behind what they read of shared
            // memory, and their queue is short.
            if (++stage == kStages) {
              stage = 0;
              ph ^= 1u;
            }
            const bool there = mbar_test(&full[stage], ph);
#pragma unroll
            for (int kk = 0; kk < kBlockK / 16; ++kk)
              umma_by(leader, d, a0 + kk * a_step, b0 + kk * b_step, idesc, (kb == kc && kk == 0) ? 0u : 1u);
            commit_pair(leader, free);
            ready = __all_sync(0xFFFFFFFFu, there);
          }
          if (!ok) break;
          commit_pair(leader, &accfull[ab]);
          ab ^= 1;
          if (ab == 0) aph ^= 1u;
          kc = ke;
        }
      }
      if (leader) {
        if (!ok) *abort_flag = 1;
        umma_commit_local(done);   // all issued MMAs complete before TMEM is released
        volatile int never = 0;
        await(done, 0, &never, kCleanupWaitNs);
      }
    }
  } else if (warp >= kFirstEpi) {
    // --------------------------------- epilogue ----------------------------------
    many_registers<Epi::kFewRegs>();
    Place at;
    at.lane = lane;
    at.half = (warp - kFirstEpi) >> 2;
    at.box = smem_u32(smem + Smem<Epi>::kBoxes + (size_t)(warp - kFirstEpi) * Epi::kBoxes * kBoxBytes);
    const int q = warp & 3, r0 = (int)rank * kHalf + q * 32;      // the warp's first row of the tile
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const float nan = __int_as_float(0x7FC00000);
    int ab = 0;
    uint32_t aph = 0;
    bool ok = true;
    Items items(sch, pair);
    Item it;
    at.tm = at.tn = at.row = at.col = 0;
    typename Epi::template Warp<Params<Epi>> epi(p, at);
    while (items.next(sch, it)) {
      at.tm = it.tm;
      at.tn = it.tn;
      at.row = it.tm * kTileM + r0;
      at.col = it.tn * kTileN + at.half * 128;
      float acc[4][32];
      for (int kc = it.kb0; kc < it.kb1; kc += kChunk) {
        // one answer for the warp: the TMEM loads below are taken by all lanes or none
        ok = ok && __all_sync(0xFFFFFFFFu, await(&accfull[ab], aph, abort_flag, wait_ns));
        if (!ok) {
          *abort_flag = 1;
          break;
        }
        tc_fence_after();
        const uint32_t from = tmem_base + (uint32_t)(ab * kTileN + at.half * 128) + lanes;
        if (kc == it.kb0) {
#pragma unroll
          for (int b = 0; b < 4; ++b) tmem_load(from + 32 * b, acc[b]);
#pragma unroll
          for (int b = 0; b < 4; ++b) tmem_wait(acc[b]);
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            float r[32];
            tmem_load(from + 32 * b, r);
            tmem_wait(r);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 v = add2(make_float2(acc[b][e], acc[b][e + 1]), make_float2(r[e], r[e + 1]));
              acc[b][e] = v.x;
              acc[b][e + 1] = v.y;
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_cta0(&accempty[ab]);
        ab ^= 1;
        if (ab == 0) aph ^= 1u;
      }
      if (!ok) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = nan;
      }
      epi.tile(p, it, at, acc);
    }
    if (lane == 0) bulk_wait_all();   // stores from the boxes
  } else {
    few_registers<Epi::kFewRegs>();
  }

  __syncwarp();
  pair_finish<kStages>(*log, abort_flag, full, armed, rank);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
}

// Left-over tiles that several pairs shared: the parts added in the order of
// the sum, then stored like a whole tile.
struct JoinParts {
  Schedule sch;
  int32_t m, n;
  const float* parts;
  Store out;
};
template <int kN>
__global__ void __launch_bounds__(kN) join_kernel(const __grid_constant__ JoinParts p) {
  constexpr int kRow = kN / 4;      // threads of a row; four rows a block
  const Schedule& s = p.sch;
  const int t = blockIdx.x;
  griddep_wait();
  griddep_launch_dependents();
  const int64_t u0 = (int64_t)t * s.nkb, u1 = u0 + s.nkb;
  int k = (int)((int64_t)t * s.sharers / s.rest);   // the sharer whose range holds unit u0
  while (k > 0 && s.begin[k] > u0) --k;
  while (s.begin[k + 1] <= u0) ++k;
  if (s.begin[k] <= u0 && s.begin[k + 1] >= u1) return;   // one pair stored it whole
  int tm, tn;
  unit_place(s, s.units + t, tm, tn);
  const int column = blockIdx.z;
  tn += column;
  int last = k;   // the last sharer of the tile
  while (last + 1 < s.sharers && s.begin[last + 1] < u1) ++last;
  const int rows = min(kTileM, p.m - tm * kTileM), cols = min(kN, p.n - tn * kN);
  // the first part may be its pair's second item; every later one is a first
  const float* part0 = p.parts + (size_t)(2 * (k * s.team + column) + (s.begin[k] >= u0 ? 0 : 1)) * (kTileM * kN);
  const int r = blockIdx.y * 4 + (threadIdx.x / kRow), c = 4 * (threadIdx.x % kRow);
  if (r >= rows || c >= cols) return;
  const size_t at = (size_t)r * kN + c;
  float4 sum = *reinterpret_cast<const float4*>(part0 + at);
#pragma unroll 4
  for (int j = k + 1; j <= last; ++j) {
    const float4 v = *reinterpret_cast<const float4*>(p.parts + (size_t)(2 * (j * s.team + column)) * (kTileM * kN) + at);
    sum.x += v.x;
    sum.y += v.y;
    sum.z += v.z;
    sum.w += v.w;
  }
  p.out.put(tm * kTileM + r, tn * kN + c, sum, cols - c);
}

// D of an empty sum.
__global__ void __launch_bounds__(256) zero_kernel(Mat d, int dt, int64_t rows, int cols) {
  griddep_wait();
  griddep_launch_dependents();
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += 256) {
      if (dt == LM_F32) static_cast<float*>(d.data)[r * d.ld + c] = 0.f;
      else static_cast<__nv_bfloat16*>(d.data)[r * d.ld + c] = __float2bfloat16_rn(0.f);
    }
}

inline PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = []() {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                    q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f) : nullptr;
  }();
  return fn;
}

// A map of (cols, rows, planes) elements whose boxes are 128 bytes x box_rows, 128-byte swizzle.
inline cudaError_t encode_boxes(CUtensorMap* m, int dt, const void* base, int64_t cols, int64_t rows, int64_t planes, int64_t ld, int64_t plane, int box_rows) {
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
  if (enc == nullptr) return cudaErrorNotSupported;
  const cuuint64_t size = dt == LM_F32 ? 4 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)ld * size, (cuuint64_t)plane * size};
  const cuuint32_t box[3] = {dt == LM_F32 ? 32u : 64u, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
  return enc(m, dt == LM_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}
// The rows of a bf16 matrix as an operand, and its 64-column blocks (block, row, 64).
inline cudaError_t encode_operand(CUtensorMap* m, const void* base, int64_t cols, int64_t rows, int64_t ld, bool mn_major, int box_rows = kHalf) {
  return encode_boxes(m, LM_BF16, base, cols, rows, 1, ld, ld * rows, mn_major ? 64 : box_rows);
}
inline cudaError_t encode_blocks(CUtensorMap* m, const void* base, int64_t cols, int64_t rows, int box_rows) {
  return encode_boxes(m, LM_BF16, base, 64, rows, (cols + 63) / 64, 64, 64 * rows, box_rows);
}

// Whether the TMA takes the rows of a bf16 matrix as they lie.
inline bool tma_rows(const Mat& m, int64_t rows, int64_t cols) {
  return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (rows > 1 ? m.ld % 8 == 0 : cols % 8 == 0);
}

// Units of `strip` tiles dealt in turn, no sum split.
inline Schedule plain_schedule(int64_t m, int64_t n, int64_t k, int strip, int tile_n = kTileN, int block_k = kBlockK) {
  Schedule s{};
  s.tiles_m = (int32_t)((m + kTileM - 1) / kTileM);
  s.tiles_n = (int32_t)((n + tile_n - 1) / tile_n);
  s.nkb = (int32_t)((k + block_k - 1) / block_k);
  s.team = 1;
  s.strip = strip;
  s.strips = (s.tiles_n + strip - 1) / strip;
  s.units = s.tiles_m * s.strips;
  return s;
}
// Whole waves of units, the rest shared by ranges of the sum.
constexpr int kMostTeam = 8;      // where more columns would leave many pairs out, each is for itself
inline Schedule split_schedule(int64_t m, int64_t n, int64_t k, int tile_n = kTileN, int block_k = kBlockK, int least = kLeast) {
  Schedule s = plain_schedule(m, n, k, 1, tile_n, block_k);
  if (s.tiles_n <= kMostTeam && s.tiles_m > 1) {
    s.team = s.tiles_n;
    s.strips = 1;
    s.units = s.tiles_m;
  }
  const int32_t all = s.units, teams = kPairs / s.team;
  s.units = all / teams * teams;
  s.rest = all - s.units;
  if (s.rest > 0) {
    // a share of at least `least` blocks, and never more sharers than teams
    const int64_t most = (int64_t)s.rest * s.nkb / least;
    s.sharers = (int32_t)(most < s.rest ? s.rest : most < teams ? most : teams);
    // Equal cuts of every unit, where they leave few teams out: those of one range of
    // the sum then read the same blocks of A and B at the same time, from L2 (dh of
    // 700 x 2500 over 150000: 723 us with equal ranges of the line, each operand from
    // memory several times).
    const int32_t cuts = (int32_t)std::min<int64_t>(teams / s.rest, std::max<int64_t>(1, s.nkb / least));
    if (4 * s.rest * cuts >= 3 * s.sharers) {
      s.cuts = cuts;
      s.sharers = s.rest * cuts;
    }
  }
  return s;
}
// Where the sharers' ranges begin (for the launch alone).
inline void share(Schedule& s) {
  for (int k = 0; s.sharers > 0 && k <= s.sharers; ++k)
    s.begin[k] = s.cuts > 0 ? (int64_t)(k / s.cuts) * s.nkb + (int64_t)s.nkb * (k % s.cuts) / s.cuts : (int64_t)s.rest * s.nkb * k / s.sharers;
}
inline bool has_parts(const Schedule& s) { return s.rest > 0 && s.sharers > s.rest; }
inline size_t parts_bytes(const Schedule& s, int tile_n = kTileN) { return has_parts(s) ? 2 * (size_t)s.sharers * s.team * kTileM * tile_n * 4 : 0; }
inline int pairs_of(const Schedule& s) { return std::min(kPairs / s.team, std::max(s.units, s.sharers)) * s.team; }

// A launch whose set-up may overlap the end of the kernel before it (which it
// waits for itself, griddepcontrol.wait).
template <typename Kernel, typename... Args>
cudaError_t launch_after(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int kALie, int kBLie, typename Epi>
cudaError_t start(const Params<Epi>& p, cudaStream_t st) {
  const int dev = device_slot();
  static bool ready[kMaxDevices];
  if (dev < 0 || !ready[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(gemm_kernel<kALie, kBLie, Epi>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Smem<Epi>::kBytes);
    if (e != cudaSuccess) return e;
    if (dev >= 0) ready[dev] = true;
  }
  return launch_after(gemm_kernel<kALie, kBLie, Epi>, dim3(2 * pairs_of(p.sch)), kThreads, Smem<Epi>::kBytes, st, p);
}
inline cudaError_t start_zero(const Mat& d, int dt, int64_t rows, int cols, cudaStream_t st) {
  return launch_after(zero_kernel, dim3((unsigned)std::min<int64_t>(rows, 152 * 8)), 256, 0, st, d, dt, rows, cols);
}
template <int kN>
cudaError_t start_join(const Schedule& s, int32_t m, int32_t n, const float* parts, const Store& out, cudaStream_t st) {
  const JoinParts j{s, m, n, parts, out};
  return launch_after(join_kernel<kN>, dim3(s.rest, kTileM / 4, s.team), kN, 0, st, j);
}
// Whether the TMA may store a result's tiles: it stores rows in whole 16 bytes, past
// the last column of a row that ends between them, over what a wider buffer has there.
inline bool tma_stores(const void* data, int64_t rows, int64_t cols, int64_t ld, int64_t size) {
  return reinterpret_cast<uintptr_t>(data) % 16 == 0 && ld * size % 16 == 0 && cols * size % 16 == 0 && ld < ((int64_t)1 << 37) / rows;
}
// A product whose sums may be split: the kernel, and the join where parts are left.
template <int kALie, int kBLie>
cudaError_t start_store(Params<StoreEpi>& p, cudaStream_t st) {
  share(p.sch);
  const Store& o = p.epi.out;
  const int64_t size = o.dt == LM_F32 ? 4 : 2;
  cudaError_t e = cudaSuccess;
  const int64_t ld = p.m > 1 ? o.d.ld : (int64_t)p.n;
  if ((!o.accumulate || o.dt == LM_F32) && tma_stores(o.d.data, p.m, p.n, ld, size)) {
    e = encode_boxes(&p.out, o.dt, o.d.data, p.n, p.m, 1, ld, ld * p.m, 32);
    p.epi.out.tma = 1;
  }
  if (e == cudaSuccess) e = start<kALie, kBLie, StoreEpi>(p, st);
  if (e != cudaSuccess || !has_parts(p.sch)) return e;
  return start_join<kTileN>(p.sch, p.m, p.n, p.parts, p.epi.out, st);
}

}  // namespace
}  // namespace gemm
}  // namespace lm
