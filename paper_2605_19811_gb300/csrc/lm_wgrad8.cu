// Weight gradient of a linear layer whose input was kept in 8 bits:
//   dW (+)= dY^T X,   dW: out x in, dY: T x out, X = code * scale: T x in
// (lm_linear_wgrad8 in lionmuon.h) on the tensor cores: tcgen05.mma on CTA
// pairs, one 256 x 256 tile of dW per pair, a sum over tokens 64 at a time.
//
// A code times its power-of-two scale is a bf16 number, so a first kernel
// writes X as bf16 into the workspace without a rounding; dY is taken as it is
// (bf16), or laid out as three bf16 planes whose sum is the fp32 value (8 + 8 +
// 8 significant bits, summed as three times as many tokens; below 2^-110 the
// last ones pass bf16's least number, 2^-133).  Every product is then exact and
// only the sums are rounded.
// (The codes made bf16 inside the product's kernel, by warps of their own,
// cost more: the conversion shares the shared memory's bandwidth with the MMA,
// 440 ns instead of 350 for a pair's 64 tokens.)
//
// Measured (X made bf16, product, join; kernels alone): 16384 x 768 x 2304
// e4m3 to bf16 10 + 54 + 9 us, a call 64 us; 16384 x 4096 x 14336 int8 to fp32
// 42 + 1076 + 12 us, a call 1117 to 1140 us by itself (1.7 PFLOP/s) and 1230 to
// 1290 us among others (1.5); 16384 x 4096 x 4096 from bf16 dY 362 us, from fp32
// 1210 us.  Bound by the tensor pipe where dW has many tiles, else by the three
// launches.
//
// Both operands lie token by token in memory, so both are MN-major: rows of
// 64 channels (128 bytes, 128-byte swizzle), one row a token.  CTA r of the
// pair holds output channels 128 r .. of the tile (A, from dY) and input
// channels 128 r .. (B, from X), both by TMA.
//
// CTA roles (12 warps, one CTA per SM):
//   warp 0      TMA producer (one lane); both CTAs' copies signal CTA 0
//   warp 1      TMEM allocation; MMA issuer (CTA 0, one lane)
//   warps 4-11  epilogue: one TMEM lane quadrant and half of the columns each
//
// Accumulation: the tensor cores drop up to a unit of the last place of the
// accumulator at each addition (16 tokens), always towards zero, so what a long
// sum loses grows with its length (left in TMEM to its end, 16384 tokens of fp32
// dY lost 5e-5 to 7e-5 of a result).  A sum of more than kChunk blocks (512
// tokens, at most 2^-19 of them lost on average) is therefore cut every kChunk
// blocks, for bf16 results too: the epilogue adds the accumulator, in fp32, to
// sums it holds in registers while the MMA fills the other accumulator.  That
// costs a bf16 result 3 to 10% (16384 x 4096 x 14336: 1091 -> 1130 us).
//
// Schedule: as many tiles as fill whole waves of the pairs go one to a pair.
// The tiles left over are one line of (tile, token block) work cut into equal
// ranges, one a pair; a tile that falls to several pairs is summed from their
// fp32 parts, in order, by a second kernel.
//
// Every wait is bounded (LM_WAIT_LIMIT_NS).  A tile whose wait gave up, and
// what its CTA had yet to write, is filled with NaN.
#include <cuda_bf16.h>
#include <cudaTypedefs.h>
#include <math.h>

#include <algorithm>

#include "lm_code8.cuh"
#include "lm_ns_tc_shared.cuh"
#include "lm_train.h"

namespace lm {
namespace {

using namespace tc;
using tcs::ProducerLog;
using tcs::pair_finish;
using tcs::kCleanupWaitNs;

constexpr int kTileM = 256, kTileN = 256, kBlockK = 64;
constexpr int kHalf = 128;
constexpr int kABytes = kHalf * kBlockK * 2, kBBytes = kHalf * kBlockK * 2;
constexpr int kStages = 6, kStageBytes = kABytes + kBBytes;
constexpr int kFirstEpi = 4, kEpiWarps = 8;            // whole warpgroups: a warp reads the TMEM lanes of its number mod 4
constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
constexpr int kChunk = 8;                              // most token blocks summed in one accumulator
constexpr int kPairs = 76;                             // CTA pairs of the GPU (152 SMs)
constexpr int kTmemCols = 512;
constexpr int kTransBytes = 32 * 20 * 4;               // an epilogue warp's transpose tile: 32 rows x 16 columns, 80-byte rows
constexpr size_t kTransOffset = (size_t)kStages * kStageBytes;
constexpr size_t kBarOffset = kTransOffset + (size_t)kEpiWarps * kTransBytes;
constexpr size_t kSmemBytes = 1024 + kBarOffset + 512;
static_assert(kSmemBytes <= 232448, "shared memory of one SM");
constexpr size_t kPartBytes = (size_t)kTileM * kTileN * 4;

// How the work falls to the pairs.
struct Schedule {
  int32_t tiles_m, tiles_n;
  int32_t nkb;          // token blocks of a tile (three times as many for fp32 dY)
  int32_t nkb_plane;    // token blocks of one plane of dY
  int32_t waves;        // whole waves: tiles [0, waves * kPairs) go one to a pair
  int32_t rest;         // tiles left over
  int32_t sharers;      // pairs that share them; 0: none left over
  int64_t begin[kPairs + 1];   // sharer k's first unit (tile, token block) in the line of left-over work
};
struct KernelParams {
  CUtensorMap dy, x;
  Schedule sch;
  int32_t out, in;
  Mat dw;
  int32_t dwdt;
  int32_t accumulate;
  int32_t vec;          // dW takes four elements at a time
  float* parts;
  uint64_t wait_ns;
};

// Tile indices run over groups of 8 tile rows, column by column, so that the
// tiles of a wave cover a compact block of dW and share its operands in L2.
__device__ __forceinline__ void tile_place(const Schedule& s, int tile, int& tm, int& tn) {
  constexpr int kGroup = 8;
  const int per = kGroup * s.tiles_n, g = tile / per, r = tile - g * per;
  const int rows = min(kGroup, s.tiles_m - g * kGroup);
  tn = r / rows;
  tm = g * kGroup + r - tn * rows;
}
// A pair's work items in order: a tile, its token blocks, and where the sum goes.
struct Item {
  int tile, kb0, kb1;
  int slot;             // -1: the whole tile, straight to dW; else part slot of the workspace
};
struct Items {
  int pair, wave;
  int64_t at, end;      // left-over units yet to do
  bool first;
  __device__ __forceinline__ Items(const Schedule& s, int p) : pair(p), wave(0), at(0), end(0), first(true) {
    if (s.sharers > 0 && p < s.sharers) {
      at = s.begin[p];
      end = s.begin[p + 1];
    }
  }
  __device__ __forceinline__ bool next(const Schedule& s, Item& it) {
    if (wave < s.waves) {
      it = Item{wave * kPairs + pair, 0, s.nkb, -1};
      ++wave;
      return true;
    }
    if (at >= end) return false;
    const int t = (int)(at / s.nkb), kb0 = (int)(at - (int64_t)t * s.nkb);
    const int kb1 = (int)min((int64_t)s.nkb, kb0 + (end - at));
    it = Item{s.waves * kPairs + t, kb0, kb1, (kb0 == 0 && kb1 == s.nkb) ? -1 : 2 * pair + (first ? 0 : 1)};
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

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32"
      " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

// Arrive on a barrier of CTA 0.  What the arrival announces is TMEM columns of the
// arriving CTA read to the end (tcgen05.wait::ld, fence before_thread_sync).
// Nothing in global memory hangs on it, so the arrival needs no fence of cluster
// scope; with one (.release.cluster) it took 1300 cycles, against 512 of a token
// block's MMA.
__device__ __forceinline__ void arrive_cta0(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(bar, 0)) : "memory");
}

// Four codes (one word) to four bf16 values times the scale (twice in s2).
template <int kFormat>
__device__ __forceinline__ uint2 convert4(uint32_t w, uint32_t s2) {
  uint32_t r[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __nv_bfloat162 v;
    if (kFormat == LM_CODE_I8) {
      // 0x43 above the code: 128 + its low seven bits; the sign bit selects 128
      // or 256 to take away (128 + (b & 127)) - (b & 128 ? 256 : 128), exactly
      const uint32_t x = __byte_perm(w, 0x43434343u, h == 0 ? 0x4140 : 0x4342);
      const uint32_t c = x & 0xFF7FFF7Fu, b = x & 0xFF80FF80u;
      v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&c), *reinterpret_cast<const __nv_bfloat162*>(&b));
    } else {
      // exponent and fraction moved to a bf16's places: the value times 2^-120
      const uint32_t x = __byte_perm(w, 0u, h == 0 ? 0x1404 : 0x3424);
      const uint32_t c = ((x >> 4) & 0x07F007F0u) | (x & 0x80008000u);
      const uint32_t k = 0x7B807B80u;   // 2^120
      v = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&c), *reinterpret_cast<const __nv_bfloat162*>(&k));
    }
    v = __hmul2(v, *reinterpret_cast<const __nv_bfloat162*>(&s2));
    r[h] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint2(r[0], r[1]);
}

__device__ __forceinline__ void put_dw(const KernelParams& p, int64_t at, float v) {
  if (p.dwdt == LM_F32) {
    float* d = static_cast<float*>(p.dw.data) + at;
    *d = p.accumulate ? *d + v : v;
  } else {
    __nv_bfloat16* d = static_cast<__nv_bfloat16*>(p.dw.data) + at;
    *d = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*d) + v : v);
  }
}

// Four elements of a row of dW, `left` of them inside.
__device__ __forceinline__ void put_dw4(const KernelParams& p, int64_t at, float4 v, int left) {
  if (!p.vec || left < 4) {
    const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) put_dw(p, at + k, e[k]);
  } else if (p.dwdt == LM_F32) {
    float4* d = reinterpret_cast<float4*>(static_cast<float*>(p.dw.data) + at);
    if (p.accumulate) {
      const float4 o = *d;
      v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
    }
    *d = v;
  } else {
    uint2* d = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.dw.data) + at);
    if (p.accumulate) {
      const uint2 o = *d;
      v = make_float4(bf_lo(o.x) + v.x, bf_hi(o.x) + v.y, bf_lo(o.y) + v.z, bf_hi(o.y) + v.w);
    }
    *d = make_uint2(pack_bf2(v.x, v.y), pack_bf2(v.z, v.w));
  }
}

// 32 rows (one a lane) x 32 columns of a tile, row r0 / column c0 of the tile:
// through the warp's transpose tile, 16 columns at a time, then eight rows a
// step, four columns a lane.
__device__ __forceinline__ void put_block(const KernelParams& p, const Item& it, int tm, int tn, int r0, int c0,
                                          const float (&v)[32], float* stg, int lane) {
  const int row0 = tm * kTileM + r0, rows = min(32, p.out - row0);
  const int q = 4 * (lane & 3), r8 = lane >> 2;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<float4*>(stg + lane * 20 + e) = make_float4(v[16 * h + e], v[16 * h + e + 1], v[16 * h + e + 2], v[16 * h + e + 3]);
    __syncwarp();
    const int c = c0 + 16 * h + q, left = p.in - (tn * kTileN + c);
    if (left > 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = r8 + 8 * k;
        const float4 x = *reinterpret_cast<const float4*>(stg + r * 20 + q);
        if (r >= rows) continue;
        if (it.slot >= 0) *reinterpret_cast<float4*>(p.parts + (size_t)it.slot * (kTileM * kTileN) + (size_t)(r0 + r) * kTileN + c) = x;
        else put_dw4(p, (int64_t)(row0 + r) * p.dw.ld + tn * kTileN + c, x, left);
      }
    }
    __syncwarp();
  }
}

// kLong: some item sums more than kChunk token blocks, and the sums are cut.  Where
// none does, the accumulator is stored as it is (512 x 768 x 50304, bf16: 56 us so,
// 70 through the registers' sums).
template <bool kLong>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) wgrad8_kernel(const __grid_constant__ KernelParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + kBarOffset);
  uint64_t* empty = full + kStages;
  uint64_t* accfull = empty + kStages;
  uint64_t* accempty = accfull + 2;
  uint64_t* done = accempty + 2;
  ProducerLog<kStages>* log = reinterpret_cast<ProducerLog<kStages>*>(done + 1);
  int* armed = reinterpret_cast<int*>(log + 1);       // last phase CTA 0 armed on each stage, or -1 (producer lane)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(armed + kStages);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
    if (lane == 0) {
      int stage = 0;
      uint32_t ph = 0;
      bool ok = true;
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        int tm, tn;
        tile_place(sch, it.tile, tm, tn);
        const int row = tm * kTileM + (int)rank * kHalf, col = tn * kTileN + (int)rank * kHalf;
        int plane = it.kb0 / sch.nkb_plane, tb = it.kb0 - plane * sch.nkb_plane;
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
          tma_load_3d(sa, &p.dy, fb, row, tb * kBlockK, plane);
          tma_load_3d(sa + kABytes / 2, &p.dy, fb, row + 64, tb * kBlockK, plane);
          tma_load_3d(sb, &p.x, fb, col, tb * kBlockK, 0);
          tma_load_3d(sb + kBBytes / 2, &p.x, fb, col + 64, tb * kBlockK, 0);
          if (++tb == sch.nkb_plane) {
            tb = 0;
            ++plane;
          }
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
    if (lane == 0 && rank == 0) {
      const uint32_t idesc = make_idesc(kTileM, kTileN, true, true);
      int stage = 0, ab = 0;
      uint32_t ph = 0, aph = 0;
      bool ok = true;
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        for (int kc = it.kb0; ok && kc < it.kb1;) {
          const int ke = kLong ? min(kc + kChunk, it.kb1) : it.kb1;
          if (!await(&accempty[ab], aph ^ 1u, abort_flag, wait_ns)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem_base + (uint32_t)(ab * kTileN);
          for (int kb = kc; kb < ke; ++kb) {
            if (!await(&full[stage], ph, abort_flag, wait_ns)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t sa = smem_u32(smem + (size_t)stage * kStageBytes);
            const uint64_t a0 = sw128_desc(sa, kABytes / 2, 1024), b0 = sw128_desc(sa + kABytes, kBBytes / 2, 1024);
#pragma unroll
            for (int kk = 0; kk < kBlockK / 16; ++kk)
              umma_bf16(d, a0 + (uint64_t)(kk * 2048 >> 4), b0 + (uint64_t)(kk * 2048 >> 4), idesc, (kb == kc && kk == 0) ? 0u : 1u);
            umma_commit_pair(&empty[stage]);
            if (++stage == kStages) {
              stage = 0;
              ph ^= 1u;
            }
          }
          if (!ok) break;
          umma_commit_pair(&accfull[ab]);
          ab ^= 1;
          if (ab == 0) aph ^= 1u;
          kc = ke;
        }
      }
      if (!ok) *abort_flag = 1;
      umma_commit_local(done);   // all issued MMAs complete before TMEM is released
      volatile int never = 0;
      await(done, 0, &never, kCleanupWaitNs);
    }
  } else if (warp >= kFirstEpi) {
    // --------------------------------- epilogue ----------------------------------
    const int q = warp & 3, half = (warp - kFirstEpi) >> 2;
    float* stg = reinterpret_cast<float*>(smem + kTransOffset + (size_t)(warp - kFirstEpi) * kTransBytes);
    const int r0 = (int)rank * kHalf + q * 32;      // the warp's first row of the tile
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const float nan = __int_as_float(0x7FC00000);
    int ab = 0;
    uint32_t aph = 0;
    bool ok = true;
    Items items(sch, pair);
    Item it;
    while (items.next(sch, it)) {
      int tm, tn;
      tile_place(sch, it.tile, tm, tn);
      const int c_tile = half * 128;
      if constexpr (kLong) {
        float acc[4][32];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = 0.f;
        for (int kc = it.kb0; kc < it.kb1; kc += kChunk) {
          // one answer for the warp: the TMEM loads below are taken by all lanes or none
          ok = ok && __all_sync(0xFFFFFFFFu, await(&accfull[ab], aph, abort_flag, wait_ns));
          if (!ok) {
            *abort_flag = 1;
            break;
          }
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int o = 0; o < 32; o += 16) {
              uint32_t r[16];
              tmem_ld16(tmem_base + (uint32_t)(ab * kTileN + c_tile + 32 * b + o) + lanes, r);
#pragma unroll
              for (int e = 0; e < 16; ++e) acc[b][o + e] += __uint_as_float(r[e]);
            }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cta0(&accempty[ab]);
          ab ^= 1;
          if (ab == 0) aph ^= 1u;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = ok ? acc[b][e] : nan;
          put_block(p, it, tm, tn, r0, c_tile + 32 * b, acc[b], stg, lane);
        }
      } else {
        ok = ok && __all_sync(0xFFFFFFFFu, await(&accfull[ab], aph, abort_flag, wait_ns));
        if (ok) tc_fence_after();
        else *abort_flag = 1;
        for (int b = 0; b < 4; ++b) {
          float v[32];
          if (ok) {
            uint32_t r[32];
            tmem_ld32(tmem_base + (uint32_t)(ab * kTileN + c_tile + 32 * b) + lanes, r);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[e]);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = nan;
          }
          if (ok && b == 3) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_cta0(&accempty[ab]);
          }
          put_block(p, it, tm, tn, r0, c_tile + 32 * b, v, stg, lane);
        }
        ab ^= 1;
        if (ab == 0) aph ^= 1u;
      }
    }
  }

  __syncwarp();
  pair_finish<kStages>(*log, abort_flag, full, armed, rank);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
}

// Left-over tiles that several pairs shared: the parts added in the order of
// the tokens, then written like a whole tile.
__global__ void __launch_bounds__(256) wgrad8_join_kernel(const __grid_constant__ KernelParams p) {
  const Schedule& s = p.sch;
  const int t = blockIdx.x;
  griddep_wait();
  const int64_t u0 = (int64_t)t * s.nkb, u1 = u0 + s.nkb;
  int k = (int)((int64_t)t * s.sharers / s.rest);   // the sharer whose range holds unit u0
  while (k > 0 && s.begin[k] > u0) --k;
  while (s.begin[k + 1] <= u0) ++k;
  if (s.begin[k] <= u0 && s.begin[k + 1] >= u1) return;   // one pair wrote it whole
  int tm, tn;
  tile_place(s, s.waves * kPairs + t, tm, tn);
  int last = k;   // the last sharer of the tile
  while (last + 1 < s.sharers && s.begin[last + 1] < u1) ++last;
  const int rows = min(kTileM, p.out - tm * kTileM), cols = min(kTileN, p.in - tn * kTileN);
  // the first part may be its pair's second item; every later one is a first
  const float* part0 = p.parts + (size_t)(2 * k + (s.begin[k] >= u0 ? 0 : 1)) * (kTileM * kTileN);
  const int r = blockIdx.y * 4 + (threadIdx.x >> 6), c = 4 * (threadIdx.x & 63);
  if (r >= rows || c >= cols) return;
  const size_t at = (size_t)r * kTileN + c;
  float4 sum = *reinterpret_cast<const float4*>(part0 + at);
#pragma unroll 4
  for (int j = k + 1; j <= last; ++j) {
    const float4 v = *reinterpret_cast<const float4*>(p.parts + (size_t)(2 * j) * (kTileM * kTileN) + at);
    sum.x += v.x;
    sum.y += v.y;
    sum.z += v.z;
    sum.w += v.w;
  }
  put_dw4(p, (int64_t)(tm * kTileM + r) * p.dw.ld + tn * kTileN + c, sum, cols - c);
}

// dW of no tokens.
__global__ void __launch_bounds__(256) wgrad8_zero_kernel(Mat dw, int dwdt, int out, int in) {
  for (int r = blockIdx.x; r < out; r += gridDim.x)
    for (int c = threadIdx.x; c < in; c += 256) {
      if (dwdt == LM_F32) static_cast<float*>(dw.data)[r * dw.ld + c] = 0.f;
      else static_cast<__nv_bfloat16*>(dw.data)[r * dw.ld + c] = __float2bfloat16_rn(0.f);
    }
}

// The operands as the TMA takes them.  Blocks below x_blocks: X = code * scale
// as bf16.  The others: dY in rows of a 16-byte
// pitch where its own are not; fp32 values as three planes whose sum is
// exactly the value, from 2^-110 up (each takes the next 8 significant bits by truncation, so
// that no piece rounds up to infinity; an infinity or a NaN is its own first
// piece, with zeros in the others).
template <int kFormat, typename T>
__global__ void __launch_bounds__(256) wgrad8_operands_kernel(Codes x, __nv_bfloat16* xdst, int64_t ldx, unsigned x_blocks, Mat dy, int64_t tokens,
                                                              int out, __nv_bfloat16* dst, int64_t ld) {
  griddep_launch_dependents();
  if (blockIdx.x < x_blocks) {
    // a warp takes 512 channels of a token, 16 a lane, kAhead such pieces at once
    constexpr int kAhead = 4, kPiece = 512;
    const int per = (int)((ldx + kPiece - 1) / kPiece);
    const int64_t first = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), warps = (int64_t)x_blocks * 8;
    int64_t row = first / per;
    int piece = (int)(first - row * per);
    const int64_t drow = warps / per;
    const int dpiece = (int)(warps - drow * per);
    while (row < tokens) {
      uint4 q[kAhead];
      float sc[kAhead];
      int64_t t[kAhead];
      int c[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        t[k] = row;
        c[k] = piece * kPiece + 16 * (int)(threadIdx.x & 31);
        if (row < tokens && c[k] < ldx) {
          q[k] = __ldcs(reinterpret_cast<const uint4*>(x.data + row * x.ld + c[k]));
          sc[k] = x.scales[(int64_t)(c[k] / LM_CODE_GROUP) * x.ld_scales + row];
        }
        row += drow;
        piece += dpiece;
        if (piece >= per) {
          piece -= per;
          ++row;
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (t[k] >= tokens || c[k] >= ldx) continue;
        const uint32_t s2 = __byte_perm(__float_as_uint(sc[k]), __float_as_uint(sc[k]), 0x3232);
        const uint2 w0 = convert4<kFormat>(q[k].x, s2), w1 = convert4<kFormat>(q[k].y, s2);
        const uint2 w2 = convert4<kFormat>(q[k].z, s2), w3 = convert4<kFormat>(q[k].w, s2);
        uint4* d = reinterpret_cast<uint4*>(xdst + t[k] * ldx + c[k]);
        d[0] = make_uint4(w0.x, w0.y, w1.x, w1.y);
        d[1] = make_uint4(w2.x, w2.y, w3.x, w3.y);
      }
    }
    return;
  }
  const int64_t plane = tokens * ld;
  for (int64_t t = blockIdx.x - x_blocks; t < tokens; t += gridDim.x - x_blocks) {
    const T* src = static_cast<const T*>(dy.data) + t * dy.ld;
    for (int c = threadIdx.x; c < out; c += 256) {
      __nv_bfloat16* d = dst + t * ld + c;
      if constexpr (sizeof(T) == 2) {
        *d = src[c];
      } else {
        const float v = src[c];
        const bool finite = fabsf(v) < INFINITY;
        const float hi = finite ? __uint_as_float(__float_as_uint(v) & 0xFFFF0000u) : v, r = finite ? v - hi : 0.f;
        const float mid = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
        d[0] = __float2bfloat16_rn(hi);
        d[plane] = __float2bfloat16_rn(mid);
        d[2 * plane] = __float2bfloat16_rn(r - mid);
      }
    }
  }
}

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = []() {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                    q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f) : nullptr;
  }();
  return fn;
}

Schedule make_schedule(int64_t tokens, int64_t out, int64_t in, int planes) {
  Schedule s{};
  s.tiles_m = (int32_t)((out + kTileM - 1) / kTileM);
  s.tiles_n = (int32_t)((in + kTileN - 1) / kTileN);
  s.nkb_plane = (int32_t)((tokens + kBlockK - 1) / kBlockK);
  s.nkb = s.nkb_plane * planes;
  const int64_t tiles = (int64_t)s.tiles_m * s.tiles_n;
  s.waves = (int32_t)(tiles / kPairs);
  s.rest = (int32_t)(tiles % kPairs);
  if (s.rest > 0) {
    // a share of at least kChunk blocks, and never more sharers than pairs
    const int64_t most = (int64_t)s.rest * s.nkb / kChunk;
    s.sharers = (int32_t)(most < s.rest ? s.rest : most < kPairs ? most : kPairs);
    for (int k = 0; k <= s.sharers; ++k) s.begin[k] = (int64_t)s.rest * s.nkb * k / s.sharers;
  }
  return s;
}
// Token blocks of the longest item.
int64_t longest_item(const Schedule& s) {
  int64_t most = s.waves > 0 ? s.nkb : 0;
  for (int k = 0; k < s.sharers; ++k) most = std::max(most, std::min<int64_t>(s.nkb, s.begin[k + 1] - s.begin[k]));
  return most;
}
// Whether any left-over tile falls to more than one pair.
bool has_parts(const Schedule& s) { return s.rest > 0 && s.sharers > s.rest; }

struct Layout {
  bool copy;          // dY is laid out anew in the workspace
  int planes;
  int64_t ld, ldx;    // of the copies of dY and X
  size_t parts, dy, total;   // bytes: parts, then dY, then X
};
Layout make_layout(const Schedule& s, int64_t tokens, int64_t out, int64_t in, int dydt, const Mat& dy) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Layout l{};
  l.planes = dydt == LM_F32 ? 3 : 1;
  l.copy = dydt == LM_F32 || reinterpret_cast<uintptr_t>(dy.data) % 16 != 0 || (tokens > 1 && dy.ld % 8 != 0) || (tokens == 1 && out % 8 != 0);
  l.ld = (out + 7) / 8 * 8;
  l.ldx = (in + 15) / 16 * 16;
  l.parts = has_parts(s) ? 2 * (size_t)s.sharers * kPartBytes : 0;
  l.dy = l.copy ? up((size_t)l.planes * tokens * l.ld * 2) : 0;
  l.total = l.parts + l.dy + up((size_t)tokens * l.ldx * 2);
  return l;
}

// A 3-D map (columns, rows, planes) of boxes of 64 columns x 64 tokens, bf16, 128-byte swizzle.
CUresult encode_operand(PFN_cuTensorMapEncodeTiled_v12000 enc, CUtensorMap* m, void* base, int64_t cols, int64_t rows, int64_t ld, int planes) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)rows};
  const cuuint32_t box[3] = {64, kBlockK, 1}, estr[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// A launch whose set-up may overlap the end of the kernel before it (which it
// waits for itself, griddepcontrol.wait).
template <typename Kernel>
cudaError_t launch_after(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, const KernelParams& p) {
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
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <bool kLong>
cudaError_t start(const KernelParams& p, int pairs, cudaStream_t st) {
  const int dev = device_slot();
  static bool ready[kMaxDevices];
  if (dev < 0 || !ready[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(wgrad8_kernel<kLong>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
    if (e != cudaSuccess) return e;
    if (dev >= 0) ready[dev] = true;
  }
  return launch_after(wgrad8_kernel<kLong>, dim3(2 * pairs), kThreads, kSmemBytes, st, p);
}

}  // namespace

size_t wgrad8_workspace(const Mat& dy, int dydt, int64_t tokens, int64_t out, int64_t in) {
  if (tokens <= 0) return 0;
  const Schedule s = make_schedule(tokens, out, in, dydt == LM_F32 ? 3 : 1);
  return make_layout(s, tokens, out, in, dydt, dy).total;
}

cudaError_t launch_wgrad8(const WgradParams& w, cudaStream_t st) {
  if (w.tokens == 0) {
    count_launch();
    wgrad8_zero_kernel<<<w.out < 2048 ? w.out : 2048, 256, 0, st>>>(w.dw, w.dwdt, w.out, w.in);
    return cudaGetLastError();
  }
  const int planes = w.dydt == LM_F32 ? 3 : 1;
  KernelParams p{};
  p.sch = make_schedule(w.tokens, w.out, w.in, planes);
  p.out = w.out;
  p.in = w.in;
  p.dw = w.dw;
  p.dwdt = w.dwdt;
  p.accumulate = w.accumulate;
  const uintptr_t four = w.dwdt == LM_F32 ? 16 : 8;   // bytes of four elements
  p.vec = reinterpret_cast<uintptr_t>(w.dw.data) % four == 0 && (w.out == 1 || w.dw.ld % 4 == 0);
  p.wait_ns = env_wait_limit_ns();
  const Layout l = make_layout(p.sch, w.tokens, w.out, w.in, w.dydt, w.dy);
  p.parts = static_cast<float*>(w.workspace);
  void* dy = w.dy.data;
  int64_t ld = w.dy.ld;
  if (l.copy) {
    dy = static_cast<uint8_t*>(w.workspace) + l.parts;
    ld = l.ld;
  }
  __nv_bfloat16* x = reinterpret_cast<__nv_bfloat16*>(static_cast<uint8_t*>(w.workspace) + l.parts + l.dy);
  {
    const int64_t pieces = w.tokens * ((l.ldx + 511) / 512), steps = (pieces + 7) / 8;   // a warp's pieces, blocks of eight warps
    const unsigned x_blocks = (unsigned)(steps < 152 * 8 ? steps : 152 * 8);
    const unsigned dy_blocks = l.copy ? (unsigned)(w.tokens < 152 * 8 ? w.tokens : 152 * 8) : 0u;
    using Operands = void (*)(Codes, __nv_bfloat16*, int64_t, unsigned, Mat, int64_t, int, __nv_bfloat16*, int64_t);
    const Operands kernels[2][2] = {{wgrad8_operands_kernel<LM_CODE_I8, float>, wgrad8_operands_kernel<LM_CODE_I8, __nv_bfloat16>},
                                    {wgrad8_operands_kernel<LM_CODE_E4M3, float>, wgrad8_operands_kernel<LM_CODE_E4M3, __nv_bfloat16>}};
    count_launch();
    kernels[w.x.format == LM_CODE_I8 ? 0 : 1][w.dydt == LM_F32 ? 0 : 1]<<<x_blocks + dy_blocks, 256, 0, st>>>(
        w.x, x, l.ldx, x_blocks, w.dy, w.tokens, w.out, static_cast<__nv_bfloat16*>(dy), ld);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
  if (enc == nullptr) return cudaErrorNotSupported;
  if (encode_operand(enc, &p.dy, dy, w.out, w.tokens, ld, planes) != CUDA_SUCCESS) return cudaErrorInvalidValue;
  if (encode_operand(enc, &p.x, x, w.in, w.tokens, l.ldx, 1) != CUDA_SUCCESS) return cudaErrorInvalidValue;
  const int pairs = p.sch.waves > 0 ? kPairs : p.sch.sharers;
  const cudaError_t e = longest_item(p.sch) > kChunk ? start<true>(p, pairs, st) : start<false>(p, pairs, st);
  if (e != cudaSuccess || !has_parts(p.sch)) return e;
  return launch_after(wgrad8_join_kernel, dim3(p.sch.rest, kTileM / 4), 256, 0, st, p);
}

}  // namespace lm
