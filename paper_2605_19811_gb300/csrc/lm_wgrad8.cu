// Weight gradient of a linear layer whose input was kept in 8 bits:
//   dW (+)= dY^T X,   dW: out x in, dY: T x out, X = code * scale: T x in
// (lm_linear_wgrad8 in lionmuon.h) on the tensor cores: tcgen05.mma on CTA
// pairs, one 256 x 256 tile of dW per pair, a sum over tokens 64 at a time.
//
// A code times its power-of-two scale is a bf16 number, so X enters the
// product exactly; dY does too, as itself (bf16) or as three bf16 pieces
// (fp32: 8 + 8 + 8 significant bits, summed as three times as many tokens).
// Every product is then exact and only the sums are rounded.
//
// Both operands lie token by token in memory, so both are MN-major: rows of
// 64 channels (128 bytes, 128-byte swizzle), one row a token.  CTA r of the
// pair holds output channels 128 r .. of the tile (A, from dY by TMA) and input
// channels 128 r .. (B): exactly one scale group, so one scale a token.  The
// codes come by TMA and the scales by cp.async into a ring of their own; eight
// converter warps make B from them: code -> bf16 by integer operations on
// pairs, times the scale, 16-byte stores into the swizzled stage.
//
// CTA roles (20 warps, one CTA per SM):
//   warp 0       TMA producer of A (one lane); both CTAs' copies signal CTA 0
//   warp 1       TMEM allocation; MMA issuer (CTA 0, one lane)
//   warp 2       codes (TMA) and scales (cp.async) of B
//   warps 4-11   converters of B
//   warps 12-19  epilogue: one TMEM lane quadrant and half of the columns each
//
// Accumulation: the tensor cores lose up to a unit of the last place of the
// accumulator at each addition (16 tokens).  For a bf16 result that is far
// below its own rounding and a tile's whole sum stays in TMEM.  For an fp32
// result the sum is cut every kChunk blocks (512 tokens): the epilogue adds
// the accumulator to sums it holds in registers while the MMA fills the other
// accumulator.
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
constexpr int kStages = 5;
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kCodeBytes = kBlockK * kHalf;            // a token block's codes of one CTA
constexpr int kCodeStage = kCodeBytes + kBlockK * 4;   // and their scales
constexpr int kConvWarps = 8, kEpiWarps = 8;
constexpr int kTeams = 2, kTeamWarps = kConvWarps / kTeams;   // converter teams take token blocks in turn
constexpr int kCodeWarp = 2;
constexpr int kFirstConv = 4, kFirstEpi = kFirstConv + kConvWarps;
constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
constexpr int kChunk = 8;                              // token blocks summed in one accumulator (fp32 results)
constexpr int kPairs = 76;                             // CTA pairs of the GPU (152 SMs)
constexpr int kTmemCols = 512;
constexpr size_t kTransBytes = 32 * 17 * 4;            // an epilogue warp's transpose tile
constexpr size_t kCodeOffset = (size_t)kStages * kStageBytes;
constexpr size_t kTransOffset = kCodeOffset + (size_t)kStages * kCodeStage;
constexpr size_t kBarOffset = kTransOffset + kEpiWarps * kTransBytes;
constexpr size_t kSmemBytes = 1024 + kBarOffset + 512;
constexpr size_t kPartBytes = (size_t)kTileM * kTileN * 4;
static_assert(kSmemBytes <= 232448, "shared memory of one SM");

// How the work falls to the pairs.
struct Schedule {
  int32_t tiles_m, tiles_n;
  int32_t nkb;          // token blocks of a tile (three times as many for fp32 dY)
  int32_t nkb_plane;    // token blocks of one plane of dY
  int32_t waves;        // whole waves: tiles [0, waves * kPairs) go one to a pair
  int32_t rest;         // tiles left over
  int32_t sharers;      // pairs that share them; 0: none left over
};
struct KernelParams {
  CUtensorMap dy, codes;
  Schedule sch;
  int64_t tokens;
  int32_t out, in;
  Codes x;
  Mat dw;
  int32_t dwdt;
  int32_t accumulate;
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
// First unit (tile, token block) of sharer k in the line of left-over work.
__host__ __device__ __forceinline__ int64_t share_begin(const Schedule& s, int k) {
  return (int64_t)s.rest * s.nkb * k / s.sharers;
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
      at = share_begin(s, p);
      end = share_begin(s, p + 1);
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

__device__ __forceinline__ void tma_load_dy(void* dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
  tma_load_3d(dst, map, bar, c0, c1, c2);
}
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

// Arrive on a barrier of CTA 0.  What the arrival announces is in the arriving
// CTA's own SM: operand bytes in its shared memory, which the arriving threads
// have fenced towards the tensor core (fence.proxy.async) before, or TMEM
// columns read to the end (tcgen05.wait::ld).  Nothing in global memory hangs
// on it, so the arrival needs no fence of cluster scope; with one
// (.release.cluster) it took 1300 cycles, against 512 of a token block's MMA.
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

// 128 codes x 64 tokens into this CTA's shared memory.
__device__ __forceinline__ void tma_load_codes(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1)
      : "memory");
}
// One scale into shared memory, zero where there is none.
__device__ __forceinline__ void copy_scale(float* dst, const float* src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
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

// 32 rows (one a lane) x 32 columns of a tile, row r0 / column c0 of the tile:
// through the warp's transpose tile, 16 columns at a time, then two rows a
// step, a column a lane.
__device__ __forceinline__ void put_block(const KernelParams& p, const Item& it, int tm, int tn, int r0, int c0,
                                          const float (&v)[32], float* stg, int lane) {
  const int row0 = tm * kTileM + r0, rows = min(32, p.out - row0);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 16; ++e) stg[lane * 17 + e] = v[16 * h + e];
    __syncwarp();
    const int c = c0 + 16 * h + (lane & 15), col = tn * kTileN + c;
    if (col < p.in) {
      float* part = it.slot >= 0 ? p.parts + (size_t)it.slot * (kTileM * kTileN) + (size_t)r0 * kTileN + c : nullptr;
      for (int r = lane >> 4; r < rows; r += 2) {
        const float x = stg[r * 17 + (lane & 15)];
        if (part != nullptr) part[(size_t)r * kTileN] = x;
        else put_dw(p, (int64_t)(row0 + r) * p.dw.ld + col, x);
      }
    }
    __syncwarp();
  }
}

// Before the register split is taken back: a warp that asked for its registers
// back earlier could take what an epilogue warp still waits for, and neither
// would go on.
__device__ __forceinline__ void all_roles_done() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); }

// kLong: sums of fp32 results, cut every kChunk token blocks.
template <int kFormat, bool kLong>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) wgrad8_kernel(const __grid_constant__ KernelParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_a = reinterpret_cast<uint64_t*>(smem + kBarOffset);
  uint64_t* full_b = full_a + kStages;
  uint64_t* empty = full_b + kStages;
  uint64_t* code_full = empty + kStages;
  uint64_t* code_empty = code_full + kStages;
  uint64_t* accfull = code_empty + kStages;
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
      mbar_init(&full_a[s], 1);
      mbar_init(&full_b[s], 2 * kTeamWarps);
      mbar_init(&empty[s], 1);
      mbar_init(&code_full[s], 1 + 32);
      mbar_init(&code_empty[s], kTeamWarps);
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
  const uint32_t tmem_base = *tmem_slot;
  const uint64_t wait_ns = p.wait_ns;

  if (warp < kFirstConv) {
    // Registers: 640 threads x 96 at launch = 128 x 32 + 256 x 64 + 256 x 160 after the split.
    if (kLong) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (warp == 0 && lane == 0) {
      // ------------------------------ producer of A ------------------------------
      int stage = 0;
      uint32_t ph = 0;
      bool ok = true;
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        int tm, tn;
        tile_place(sch, it.tile, tm, tn);
        const int row = tm * kTileM + (int)rank * kHalf;
        int plane = it.kb0 / sch.nkb_plane, tb = it.kb0 - plane * sch.nkb_plane;
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
          if (!await(&empty[stage], ph ^ 1u, abort_flag, wait_ns)) {
            ok = false;
            break;
          }
          uint8_t* sa = smem + (size_t)stage * kStageBytes;
          const uint32_t fb = peer_addr(&full_a[stage], 0);
          if (rank == 0) {
            mbar_arrive_expect_tx(&full_a[stage], 2u * kABytes);
            armed[stage] = (int)ph;
          }
          log->bytes[stage] = kABytes;
          log->n += 1u;
          tma_load_dy(sa, &p.dy, fb, row, tb * kBlockK, plane);
          tma_load_dy(sa + kABytes / 2, &p.dy, fb, row + 64, tb * kBlockK, plane);
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
    } else if (warp == 1 && lane == 0 && rank == 0) {
      // -------------------------------- MMA issuer -------------------------------
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
            if (!await(&full_a[stage], ph, abort_flag, wait_ns) || !await(&full_b[stage], ph, abort_flag, wait_ns)) {
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
    if (warp == kCodeWarp) {
      // ------------------------- codes and scales of B ---------------------------
      // By TMA and cp.async, into a ring of their own: the converters then have no
      // load in flight when they fence their stores (the fence would wait for it).
      int stage = 0, issued = 0;   // issued: token blocks, counted up to kStages
      uint32_t ph = 0;
      bool ok = true;
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        int tm, tn;
        tile_place(sch, it.tile, tm, tn);
        const int col = tn * kTileN + (int)rank * kHalf;
        const float* cs = p.x.scales + (int64_t)(col / LM_CODE_GROUP) * p.x.ld_scales;
        int tb = it.kb0 % sch.nkb_plane;
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
          if (!await(&code_empty[stage], ph ^ 1u, abort_flag, wait_ns)) {
            ok = false;
            break;
          }
          uint8_t* c = smem + kCodeOffset + (size_t)stage * kCodeStage;
          if (lane == 0) {
            mbar_arrive_expect_tx(&code_full[stage], kCodeBytes);
            tma_load_codes(c, &p.codes, &code_full[stage], col, tb * kBlockK);
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int64_t t = (int64_t)tb * kBlockK + 32 * j + lane;
            const bool in = col < p.in && t < p.tokens;
            copy_scale(reinterpret_cast<float*>(c + kCodeBytes) + 32 * j + lane, in ? cs + t : p.x.scales, in);
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&code_full[stage])) : "memory");
          if (issued < kStages) ++issued;
          if (++tb == sch.nkb_plane) tb = 0;
          if (++stage == kStages) {
            stage = 0;
            ph ^= 1u;
          }
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (!ok) {
        // nothing may be in flight into a CTA that leaves: wait (bounded) for the
        // newest phase of every stage that was used
        *abort_flag = 1;
        volatile int never = 0;
        for (int s = 0; s < kStages && s < issued; ++s) await(&code_full[s], s < stage ? ph : ph ^ 1u, &never, kCleanupWaitNs);
      }
    }
    __syncwarp();
    if (kLong) {
      all_roles_done();
      asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
    }
  } else if (warp < kFirstEpi) {
    // ------------------------------ converters of B ------------------------------
    // Two teams of four warps take the token blocks in turn.  Warp w of a team
    // makes tokens 16 w .. 16 w + 15 of a block: lane l reads 16 codes (columns
    // 16 (l % 8) ..) of tokens l / 8 + 4 j.  The two atoms of 64 columns store
    // their halves in opposite order, so that the eight lanes of a 16-byte store
    // phase touch all banks.
    if (kLong) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const int team = (warp - kFirstConv) / kTeamWarps;
    const int tok = 16 * ((warp - kFirstConv) % kTeamWarps) + (lane >> 3);
    const int atom = (lane & 7) >> 2, chunk = 2 * (lane & 3);
    uint32_t off[2][2];   // of tokens j = 0 and 1; j = 2 and 3 lie 8 rows further
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = tok + 4 * j, c = chunk + (h ^ atom);
        off[j][h] = (uint32_t)(kABytes + atom * (kBBytes / 2) + k * 128 + ((c ^ (k & 7)) << 4));
      }
    int64_t blocks = (int64_t)sch.waves * sch.nkb;   // token blocks of this pair
    if (pair < sch.sharers) blocks += share_begin(sch, pair + 1) - share_begin(sch, pair);
    int stage = team;
    uint32_t ph = 0;
    for (int64_t n = team; n < blocks; n += kTeams) {
      if (!await(&code_full[stage], ph, abort_flag, wait_ns) || !await(&empty[stage], ph ^ 1u, abort_flag, wait_ns)) {
        *abort_flag = 1;
        break;
      }
      const uint8_t* code = smem + kCodeOffset + (size_t)stage * kCodeStage;
      uint8_t* st = smem + (size_t)stage * kStageBytes;
      uint4 q[4];
      uint32_t s2[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        q[j] = *reinterpret_cast<const uint4*>(code + (tok + 4 * j) * kHalf + 16 * (lane & 7));
        const uint32_t sb = *reinterpret_cast<const uint32_t*>(code + kCodeBytes + 4 * (tok + 4 * j));
        s2[j] = __byte_perm(sb, sb, 0x3232);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint2 w0 = convert4<kFormat>(q[j].x, s2[j]), w1 = convert4<kFormat>(q[j].y, s2[j]);
        const uint2 w2 = convert4<kFormat>(q[j].z, s2[j]), w3 = convert4<kFormat>(q[j].w, s2[j]);
        const uint4 lo = make_uint4(w0.x, w0.y, w1.x, w1.y), hi = make_uint4(w2.x, w2.y, w3.x, w3.y);
        *reinterpret_cast<uint4*>(st + off[j & 1][0] + (j >> 1) * 1024) = atom == 0 ? lo : hi;
        *reinterpret_cast<uint4*>(st + off[j & 1][1] + (j >> 1) * 1024) = atom == 0 ? hi : lo;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&code_empty[stage]);
        arrive_cta0(&full_b[stage]);
      }
      stage += kTeams;
      if (stage >= kStages) {
        stage -= kStages;
        ph ^= 1u;
      }
    }
    __syncwarp();
    if (kLong) {
      all_roles_done();
      asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
    }
  } else {
    // --------------------------------- epilogue ----------------------------------
    if (kLong) asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
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
      if (kLong) {
        float acc[4][32];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = 0.f;
        for (int kc = it.kb0; kc < it.kb1; kc += kChunk) {
          if (ok && !await(&accfull[ab], aph, abort_flag, wait_ns)) ok = false;
          if (!ok) {
            *abort_flag = 1;
            break;
          }
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int o = 0; o < 4; ++o) {
              uint32_t r[8];
              asm volatile(
                  "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
                  "tcgen05.wait::ld.sync.aligned;"
                  : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                  : "r"(tmem_base + (uint32_t)(ab * kTileN + c_tile + 32 * b + 8 * o) + lanes)
                  : "memory");
#pragma unroll
              for (int e = 0; e < 8; ++e) acc[b][8 * o + e] += __uint_as_float(r[e]);
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
        if (ok && !await(&accfull[ab], aph, abort_flag, wait_ns)) {
          ok = false;
          *abort_flag = 1;
        }
        if (ok) tc_fence_after();
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
    __syncwarp();
    if (kLong) {
      all_roles_done();
      asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    }
  }

  __syncwarp();
  pair_finish<kStages>(*log, abort_flag, full_a, armed, rank);
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
  const int64_t u0 = (int64_t)t * s.nkb, u1 = u0 + s.nkb;
  // the sharer whose range holds unit u0
  int k = (int)(u0 * s.sharers / ((int64_t)s.rest * s.nkb));
  while (k > 0 && share_begin(s, k) > u0) --k;
  while (share_begin(s, k + 1) <= u0) ++k;
  if (share_begin(s, k) <= u0 && share_begin(s, k + 1) >= u1) return;   // one pair wrote it whole
  int tm, tn;
  tile_place(s, s.waves * kPairs + t, tm, tn);
  int last = k;   // the last sharer of the tile
  while (last + 1 < s.sharers && share_begin(s, last + 1) < u1) ++last;
  const int rows = min(kTileM, p.out - tm * kTileM), cols = min(kTileN, p.in - tn * kTileN);
  // the first part may be its pair's second item; every later one is a first
  const float* part0 = p.parts + (size_t)(2 * k + (share_begin(s, k) / s.nkb == t ? 0 : 1)) * (kTileM * kTileN);
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
  const float out[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c + e < cols) put_dw(p, (int64_t)(tm * kTileM + r) * p.dw.ld + tn * kTileN + c + e, out[e]);
}

// dW of no tokens.
__global__ void __launch_bounds__(256) wgrad8_zero_kernel(Mat dw, int dwdt, int out, int in) {
  for (int r = blockIdx.x; r < out; r += gridDim.x)
    for (int c = threadIdx.x; c < in; c += 256) {
      if (dwdt == LM_F32) static_cast<float*>(dw.data)[r * dw.ld + c] = 0.f;
      else static_cast<__nv_bfloat16*>(dw.data)[r * dw.ld + c] = __float2bfloat16_rn(0.f);
    }
}

// dY as the TMA wants it: rows of a 16-byte pitch, bf16; fp32 values as three
// planes whose sum is exactly the value (each takes the next 8 significant
// bits by truncation, so that no piece rounds up to infinity; a non-finite
// value keeps its first piece and has NaN or infinity in the others).
template <typename T>
__global__ void __launch_bounds__(256) wgrad8_layout_kernel(Mat dy, int64_t tokens, int out, __nv_bfloat16* dst, int64_t ld) {
  const int64_t plane = tokens * ld;
  for (int64_t t = blockIdx.y; t < tokens; t += gridDim.y) {
    const T* src = static_cast<const T*>(dy.data) + t * dy.ld;
    for (int c = blockIdx.x * 256 + threadIdx.x; c < out; c += gridDim.x * 256) {
      __nv_bfloat16* d = dst + t * ld + c;
      if constexpr (sizeof(T) == 2) {
        *d = src[c];
      } else {
        const float v = src[c];
        const float hi = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u), r = v - hi;
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
  }
  return s;
}
// Whether any left-over tile falls to more than one pair.
bool has_parts(const Schedule& s) { return s.rest > 0 && s.sharers > s.rest; }

struct Layout {
  bool copy;          // dY is laid out anew in the workspace
  int planes;
  int64_t ld;         // of the copy
  size_t parts, total;
};
Layout make_layout(const Schedule& s, int64_t tokens, int64_t out, int dydt, const Mat& dy) {
  Layout l{};
  l.planes = dydt == LM_F32 ? 3 : 1;
  l.copy = dydt == LM_F32 || reinterpret_cast<uintptr_t>(dy.data) % 16 != 0 || (tokens > 1 && dy.ld % 8 != 0) || (tokens == 1 && out % 8 != 0);
  l.ld = (out + 7) / 8 * 8;
  l.parts = has_parts(s) ? 2 * (size_t)s.sharers * kPartBytes : 0;
  l.total = l.parts + (l.copy ? (size_t)l.planes * tokens * l.ld * 2 : 0);
  return l;
}

}  // namespace

size_t wgrad8_workspace(const Mat& dy, int dydt, int64_t tokens, int64_t out, int64_t in) {
  if (tokens <= 0) return 0;
  const Schedule s = make_schedule(tokens, out, in, dydt == LM_F32 ? 3 : 1);
  return make_layout(s, tokens, out, dydt, dy).total;
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
  p.tokens = w.tokens;
  p.out = w.out;
  p.in = w.in;
  p.x = w.x;
  p.dw = w.dw;
  p.dwdt = w.dwdt;
  p.accumulate = w.accumulate;
  p.wait_ns = env_wait_limit_ns();
  const Layout l = make_layout(p.sch, w.tokens, w.out, w.dydt, w.dy);
  p.parts = static_cast<float*>(w.workspace);
  void* dy = w.dy.data;
  int64_t ld = w.dy.ld;
  if (l.copy) {
    dy = static_cast<uint8_t*>(w.workspace) + l.parts;
    ld = l.ld;
    const dim3 grid((unsigned)((w.out + 255) / 256), (unsigned)(w.tokens < 8192 ? w.tokens : 8192));
    count_launch();
    if (w.dydt == LM_F32) wgrad8_layout_kernel<float><<<grid, 256, 0, st>>>(w.dy, w.tokens, w.out, static_cast<__nv_bfloat16*>(dy), ld);
    else wgrad8_layout_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(w.dy, w.tokens, w.out, static_cast<__nv_bfloat16*>(dy), ld);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
  if (enc == nullptr) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {(cuuint64_t)w.out, (cuuint64_t)w.tokens, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)w.tokens};
  const cuuint32_t box[3] = {64, kBlockK, 1}, estr[3] = {1, 1, 1};
  if (enc(&p.dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, dy, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;

  const cuuint64_t cdims[2] = {(cuuint64_t)w.in, (cuuint64_t)w.tokens};
  const cuuint64_t cstride[1] = {(cuuint64_t)w.x.ld};
  const cuuint32_t cbox[2] = {kHalf, kBlockK};
  if (enc(&p.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, w.x.data, cdims, cstride, cbox, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;

  using Kernel = void (*)(KernelParams);
  const Kernel kernels[2][2] = {{wgrad8_kernel<LM_CODE_I8, false>, wgrad8_kernel<LM_CODE_I8, true>},
                                {wgrad8_kernel<LM_CODE_E4M3, false>, wgrad8_kernel<LM_CODE_E4M3, true>}};
  const int dev = device_slot();
  static bool ready[kMaxDevices];
  if (dev < 0 || !ready[dev]) {
    for (const auto& row : kernels)
      for (const Kernel k : row) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
        if (e != cudaSuccess) return e;
      }
    if (dev >= 0) ready[dev] = true;
  }
  const int pairs = p.sch.waves > 0 ? kPairs : p.sch.sharers;
  count_launch();
  kernels[w.x.format == LM_CODE_I8 ? 0 : 1][w.dwdt == LM_F32 ? 1 : 0]<<<2 * pairs, kThreads, kSmemBytes, st>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !has_parts(p.sch)) return e;
  count_launch();
  wgrad8_join_kernel<<<dim3(p.sch.rest, kTileM / 4), 256, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace lm
