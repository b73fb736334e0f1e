// Linear layers in 8 bits (lm_weight8, lm_linear8 and lm_linear8_grad in
// lionmuon.h):
//   y = x W^T (tokens x out),  dx = dy W (tokens x in)
// with activations of one scale for each token's 128 channels and weights of one
// scale for each block of 128 x 128, on the tensor cores: tcgen05.mma
// (kind::mxf8f6f4) on CTA pairs takes the e4m3 codes as they are and multiplies
// each 32 of the sum by two powers of two, here the same for four such steps.  A
// power-of-two float's exponent bits are that scale; they are put, a byte a row, into
// the order in which the tensor memory holds them: by a first kernel, from which they
// are loaded like the codes, or, where there is little work, by two warps of each CTA
// (kMake).
//
// A pair takes a tile of 256 tokens x 256 columns, 256 of the sum at a time.  CTA r
// holds tokens 128 r .. (A) and columns 128 r .. (B); W lies K-major for the product
// with W^T and MN-major for the one with W, so the same codes serve both.  The sum
// is cut every 2048 (64 additions, each of which may drop 2^-23 of what is there)
// and goes on in fp32 registers, as in lm_gemm_tc.cuh, whose schedules are used
// here.  (Cut every 1024: 631 us where 597 were taken; not cut: 584.)
//
// Measured: 16384 x 4096 x 14336 580 us (3.3 PFLOP/s), by itself; bound by what the
// SMs take from L2 (473 us without the TMA's loads) and by the copies of the scales
// (15 us) and the accumulators' turns (13).  16384 x 5120 by W of 5120 x 1280 76 us.
// One token by 14336 x 4096 19.5 us (59 MB, 3 TB/s): 2 us until the first bytes are
// there, 3 us at the end, and the scales' way.  Packing 14336 x 4096 bf16 42 us (4.2 TB/s, instructions), back 31 us
// (5.7 TB/s).
//
// Two accumulators of 256 columns would leave the tensor memory no room for the
// scales, so they share 32 columns: the second begins where the first has 32 left,
// and the next 2048 of the sum begin once the epilogue has taken those.  (Tiles of
// 192 columns, two whole accumulators, 128 of the sum a stage: 16384 x 4096 x 14336
// 718 us.  What a stage costs the issuing warp beside its MMAs, 250 cycles, is not
// hidden, as the queue of MMAs is short, so stages are long.)
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
    // code8::encode2's two exceptions are the block's: a NaN scale, and the largest
    const bool plain = inv != 0.f && inv != __uint_as_float(7u << 23);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t r = r0 + 2 * k;
      if (r >= rows || left <= 0) continue;
      float v[8];
      raw[k].get(v);
      uint32_t q[4];
      if (plain) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          q[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2 * i] * inv, v[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = code8::encode2<LM_CODE_E4M3>(v[2 * i], v[2 * i + 1], inv);
      }
      // the pitch is a multiple of 16: eight codes are inside the row wherever one is
      __stcs(reinterpret_cast<uint2*>(out.data + r * out.ld + c), make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16));
    }
  }
}

// Codes back to values: a warp takes 256 columns of a row, eight a lane, kAhead rows
// at once.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) values_kernel(Blocks w, int64_t nrows, int64_t cols, Mat to) {
  constexpr int kAhead = 4;
  griddep_wait();
  griddep_launch_dependents();
  const int64_t c = (int64_t)blockIdx.x * 256 + 8 * (threadIdx.x & 31);
  const int left = (int)max((int64_t)0, min((int64_t)8, cols - c));
  for (int64_t r0 = ((int64_t)blockIdx.y * 8 + (threadIdx.x >> 5)) * kAhead; r0 < nrows; r0 += (int64_t)gridDim.y * 8 * kAhead) {
    uint2 q[kAhead];
    float s[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      q[k] = make_uint2(0u, 0u);
      s[k] = 0.f;
      if (r0 + k >= nrows || left == 0) continue;
      q[k] = __ldcs(reinterpret_cast<const uint2*>(w.data + (r0 + k) * w.ld + c));
      s[k] = w.scales[(r0 + k) / kBlock * w.ld_scales + c / kBlock];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (r0 + k >= nrows) break;
      const uint32_t two[4] = {q[k].x, q[k].x >> 16, q[k].y, q[k].y >> 16};
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 d = code8::decode2<LM_CODE_E4M3>(two[i]);
        v[2 * i] = d.x * s[k];
        v[2 * i + 1] = d.y * s[k];
      }
      rows::Raw<T> o;
      o.set(v);
      o.template store<kVec>(static_cast<T*>(to.data) + (r0 + k) * to.ld + c, left);
    }
  }
}

// --- the product ---

constexpr int kN = 256, kHalfN = kN / 2, kK = 256;      // tile columns; of the sum at a time
constexpr int kSub = 128, kSubs = kK / kSub;            // of the sum: a swizzled row's bytes, a scale's group
constexpr int kFewTokens = 32;
constexpr int kLeastShare = 8;                          // stages of a split sum's part: the parts and their join cost as much as ten
constexpr int kChunk8 = 8;                              // most stages summed in one accumulator: 64 additions
constexpr int kScaleBytes = 512 + 1024;                 // of two stages: the CTA's rows', the tile's columns'
constexpr int kScaleRing = 4;                           // kMake: how many are under way
// The kernel makes the scales itself where a pair takes at most so many stages.  One
// launch less: one token by 14336 x 4096 20.4 us a call instead of 25 (the kernel
// 19.5 instead of 17.1 and 1.8); 1021 x 517 by 1283 the kernel 17.1 us instead of 15.3
// and 1.7, calls one after another 4 us less.  But these warps' loads cost 6% of the
// rate: 16384 x 5120 by 1280 83 us instead of 76 and 3.7.
constexpr int kMakeStages = 32;
constexpr int kWarpBytes = 32 * 64;                     // an epilogue warp's box: 32 columns in bf16, 16 in fp32
constexpr int kShared = 32, kSecond = kN - kShared;     // TMEM: the second accumulator's first column
constexpr int kScaleCol = kSecond + kN, kScaleSlots = 2;    // then 16 columns for each two stages' scales
static_assert(kScaleCol + 16 * kScaleSlots <= kTmemCols, "tensor memory");
// Shared memory.  kFew: at most kFewTokens tokens.  Then the weights' bytes are all
// that counts, and more of them are under way: A is loaded, and has room, for those
// rows alone.  The MMA reads 128 rows from A's place all the same; the others are
// bytes of B, and the rows of the result that they reach are never stored.
template <bool kFew, bool kMake>
struct Ring {
  static constexpr int kStages = kFew ? 5 : 3, kRowsA = kFew ? kFewTokens : kHalf, kSubA = kRowsA * kSub, kSubB = kHalfN * kSub;
  static constexpr int kStage = kSubs * (kSubA + kSubB);
  static constexpr size_t kBoxes = (size_t)kStages * kStage, kScales = kBoxes + (size_t)kEpiWarps * kWarpBytes;
  static constexpr size_t kBars = kScales + (size_t)(kMake ? kScaleRing : kStages) * kScaleBytes, kBytes = 1024 + kBars + 512;
  static_assert(kBytes <= 232448, "shared memory of one SM");
  static_assert(kSubA % 1024 == 0 && kSubB % 1024 == 0 && kWarpBytes % 512 == 0 && kScaleBytes % 128 == 0, "swizzled boxes");
  static_assert(kSubs * kSubA + kSubs * kSubB >= (kSubs - 1) * kSubA + kHalf * kSub, "128 rows from A's last place on are inside the stage");
};


// The scales' source.
struct Scales {
  const float *x, *w;
  int64_t ldx, ldw, tokens;
  int32_t n, groups;
};
// The byte that the tensor cores multiply by 2^(byte - 127) for, 255 being NaN: of NaN, and
// of whatever is no power of two (its fraction would be lost, and a sign's bit would reach
// the next group's byte).
__device__ __forceinline__ uint32_t exponent(float s) {
  const uint32_t bits = __float_as_uint(s);
  return (bits & 0x807FFFFFu) != 0 ? 255u : bits >> 23;
}
// As the tensor memory takes them: the 128 of a block of rows as 32 x 16 bytes,
// row 32 j + l at word 4 l + j, four groups of the sum in a word's bytes.  kMake: lane l
// reads those of rows l, 32 + l, 64 + l, 96 + l of its CTA's tokens, and those of the
// tile's two blocks of 128 columns, from group 4 `four` on; 0 where there are none.
struct FourScales {
  float x[4][4], w[2][4];
  template <bool kGrad>
  __device__ __forceinline__ void load(const Scales& p, int four, int64_t row, int64_t col, int lane) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t g = 4 * (int64_t)four + k;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t token = row + 32 * j + lane;
        x[j][k] = g < p.groups && token < p.tokens ? p.x[g * p.ldx + token] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t block = col / kBlock + j;
        w[j][k] = g < p.groups && block * kBlock < p.n ? (kGrad ? p.w[g * p.ldw + block] : p.w[block * p.ldw + g]) : 0.f;
      }
    }
  }
  static __device__ __forceinline__ uint32_t word(const float (&v)[4]) {
    return exponent(v[0]) | exponent(v[1]) << 8 | exponent(v[2]) << 16 | exponent(v[3]) << 24;
  }
};
static_assert(kN == 2 * kBlock, "two blocks of the weights' scales a tile");

// The first kernel's: activations (four groups, 128 tokens), weights (four groups,
// tile of columns, two blocks of 128).
struct ScaleParams {
  Scales from;
  int32_t fours, row_blocks, tiles_n;
  bool grad;
  uint32_t *sa, *sb;
};
__global__ void __launch_bounds__(128) scales_kernel(const ScaleParams p) {
  griddep_wait();
  griddep_launch_dependents();
  const int t = threadIdx.x;
  const uint32_t a = (uint32_t)p.fours * (uint32_t)p.row_blocks, all = a + (uint32_t)p.fours * 2u * (uint32_t)p.tiles_n;
  for (uint32_t block = blockIdx.x; block < all; block += gridDim.x) {     // 128 words each
    uint32_t v = 0;
    if (block < a) {       // threads in the order of the rows
      const int four = (int)(block / (uint32_t)p.row_blocks);
      const int64_t token = (int64_t)(block - (uint32_t)four * (uint32_t)p.row_blocks) * 128 + t;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (token < p.from.tokens && 4 * four + k < p.from.groups) v |= exponent(p.from.x[(int64_t)(4 * four + k) * p.from.ldx + token]) << (8 * k);
      p.sa[(size_t)block * 128 + (t & 31) * 4 + (t >> 5)] = v;
    } else {               // in the order of the words: word t holds this column
      const uint32_t b = block - a, four = b / (2u * (uint32_t)p.tiles_n), tile = b - four * 2u * (uint32_t)p.tiles_n;
      const int64_t col = (int64_t)tile * 128 + (t & 3) * 32 + (t >> 2);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t g = 4 * (int64_t)four + k;
        if (col < p.from.n && g < p.from.groups) v |= exponent(p.grad ? p.from.w[g * p.from.ldw + col / kBlock] : p.from.w[col / kBlock * p.from.ldw + g]) << (8 * k);
      }
      p.sb[(size_t)b * 128 + t] = v;
    }
  }
}

struct Params8 {
  CUtensorMap a, b, sa, sb, y;                        // sa, sb: from the first kernel
  Schedule sch;
  Scales scales;                                      // kMake
  int32_t m, n;
  float* parts;
  uint64_t wait_ns;
  Store out;
};

// Instruction descriptor, kind::mxf8f6f4: A and B e4m3, scales ue8m0 (bit 23),
// the byte of a scale's word at bits 4 (B) and 29 (A), N >> 3 at bit 17, M >> 7
// at bit 27.
constexpr uint32_t idesc8(bool b_mn_major) {
  return ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(kN >> 3) << 17) | (1u << 23) | ((uint32_t)(kTileM >> 7) << 27);
}
// The whole warp comes here, so that what the instruction takes is the same in
// every lane and needs no move from a lane's registers; the leader issues it.
__device__ __forceinline__ void umma_mx8(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate), "r"(leader)
      : "memory");
}
// await and mbar_test for a barrier on which the other CTA's scales arrive: what
// that CTA wrote before is visible too.
__device__ __forceinline__ bool mbar_test_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool await_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t limit_ns) {
  return await(bar, parity, abort_flag, limit_ns) && mbar_test_cluster(bar, parity);
}
// 32 x 16 bytes of shared memory to four columns of every lane quadrant, in both
// CTAs; MMAs issued after it by the same thread see them.
__device__ __forceinline__ void copy_scales(uint32_t leader, uint32_t tmem, uint32_t smem) {
  // no swizzle: eight rows of 16 bytes side by side, 128 bytes apart
  const uint64_t desc = (uint64_t)((smem >> 4) & 0x3FFFu) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem), "l"(desc), "r"(leader) : "memory");
}

// 32 rows (one a lane) x 32 columns through a box, 16 columns at a time, then
// eight rows a step, four columns a lane.
template <typename Put>
__device__ __forceinline__ void put16(const float (&v)[32], uint32_t box, int lane, int rows, const Put& put) {
  const int q = lane & 3, r8 = lane >> 2;
  auto at = [&](int row, int chunk) { return box + row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4); };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* f = v + 16 * h + 4 * e;
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at(lane, e)), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = r8 + 8 * k;
      if (r >= rows) continue;
      float4 x;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at(r, q)) : "memory");
      put(r, 16 * h + 4 * q, x);
    }
    __syncwarp();
  }
}

// The same straight to y, as gemm::put_plain_block: eight rows a step and four
// columns a lane, or two rows and a column.
template <typename T>
__device__ __forceinline__ void put16_plain(const float (&v)[32], uint32_t box, int lane, int row0, int rows, int c, int n, const Store& out) {
  auto at = [&](int row, int chunk) { return box + row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4); };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float* f = v + 16 * h + 4 * k;
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at(lane, k)), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
    }
    __syncwarp();
    T* o = static_cast<T*>(out.d.data) + (int64_t)row0 * out.d.ld + c + 16 * h;
    if (out.vec && c + 16 * h + 16 <= n) {
      const int q = lane & 3, r8 = lane >> 2;
      o += r8 * out.d.ld + 4 * q;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float4 x;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at(r8 + 8 * k, q)) : "memory");
        if (r8 + 8 * k < rows) put_plain4(o, x);
        o += 8 * out.d.ld;
      }
    } else {
      const int e = lane & 15;
      const bool in = c + 16 * h + e < n;
      o += (lane >> 4) * out.d.ld + e;
#pragma unroll 8
      for (int r = lane >> 4; r < rows; r += 2) {
        float x;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at(r, e >> 2) + 4 * (e & 3)) : "memory");
        if (in) put_plain(o, x);
        o += 2 * out.d.ld;
      }
    }
    __syncwarp();
  }
}

template <bool kGrad, bool kFew, bool kMake>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) linear8_kernel(const __grid_constant__ Params8 p) {
  using R = Ring<kFew, kMake>;
  constexpr int kStages = R::kStages, kStage = R::kStage, kSubA = R::kSubA, kSubB = R::kSubB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + R::kBars);
  uint64_t* empty = full + kStages;
  uint64_t* accfull = empty + kStages;
  uint64_t* accempty = accfull + 2;
  uint64_t* shared = accempty + 2;                    // the columns that both accumulators have are read
  uint64_t* sfull = shared + 2;                       // kMake: both CTAs' scales are there, and copied
  uint64_t* sempty = sfull + kScaleRing;
  uint64_t* done = sempty + kScaleRing;
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
      mbar_init(&shared[b], kEpiWarps);               // the warps of one half, in both CTAs
    }
    for (int b = 0; b < kScaleRing; ++b) {
      mbar_init(&sfull[b], 2);
      mbar_init(&sempty[b], 1);
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
    few_registers<96>();
    if (lane == 0) {
      int stage = 0;
      uint32_t ph = 0;
      bool ok = true;
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        const int row = it.tm * kTileM + (int)rank * kHalf, col = it.tn * kN + (int)rank * kHalfN;
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
          if (!await(&empty[stage], ph ^ 1u, abort_flag, wait_ns)) {
            ok = false;
            break;
          }
          uint8_t* sa = smem + (size_t)stage * kStage;
          uint8_t* sb = sa + kSubs * kSubA;
          const uint32_t fb = peer_addr(&full[stage], 0);
          const bool scales = !kMake && (kb == it.kb0 || (kb & 1) == 0);      // four groups', of two stages
          const uint32_t tx = kStage + (scales ? kScaleBytes : 0);
          if (rank == 0) {
            mbar_arrive_expect_tx(&full[stage], 2u * tx);
            armed[stage] = (int)ph;
          }
          log->bytes[stage] = tx;
          log->n += 1u;
#pragma unroll
          for (int k = 0; k < kSubs; ++k) {
            const int at = (kb * kSubs + k) * kSub;
            tma_load_3d(sa + k * kSubA, &p.a, fb, at, row, 0);
            if (kGrad) tma_load_3d(sb + k * kSubB, &p.b, fb, col, at, 0);
            else tma_load_3d(sb + k * kSubB, &p.b, fb, at, col, 0);
          }
          if (scales) {
            uint8_t* ss = smem + R::kScales + (size_t)stage * kScaleBytes;
            tma_load_3d(ss, &p.sa, fb, 0, row / 128, kb >> 1);
            tma_load_3d(ss + 512, &p.sb, fb, 0, it.tn, kb >> 1);
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
    few_registers<96>();
    if (rank == 0) {
      constexpr uint32_t idesc = idesc8(kGrad);
      // 32 of the sum: 32 bytes of a row (K-major), 32 rows of 128 bytes (MN-major)
      constexpr uint64_t a_step = 32 >> 4, b_step = (kGrad ? 4096 : 32) >> 4;
      const uint32_t leader = lane == 0 ? 1u : 0u, smem0 = smem_u32(smem), tmem0 = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
      int stage = 0, ab = 0;
      uint32_t ph = 0, aph = 0, ta = 0, blocks = 0, slot = 0, last_use[kScaleSlots] = {0, 0};   // blocks: issued so far
      int sslot = 0;
      uint32_t sph = 0;
      bool ok = true, ready = false, sready = false;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (!__all_sync(0xFFFFFFFFu, await(bar, parity, abort_flag, wait_ns))) ok = false;
        return ok;
      };
      Items items(sch, pair);
      Item it;
      while (ok && items.next(sch, it)) {
        for (int kc = it.kb0; ok && kc < it.kb1;) {
          const int ke = min(kc + kChunk8, it.kb1);
          // this accumulator read to its end, and the other one's columns that it shares
          // (the one before the first has none: that wait passes)
          if (!wait(&accempty[ab], aph ^ 1u) || !wait(&shared[ab ^ 1], ab ? aph : aph ^ 1u)) break;
          tc_fence_after();
          const uint32_t d = tmem0 + (uint32_t)(ab * kSecond);
          for (int kb = kc; kb < ke; ++kb) {
            if (!ready && !wait(&full[stage], ph)) break;
            tc_fence_after();
            if (kb == it.kb0 || (kb & 1) == 0) {
              // MMAs of kStages blocks ago are done, as their stage is filled again; of
              // later ones (an item that began or ended between two) the slot's are waited for
              slot ^= 1u;
              if (last_use[slot] > 0 && blocks + 1 - last_use[slot] < (uint32_t)kStages &&
                  !wait(&empty[(last_use[slot] - 1) % kStages], ((last_use[slot] - 1) / kStages) & 1u))
                break;
              if (kMake && !sready && !__all_sync(0xFFFFFFFFu, await_cluster(&sfull[sslot], sph, abort_flag, wait_ns))) {
                ok = false;
                break;
              }
              const uint32_t ss = smem0 + (uint32_t)(R::kScales + (size_t)(kMake ? sslot : stage) * kScaleBytes);
              ta = tmem0 + (uint32_t)kScaleCol + 16u * slot;
              copy_scales(leader, ta, ss);
              copy_scales(leader, ta + 4, ss + 512);
              copy_scales(leader, ta + 8, ss + 1024);
              if (kMake) {
                commit_pair(leader, &sempty[sslot]);
                if (++sslot == kScaleRing) {
                  sslot = 0;
                  sph ^= 1u;
                }
              }
            }
            last_use[slot] = ++blocks;
            const uint32_t sa = smem0 + (uint32_t)(stage * kStage);
            uint64_t* const free = &empty[stage];
            // Whether the next block is there is asked now and known after this
            // block's MMAs: the answer comes late, behind what they read of shared
            // memory.
            if (++stage == kStages) {
              stage = 0;
              ph ^= 1u;
            }
            const bool there = mbar_test(&full[stage], ph), sthere = kMake && mbar_test_cluster(&sfull[sslot], sph);
#pragma unroll
            for (int k = 0; k < kSubs; ++k) {
              const uint64_t a0 = sw128_desc(sa + k * kSubA, 16, 1024), b0 = sw128_desc(sa + kSubs * kSubA + k * kSubB, 16, 1024);
              const uint32_t byte = (uint32_t)((kb & 1) * kSubs + k), id = idesc | byte << 4 | byte << 29;
#pragma unroll
              for (int kk = 0; kk < kSub / 32; ++kk)
                umma_mx8(leader, d, a0 + kk * a_step, b0 + kk * b_step, id, ta, ta + 4, (kb == kc && k == 0 && kk == 0) ? 0u : 1u);
            }
            commit_pair(leader, free);
            ready = __all_sync(0xFFFFFFFFu, there);
            if (kMake) sready = __all_sync(0xFFFFFFFFu, sthere);
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
    many_registers<96>();
    const int half = (warp - kFirstEpi) >> 2, q = warp & 3, r0 = (int)rank * kHalf + q * 32;
    const uint32_t box = smem_u32(smem + R::kBoxes + (size_t)(warp - kFirstEpi) * kWarpBytes);
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const float nan = __int_as_float(0x7FC00000);
    int ab = 0;
    uint32_t aph = 0;
    bool ok = true;
    Items items(sch, pair);
    Item it;
    while (items.next(sch, it)) {
      const int row0 = it.tm * kTileM + r0, c0 = half * kHalfN, col0 = it.tn * kN + c0, rows = min(32, p.m - row0);
      float acc[4][32];
      for (int kc = it.kb0; kc < it.kb1; kc += kChunk8) {
        // one answer for the warp: the TMEM loads below are taken by all lanes or none
        ok = ok && __all_sync(0xFFFFFFFFu, await(&accfull[ab], aph, abort_flag, wait_ns));
        if (!ok) {
          *abort_flag = 1;
          break;
        }
        tc_fence_after();
        const uint32_t from = tmem_base + (uint32_t)(ab * kSecond + c0) + lanes;
        const bool fresh = kc == it.kb0;
        auto take = [&](float (&a)[32], int b) {
          float r[32];
          tmem_load(from + 32 * b, r);
          tmem_wait(r);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 v = add2(fresh ? make_float2(0.f, 0.f) : make_float2(a[e], a[e + 1]), make_float2(r[e], r[e + 1]));
            a[e] = v.x;
            a[e + 1] = v.y;
          }
        };
        auto arrive = [&](uint64_t* bar) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cta0(bar);
        };
        // the first accumulator's last 32 columns are the second one's first
        const bool last_first = ab == 0 && half == 1;
        if (last_first) {
          take(acc[3], 3);
          arrive(&shared[0]);
        }
        take(acc[0], 0);
        if (ab == 1 && half == 0) arrive(&shared[1]);
        take(acc[1], 1);
        take(acc[2], 2);
        if (!last_first) take(acc[3], 3);
        arrive(&accempty[ab]);
        ab ^= 1;
        if (ab == 0) aph ^= 1u;
      }
      if (!ok) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[b][e] = nan;
      }
      if (rows <= 0) continue;
      const bool whole = it.slot < 0 && p.out.tma;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = col0 + 32 * b;
        if (c >= p.n) continue;
        if (whole) {
          // boxes of 32 rows x 64 bytes, 64-byte swizzle: 32 columns in bf16, 16 in fp32
          const int boxes = p.out.dt == LM_BF16 ? 1 : 2;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h >= boxes || c + 16 * h >= p.n) continue;
            box_free(lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float *v = &acc[b][8 * e], *f = &acc[b][16 * h + 4 * e];
              const bool two = boxes == 1;
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)),
                           "r"(two ? pack_bf2(v[0], v[1]) : __float_as_uint(f[0])), "r"(two ? pack_bf2(v[2], v[3]) : __float_as_uint(f[1])),
                           "r"(two ? pack_bf2(v[4], v[5]) : __float_as_uint(f[2])), "r"(two ? pack_bf2(v[6], v[7]) : __float_as_uint(f[3]))
                           : "memory");
            }
            box_ready();
            if (lane == 0) {
              box_store(&p.y, box, c + 16 * h, row0, 0);
              bulk_commit();
            }
          }
        } else if (it.slot < 0) {
          if (p.out.dt == LM_F32) put16_plain<float>(acc[b], box, lane, row0, rows, c, p.n, p.out);
          else put16_plain<__nv_bfloat16>(acc[b], box, lane, row0, rows, c, p.n, p.out);
        } else {
          box_free(lane);
          float* part = p.parts + (size_t)it.slot * (kTileM * kN) + (size_t)r0 * kN + c0 + 32 * b;
          put16(acc[b], box, lane, rows, [&](int r, int e, float4 v) { *reinterpret_cast<float4*>(part + r * kN + e) = v; });
        }
      }
    }
    if (lane == 0) bulk_wait_all();   // stores from the boxes
  } else if constexpr (!kMake) {
    few_registers<96>();
  } else {
    // ---------------------------------- scales -----------------------------------
    // In the order in which the MMA issuer takes them: an item's first stage's, then
    // each even stage's.  The two warps take turns, and load a turn's before they
    // wait for the room of the last one's: a load's time is that of two stages.
    few_registers<96>();
    Items items(sch, pair);
    Item it{};
    int kb = 0;
    auto step = [&]() {
      kb = (kb | 1) + 1;
      if (kb < it.kb1) return true;
      if (!items.next(sch, it)) return false;
      kb = it.kb0;
      return true;
    };
    FourScales now;
    auto load = [&]() { now.load<kGrad>(p.scales, kb >> 1, (int64_t)it.tm * kTileM + (int)rank * kHalf, (int64_t)it.tn * kN, lane); };
    bool more = step() && (warp == 2 || step()), ok = true;
    if (more) load();
    for (uint32_t turn = warp - 2; more; turn += 2) {
      const uint32_t x0 = now.word(now.x[0]), x1 = now.word(now.x[1]), x2 = now.word(now.x[2]), x3 = now.word(now.x[3]);
      const uint32_t w[2] = {now.word(now.w[0]), now.word(now.w[1])};
      more = step() && step();
      if (more) load();
      const uint32_t slot = turn % kScaleRing, ph = turn / kScaleRing & 1u;
      if (!__all_sync(0xFFFFFFFFu, await(&sempty[slot], ph ^ 1u, abort_flag, wait_ns))) {
        ok = false;
        break;
      }
      const uint32_t to = smem_u32(smem + R::kScales + (size_t)slot * kScaleBytes) + 16 * lane;
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(x0), "r"(x1), "r"(x2), "r"(x3) : "memory");
#pragma unroll
      for (int j = 0; j < 2; ++j) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + 512 * (j + 1)), "r"(w[j]) : "memory");
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(peer_addr(&sfull[slot], 0));
    }
    if (!ok && lane == 0) *abort_flag = 1;
  }

  __syncwarp();
  pair_finish<kStages>(*log, abort_flag, full, armed, rank);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
}

cudaError_t encode(CUtensorMap* m, CUtensorMapDataType type, int size, const void* base, int64_t cols, int64_t rows, int64_t planes, int64_t ld, int64_t plane,
                   int box_cols, int box_rows, CUtensorMapSwizzle swizzle) {
  const PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
  if (enc == nullptr) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(plane * size)};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
  return enc(m, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

struct Layout {
  int64_t k, n;
  int32_t groups, fours, row_blocks;
  Schedule sch;
  bool few, make;
  size_t sb, parts, total;     // the activations' scales, the weights', partial sums
};
Layout make_layout(const Linear8Params& q) {
  Layout l{};
  l.k = q.grad ? q.out : q.in;
  l.n = q.grad ? q.in : q.out;
  l.groups = (int32_t)((l.k + kBlock - 1) / kBlock);
  l.fours = (l.groups + 3) / 4;
  l.row_blocks = (int32_t)((q.tokens + 127) / 128);
  l.few = q.tokens <= kFewTokens;
  // few tokens: half of the pairs draw the weights as fast as all, and a sum that is
  // not split needs no second kernel
  l.sch = plain_schedule(q.tokens, l.n, l.k, 1, kN, kK);
  if (!l.few || l.sch.units < kPairs / 2) l.sch = split_schedule(q.tokens, l.n, l.k, kN, kK, kLeastShare);
  l.make = l.few || (int64_t)l.sch.tiles_m * l.sch.tiles_n * ((l.k + kK - 1) / kK) <= (int64_t)kPairs * kMakeStages;
  l.sb = l.make ? 0 : (size_t)l.fours * l.row_blocks * 512;
  l.parts = l.make ? 0 : l.sb + (size_t)l.fours * l.sch.tiles_n * 1024;
  l.total = l.parts + parts_bytes(l.sch, kN);
  return l;
}

template <bool kGrad, bool kFew, bool kMake>
cudaError_t start8(const Params8& p, cudaStream_t st) {
  const int dev = device_slot();
  static bool ready[kMaxDevices];
  if (dev < 0 || !ready[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(linear8_kernel<kGrad, kFew, kMake>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Ring<kFew, kMake>::kBytes);
    if (e != cudaSuccess) return e;
    if (dev >= 0) ready[dev] = true;
  }
  return launch_after(linear8_kernel<kGrad, kFew, kMake>, dim3(2 * pairs_of(p.sch)), kThreads, Ring<kFew, kMake>::kBytes, st, p);
}

}  // namespace

cudaError_t launch_weight8_pack(lm_dtype dt, const Mat& w, int64_t nrows, int64_t cols, const Blocks& c, cudaStream_t st) {
  const dim3 grid((unsigned)((cols + kBlock - 1) / kBlock), (unsigned)std::min<int64_t>((nrows + kBlock - 1) / kBlock, 65535));
  const bool vec = rows::aligned(w, dt == LM_F32 ? 4 : 2, nrows);
  if (dt == LM_F32) return launch_after(vec ? weight8_pack_kernel<float, true> : weight8_pack_kernel<float, false>, grid, 256, 0, st, w, nrows, cols, c);
  return launch_after(vec ? weight8_pack_kernel<__nv_bfloat16, true> : weight8_pack_kernel<__nv_bfloat16, false>, grid, 256, 0, st, w, nrows, cols, c);
}

cudaError_t launch_weight8_unpack(lm_dtype dt, const Blocks& c, int64_t nrows, int64_t cols, const Mat& w, cudaStream_t st) {
  const bool vec = rows::aligned(w, dt == LM_F32 ? 4 : 2, nrows);
  const dim3 grid((unsigned)((cols + 255) / 256), (unsigned)std::min<int64_t>((nrows + 31) / 32, 65535));
  if (dt == LM_F32) return launch_after(vec ? values_kernel<float, true> : values_kernel<float, false>, grid, 256, 0, st, c, nrows, cols, w);
  return launch_after(vec ? values_kernel<__nv_bfloat16, true> : values_kernel<__nv_bfloat16, false>, grid, 256, 0, st, c, nrows, cols, w);
}

size_t linear8_workspace(const Linear8Params& q) { return q.tokens <= 0 || q.in <= 0 || q.out <= 0 ? 0 : make_layout(q).total; }

cudaError_t launch_linear8(const Linear8Params& q, cudaStream_t st) {
  if ((q.grad ? q.out : q.in) == 0) return start_zero(q.y, q.ydt, q.tokens, q.grad ? q.in : q.out, st);
  const Layout l = make_layout(q);
  uint8_t* ws = static_cast<uint8_t*>(q.workspace);
  uint32_t *sa = reinterpret_cast<uint32_t*>(ws), *sb = reinterpret_cast<uint32_t*>(ws + l.sb);
  Params8 p{};
  p.scales = Scales{q.x.scales, q.w.scales, q.x.ld_scales, q.w.ld_scales, q.tokens, (int32_t)l.n, l.groups};
  cudaError_t e;
  if (!l.make) {
    const ScaleParams sp{p.scales, l.fours, l.row_blocks, l.sch.tiles_n, q.grad, sa, sb};
    const int64_t words = (int64_t)l.fours * (l.row_blocks + 2 * (int64_t)l.sch.tiles_n);      // blocks of 128
    if ((e = launch_after(scales_kernel, dim3((unsigned)std::min<int64_t>(words, 152 * 32)), 128, 0, st, sp)) != cudaSuccess) return e;
  }
  p.sch = l.sch;
  share(p.sch);
  p.m = (int32_t)q.tokens;
  p.n = (int32_t)l.n;
  p.wait_ns = env_wait_limit_ns();
  p.parts = reinterpret_cast<float*>(ws + l.parts);
  p.out = make_store(q.y, q.ydt, q.tokens, false);
  const int64_t ld = q.tokens > 1 ? q.y.ld : l.n, size = q.ydt == LM_F32 ? 4 : 2;
  if (tma_stores(q.y.data, q.tokens, l.n, ld, size)) {
    e = q.ydt == LM_F32 ? encode(&p.y, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, q.y.data, l.n, q.tokens, 1, ld, ld * q.tokens, 16, 32, CU_TENSOR_MAP_SWIZZLE_64B)
                        : encode(&p.y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, q.y.data, l.n, q.tokens, 1, ld, ld * q.tokens, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
    if (e != cudaSuccess) return e;
    p.out.tma = 1;
  }
  const CUtensorMapDataType u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8, u32 = CU_TENSOR_MAP_DATA_TYPE_UINT32;
  const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B, none = CU_TENSOR_MAP_SWIZZLE_NONE;
  if ((e = encode(&p.a, u8, 1, q.x.data, l.k, q.tokens, 1, q.x.ld, q.x.ld * q.tokens, kSub, l.few ? kFewTokens : kHalf, sw)) != cudaSuccess) return e;
  if ((e = encode(&p.b, u8, 1, q.w.data, q.in, q.out, 1, q.w.ld, q.w.ld * q.out, 128, q.grad ? kSub : kHalfN, sw)) != cudaSuccess) return e;
  if (!l.make && (e = encode(&p.sa, u32, 4, sa, 128, l.row_blocks, l.fours, 128, 128 * (int64_t)l.row_blocks, 128, 1, none)) != cudaSuccess) return e;
  if (!l.make && (e = encode(&p.sb, u32, 4, sb, 256, l.sch.tiles_n, l.fours, 256, 256 * (int64_t)l.sch.tiles_n, 256, 1, none)) != cudaSuccess) return e;
  if (l.few) e = q.grad ? start8<true, true, true>(p, st) : start8<false, true, true>(p, st);
  else if (l.make) e = q.grad ? start8<true, false, true>(p, st) : start8<false, false, true>(p, st);
  else e = q.grad ? start8<true, false, false>(p, st) : start8<false, false, false>(p, st);
  if (e != cudaSuccess || !has_parts(p.sch)) return e;
  return start_join<kN>(p.sch, p.m, p.n, p.parts, p.out, st);
}

}  // namespace lm
