// Internal declarations of the training-step operators: the launch parameters
// that lm_train_api.cu fills from checked arguments, and the launchers of
// lm_logprob.cu, lm_linlogp.cu, lm_rmsnorm.cu, lm_rotary.cu, lm_checkpoint8.cu,
// lm_wgrad8.cu and lm_linear8.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "lm_internal.h"

namespace lm {

// A checked matrix: row r at data + r * ld elements.
struct Mat {
  void* data;
  int64_t ld;
};
// A checked 8-bit checkpoint (data NULL: none).
struct Codes {
  uint8_t* data;
  float* scales;
  int64_t ld, ld_scales;
  int format;
};

struct LogprobParams {
  const void* logits;
  int64_t ld;
  int64_t rows;
  int32_t vocab;
  int32_t top_k;
  const int64_t* targets;
  float *logp, *entropy, *lse, *top_logp;
  int64_t* top_index;
  const float *g_logp, *g_entropy, *g_lse;
  void* dlogits;        // NULL: no gradient
  int64_t ld_d;
  int32_t cluster;      // blocks a row, set by the launcher
};
cudaError_t launch_logprob(lm_dtype dt, const LogprobParams& p, cudaStream_t st);
// p.lse and p.entropy are read
cudaError_t launch_logprob_grad(lm_dtype dt, const LogprobParams& p, cudaStream_t st);

struct NormParams {
  int64_t rows;
  int32_t cols;
  int32_t wdt;          // dtype of weight / dweight
  Mat x, residual, h, y;   // data NULL where absent
  const void* weight;
  float eps;
  float* rstd;
  Codes kept;
};
cudaError_t launch_rmsnorm(lm_dtype dt, const NormParams& p, cudaStream_t st);

struct NormGradParams {
  int64_t rows;
  int32_t cols;
  int32_t wdt;          // dtype of weight
  int32_t dwdt;         // dtype of dweight
  Mat dy, h, dh, dx;
  Codes h8;
  const float* rstd;
  const void* weight;
  void* dweight;
  float* parts;         // dweight summed over each block's rows: blocks x cols
};
constexpr int kNormGradParts = 608;    // most blocks of a norm's gradient
cudaError_t launch_rmsnorm_grad(lm_dtype dt, const NormGradParams& p, cudaStream_t st);

cudaError_t launch_pack8(lm_dtype dt, const Mat& x, int64_t rows, int64_t cols, const Codes& c, cudaStream_t st);
cudaError_t launch_unpack8(lm_dtype dt, const Codes& c, int64_t rows, int64_t cols, const Mat& x, cudaStream_t st);

struct WgradParams {
  int64_t tokens;
  int32_t out, in;
  int32_t dydt, dwdt;
  Mat dy, dw;
  Codes x;
  int32_t accumulate;
  void* workspace;
};
size_t wgrad8_workspace(const Mat& dy, int dydt, int64_t tokens, int64_t out, int64_t in);
cudaError_t launch_wgrad8(const WgradParams& p, cudaStream_t st);

struct LinLogpParams {
  int64_t rows;
  int32_t vocab, width;
  Mat h, w;             // bf16
  const int64_t* targets;
  float *logp, *entropy, *lse;
  const float *g_logp, *g_entropy, *g_lse;
  bool gradient_only;   // lse and entropy are read
  Mat dh, dw;           // data NULL where absent; dh bf16
  int dwdt;
  int accumulate;       // adds to dw
  void* workspace;
};
size_t linlogp_workspace(const LinLogpParams& p);
cudaError_t launch_linlogp(const LinLogpParams& p, cudaStream_t st);

// A checked 8-bit weight matrix.
struct Blocks {
  uint8_t* data;
  float* scales;
  int64_t ld, ld_scales;
};
cudaError_t launch_weight8_pack(lm_dtype dt, const Mat& w, int64_t rows, int64_t cols, const Blocks& c, cudaStream_t st);
cudaError_t launch_weight8_unpack(lm_dtype dt, const Blocks& c, int64_t rows, int64_t cols, const Mat& w, cudaStream_t st);

struct Linear8Params {
  int64_t tokens;
  int32_t out, in;      // of the weights
  Codes x;              // tokens x in; tokens x out for the input gradient
  Blocks w;
  Mat y;
  int ydt;
  bool grad;
  void* workspace;
};
size_t linear8_workspace(const Linear8Params& p);
cudaError_t launch_linear8(const Linear8Params& p, cudaStream_t st);

// Heads of one tensor: channel c of head h of token t at data[t * ld_token + h * ld_head + c].
struct Heads {
  void* data;
  int64_t ld_token, ld_head;
};
struct RotaryPart {
  int32_t heads;        // 0: absent
  Heads x, y, dy, dx;   // forward: x -> y; gradient: dy (and x with the norm) -> dx
  const void* weight;   // NULL for ones
  int wdt;
  void* dweight;        // NULL: not wanted
  int dwdt;
};
struct RotaryParams {
  int64_t tokens;
  int32_t dim, turned;
  const int64_t* positions;
  const float* table;   // table_rows x turned / 2 x (cos, sin)
  int64_t table_rows;
  RotaryPart part[2];   // queries, keys
  bool norm, interleaved;
  float eps;
  float* sums;          // dweight's parts: blocks x dim for each part
};
size_t rotary_grad_workspace(int64_t tokens, int64_t heads, int32_t dim);
cudaError_t launch_rotary(lm_dtype dt, const RotaryParams& p, cudaStream_t st);
cudaError_t launch_rotary_grad(lm_dtype dt, const RotaryParams& p, cudaStream_t st);

}  // namespace lm
