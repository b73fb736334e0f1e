// C entry points of the training-step operators: every argument is checked
// here, before anything is enqueued; the kernels see only what passed.
#include <cuda_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "lm_train.h"

namespace lm {
namespace {

lm_status fail(lm_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
lm_status fail(lm_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return set_error(st, buf);
}
#define LM_TRY(call)                       \
  do {                                     \
    const lm_status st_ = (call);          \
    if (st_ != LM_OK) return st_;          \
  } while (0)

lm_status launched(cudaError_t e, const char* what) {
  return e == cudaSuccess ? LM_OK : fail(LM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Extents are bounded so that every index fits: columns in 31 bits, and the
// last byte of a matrix in 63.
constexpr int64_t kMaxCols = 0x7FFFFF00ll;
constexpr int64_t kMaxBytes = (int64_t)1 << 62;
// The norm's kernels count channels in whole rounds of a block's threads (8192
// channels at most), past the row's end.
constexpr int64_t kMaxNormCols = 0x7FFF0000ll;

lm_status current_device(int* dev) {
  if (cudaGetDevice(dev) != cudaSuccess) return fail(LM_ERR_CUDA, "no CUDA device");
  int major = 0, minor = 0;
  cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev);
  cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, *dev);
  if (major != 10 || minor != 3)
    return fail(LM_ERR_UNSUPPORTED, "device %d is sm_%d%d; this library is built for sm_103a", *dev, major, minor);
  return LM_OK;
}

lm_status check_extent(int64_t rows, int64_t cols, const char* what) {
  if (rows < 0 || cols < 0) return fail(LM_ERR_INVALID_ARG, "%s: negative extent", what);
  if (cols > kMaxCols || rows > kMaxCols) return fail(LM_ERR_UNSUPPORTED, "%s: more than 2^31 - 256 rows or columns", what);
  return LM_OK;
}

lm_status check_norm_cols(int64_t cols) {
  return cols > kMaxNormCols ? fail(LM_ERR_UNSUPPORTED, "%lld channels, more than 2^31 - 2^16", (long long)cols) : LM_OK;
}

// Shape, type, pitch and element alignment of a matrix argument (no device access).
lm_status check_matrix(const lm_matrix& m, int64_t rows, int64_t cols, const char* what) {
  if (m.dtype != LM_F32 && m.dtype != LM_BF16) return fail(LM_ERR_DTYPE, "%s: dtype %d is not LM_F32 or LM_BF16", what, (int)m.dtype);
  if (m.rows != rows || m.cols != cols)
    return fail(LM_ERR_INVALID_ARG, "%s is %lld x %lld, expected %lld x %lld", what, (long long)m.rows, (long long)m.cols,
                (long long)rows, (long long)cols);
  LM_TRY(check_extent(rows, cols, what));
  if (rows == 0 || cols == 0) return LM_OK;
  if (m.data == nullptr) return fail(LM_ERR_INVALID_ARG, "%s: NULL data", what);
  if (rows > 1 && m.ld < cols) return fail(LM_ERR_INVALID_ARG, "%s: row pitch %lld is below its %lld columns", what, (long long)m.ld, (long long)cols);
  const int64_t size = m.dtype == LM_F32 ? 4 : 2;
  if (rows > 1 && m.ld > kMaxBytes / size / rows) return fail(LM_ERR_UNSUPPORTED, "%s: row pitch too large", what);
  if (reinterpret_cast<uintptr_t>(m.data) % size != 0) return fail(LM_ERR_ALIGN, "%s: data is not aligned to its element", what);
  return LM_OK;
}

lm_status check_codes(const lm_checkpoint8& c, int64_t rows, int64_t cols, const char* what) {
  if (c.format != LM_CODE_I8 && c.format != LM_CODE_E4M3) return fail(LM_ERR_DTYPE, "%s: unknown code format %d", what, (int)c.format);
  if (c.rows != rows || c.cols != cols)
    return fail(LM_ERR_INVALID_ARG, "%s is %lld x %lld, expected %lld x %lld", what, (long long)c.rows, (long long)c.cols,
                (long long)rows, (long long)cols);
  LM_TRY(check_extent(rows, cols, what));
  if (rows == 0 || cols == 0) return LM_OK;
  if (c.codes == nullptr || c.scales == nullptr) return fail(LM_ERR_INVALID_ARG, "%s: NULL codes or scales", what);
  if (c.ld_codes < cols || c.ld_scales < rows) return fail(LM_ERR_INVALID_ARG, "%s: pitch of codes or scales below the extent", what);
  if (c.ld_codes % 16 != 0 || reinterpret_cast<uintptr_t>(c.codes) % 16 != 0 || reinterpret_cast<uintptr_t>(c.scales) % 4 != 0)
    return fail(LM_ERR_ALIGN, "%s: codes and their pitch must be multiples of 16 bytes, scales of 4", what);
  if (c.ld_codes > kMaxBytes / rows || c.ld_scales > kMaxBytes / 4 / ((cols + LM_CODE_GROUP - 1) / LM_CODE_GROUP))
    return fail(LM_ERR_UNSUPPORTED, "%s: pitch too large", what);
  return LM_OK;
}

// A vector of n elements given as an lm_tensor (1 x n or n x 1).
lm_status check_vector(const lm_tensor& v, int64_t n, const char* what) {
  if (v.dtype != LM_F32 && v.dtype != LM_BF16) return fail(LM_ERR_DTYPE, "%s: dtype %d is not LM_F32 or LM_BF16", what, (int)v.dtype);
  if (!((v.rows == 1 && v.cols == n) || (v.cols == 1 && v.rows == n)))
    return fail(LM_ERR_INVALID_ARG, "%s is %lld x %lld, expected a vector of %lld", what, (long long)v.rows, (long long)v.cols, (long long)n);
  if (n == 0) return LM_OK;
  if (v.data == nullptr) return fail(LM_ERR_INVALID_ARG, "%s: NULL data", what);
  if (reinterpret_cast<uintptr_t>(v.data) % (v.dtype == LM_F32 ? 4 : 2) != 0) return fail(LM_ERR_ALIGN, "%s: data is not aligned to its element", what);
  return LM_OK;
}

lm_status check_aligned(const void* p, size_t to, const char* what) {
  return reinterpret_cast<uintptr_t>(p) % to != 0 ? fail(LM_ERR_ALIGN, "%s: not aligned to %zu bytes", what, to) : LM_OK;
}

// NULL, or device (or managed) memory of device dev.
lm_status check_memory(const void* p, int dev, const char* what) {
  if (p == nullptr) return LM_OK;
  cudaPointerAttributes a{};
  const cudaError_t e = cudaPointerGetAttributes(&a, p);
  if (e != cudaSuccess) {
    cudaGetLastError();   // an unknown pointer is an argument error, not a sticky CUDA error
    return fail(LM_ERR_INVALID_ARG, "%s: not a CUDA pointer (%s)", what, cudaGetErrorString(e));
  }
  if (a.type != cudaMemoryTypeDevice && a.type != cudaMemoryTypeManaged)
    return fail(LM_ERR_INVALID_ARG, "%s: %s memory, not device memory", what, a.type == cudaMemoryTypeHost ? "page-locked host" : "unregistered host");
  if (a.type == cudaMemoryTypeDevice && a.device != dev)
    return fail(LM_ERR_INVALID_ARG, "%s: memory of device %d, the call runs on device %d", what, a.device, dev);
  return LM_OK;
}

// A one-row matrix's pitch is not read by the caller's contract.
Mat mat(const lm_matrix* m) { return m == nullptr ? Mat{nullptr, 0} : Mat{m->data, m->rows > 1 ? m->ld : m->cols}; }
Codes codes(const lm_checkpoint8* c) {
  if (c == nullptr) return Codes{nullptr, nullptr, 0, 0, 0};
  return Codes{static_cast<uint8_t*>(c->codes), c->scales, c->ld_codes, c->ld_scales, (int)c->format};
}

lm_status logprob_call(const lm_token_logprob_args* a, bool gradient_only, void* cuda_stream) {
  if (a == nullptr) return fail(LM_ERR_INVALID_ARG, "args is NULL");
  const int64_t n = a->logits.rows, v = a->logits.cols;
  LM_TRY(check_matrix(a->logits, n, v, "logits"));
  const bool grad = a->dlogits.data != nullptr;
  if (gradient_only && !grad && n > 0 && v > 0) return fail(LM_ERR_INVALID_ARG, "dlogits is NULL");
  if (grad) {
    LM_TRY(check_matrix(a->dlogits, n, v, "dlogits"));
    if (a->dlogits.dtype != a->logits.dtype) return fail(LM_ERR_DTYPE, "dlogits and logits differ in dtype");
    if (a->g_logp == nullptr && a->g_entropy == nullptr && a->g_lse == nullptr)
      return fail(LM_ERR_INVALID_ARG, "dlogits without any of g_logp, g_entropy, g_lse");
    if (a->dlogits.data == a->logits.data && n > 1 && a->dlogits.ld != a->logits.ld)
      return fail(LM_ERR_INVALID_ARG, "dlogits written over logits needs the same row pitch");
  } else if (a->g_logp != nullptr || a->g_entropy != nullptr || a->g_lse != nullptr) {
    return fail(LM_ERR_INVALID_ARG, "g_logp, g_entropy or g_lse without dlogits");
  }
  const float* logp = gradient_only ? nullptr : a->logp;
  const int k = gradient_only ? 0 : a->top_k;
  if (a->targets == nullptr && n > 0 && (logp != nullptr || a->g_logp != nullptr)) return fail(LM_ERR_INVALID_ARG, "targets is NULL");
  if (k < 0 || k > 32 || k > v) return fail(LM_ERR_INVALID_ARG, "top_k %d is outside 0 .. min(32, vocabulary)", k);
  if (!gradient_only && n > 0 && ((a->top_logp != nullptr) != (k > 0) || (a->top_index != nullptr) != (k > 0)))
    return fail(LM_ERR_INVALID_ARG, "top_logp and top_index go with top_k > 0");
  if (gradient_only && n > 0 && (a->lse == nullptr || (a->g_entropy != nullptr && a->entropy == nullptr)))
    return fail(LM_ERR_INVALID_ARG, "the gradient reads lse, and entropy with g_entropy");
  if (n > 0 && v == 0) return fail(LM_ERR_INVALID_ARG, "an empty vocabulary");
  LM_TRY(check_aligned(a->targets, 8, "targets"));
  const void* floats[] = {logp, a->entropy, a->lse, a->g_logp, a->g_entropy, a->g_lse, k > 0 ? a->top_logp : nullptr};
  for (const void* f : floats) LM_TRY(check_aligned(f, 4, "a float array"));
  if (k > 0) LM_TRY(check_aligned(a->top_index, 8, "top_index"));
  if (n == 0) return LM_OK;
  int dev = 0;
  LM_TRY(current_device(&dev));
  LM_TRY(check_memory(a->logits.data, dev, "logits"));
  if (a->dlogits.data != a->logits.data) LM_TRY(check_memory(a->dlogits.data, dev, "dlogits"));
  LM_TRY(check_memory(a->targets, dev, "targets"));
  for (const void* f : floats) LM_TRY(check_memory(f, dev, "a float array"));
  if (k > 0) LM_TRY(check_memory(a->top_index, dev, "top_index"));
  LogprobParams p{};
  p.logits = a->logits.data;
  p.ld = mat(&a->logits).ld;
  p.rows = n;
  p.vocab = (int32_t)v;
  p.top_k = k;
  p.targets = a->targets;
  p.logp = a->logp;
  p.entropy = a->entropy;
  p.lse = a->lse;
  p.top_logp = a->top_logp;
  p.top_index = a->top_index;
  p.g_logp = a->g_logp;
  p.g_entropy = a->g_entropy;
  p.g_lse = a->g_lse;
  p.dlogits = a->dlogits.data;
  p.ld_d = n > 1 ? a->dlogits.ld : v;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return gradient_only ? launched(launch_logprob_grad(a->logits.dtype, p, st), "lm_token_logprob_grad")
                       : launched(launch_logprob(a->logits.dtype, p, st), "lm_token_logprob");
}

}  // namespace
}  // namespace lm

using namespace lm;

extern "C" {

lm_status lm_token_logprob(const lm_token_logprob_args* a, void* cuda_stream) { return logprob_call(a, false, cuda_stream); }
lm_status lm_token_logprob_grad(const lm_token_logprob_args* a, void* cuda_stream) { return logprob_call(a, true, cuda_stream); }

lm_status lm_checkpoint8_pack(const lm_matrix* x, const lm_checkpoint8* c, void* cuda_stream) {
  if (x == nullptr || c == nullptr) return fail(LM_ERR_INVALID_ARG, "x or c is NULL");
  LM_TRY(check_matrix(*x, x->rows, x->cols, "x"));
  LM_TRY(check_codes(*c, x->rows, x->cols, "c"));
  if (x->rows == 0 || x->cols == 0) return LM_OK;
  int dev = 0;
  LM_TRY(current_device(&dev));
  LM_TRY(check_memory(x->data, dev, "x"));
  LM_TRY(check_memory(c->codes, dev, "codes"));
  LM_TRY(check_memory(c->scales, dev, "scales"));
  return launched(launch_pack8(x->dtype, mat(x), x->rows, x->cols, codes(c), static_cast<cudaStream_t>(cuda_stream)), "lm_checkpoint8_pack");
}

lm_status lm_checkpoint8_unpack(const lm_checkpoint8* c, const lm_matrix* x, void* cuda_stream) {
  if (x == nullptr || c == nullptr) return fail(LM_ERR_INVALID_ARG, "x or c is NULL");
  LM_TRY(check_matrix(*x, x->rows, x->cols, "x"));
  LM_TRY(check_codes(*c, x->rows, x->cols, "c"));
  if (x->rows == 0 || x->cols == 0) return LM_OK;
  int dev = 0;
  LM_TRY(current_device(&dev));
  LM_TRY(check_memory(x->data, dev, "x"));
  LM_TRY(check_memory(c->codes, dev, "codes"));
  LM_TRY(check_memory(c->scales, dev, "scales"));
  return launched(launch_unpack8(x->dtype, codes(c), x->rows, x->cols, mat(x), static_cast<cudaStream_t>(cuda_stream)), "lm_checkpoint8_unpack");
}

lm_status lm_rmsnorm(const lm_matrix* x, const lm_matrix* residual, const lm_tensor* weight, double eps,
                     const lm_matrix* h, const lm_matrix* y, float* rstd, const lm_checkpoint8* kept,
                     void* cuda_stream) {
  if (x == nullptr) return fail(LM_ERR_INVALID_ARG, "x is NULL");
  if (!(eps >= 0.0) || !isfinite(eps)) return fail(LM_ERR_INVALID_ARG, "eps must be finite and >= 0");
  const int64_t rows = x->rows, cols = x->cols;
  LM_TRY(check_matrix(*x, rows, cols, "x"));
  LM_TRY(check_norm_cols(cols));
  if (h != nullptr && residual == nullptr) return fail(LM_ERR_INVALID_ARG, "h is x itself without a residual");
  const lm_matrix* others[] = {residual, h, y};
  const char* names[] = {"residual", "h", "y"};
  for (int i = 0; i < 3; ++i) {
    if (others[i] == nullptr) continue;
    LM_TRY(check_matrix(*others[i], rows, cols, names[i]));
    if (others[i]->dtype != x->dtype) return fail(LM_ERR_DTYPE, "%s and x differ in dtype", names[i]);
  }
  for (int i = 0; h != nullptr && i < 2; ++i) {
    const lm_matrix* in = i == 0 ? x : residual;
    if (rows > 1 && h->data == in->data && h->ld != in->ld) return fail(LM_ERR_INVALID_ARG, "h written over an input needs the same row pitch");
  }
  if (weight != nullptr) LM_TRY(check_vector(*weight, cols, "weight"));
  if (kept != nullptr) LM_TRY(check_codes(*kept, rows, cols, "kept"));
  LM_TRY(check_aligned(rstd, 4, "rstd"));
  if (rows == 0 || (cols == 0 && rstd == nullptr)) return LM_OK;
  int dev = 0;
  LM_TRY(current_device(&dev));
  if (cols > 0) {   // (without channels rstd alone is written, nothing is read)
    LM_TRY(check_memory(x->data, dev, "x"));
    for (int i = 0; i < 3; ++i)
      if (others[i] != nullptr) LM_TRY(check_memory(others[i]->data, dev, names[i]));
    if (weight != nullptr) LM_TRY(check_memory(weight->data, dev, "weight"));
  }
  LM_TRY(check_memory(rstd, dev, "rstd"));
  if (kept != nullptr && cols > 0) {
    LM_TRY(check_memory(kept->codes, dev, "codes"));
    LM_TRY(check_memory(kept->scales, dev, "scales"));
  }
  NormParams p{};
  p.rows = rows;
  p.cols = (int32_t)cols;
  p.x = mat(x);
  p.residual = mat(residual);
  p.h = mat(h);
  p.y = mat(y);
  p.weight = weight != nullptr ? weight->data : nullptr;
  p.wdt = weight != nullptr ? (int)weight->dtype : LM_F32;
  p.eps = (float)eps;
  p.rstd = rstd;
  p.kept = codes(kept);
  return launched(launch_rmsnorm(x->dtype, p, static_cast<cudaStream_t>(cuda_stream)), "lm_rmsnorm");
}

size_t lm_rmsnorm_grad_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return 0;
  const int64_t blocks = rows < kNormGradParts ? rows : kNormGradParts;
  return (size_t)blocks * (size_t)cols * sizeof(float);
}

lm_status lm_rmsnorm_grad(const lm_matrix* dy, const lm_matrix* h, const lm_checkpoint8* h8, const float* rstd,
                          const lm_tensor* weight, const lm_matrix* dh, const lm_matrix* dx, const lm_tensor* dweight,
                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (dy == nullptr) return fail(LM_ERR_INVALID_ARG, "dy is NULL");
  if ((h == nullptr) == (h8 == nullptr)) return fail(LM_ERR_INVALID_ARG, "exactly one of h and h8 must be given");
  if (dx == nullptr && dweight == nullptr) return fail(LM_ERR_INVALID_ARG, "dx and dweight are both NULL");
  const int64_t rows = dy->rows, cols = dy->cols;
  LM_TRY(check_matrix(*dy, rows, cols, "dy"));
  LM_TRY(check_norm_cols(cols));
  if (h != nullptr) LM_TRY(check_matrix(*h, rows, cols, "h"));
  else LM_TRY(check_codes(*h8, rows, cols, "h8"));
  const lm_matrix* same[] = {h, dh, dx};
  const char* names[] = {"h", "dh", "dx"};
  for (int i = 0; i < 3; ++i) {
    if (same[i] == nullptr) continue;
    LM_TRY(check_matrix(*same[i], rows, cols, names[i]));
    if (same[i]->dtype != dy->dtype) return fail(LM_ERR_DTYPE, "%s and dy differ in dtype", names[i]);
  }
  for (int i = 0; dx != nullptr && i < 2; ++i) {
    const lm_matrix* in = i == 0 ? dy : dh;
    if (in != nullptr && rows > 1 && dx->data == in->data && dx->ld != in->ld)
      return fail(LM_ERR_INVALID_ARG, "dx written over an input needs the same row pitch");
  }
  if (weight != nullptr) LM_TRY(check_vector(*weight, cols, "weight"));
  if (dweight != nullptr) LM_TRY(check_vector(*dweight, cols, "dweight"));
  if (rstd == nullptr && rows > 0 && cols > 0) return fail(LM_ERR_INVALID_ARG, "rstd is NULL");
  LM_TRY(check_aligned(rstd, 4, "rstd"));
  if (cols == 0 || (rows == 0 && dweight == nullptr)) return LM_OK;
  if (dweight != nullptr && rows > 0) {
    const size_t need = lm_rmsnorm_grad_workspace(rows, cols);
    if (workspace == nullptr || workspace_bytes < need)
      return fail(LM_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", workspace == nullptr ? (size_t)0 : workspace_bytes, need);
    LM_TRY(check_aligned(workspace, 16, "workspace"));
  }
  int dev = 0;
  LM_TRY(current_device(&dev));
  if (rows > 0) {
    LM_TRY(check_memory(dy->data, dev, "dy"));
    if (h != nullptr) LM_TRY(check_memory(h->data, dev, "h"));
    if (h8 != nullptr) {
      LM_TRY(check_memory(h8->codes, dev, "codes"));
      LM_TRY(check_memory(h8->scales, dev, "scales"));
    }
    if (dh != nullptr) LM_TRY(check_memory(dh->data, dev, "dh"));
    if (dx != nullptr) LM_TRY(check_memory(dx->data, dev, "dx"));
    LM_TRY(check_memory(rstd, dev, "rstd"));
    if (weight != nullptr) LM_TRY(check_memory(weight->data, dev, "weight"));
    if (dweight != nullptr) LM_TRY(check_memory(workspace, dev, "workspace"));
  }
  if (dweight != nullptr) LM_TRY(check_memory(dweight->data, dev, "dweight"));
  NormGradParams p{};
  p.rows = rows;
  p.cols = (int32_t)cols;
  p.dy = mat(dy);
  p.h = mat(h);
  p.h8 = codes(h8);
  p.dh = mat(dh);
  p.dx = mat(dx);
  p.rstd = rstd;
  p.weight = weight != nullptr ? weight->data : nullptr;
  p.wdt = weight != nullptr ? (int)weight->dtype : LM_F32;
  p.dweight = dweight != nullptr ? dweight->data : nullptr;
  p.dwdt = dweight != nullptr ? (int)dweight->dtype : LM_F32;
  p.parts = static_cast<float*>(workspace);
  return launched(launch_rmsnorm_grad(dy->dtype, p, static_cast<cudaStream_t>(cuda_stream)), "lm_rmsnorm_grad");
}

size_t lm_linear_wgrad8_workspace(const lm_matrix* dy, const lm_checkpoint8* x, const lm_matrix* dw) {
  if (dy == nullptr || x == nullptr || dw == nullptr) return 0;
  if (dy->rows < 0 || dy->cols <= 0 || x->cols <= 0) return 0;
  return wgrad8_workspace(mat(dy), (int)dy->dtype, dy->rows, dy->cols, x->cols);
}

lm_status lm_linear_wgrad8(const lm_matrix* dy, const lm_checkpoint8* x, const lm_matrix* dw, int accumulate,
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (dy == nullptr || x == nullptr || dw == nullptr) return fail(LM_ERR_INVALID_ARG, "dy, x or dw is NULL");
  const int64_t tokens = dy->rows, out = dy->cols, in = x->cols;
  LM_TRY(check_matrix(*dy, tokens, out, "dy"));
  LM_TRY(check_codes(*x, tokens, in, "x"));
  LM_TRY(check_matrix(*dw, out, in, "dw"));
  if (out == 0 || in == 0 || (tokens == 0 && accumulate != 0)) return LM_OK;
  // the tensor maps hold strides below 2^40 bytes
  constexpr int64_t kMost = (int64_t)1 << 38;
  if (tokens > 0 && ((tokens > 1 && dy->ld > kMost / tokens) || out > kMost / tokens || in > kMost / tokens || x->ld_codes > kMost / tokens))
    return fail(LM_ERR_UNSUPPORTED, "dy or x of 2^38 elements or more");
  const size_t need = lm_linear_wgrad8_workspace(dy, x, dw);
  if (need > 0) {
    if (workspace == nullptr || workspace_bytes < need)
      return fail(LM_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", workspace == nullptr ? (size_t)0 : workspace_bytes, need);
    LM_TRY(check_aligned(workspace, 256, "workspace"));
  }
  int dev = 0;
  LM_TRY(current_device(&dev));
  if (tokens > 0) {
    LM_TRY(check_memory(dy->data, dev, "dy"));
    LM_TRY(check_memory(x->codes, dev, "codes"));
    LM_TRY(check_memory(x->scales, dev, "scales"));
    if (need > 0) LM_TRY(check_memory(workspace, dev, "workspace"));
  }
  LM_TRY(check_memory(dw->data, dev, "dw"));
  WgradParams p{};
  p.tokens = tokens;
  p.out = (int32_t)out;
  p.in = (int32_t)in;
  p.dydt = (int)dy->dtype;
  p.dwdt = (int)dw->dtype;
  p.dy = mat(dy);
  p.dw = mat(dw);
  p.x = codes(x);
  p.accumulate = accumulate != 0;
  p.workspace = workspace;
  return launched(launch_wgrad8(p, static_cast<cudaStream_t>(cuda_stream)), "lm_linear_wgrad8");
}

}  // extern "C"
