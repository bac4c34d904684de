// C ABI of the training step around the codec: argument checks of the embedding
// lookup and gradient, the gradient norm and the AdamW step.

#include <math.h>

#include <string>

#include "gift_internal.h"

namespace gift {

namespace {

constexpr int64_t kMaxIds = (1LL << 31) - 1;       // positions of all ranks; sort places are 32-bit
constexpr int64_t kMaxVocab = (1LL << 31) - 2;
constexpr int64_t kMaxWidth = 1LL << 20;
constexpr int64_t kMaxElements = 1LL << 33;      // of a tensor: one launch takes its chunks

bool is_dtype(int t) { return t == GIFT_F32 || t == GIFT_BF16; }

gift_status fail(gift_status st, const char *call, const char *what) {
  return set_error(st, std::string(call) + ": " + what);
}

// binds the context to the current device, or checks that its device is current
gift_status enter(gift_ctx *ctx, const char *call) {
  gift_status st = bind_device(ctx);
  if (st != GIFT_OK) return st;
  int dev = -1;
  GIFT_HIP_TRY(hipGetDevice(&dev));
  if (dev != ctx->device) return fail(GIFT_EINVAL, call, "the context's device is not the current one");
  return GIFT_OK;
}

// No events are recorded into a graph: while the stream is being captured the
// call's launches are not timed.
struct QuietCapture {
  gift_ctx *ctx;
  bool was;
  explicit QuietCapture(gift_ctx *c) : ctx(c), was(c->no_alloc_call) {
    if (!ctx->profile) return;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(ctx->stream, &capture) != hipSuccess) {
      (void)hipGetLastError();
      return;
    }
    if (capture != hipStreamCaptureStatusNone) ctx->no_alloc_call = true;
  }
  ~QuietCapture() { ctx->no_alloc_call = was; }
};

// the caller's scratch, or the context's workspace outside of a capture
gift_status take_scratch(gift_ctx *ctx, const char *call, void *scratch, uint64_t have, size_t need, uintptr_t align,
                         void **out) {
  if (scratch) {
    if (have < need) return fail(GIFT_EINVAL, call, "scratch is too small");
    if (!aligned(scratch, align)) return fail(GIFT_EINVAL, call, "scratch is misaligned");
    *out = scratch;
    return GIFT_OK;
  }
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  GIFT_HIP_TRY(hipStreamIsCapturing(ctx->stream, &capture));
  if (capture != hipStreamCaptureStatusNone)
    return fail(GIFT_EUNSUPPORTED, call, "a captured call needs scratch of the caller's");
  return workspace(ctx, need, out);
}

gift_status check_table(const char *call, int64_t V, int64_t d) {
  if (V < 1 || V > kMaxVocab) return fail(GIFT_ESHAPE, call, "V must be in [1, 2^31 - 2]");
  if (d < 1 || d > kMaxWidth) return fail(GIFT_ESHAPE, call, "d must be in [1, 2^20]");
  return GIFT_OK;
}

}  // namespace
}  // namespace gift

using namespace gift;

extern "C" {

gift_status gift_embedding(gift_ctx *ctx, const void *table, gift_dtype table_dtype, int64_t V, int64_t d,
                           const void *tokens, gift_index_type token_type, int64_t T, float scale, void *out,
                           gift_dtype out_dtype) {
  const char *call = "gift_embedding";
  if (!ctx || !table) return fail(GIFT_EINVAL, call, "NULL argument");
  if (!is_dtype(table_dtype) || !is_dtype(out_dtype))
    return fail(GIFT_EINVAL, call, "dtypes must be GIFT_F32 or GIFT_BF16");
  if (token_type != GIFT_I32 && token_type != GIFT_I64)
    return fail(GIFT_EINVAL, call, "token_type must be GIFT_I32 or GIFT_I64");
  if (!isfinite(scale)) return fail(GIFT_EINVAL, call, "scale must be finite");
  if (T < 0 || T > kMaxIds) return fail(GIFT_ESHAPE, call, "T must be in [0, 2^31)");
  gift_status st = check_table(call, V, d);
  if (st != GIFT_OK) return st;
  if (T == 0) return GIFT_OK;
  if (!tokens || !out) return fail(GIFT_EINVAL, call, "NULL argument");
  if (!aligned(table, table_dtype == GIFT_F32 ? 4 : 2) || !aligned(out, out_dtype == GIFT_F32 ? 4 : 2) ||
      !aligned(tokens, token_type == GIFT_I64 ? 8 : 4))
    return fail(GIFT_EINVAL, call, "a tensor is not aligned to its element");
  if ((st = enter(ctx, call)) != GIFT_OK) return st;
  LookupJob j;
  j.table = table;
  j.tokens = tokens;
  j.out = out;
  j.T = T;
  j.V = V;
  j.d = d;
  j.scale = scale;
  j.table_bf16 = table_dtype == GIFT_BF16;
  j.out_bf16 = out_dtype == GIFT_BF16;
  j.wide = token_type == GIFT_I64;
  QuietCapture quiet(ctx);
  return launch_lookup(ctx, j);
}

uint64_t gift_embedding_grad_scratch(int32_t N, int64_t T, int64_t V, int64_t d) {
  if (N < 1 || N > 65535 || T <= 0 || T > kMaxIds / N || V < 1 || V > kMaxVocab || d < 1 || d > kMaxWidth) return 0;
  EmbGradJob j;
  j.N = N;
  j.T = T;
  j.V = V;
  j.d = d;
  j.accumulate = true;    // (the form with fewer workgroups)
  if (embgrad_blocks(j) > kMaxBlocks) return 0;
  return embgrad_scratch(N, T, V, d);
}

gift_status gift_embedding_grad(gift_ctx *ctx, const void *tokens, gift_index_type token_type, const void *dout,
                                gift_dtype dtype, int32_t N, int64_t T, int64_t V, int64_t d, float scale,
                                int32_t accumulate, float *grads, void *scratch, uint64_t scratch_bytes) {
  const char *call = "gift_embedding_grad";
  if (!ctx || !grads) return fail(GIFT_EINVAL, call, "NULL argument");
  if (!is_dtype(dtype)) return fail(GIFT_EINVAL, call, "dtype must be GIFT_F32 or GIFT_BF16");
  if (token_type != GIFT_I32 && token_type != GIFT_I64)
    return fail(GIFT_EINVAL, call, "token_type must be GIFT_I32 or GIFT_I64");
  if (!isfinite(scale)) return fail(GIFT_EINVAL, call, "scale must be finite");
  if (N < 1 || N > 65535) return fail(GIFT_ESHAPE, call, "N must be in [1, 65535]");
  if (T < 0 || T > kMaxIds / N) return fail(GIFT_ESHAPE, call, "T must be >= 0 and N T < 2^31");
  gift_status st = check_table(call, V, d);
  if (st != GIFT_OK) return st;
  if (T > 0 && (!tokens || !dout)) return fail(GIFT_EINVAL, call, "NULL argument");
  if (!aligned(grads, 4) || !aligned(dout, dtype == GIFT_F32 ? 4 : 2) || !aligned(tokens, token_type == GIFT_I64 ? 8 : 4))
    return fail(GIFT_EINVAL, call, "a tensor is not aligned to its element");
  EmbGradJob j;
  j.tokens = tokens;
  j.dout = dout;
  j.grads = grads;
  j.N = N;
  j.T = T;
  j.V = V;
  j.d = d;
  j.scale = scale;
  j.bf16 = dtype == GIFT_BF16;
  j.wide = token_type == GIFT_I64;
  j.accumulate = accumulate != 0;
  if (T == 0 && accumulate) return GIFT_OK;
  if (embgrad_blocks(j) > kMaxBlocks) return fail(GIFT_ESHAPE, call, "more work than one launch takes");
  if ((st = enter(ctx, call)) != GIFT_OK) return st;
  void *ws = nullptr;
  if (T > 0 && (st = take_scratch(ctx, call, scratch, scratch_bytes, embgrad_scratch(N, T, V, d), 256, &ws)) != GIFT_OK)
    return st;
  QuietCapture quiet(ctx);
  return launch_embgrad(ctx, j, static_cast<char *>(ws));
}

gift_status gift_grad_norm(gift_ctx *ctx, int32_t count, const void *const *grads, const int64_t *numel,
                           gift_dtype dtype, double max_norm, float *out, void *scratch, uint64_t scratch_bytes) {
  const char *call = "gift_grad_norm";
  if (!ctx || !out) return fail(GIFT_EINVAL, call, "NULL argument");
  if (!is_dtype(dtype)) return fail(GIFT_EINVAL, call, "dtype must be GIFT_F32 or GIFT_BF16");
  if (!(max_norm > 0.0)) return fail(GIFT_EINVAL, call, "max_norm must be > 0");
  if (count < 0) return fail(GIFT_ESHAPE, call, "count must be >= 0");
  if (count > 0 && (!grads || !numel)) return fail(GIFT_EINVAL, call, "NULL argument");
  for (int32_t i = 0; i < count; ++i) {
    if (numel[i] < 0 || numel[i] > kMaxElements)
      return fail(GIFT_ESHAPE, call, "element counts must be in [0, 2^33]");
    if (numel[i] > 0 && !grads[i]) return fail(GIFT_EINVAL, call, "NULL gradient");
    if (!aligned(grads[i], dtype == GIFT_F32 ? 4 : 2))
      return fail(GIFT_EINVAL, call, "a gradient is not aligned to its element");
  }
  if (!aligned(out, 4)) return fail(GIFT_EINVAL, call, "out is not aligned to its element");
  gift_status st = enter(ctx, call);
  if (st != GIFT_OK) return st;
  void *part = nullptr;
  if ((st = take_scratch(ctx, call, scratch, scratch_bytes, grad_norm_scratch(), 8, &part)) != GIFT_OK) return st;
  QuietCapture quiet(ctx);
  return launch_grad_norm(ctx, count, grads, numel, dtype == GIFT_BF16, max_norm, out, static_cast<double *>(part));
}

gift_status gift_adamw_step(gift_ctx *ctx, int32_t count, const gift_adamw_tensor *tensors,
                            const gift_adamw_options *options) {
  const char *call = "gift_adamw_step";
  if (!ctx || !options) return fail(GIFT_EINVAL, call, "NULL argument");
  if (count < 0) return fail(GIFT_ESHAPE, call, "count must be >= 0");
  if (count > 0 && !tensors) return fail(GIFT_EINVAL, call, "NULL argument");
  const gift_adamw_options &o = *options;
  if (!is_dtype(o.grad_dtype)) return fail(GIFT_EINVAL, call, "grad_dtype must be GIFT_F32 or GIFT_BF16");
  if (o.moments != GIFT_MOMENTS_F32 && o.moments != GIFT_MOMENTS_FP8)
    return fail(GIFT_EINVAL, call, "moments must be GIFT_MOMENTS_F32 or GIFT_MOMENTS_FP8");
  if (!o.lr_dev && !(o.lr >= 0.0 && isfinite(o.lr))) return fail(GIFT_EINVAL, call, "lr must be finite and >= 0");
  if (!(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0))
    return fail(GIFT_EINVAL, call, "betas must be in [0, 1)");
  if (!((float)o.eps >= 1.17549435e-38f) || !isfinite((float)o.eps))
    return fail(GIFT_EINVAL, call, "eps must be a normal positive float32");
  if (!o.step_dev && o.step < 1) return fail(GIFT_EINVAL, call, "step must be >= 1");
  if (!aligned(o.lr_dev, 4) || !aligned(o.step_dev, 8) || !aligned(o.grad_scale, 4))
    return fail(GIFT_EINVAL, call, "a device scalar is misaligned");
  const bool eight = o.moments == GIFT_MOMENTS_FP8;
  for (int32_t i = 0; i < count; ++i) {
    const gift_adamw_tensor &t = tensors[i];
    if (t.numel < 0 || t.numel > kMaxElements)
      return fail(GIFT_ESHAPE, call, "element counts must be in [0, 2^33]");
    if (t.numel == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scales || !t.v_scales)))
      return fail(GIFT_EINVAL, call, "NULL tensor");
    if (!(t.weight_decay >= 0.0) || !isfinite(t.weight_decay))
      return fail(GIFT_EINVAL, call, "weight decays must be finite and >= 0");
    if (!aligned(t.param, 4) || !aligned(t.grad, o.grad_dtype == GIFT_F32 ? 4 : 2) || !aligned(t.copy, 2) ||
        (eight ? !aligned(t.m_scales, 4) || !aligned(t.v_scales, 4) : !aligned(t.m, 4) || !aligned(t.v, 4)))
      return fail(GIFT_EINVAL, call, "a tensor is not aligned to its element");
  }
  gift_status st = enter(ctx, call);
  if (st != GIFT_OK) return st;
  QuietCapture quiet(ctx);
  return launch_adamw(ctx, count, tensors, o);
}

}  // extern "C"
