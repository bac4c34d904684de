// Global gradient norm and the AdamW step over many tensors.
//
// Both take their tensors' pointers in the kernel arguments, up to kNormTensors
// or kAdamTensors a launch: no device table, nothing to upload, and a captured
// launch holds all it needs.  A workgroup finds its tensor from the tensors'
// first chunks with one vector load and a ballot.

#include <math.h>

#include "bf16.h"
#include "fp8_e4m3.h"
#include "gift_internal.h"
#include "philox.h"

namespace gift {

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

// index of the last of `count` ascending first chunks that is <= chunk
__device__ __forceinline__ int find_tensor(const uint32_t *first, int count, uint32_t chunk) {
  const int lane = threadIdx.x & 63;
  int below = 0;
  for (int at = 0; at < count; at += 64)
    below += __popcll(__ballot(at + lane < count && first[at + lane < count ? at + lane : 0] <= chunk));
  return below - 1;
}

// ---------------------------------------------------------------------------
// Norm
// ---------------------------------------------------------------------------
// Squares and sums in float64: no overflow of a square, and the result does
// not depend on how the elements are spread over the workgroups beyond its
// last bits.  Bound by reading the gradients once: past the caches, 374 M
// float32 elements in 224 us, 6.7 TB/s (through them 247 us).  Tensors that do
// not start on 16 bytes are read element by element: 315 M float32 elements 351
// instead of 183 us, bfloat16 318 instead of 102.
constexpr int kNormTensors = 128;
constexpr int kNormChunk = 4096;      // elements of a workgroup's step
constexpr int kNormGroups = 2048;     // workgroups, one partial sum each

struct NormArgs {
  const void *ptr[kNormTensors];
  int64_t n[kNormTensors];
  uint32_t first[kNormTensors];       // first chunk of each tensor
  int count;
  uint32_t chunks;
  bool bf16, add;                     // add: the partials hold earlier launches' sums
  double *part;
};

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double wave_sum[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x / 64] = x;
  __syncthreads();
  return wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
}

__device__ __forceinline__ void add_square(double &acc, float x) {
  const double v = x;
  acc = __builtin_fma(v, v, acc);
}

__global__ __launch_bounds__(256) void norm_kernel(NormArgs a) {
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const int t = find_tensor(a.first, a.count, chunk);
    const int64_t at = (int64_t)(chunk - a.first[t]) * kNormChunk;
    const int n = (int)(a.n[t] - at < kNormChunk ? a.n[t] - at : kNormChunk);
    if (a.bf16) {
      const uint16_t *p = static_cast<const uint16_t *>(a.ptr[t]) + at;
      const int vec = (reinterpret_cast<uintptr_t>(p) & 15) == 0 ? n / 8 : 0;
      for (int i = threadIdx.x; i < vec; i += 256) {
        const uintx4 x = __builtin_nontemporal_load(reinterpret_cast<const uintx4 *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) add_square(acc[k], bf16_lo(x[k])), add_square(acc[k], bf16_hi(x[k]));
      }
      for (int i = 8 * vec + threadIdx.x; i < n; i += 256) add_square(acc[0], bf16_lo(p[i]));
    } else {
      const float *p = static_cast<const float *>(a.ptr[t]) + at;
      const int vec = (reinterpret_cast<uintptr_t>(p) & 15) == 0 ? n / 4 : 0;
      for (int i = threadIdx.x; i < vec; i += 256) {
        const floatx4 x = __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) add_square(acc[k], x[k]);
      }
      for (int i = 4 * vec + threadIdx.x; i < n; i += 256) add_square(acc[0], p[i]);
    }
  }
  const double sum = block_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (threadIdx.x == 0) a.part[blockIdx.x] = a.add ? a.part[blockIdx.x] + sum : sum;
}

__global__ __launch_bounds__(256) void norm_finish_kernel(const double *part, int count, double max_norm, float *out) {
  double x = 0.0;
  for (int i = threadIdx.x; i < count; i += 256) x += part[i];
  const double norm = sqrt(block_sum(x));
  if (threadIdx.x == 0) {
    const double ratio = max_norm / (norm + 1e-6);
    const bool finite = norm <= 1.7976931348623157e308;
    out[0] = (float)norm;
    out[1] = !finite ? __uint_as_float(0x7fc00000u) : ratio < 1.0 ? (float)ratio : 1.0f;
  }
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
// With g' = grad_scale g:
//   m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// One pass over all of it, every array streamed past the caches (non-temporal):
// bound by HBM (28 bytes an element with float32 moments and gradients, 16
// with 8-bit moments, 2 more with a bfloat16 copy).
constexpr int kAdamTensors = 44;
constexpr int kAdamChunk = 1024;      // elements of a workgroup, float32 moments
constexpr int kGroup = 512;           // elements of a wave, 8-bit moments
constexpr int kBlock = 256;           // elements under one scale
constexpr int kAdamChunk8 = 4 * kGroup;

struct AdamTensor {
  float *p;
  const void *g;
  void *m, *v;
  float *ms, *vs;
  uint16_t *copy;
  int64_t n;
  double decay;        // weight decay
  float keep;          // 1 - lr decay, for a learning rate of the host's
  uint32_t index;      // place in the caller's list (random numbers)
};

// the step's scalars
struct AdamStep {
  float size;          // lr / (1 - b1^t)
  float vscale;        // 1 / sqrt(1 - b2^t)
  float gscale;
  uint32_t step;
};

struct AdamArgs {
  AdamTensor t[kAdamTensors];
  uint32_t first[kAdamTensors];       // first chunk of each tensor
  uint64_t vec;                       // bit i: tensor i's arrays are aligned for 4-element accesses
  int count;
  AdamStep host;                      // of the host's learning rate and step
  double lr, log_beta1, log_beta2;
  int64_t step;
  const float *lr_dev;
  const int64_t *step_dev;
  const float *grad_scale;
  double b1, c1, b2, c2;              // betas, 1 - betas
  float eps;
  uint32_t seed_lo, seed_hi;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

__host__ __device__ __forceinline__ void bias_corrections(double lr, int64_t step, double log_beta1, double log_beta2,
                                                          AdamStep &s) {
  s.size = (float)(lr / -expm1((double)step * log_beta1));
  s.vscale = (float)(1.0 / sqrt(-expm1((double)step * log_beta2)));
  s.step = (uint32_t)step;
}

// A learning rate or step of the device's is worked out by every lane, beside
// the other waves' loads: 315 M elements in a replayed graph 1640 us with float32
// and 957 with 8-bit moments, by the host's scalars 1675 and 968.
__device__ __forceinline__ AdamStep adam_step(const AdamArgs &a, const AdamTensor &t, float &keep) {
  AdamStep s = a.host;
  keep = t.keep;
  s.gscale = a.grad_scale ? *a.grad_scale : 1.0f;
  if (a.lr_dev || a.step_dev) {
    const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    const int64_t step = a.step_dev ? *a.step_dev : a.step;
    bias_corrections(lr, step, a.log_beta1, a.log_beta2, s);
    keep = (float)(1.0 - lr * t.decay);
    if (step < 1) s.gscale = __uint_as_float(0x7fc00000u);   // no such step: skipped
  }
  return s;
}

// one element, float32 moments: m, v updated in place, the new parameter returned
__device__ __forceinline__ float adam_element(const AdamArgs &a, const AdamStep &s, float keep, float p, float g,
                                              float &m, float &v) {
  g *= s.gscale;
  m = m * (float)a.b1 + g * (float)a.c1;
  v = v * (float)a.b2 + (g * g) * (float)a.c2;
  const float update = m / (sqrtf(v) * s.vscale + a.eps);
  return p * keep - update * s.size;
}

// float32 of four gradients
template <bool BF16>
__device__ __forceinline__ floatx4 load_grad4(const void *g, int64_t i) {
  if constexpr (BF16) {
    const uintx2 x = __builtin_nontemporal_load(reinterpret_cast<const uintx2 *>(static_cast<const uint16_t *>(g) + i));
    return floatx4{bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]), bf16_hi(x[1])};
  } else {
    return __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(static_cast<const float *>(g) + i));
  }
}

template <bool BF16>
__device__ __forceinline__ float load_grad(const void *g, int64_t i) {
  return BF16 ? bf16_lo(static_cast<const uint16_t *>(g)[i]) : static_cast<const float *>(g)[i];
}

__device__ __forceinline__ floatx4 load4(const float *p) {
  return __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(p));
}

__device__ __forceinline__ void store4(float *p, const float v[4]) {
  __builtin_nontemporal_store(floatx4{v[0], v[1], v[2], v[3]}, reinterpret_cast<floatx4 *>(p));
}

__device__ __forceinline__ void store_copy4(uint16_t *copy, int64_t i, const float p[4]) {
  __builtin_nontemporal_store(uintx2{to_bf16(p[0]) | to_bf16(p[1]) << 16, to_bf16(p[2]) | to_bf16(p[3]) << 16},
                              reinterpret_cast<uintx2 *>(copy + i));
}

template <bool BF16>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  const int index = find_tensor(a.first, a.count, blockIdx.x);
  const AdamTensor &t = a.t[index];
  float keep;
  const AdamStep s = adam_step(a, t, keep);
  if (s.gscale != s.gscale) return;
  float *m = static_cast<float *>(t.m), *v = static_cast<float *>(t.v);
  const int64_t lo = (int64_t)(blockIdx.x - a.first[index]) * kAdamChunk;
  const int64_t hi = lo + kAdamChunk < t.n ? lo + kAdamChunk : t.n;
  if ((a.vec >> index & 1) && hi - lo == kAdamChunk) {
    const int64_t i = lo + threadIdx.x * 4;
    const floatx4 p4 = load4(t.p + i), g4 = load_grad4<BF16>(t.g, i), m4 = load4(m + i), v4 = load4(v + i);
    float pn[4], mn[4], vn[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      mn[k] = m4[k];
      vn[k] = v4[k];
      pn[k] = adam_element(a, s, keep, p4[k], g4[k], mn[k], vn[k]);
    }
    store4(t.p + i, pn);
    store4(m + i, mn);
    store4(v + i, vn);
    if (t.copy) store_copy4(t.copy, i, pn);
    return;
  }
  for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
    float mn = m[i], vn = v[i];
    const float pn = adam_element(a, s, keep, t.p[i], load_grad<BF16>(t.g, i), mn, vn);
    t.p[i] = pn;
    m[i] = mn;
    v[i] = vn;
    if (t.copy) t.copy[i] = (uint16_t)to_bf16(pn);
  }
}

// 8-bit moments.  A nearest rounding would not do: E4M3's half step is 3 to 6
// percent of a value, an update with b2 near 1 far less, so v would never
// move; rounded by random numbers the stored moments are right in the mean.
// One number of 16 bits serves both moments of an element (each is unbiased by
// itself).  A positive v keeps at least the smallest code: as 0 it would leave
// m / eps as the next update.
//
// Which of two codes a value gets hangs on y's last bits, so moments, scale and
// multiplier are float32 with one rounding per operation.
//
// A wave takes kGroup elements, two scale blocks, a lane four neighbours of
// each: the block maxima are wave maxima, and the eight numbers are one
// Philox call, counter (call lo, call hi, tensor, step): words 0, 1 for the
// first block's four elements, words 2, 3 for the second's, low half first.

// maximum over the wave's 64 lanes (all active)
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  const auto step = [](uint32_t a, int b) { return (uint32_t)b > a ? (uint32_t)b : a; };
  x = step(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));    // row_shr 1, 2, 4, 8
  x = step(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));
  x = step(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));
  x = step(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));
  x = step(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));   // last lanes of rows 0, 2 to 1, 3
  x = step(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));   // lane 31 to rows 2, 3
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// E4M3 code of |y|, y finite, rounded by r: up to the grid's next point where
// the part beyond the lower one plus (r + 1/2) 2^-16 reaches a step.  In the
// normal range a step of the 3-bit mantissa is 2^20 units of a float's last
// place; below 2^-6 the step is 2^-9, which adding 2^-6 (code 8) brings to the
// same 2^20 units.
__device__ __forceinline__ uint32_t round_code(float y, uint32_t r) {
  const float a = fabsf(y);
  const bool low = a < 0.015625f;
  const uint32_t t = __float_as_uint(low ? a + 0.015625f : a) + (16u * r + 8u);
  const uint32_t code = (t >> 20) - (low ? 968u : 960u);   // exponent bias 127 - 7, 3 mantissa bits
  return code < 126u ? code : 126u;                        // 448
}

// Codes and the stored scale of a lane's four elements of a block: m signed, v
// (SIGNED false) non-negative and kept above 0.
template <bool SIGNED>
__device__ __forceinline__ uint32_t block_codes(const float x[4], const uint32_t r[4], float &scale) {
  uint32_t mine = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t u = __float_as_uint(x[k]) & 0x7fffffffu;
    mine = u > mine ? u : mine;
  }
  const float amax = __uint_as_float(wave_max(mine));       // (a NaN's bits are the largest)
  scale = amax * (1.0f / kE4M3Max);
  uint32_t word = 0;
  if (__float_as_uint(amax) >= 0x7f800000u) {               // a NaN: all codes NaN; an infinity: that element's
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool finite = fabsf(x[k]) <= 3.402823466e38f;
      const uint32_t sign = SIGNED ? __float_as_uint(x[k]) >> 31 << 7 : 0u;
      word |= (amax == amax && finite ? sign : 0x7fu) << (8 * k);
    }
    return word;
  }
  const float mult = amax > 0.f ? fminf(kE4M3Max * (1.0f / amax), 3.402823466e38f) : 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float y = x[k] * mult;
    uint32_t code = round_code(y, r[k]);
    if (SIGNED) code |= __float_as_uint(y) >> 31 << 7;
    else if (y > 0.f && code == 0) code = 1;
    word |= code << (8 * k);
  }
  return word;
}

template <bool BF16>
__global__ __launch_bounds__(256) void adamw_e4m3_kernel(AdamArgs a) {
  const int index = find_tensor(a.first, a.count, blockIdx.x);
  const AdamTensor &t = a.t[index];
  float keep;
  const AdamStep s = adam_step(a, t, keep);
  if (s.gscale != s.gscale) return;
  const int lane = threadIdx.x & 63;
  const int64_t group = (int64_t)(blockIdx.x - a.first[index]) * (kAdamChunk8 / kGroup) +
                        __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t lo = group * kGroup;
  if (lo >= t.n) return;
  uint8_t *mc = static_cast<uint8_t *>(t.m), *vc = static_cast<uint8_t *>(t.v);
  const int blocks = lo + kBlock < t.n ? 2 : 1;
  const bool whole = (a.vec >> index & 1) && lo + kGroup <= t.n;
  float p[8], g[8], m[8], v[8];    // (outside the tensor 0)
  if (whole) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int64_t i = lo + b * kBlock + lane * 4;
      const floatx4 x = load4(t.p + i), y = load_grad4<BF16>(t.g, i);
      e4m3_decode4(__builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(mc + i)), m + 4 * b);
      e4m3_decode4(__builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(vc + i)), v + 4 * b);
#pragma unroll
      for (int k = 0; k < 4; ++k) p[4 * b + k] = x[k], g[4 * b + k] = y[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t i = lo + (k / 4) * kBlock + lane * 4 + (k & 3);
      const bool in = i < t.n;
      p[k] = in ? t.p[i] : 0.f;
      g[k] = in ? load_grad<BF16>(t.g, i) : 0.f;
      m[k] = in ? e4m3_decode(mc[i]) : 0.f;
      v[k] = in ? e4m3_decode(vc[i]) : 0.f;
    }
  }
  const uint64_t call = (uint64_t)group * 64 + lane;
  const PhiloxWords w = philox((uint32_t)call, (uint32_t)(call >> 32), t.index, s.step, a.seed_lo, a.seed_hi);
  const float b1 = (float)a.b1, c1 = (float)a.c1, b2 = (float)a.b2, c2 = (float)a.c2;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (b >= blocks) break;
    const float old_ms = t.ms[lo / kBlock + b], old_vs = t.vs[lo / kBlock + b];
    float mn[4], vn[4];
    float pn[4];
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float gk = g[4 * b + k] * s.gscale;
      mn[k] = m[4 * b + k] * old_ms * b1 + gk * c1;
      vn[k] = v[4 * b + k] * old_vs * b2 + gk * gk * c2;
      // hardware square root and reciprocal, 1 ulp each (with the exact ones 679 M elements took 11 % longer)
      const float update = mn[k] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(vn[k]) * s.vscale + a.eps);
      pn[k] = p[4 * b + k] * keep - update * s.size;
      r[k] = (w.w[2 * b + k / 2] >> (16 * (k & 1))) & 0xffffu;
    }
    float ms, vs;
    const uint32_t mw = block_codes<true>(mn, r, ms), vw = block_codes<false>(vn, r, vs);
    const int64_t i = lo + b * kBlock + lane * 4;
    if (whole) {
      store4(t.p + i, pn);
      __builtin_nontemporal_store(mw, reinterpret_cast<uint32_t *>(mc + i));
      __builtin_nontemporal_store(vw, reinterpret_cast<uint32_t *>(vc + i));
      if (t.copy) store_copy4(t.copy, i, pn);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i + k >= t.n) break;
        t.p[i + k] = pn[k];
        mc[i + k] = (uint8_t)(mw >> (8 * k));
        vc[i + k] = (uint8_t)(vw >> (8 * k));
        if (t.copy) t.copy[i + k] = (uint16_t)to_bf16(pn[k]);
      }
    }
    if (lane == 0) {
      t.ms[lo / kBlock + b] = ms;
      t.vs[lo / kBlock + b] = vs;
    }
  }
}

}  // namespace

size_t grad_norm_scratch() { return kNormGroups * sizeof(double); }

gift_status launch_grad_norm(gift_ctx *ctx, int32_t count, const void *const *grads, const int64_t *numel, bool bf16,
                             double max_norm, float *out, double *part) {
  ProfileScope prof(ctx, GIFT_KERNEL_NORM);
  NormArgs a;
  a.bf16 = bf16;
  a.part = part;
  gift_status st;
  int used = 0;   // partials that hold a sum
  for (int32_t i = 0; i < count;) {
    a.count = 0;
    a.chunks = 0;
    for (; i < count && a.count < kNormTensors; ++i) {
      if (numel[i] == 0) continue;
      const int64_t chunks = (numel[i] + kNormChunk - 1) / kNormChunk;
      if (a.count > 0 && (int64_t)a.chunks + chunks > 0x7fffffff) break;
      a.ptr[a.count] = grads[i];
      a.n[a.count] = numel[i];
      a.first[a.count++] = a.chunks;
      a.chunks += (uint32_t)chunks;
    }
    if (a.count == 0) break;
    // later launches add to the first one's partials: as many as it wrote
    const int groups = used ? used : a.chunks < (uint32_t)kNormGroups && i >= count ? (int)a.chunks : kNormGroups;
    a.add = used > 0;
    used = groups;
    hipLaunchKernelGGL(norm_kernel, dim3(groups), dim3(256), 0, ctx->stream, a);
    if ((st = check_launch("norm_kernel")) != GIFT_OK) return st;
  }
  hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(256), 0, ctx->stream, part, used, max_norm, out);
  return check_launch("norm_finish_kernel");
}

gift_status launch_adamw(gift_ctx *ctx, int32_t count, const gift_adamw_tensor *tensors, const gift_adamw_options &o) {
  ProfileScope prof(ctx, GIFT_KERNEL_OPTIMIZER);
  const bool bf16 = o.grad_dtype == GIFT_BF16, eight = o.moments == GIFT_MOMENTS_FP8;
  const int64_t per_group = eight ? kAdamChunk8 : kAdamChunk;
  AdamArgs a;
  a.lr = o.lr;
  a.log_beta1 = log(o.beta1);   // beta 0: -inf, 1 - 0^t = 1
  a.log_beta2 = log(o.beta2);
  a.step = o.step;
  a.lr_dev = o.lr_dev;
  a.step_dev = o.step_dev;
  a.grad_scale = o.grad_scale;
  bias_corrections(o.lr, o.step, a.log_beta1, a.log_beta2, a.host);   // (unused where the device has its own)
  a.b1 = o.beta1;
  a.c1 = 1.0 - o.beta1;
  a.b2 = o.beta2;
  a.c2 = 1.0 - o.beta2;
  a.eps = (float)o.eps;
  a.seed_lo = (uint32_t)o.seed;
  a.seed_hi = (uint32_t)(o.seed >> 32);
  for (int32_t i = 0; i < count;) {
    a.count = 0;
    a.vec = 0;
    int64_t chunks = 0;
    for (; i < count && a.count < kAdamTensors; ++i) {
      const gift_adamw_tensor &x = tensors[i];
      if (x.numel == 0) continue;
      const int64_t more = (x.numel + per_group - 1) / per_group;
      if (a.count > 0 && chunks + more > kMaxBlocks) break;
      AdamTensor &t = a.t[a.count];
      t.p = x.param;
      t.g = x.grad;
      t.m = x.m;
      t.v = x.v;
      t.ms = x.m_scales;
      t.vs = x.v_scales;
      t.copy = static_cast<uint16_t *>(x.copy);
      t.n = x.numel;
      t.decay = x.weight_decay;
      t.keep = (float)(1.0 - o.lr * x.weight_decay);
      t.index = (uint32_t)i;
      // else element by element: 315 M elements, each array one off, float32 moments
      // 1840 us (aligned 1685), 8-bit moments 2015 (970)
      if (aligned(x.param, 16) && aligned(x.grad, bf16 ? 8 : 16) && aligned(x.m, eight ? 4 : 16) &&
          aligned(x.v, eight ? 4 : 16) && aligned(x.copy, 8))
        a.vec |= 1ull << a.count;
      a.first[a.count++] = (uint32_t)chunks;
      chunks += more;
    }
    if (a.count == 0) break;
    const dim3 grid((unsigned)chunks), block(256);
    if (eight) {
      if (bf16) hipLaunchKernelGGL((adamw_e4m3_kernel<true>), grid, block, 0, ctx->stream, a);
      else hipLaunchKernelGGL((adamw_e4m3_kernel<false>), grid, block, 0, ctx->stream, a);
    } else {
      if (bf16) hipLaunchKernelGGL((adamw_kernel<true>), grid, block, 0, ctx->stream, a);
      else hipLaunchKernelGGL((adamw_kernel<false>), grid, block, 0, ctx->stream, a);
    }
    gift_status st = check_launch(eight ? "adamw_e4m3_kernel" : "adamw_kernel");
    if (st != GIFT_OK) return st;
  }
  return GIFT_OK;
}

}  // namespace gift
