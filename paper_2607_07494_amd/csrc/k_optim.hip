// Global gradient norm and the AdamW step over many tensors.
//
// Both take their tensors' pointers in the kernel arguments, up to kNormTensors
// or kAdamTensors a launch: no device table, nothing to upload, and a captured
// launch holds all it needs.  A workgroup finds its tensor from the tensors'
// first chunks with one vector load and a ballot.

#include <math.h>

#include "fp8_e4m3.h"
#include "gift_internal.h"
#include "philox.h"

namespace gift {

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// float32 -> bfloat16, to nearest even; a NaN stays one
__device__ __forceinline__ uint32_t to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? (u >> 16 | 0x40u) : (u + 0x7fffu + (u >> 16 & 1u)) >> 16;
}

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
// last bits.  Bound by reading the gradients once.
constexpr int kNormTensors = 128;
constexpr int kNormChunk = 8192;      // elements of a workgroup's step
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
        const uintx4 x = reinterpret_cast<const uintx4 *>(p)[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) add_square(acc[k], bf16_lo(x[k])), add_square(acc[k], bf16_hi(x[k]));
      }
      for (int i = 8 * vec + threadIdx.x; i < n; i += 256) add_square(acc[0], bf16_lo(p[i]));
    } else {
      const float *p = static_cast<const float *>(a.ptr[t]) + at;
      const int vec = (reinterpret_cast<uintptr_t>(p) & 15) == 0 ? n / 4 : 0;
      for (int i = threadIdx.x; i < vec; i += 256) {
        const floatx4 x = reinterpret_cast<const floatx4 *>(p)[i];
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
// every operation in float32, in this order.  One pass over all of it: bound
// by HBM (28 bytes an element with float32 moments and gradients, 16 with
// 8-bit moments, 2 more with a bfloat16 copy).
constexpr int kAdamTensors = 44;
constexpr int kAdamChunk = 4096;      // elements of a workgroup, float32 moments
constexpr int kGroup = 512;           // elements of a wave's step, 8-bit moments
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
  uint32_t index;      // place in the caller's list (random numbers)
  uint32_t vec;        // every array aligned for 4-element accesses
};

struct AdamArgs {
  AdamTensor t[kAdamTensors];
  uint32_t first[kAdamTensors];
  int count;
  double lr, log_beta1, log_beta2;
  int64_t step;
  const float *lr_dev;
  const int64_t *step_dev;
  const float *grad_scale;
  float b1, c1, b2, c2, eps;
  uint32_t seed_lo, seed_hi;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// the step's scalars
struct AdamStep {
  float decay;         // 1 - lr wd
  float size;          // lr / (1 - b1^t)
  float vscale;        // 1 / sqrt(1 - b2^t)
  float gscale;
  uint32_t step;
};

__device__ __forceinline__ AdamStep adam_step(const AdamArgs &a, double decay) {
  const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
  const int64_t step = a.step_dev ? *a.step_dev : a.step;
  AdamStep s;
  s.decay = (float)(1.0 - lr * decay);
  s.size = (float)(lr / -expm1((double)step * a.log_beta1));
  s.vscale = (float)(1.0 / sqrt(-expm1((double)step * a.log_beta2)));
  s.gscale = a.grad_scale ? *a.grad_scale : 1.0f;
  s.step = (uint32_t)step;
  return s;
}

// one element: moments m, v updated in place, the new parameter returned
__device__ __forceinline__ float adam_element(const AdamArgs &a, const AdamStep &s, float p, float g, float &m, float &v) {
  g *= s.gscale;
  m = m * a.b1 + g * a.c1;
  v = v * a.b2 + (g * g) * a.c2;
  const float update = m / (sqrtf(v) * s.vscale + a.eps);
  return p * s.decay - update * s.size;
}

// float32 of four gradients
template <bool BF16>
__device__ __forceinline__ floatx4 load_grad4(const void *g, int64_t i) {
  if constexpr (BF16) {
    const uintx2 x = *reinterpret_cast<const uintx2 *>(static_cast<const uint16_t *>(g) + i);
    return floatx4{bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]), bf16_hi(x[1])};
  } else {
    return *reinterpret_cast<const floatx4 *>(static_cast<const float *>(g) + i);
  }
}

template <bool BF16>
__device__ __forceinline__ float load_grad(const void *g, int64_t i) {
  return BF16 ? bf16_lo(static_cast<const uint16_t *>(g)[i]) : static_cast<const float *>(g)[i];
}

__device__ __forceinline__ void store_copy4(uint16_t *copy, int64_t i, const float p[4]) {
  *reinterpret_cast<uintx2 *>(copy + i) = uintx2{to_bf16(p[0]) | to_bf16(p[1]) << 16, to_bf16(p[2]) | to_bf16(p[3]) << 16};
}

template <bool BF16>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  const int index = find_tensor(a.first, a.count, blockIdx.x);
  const AdamTensor &t = a.t[index];
  const AdamStep s = adam_step(a, t.decay);
  if (s.gscale != s.gscale) return;
  float *m = static_cast<float *>(t.m), *v = static_cast<float *>(t.v);
  const int64_t lo = (int64_t)(blockIdx.x - a.first[index]) * kAdamChunk;
  const int64_t hi = lo + kAdamChunk < t.n ? lo + kAdamChunk : t.n;
  if (t.vec && hi - lo == kAdamChunk) {
    floatx4 p4[4], g4[4], m4[4], v4[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = lo + u * 1024 + threadIdx.x * 4;
      p4[u] = *reinterpret_cast<const floatx4 *>(t.p + i);
      g4[u] = load_grad4<BF16>(t.g, i);
      m4[u] = *reinterpret_cast<const floatx4 *>(m + i);
      v4[u] = *reinterpret_cast<const floatx4 *>(v + i);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = lo + u * 1024 + threadIdx.x * 4;
      float pn[4], mn[4], vn[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        mn[k] = m4[u][k];
        vn[k] = v4[u][k];
        pn[k] = adam_element(a, s, p4[u][k], g4[u][k], mn[k], vn[k]);
      }
      *reinterpret_cast<floatx4 *>(t.p + i) = floatx4{pn[0], pn[1], pn[2], pn[3]};
      *reinterpret_cast<floatx4 *>(m + i) = floatx4{mn[0], mn[1], mn[2], mn[3]};
      *reinterpret_cast<floatx4 *>(v + i) = floatx4{vn[0], vn[1], vn[2], vn[3]};
      if (t.copy) store_copy4(t.copy, i, pn);
    }
    return;
  }
  for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
    float mn = m[i], vn = v[i];
    const float pn = adam_element(a, s, t.p[i], load_grad<BF16>(t.g, i), mn, vn);
    t.p[i] = pn;
    m[i] = mn;
    v[i] = vn;
    if (t.copy) t.copy[i] = (uint16_t)to_bf16(pn);
  }
}

// Stochastic rounding of |y| to E4M3's grid by a 16-bit number r: the value
// rises to the grid's next one where the part below it, a fraction of the
// grid's step, plus (r + 1/2) / 2^16 reaches 1, so the mean over r is y.  In
// the normal range a step is 2^20 units of the float's last place; below 2^-6
// the step is 2^-9, which adding 2^-6 brings to the same 2^20 units.
__device__ __forceinline__ float round_e4m3(float y, uint32_t r, bool keep) {
  const float a = fabsf(y);
  const bool low = a < 0.015625f;
  const float t = low ? a + 0.015625f : a;
  float q = __uint_as_float((__float_as_uint(t) + (r * 16u + 8u)) & 0xfff00000u);
  if (low) q -= 0.015625f;
  if (keep && q == 0.f && a > 0.f) q = 0.001953125f;
  return a != a ? y : copysignf(q, y);
}

// maximum over the wave of non-negative floats' bits (a NaN's are the largest)
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)x, o);
    x = y > x ? y : x;
  }
  return x;
}

// 8-bit moments.  A nearest rounding would not do: E4M3's half step is 3 to 6
// percent of a value, an update with b2 near 1 far less, so v would never
// move; rounded by random numbers the stored moments are right in the mean.
// One number of 16 bits serves both moments of an element (each is unbiased by
// itself).  A positive v keeps at least the smallest code: as 0 it would leave
// m / eps as the next update.
//
// A wave takes kGroup elements, two scale blocks, a lane four neighbours of
// each: the block maxima are wave maxima, and the eight numbers are one
// Philox call, counter (call lo, call hi, tensor, step): words 0, 1 for the
// first block's four elements, words 2, 3 for the second's, low half first.
template <bool BF16>
__global__ __launch_bounds__(256) void adamw_e4m3_kernel(AdamArgs a) {
  const int index = find_tensor(a.first, a.count, blockIdx.x);
  const AdamTensor &t = a.t[index];
  const AdamStep s = adam_step(a, t.decay);
  if (s.gscale != s.gscale) return;
  const int lane = threadIdx.x & 63;
  const int64_t group = (int64_t)(blockIdx.x - a.first[index]) * (kAdamChunk8 / kGroup) + threadIdx.x / 64;
  const int64_t lo = group * kGroup;
  if (lo >= t.n) return;
  uint8_t *mc = static_cast<uint8_t *>(t.m), *vc = static_cast<uint8_t *>(t.v);
  const bool whole = t.vec && lo + kGroup <= t.n;
  float p[8], g[8], m[8], v[8];
  if (whole) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int64_t i = lo + b * kBlock + lane * 4;
      const floatx4 x = *reinterpret_cast<const floatx4 *>(t.p + i);
      const floatx4 y = load_grad4<BF16>(t.g, i);
      const uint32_t mw = *reinterpret_cast<const uint32_t *>(mc + i), vw = *reinterpret_cast<const uint32_t *>(vc + i);
      const float ms = t.ms[lo / kBlock + b], vs = t.vs[lo / kBlock + b];
      e4m3_decode4(mw, m + 4 * b);
      e4m3_decode4(vw, v + 4 * b);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        p[4 * b + k] = x[k];
        g[4 * b + k] = y[k];
        m[4 * b + k] *= ms;
        v[4 * b + k] *= vs;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t i = lo + (k / 4) * kBlock + lane * 4 + (k & 3);
      const bool in = i < t.n;
      p[k] = in ? t.p[i] : 0.f;
      g[k] = in ? load_grad<BF16>(t.g, i) : 0.f;
      m[k] = in ? e4m3_decode(mc[i]) * t.ms[i / kBlock] : 0.f;
      v[k] = in ? e4m3_decode(vc[i]) * t.vs[i / kBlock] : 0.f;
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) p[k] = adam_element(a, s, p[k], g[k], m[k], v[k]);
  const uint64_t call = (uint64_t)group * 64 + lane;
  const PhiloxWords w = philox((uint32_t)call, (uint32_t)(call >> 32), t.index, s.step, a.seed_lo, a.seed_hi);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    uint32_t mx = 0, vx = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t mb = __float_as_uint(m[4 * b + k]) & 0x7fffffffu, vb = __float_as_uint(v[4 * b + k]) & 0x7fffffffu;
      // (outside the tensor a lane's moments are 0)
      mx = mb > mx ? mb : mx;
      vx = vb > vx ? vb : vx;
    }
    const float mmax = __uint_as_float(wave_max(mx)), vmax = __uint_as_float(wave_max(vx));
    const float mmul = e4m3_multiplier(mmax), vmul = e4m3_multiplier(vmax);
    float mq[4], vq[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t r = (w.w[2 * b + k / 2] >> (16 * (k & 1))) & 0xffffu;
      mq[k] = round_e4m3(m[4 * b + k] * mmul, r, false);
      vq[k] = round_e4m3(v[4 * b + k] * vmul, r, true);
    }
    const uint32_t mw = e4m3_encode4(mq[0], mq[1], mq[2], mq[3]), vw = e4m3_encode4(vq[0], vq[1], vq[2], vq[3]);
    const int64_t i = lo + b * kBlock + lane * 4;
    if (whole) {
      *reinterpret_cast<floatx4 *>(t.p + i) = floatx4{p[4 * b], p[4 * b + 1], p[4 * b + 2], p[4 * b + 3]};
      *reinterpret_cast<uint32_t *>(mc + i) = mw;
      *reinterpret_cast<uint32_t *>(vc + i) = vw;
      if (t.copy) store_copy4(t.copy, i, p + 4 * b);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i + k >= t.n) break;
        t.p[i + k] = p[4 * b + k];
        mc[i + k] = (uint8_t)(mw >> (8 * k));
        vc[i + k] = (uint8_t)(vw >> (8 * k));
        if (t.copy) t.copy[i + k] = (uint16_t)to_bf16(p[4 * b + k]);
      }
    }
    if (lane == 0 && lo + b * kBlock < t.n) {
      t.ms[lo / kBlock + b] = e4m3_scale(mmax);
      t.vs[lo / kBlock + b] = e4m3_scale(vmax);
    }
  }
}

bool aligned(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

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
  a.b1 = (float)o.beta1;
  a.c1 = (float)(1.0 - o.beta1);
  a.b2 = (float)o.beta2;
  a.c2 = (float)(1.0 - o.beta2);
  a.eps = (float)o.eps;
  a.seed_lo = (uint32_t)o.seed;
  a.seed_hi = (uint32_t)(o.seed >> 32);
  for (int32_t i = 0; i < count;) {
    a.count = 0;
    int64_t chunks = 0;
    for (; i < count && a.count < kAdamTensors; ++i) {
      const gift_adamw_tensor &x = tensors[i];
      if (x.numel == 0) continue;
      const int64_t more = (x.numel + per_group - 1) / per_group;
      if (a.count > 0 && chunks + more > 0xffffff) break;   // 2^24 workgroups of 256 threads a launch
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
      t.index = (uint32_t)i;
      t.vec = aligned(x.param, 16) && aligned(x.grad, bf16 ? 8 : 16) && aligned(x.m, eight ? 4 : 16) &&
              aligned(x.v, eight ? 4 : 16) && aligned(x.copy, 8);
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
