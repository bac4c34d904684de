// Embedding lookup and its gradient.
//
// Lookup: out[t] = scale * table[tokens[t]].  Gradient, for every rank j:
//
//   grads[j][v] (+)= scale * sum over t with tokens[j][t] = v of dout[j][t]
//
// The gradient first orders each rank's positions by token (a stable radix
// sort, 8 bits a pass), so that a row's terms are neighbours and stand in
// position order.  The ordered list is cut into runs of kRun entries, one wave
// each: the work does not depend on how often a token occurs.  A wave adds its
// entries' rows in float32 and stores every row that begins and ends in its
// run; the parts of rows that cross a border go to scratch and a second kernel
// adds them in order.  No atomics on values: the same inputs give the same
// bits.  Rows without a token are zeroed by further waves of the same launch.
//
// Ids outside [0, V) (padding) get the sort key V, the largest: they end up
// behind all others and nothing reads them.

#include "gift_internal.h"

namespace gift {

namespace {

// Rows of any length and address: 16-byte accesses at the element's own
// alignment (gfx950's vector memory takes any address).
typedef float floatx4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t uintx4_u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t uintx2_u __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t uintx1_u __attribute__((aligned(2)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// float32 -> bfloat16, to nearest even; a NaN stays one
__device__ __forceinline__ uint32_t to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  return x != x ? (u >> 16 | 0x40u) : (u + 0x7fffu + (u >> 16 & 1u)) >> 16;
}

// VEC neighbouring elements of a row as float32
template <int VEC>
__device__ __forceinline__ void load_row(const float *p, float v[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const floatx4_u x = *reinterpret_cast<const floatx4_u *>(p + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[i + k] = x[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = p[i];
  }
}

template <int VEC>
__device__ __forceinline__ void load_row(const uint16_t *p, float v[VEC]) {
  if constexpr (VEC == 8) {
    const uintx4_u x = *reinterpret_cast<const uintx4_u *>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[2 * k] = bf16_lo(x[k]), v[2 * k + 1] = bf16_hi(x[k]);
  } else if constexpr (VEC == 4) {
    const uintx2_u x = *reinterpret_cast<const uintx2_u *>(p);
#pragma unroll
    for (int k = 0; k < 2; ++k) v[2 * k] = bf16_lo(x[k]), v[2 * k + 1] = bf16_hi(x[k]);
  } else if constexpr (VEC == 2) {
    const uint32_t x = *reinterpret_cast<const uintx1_u *>(p);
    v[0] = bf16_lo(x), v[1] = bf16_hi(x);
  } else {
    v[0] = bf16_lo(p[0]);
  }
}

template <int VEC>
__device__ __forceinline__ void store_row(float *p, const float v[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) *reinterpret_cast<floatx4_u *>(p + i) = floatx4_u{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = v[i];
  }
}

template <int VEC>
__device__ __forceinline__ void store_row(uint16_t *p, const float v[VEC]) {
  if constexpr (VEC == 8) {
    uintx4_u x;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = to_bf16(v[2 * k]) | to_bf16(v[2 * k + 1]) << 16;
    *reinterpret_cast<uintx4_u *>(p) = x;
  } else if constexpr (VEC == 4) {
    uintx2_u x;
#pragma unroll
    for (int k = 0; k < 2; ++k) x[k] = to_bf16(v[2 * k]) | to_bf16(v[2 * k + 1]) << 16;
    *reinterpret_cast<uintx2_u *>(p) = x;
  } else if constexpr (VEC == 2) {
    *reinterpret_cast<uintx1_u *>(p) = to_bf16(v[0]) | to_bf16(v[1]) << 16;
  } else {
    p[0] = (uint16_t)to_bf16(v[0]);
  }
}

// the same, past the caches where VEC elements are 16-byte groups or words
template <int VEC>
__device__ __forceinline__ void stream_row(float *p, const float v[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4)
      __builtin_nontemporal_store(floatx4_u{v[i], v[i + 1], v[i + 2], v[i + 3]}, reinterpret_cast<floatx4_u *>(p + i));
  } else {
    store_row<VEC>(p, v);
  }
}

template <int VEC>
__device__ __forceinline__ void stream_row(uint16_t *p, const float v[VEC]) {
  if constexpr (VEC == 8) {
    uintx4_u x;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = to_bf16(v[2 * k]) | to_bf16(v[2 * k + 1]) << 16;
    __builtin_nontemporal_store(x, reinterpret_cast<uintx4_u *>(p));
  } else {
    store_row<VEC>(p, v);
  }
}

// Columns of a lane: VEC from `first` on.  The row's last lane holds fewer:
// it loads the VEC columns that end the row and keeps the last `own` of them.
template <int VEC>
struct Columns {
  int64_t first;   // first column loaded
  int skip;        // of these, columns that belong to the lane before
  bool any;
  __device__ __forceinline__ Columns(int64_t chunk, int64_t d) {
    const int64_t c = (chunk * 64 + (threadIdx.x & 63)) * VEC;
    any = c < d;
    const int64_t last = d - VEC;
    first = c <= last ? c : last;
    skip = (int)(c - first);
  }
};

__device__ __forceinline__ int64_t read_token(const void *tokens, bool wide, int64_t i) {
  return wide ? static_cast<const int64_t *>(tokens)[i] : (int64_t)static_cast<const int32_t *>(tokens)[i];
}

// ---------------------------------------------------------------------------
// Lookup
// ---------------------------------------------------------------------------
// One wave takes 64 columns x VEC of two or four neighbouring rows, their ids
// and then their table rows in flight together.  The kernel moves bytes only:
// bound by the table's rows and the output in HBM; the output is streamed past
// the caches, which hold the frequent ids' rows.
// Rows: two where a lane's part of a row is 32 bytes, else four (65536 x 1536 from
// a float32 table: one 85 us, two 59, four 61).
template <typename TIn, int VEC>
constexpr int lookup_rows() {
  return VEC * sizeof(TIn) >= 32 ? 2 : 4;
}

template <typename TIn, typename TOut, int VEC>
__global__ __launch_bounds__(256) void lookup_kernel(const TIn *table, const void *tokens, bool wide, int64_t T,
                                                     int64_t V, int64_t d, int chunks, float scale, TOut *out) {
  constexpr int kLookupRows = lookup_rows<TIn, VEC>();
  const int64_t groups = (T + kLookupRows - 1) / kLookupRows, items = groups * chunks, stride = (int64_t)gridDim.x * 4;
  for (int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); i < items; i += stride) {
    const int64_t group = i / chunks, t0 = group * kLookupRows;
    const Columns<VEC> c(i - group * chunks, d);
    if (!c.any) continue;
    float v[kLookupRows][VEC];
    bool in[kLookupRows];
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
      const int64_t id = read_token(tokens, wide, t0 + r < T ? t0 + r : T - 1);
      in[r] = id >= 0 && id < V;
      load_row<VEC>(table + (in[r] ? id : 0) * d + c.first, v[r]);
    }
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
      if (t0 + r >= T) break;
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[r][k] = in[r] ? v[r][k] * scale : 0.f;
      // (a row's last lane rewrites columns of the one before with the same values)
      stream_row<VEC>(out + (t0 + r) * d + c.first, v[r]);
    }
  }
}

// ---------------------------------------------------------------------------
// Sort of each rank's positions by token
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 256;
constexpr int kSortPerWave = 512;                      // keys of a wave, in order
constexpr int kSortTile = 4 * kSortPerWave;            // keys of a workgroup
constexpr int kDigits = 256;

struct SortArgs {
  const void *tokens;      // first pass: [N, T] ids; else null
  bool wide;
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t *hist;          // [N][256][tiles]
  int64_t T, V;
  int tiles, shift;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs &a, int64_t rank, int64_t i) {
  if (!a.tokens) return a.key_in[rank * a.T + i];
  const int64_t id = read_token(a.tokens, a.wide, rank * a.T + i);
  return (uint32_t)(id >= 0 && id < a.V ? id : a.V);
}

__global__ __launch_bounds__(kSortThreads) void sort_hist_kernel(SortArgs a) {
  __shared__ uint32_t count[kDigits];
  const int64_t rank = blockIdx.y;
  count[threadIdx.x] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * kSortTile, hi = lo + kSortTile < a.T ? lo + kSortTile : a.T;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads)
    atomicAdd(&count[(sort_key(a, rank, i) >> a.shift) & 255u], 1u);
  __syncthreads();
  a.hist[(rank * kDigits + threadIdx.x) * a.tiles + blockIdx.x] = count[threadIdx.x];
}

// exclusive prefix sums of one rank's [256][tiles] counts, in place
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t *hist, int tiles) {
  __shared__ uint32_t wave_sum[16];
  uint32_t *h = hist + (int64_t)blockIdx.x * kDigits * tiles;
  const int64_t n = (int64_t)kDigits * tiles;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  uint32_t carry = 0;
  for (int64_t at = 0; at < n; at += 1024) {
    const int64_t i = at + threadIdx.x;
    const uint32_t own = i < n ? h[i] : 0u;
    uint32_t s = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t t = (uint32_t)__shfl_up((int)s, o);
      if (lane >= o) s += t;
    }
    if (lane == 63) wave_sum[wave] = s;
    __syncthreads();
    uint32_t before = carry, total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += wave_sum[w];
      total += wave_sum[w];
    }
    if (i < n) h[i] = before + s - own;
    carry += total;
    __syncthreads();
  }
}

// lanes of the wave that are `in` and hold the same digit as this one
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool in) {
  uint64_t m = __ballot(in);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const uint64_t ones = __ballot((digit >> b) & 1u);
    m &= (digit >> b) & 1u ? ones : ~ones;
  }
  return m;
}

// Stable scatter: a wave walks its 512 keys in order, 64 at a time; a key's
// place is its digit's next free place plus the equal digits in lower lanes.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortArgs a) {
  __shared__ uint32_t next[4][kDigits];
  const int64_t rank = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
#pragma unroll
  for (int w = 0; w < 4; ++w) next[w][threadIdx.x] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * kSortTile + wave * kSortPerWave;
  uint32_t key[kSortPerWave / 64];
#pragma unroll
  for (int it = 0; it < kSortPerWave / 64; ++it) {
    const int64_t i = lo + it * 64 + lane;
    key[it] = i < a.T ? sort_key(a, rank, i) : 0u;
    if (i < a.T) atomicAdd(&next[wave][(key[it] >> a.shift) & 255u], 1u);
  }
  __syncthreads();
  uint32_t at = a.hist[(rank * kDigits + threadIdx.x) * a.tiles + blockIdx.x];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t c = next[w][threadIdx.x];
    next[w][threadIdx.x] = at;
    at += c;
  }
  __syncthreads();
  uint32_t *key_out = a.key_out + rank * a.T, *pos_out = a.pos_out + rank * a.T;
#pragma unroll
  for (int it = 0; it < kSortPerWave / 64; ++it) {
    const int64_t i = lo + it * 64 + lane;
    const bool in = i < a.T;
    const uint32_t digit = (key[it] >> a.shift) & 255u;
    const uint64_t same = same_digit(digit, in);
    const int before = __popcll(same & ((1ull << lane) - 1ull));
    uint32_t place = 0;
    if (in) place = next[wave][digit] + before;
    __builtin_amdgcn_wave_barrier();
    if (in && before == 0) next[wave][digit] += (uint32_t)__popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (in) {
      key_out[place] = key[it];
      pos_out[place] = a.tokens ? (uint32_t)i : a.pos_in[rank * a.T + i];
    }
  }
}

// ---------------------------------------------------------------------------
// Sums over the ordered positions
// ---------------------------------------------------------------------------
constexpr int kRun = 32;          // ordered entries of one wave
constexpr int kZeroRows = 64;     // table rows looked over by one wave
constexpr int kInFlight = 8;      // rows loaded ahead

struct SumArgs {
  const uint32_t *key, *pos;   // [N][T], ordered by (key, pos)
  const void *dout;            // [N][T][d]
  float *grads;                // [N][V][d]
  float *part;                 // [N][runs][2][d4]: a run's first row, where it began before; its last, where it goes on
  int64_t T, V, d, d4;
  int64_t runs, chunks, run_waves;
  int64_t zero_groups, zero_ranks;   // waves behind run_waves: zero_ranks x zero_groups
  float scale;
  bool accumulate;
};

// the lane's own columns to p
template <int VEC>
__device__ __forceinline__ void keep_row(float *p, const Columns<VEC> &c, const float v[VEC]) {
  if (c.skip == 0) {
    store_row<VEC>(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k)
      if (k >= c.skip) p[k] = v[k];
  }
}

template <int VEC>
__device__ __forceinline__ void write_grad(const SumArgs &a, int64_t rank, uint32_t row, const Columns<VEC> &c,
                                           const float sum[VEC]) {
  if (!c.any) return;
  float *p = a.grads + ((int64_t)rank * a.V + row) * a.d + c.first;
  float v[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) v[k] = sum[k] * a.scale;
  if (a.accumulate) {
    float old[VEC];
    load_row<VEC>(p, old);
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = old[k] + v[k];
  }
  keep_row<VEC>(p, c, v);
}

// n consecutive floats set to zero by one wave
__device__ __forceinline__ void zero_span(float *p, int64_t n) {
  const int lane = threadIdx.x & 63;
  const int64_t n4 = n / 4;
  for (int64_t i = lane; i < n4; i += 64) *reinterpret_cast<floatx4_u *>(p + 4 * i) = floatx4_u{0.f, 0.f, 0.f, 0.f};
  if (lane < n - 4 * n4) p[4 * n4 + lane] = 0.f;
}

// rows without a token among kZeroRows neighbours: each lane looks one up by
// bisection, neighbouring empty rows are cleared as one span
__device__ __forceinline__ void zero_rows(const SumArgs &a, int64_t rank, int64_t group) {
  const int lane = threadIdx.x & 63;
  const int64_t row0 = group * kZeroRows, row = row0 + lane;
  const uint32_t *key = a.key + rank * a.T;
  int64_t lo = 0, hi = a.T;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if ((int64_t)key[mid] < row) lo = mid + 1;
    else hi = mid;
  }
  const bool empty = row < a.V && !(lo < a.T && (int64_t)key[lo] == row);
  uint64_t left = __ballot(empty);
  float *base = a.grads + (rank * a.V + row0) * a.d;
  while (left) {
    const int s = __ffsll((unsigned long long)left) - 1;
    const uint64_t gap = ~(left >> s);
    const int len = gap ? __ffsll((unsigned long long)gap) - 1 : 64 - s;
    zero_span(base + (int64_t)s * a.d, (int64_t)len * a.d);
    left &= len + s >= 64 ? 0ull : ~0ull << (s + len);
  }
}

template <typename TIn, int VEC>
__global__ __launch_bounds__(256) void embgrad_sum_kernel(SumArgs a) {
  const int lane = threadIdx.x & 63;
  int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (w >= a.run_waves) {
    w -= a.run_waves;
    const int64_t rank = w / a.zero_groups;
    if (rank < a.zero_ranks) zero_rows(a, rank, w - rank * a.zero_groups);
    return;
  }
  const int64_t chunk = w % a.chunks, r = w / a.chunks, rank = r / a.runs, run = r - rank * a.runs;
  const uint32_t *key = a.key + rank * a.T, *pos = a.pos + rank * a.T;
  const int64_t lo = run * kRun, hi = lo + kRun < a.T ? lo + kRun : a.T;
  const int64_t mine = lo + lane < hi ? lo + lane : hi - 1;
  const uint32_t my_key = key[mine], my_pos = pos[mine];
  // entries of ids inside the table come first
  const int count = __popcll(__ballot(lo + lane < hi && (int64_t)my_key < a.V));
  if (count == 0) return;
  const Columns<VEC> c(chunk, a.d);
  const TIn *dout = static_cast<const TIn *>(a.dout) + rank * a.T * a.d + c.first;
  const uint32_t first_key = __builtin_amdgcn_readlane(my_key, 0);
  const bool begun = lo > 0 && key[lo - 1] == first_key;
  const bool goes_on = count == hi - lo && hi < a.T && key[hi] == (uint32_t)__builtin_amdgcn_readlane(my_key, count - 1);
  float *part = a.part + ((rank * a.runs + run) * 2) * a.d4;
  auto flush = [&](uint32_t row, bool head, bool tail, const float sum[VEC]) {
    if (head || tail) {
      if (!c.any) return;
      keep_row<VEC>(part + (head ? 0 : a.d4) + c.first, c, sum);
    } else {
      write_grad<VEC>(a, rank, row, c, sum);
    }
  };
  float sum[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) sum[k] = 0.f;
  uint32_t row = first_key;
  bool head = begun;
  for (int i0 = 0; i0 < count; i0 += kInFlight) {
    float x[kInFlight][VEC];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int i = i0 + u < count ? i0 + u : count - 1;
      const uint32_t p = (uint32_t)__builtin_amdgcn_readlane(my_pos, i);
      if (c.any) load_row<VEC>(dout + (int64_t)p * a.d, x[u]);
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (i0 + u >= count) break;
      const uint32_t k = (uint32_t)__builtin_amdgcn_readlane(my_key, i0 + u);
      if (k != row) {
        flush(row, head, false, sum);
        head = false;
        row = k;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += x[u][e];
    }
  }
  flush(row, head, goes_on, sum);
}

// Rows that cross a run's border: the run where such a row begins adds the
// parts of the following runs, in order.
template <int VEC>
__global__ __launch_bounds__(256) void embgrad_join_kernel(SumArgs a) {
  const int64_t w = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (w >= a.run_waves) return;
  const int64_t chunk = w % a.chunks, r = w / a.chunks, rank = r / a.runs, run = r - rank * a.runs;
  const uint32_t *key = a.key + rank * a.T;
  const int64_t lo = run * kRun, hi = lo + kRun;
  if (hi >= a.T) return;
  const uint32_t row = key[hi - 1];
  if ((int64_t)row >= a.V || key[hi] != row) return;                     // nothing goes on
  if (key[lo] == row && lo > 0 && key[lo - 1] == row) return;            // begun in an earlier run
  // the last entry of this row
  int64_t b = hi, e = a.T;
  while (b < e) {
    const int64_t mid = (b + e) / 2;
    if (key[mid] <= row) b = mid + 1;
    else e = mid;
  }
  const int64_t last = (b - 1) / kRun;
  const Columns<VEC> c(chunk, a.d);
  if (!c.any) return;
  const float *part = a.part + rank * a.runs * 2 * a.d4 + c.first;
  float sum[VEC];
  load_row<VEC>(part + (run * 2 + 1) * a.d4, sum);
  for (int64_t u0 = run + 1; u0 <= last; u0 += kInFlight) {
    float x[kInFlight][VEC];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) load_row<VEC>(part + (u0 + u <= last ? u0 + u : last) * 2 * a.d4, x[u]);
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (u0 + u > last) break;
#pragma unroll
      for (int k = 0; k < VEC; ++k) sum[k] += x[u][k];
    }
  }
  write_grad<VEC>(a, rank, row, c, sum);
}

unsigned blocks_for(int64_t waves) { return (unsigned)((waves + 3) / 4); }

// Elements of a lane: enough lanes of a wave at work on narrow rows, 16-byte
// loads of bfloat16 on wide ones.
int lane_columns(int64_t d) { return d > 256 ? 8 : d > 128 ? 4 : d > 64 ? 2 : 1; }

int64_t column_chunks(int64_t d) {
  const int64_t width = 64 * lane_columns(d);
  return (d + width - 1) / width;
}

size_t a256(size_t b) { return (b + 255) & ~(size_t)255; }

struct GradPlan {
  size_t key[2], pos[2], hist, part, bytes;
  int64_t runs, d4;
  int tiles;
};

GradPlan grad_plan(int64_t N, int64_t T, int64_t V, int64_t d) {
  GradPlan p{};
  p.tiles = (int)((T + kSortTile - 1) / kSortTile);
  p.runs = (T + kRun - 1) / kRun;
  p.d4 = (d + 3) / 4 * 4;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += a256(bytes);
    return o;
  };
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take((size_t)N * T * 4);
    p.pos[i] = take((size_t)N * T * 4);
  }
  p.hist = take((size_t)N * kDigits * p.tiles * 4);
  p.part = take((size_t)N * p.runs * 2 * p.d4 * 4);
  p.bytes = at;
  return p;
}

template <typename TIn, typename TOut>
void lookup_launch(gift_ctx *ctx, const LookupJob &j) {
  const int vec = lane_columns(j.d);
  const int chunks = (int)column_chunks(j.d);
  const int rows = vec == 8 ? lookup_rows<TIn, 8>() : 4;
  const int64_t waves = (j.T + rows - 1) / rows * chunks;
  const dim3 grid(blocks_for(waves < 65536 * 4 ? waves : 65536 * 4));
  const TIn *table = static_cast<const TIn *>(j.table);
  TOut *out = static_cast<TOut *>(j.out);
#define GIFT_LOOKUP(VEC)                                                                                          \
  hipLaunchKernelGGL((lookup_kernel<TIn, TOut, VEC>), grid, dim3(256), 0, ctx->stream, table, j.tokens, j.wide, j.T, \
                     j.V, j.d, chunks, j.scale, out)
  if (vec == 8) GIFT_LOOKUP(8);
  else if (vec == 4) GIFT_LOOKUP(4);
  else if (vec == 2) GIFT_LOOKUP(2);
  else GIFT_LOOKUP(1);
#undef GIFT_LOOKUP
}

template <typename TIn, int VEC>
gift_status sum_launch(gift_ctx *ctx, const SumArgs &a, int64_t zero_waves) {
  hipLaunchKernelGGL((embgrad_sum_kernel<TIn, VEC>), dim3(blocks_for(a.run_waves + zero_waves)), dim3(256), 0,
                     ctx->stream, a);
  gift_status st = check_launch("embgrad_sum_kernel");
  if (st != GIFT_OK || a.runs < 2) return st;
  hipLaunchKernelGGL((embgrad_join_kernel<VEC>), dim3(blocks_for(a.run_waves)), dim3(256), 0, ctx->stream, a);
  return check_launch("embgrad_join_kernel");
}

template <typename TIn>
gift_status sum_launch(gift_ctx *ctx, const SumArgs &a, int64_t zero_waves, int vec) {
  if (vec == 8) return sum_launch<TIn, 8>(ctx, a, zero_waves);
  if (vec == 4) return sum_launch<TIn, 4>(ctx, a, zero_waves);
  if (vec == 2) return sum_launch<TIn, 2>(ctx, a, zero_waves);
  return sum_launch<TIn, 1>(ctx, a, zero_waves);
}

}  // namespace

gift_status launch_lookup(gift_ctx *ctx, const LookupJob &j) {
  ProfileScope prof(ctx, GIFT_KERNEL_EMBED);
  if (j.table_bf16) {
    if (j.out_bf16) lookup_launch<uint16_t, uint16_t>(ctx, j);
    else lookup_launch<uint16_t, float>(ctx, j);
  } else {
    if (j.out_bf16) lookup_launch<float, uint16_t>(ctx, j);
    else lookup_launch<float, float>(ctx, j);
  }
  return check_launch("lookup_kernel");
}

size_t embgrad_scratch(int64_t N, int64_t T, int64_t V, int64_t d) {
  return T > 0 ? grad_plan(N, T, V, d).bytes : 0;
}

int64_t embgrad_waves(const EmbGradJob &j) {
  const int64_t run = (int64_t)j.N * ((j.T + kRun - 1) / kRun) * column_chunks(j.d);
  return run + (j.accumulate ? 0 : (int64_t)j.N * ((j.V + kZeroRows - 1) / kZeroRows));
}

gift_status launch_embgrad(gift_ctx *ctx, const EmbGradJob &j, char *ws) {
  const GradPlan p = grad_plan(j.N, j.T, j.V, j.d);
  uint32_t *key[2], *pos[2];
  for (int i = 0; i < 2; ++i) {
    key[i] = reinterpret_cast<uint32_t *>(ws + p.key[i]);
    pos[i] = reinterpret_cast<uint32_t *>(ws + p.pos[i]);
  }
  ProfileScope prof(ctx, GIFT_KERNEL_EMBED_GRAD);
  gift_status st;
  int cur = 0;
  if (j.T > 0) {
    int bits = 0;
    while ((j.V >> bits) != 0) ++bits;   // the keys are 0 .. V
    SortArgs s{};
    s.hist = reinterpret_cast<uint32_t *>(ws + p.hist);
    s.T = j.T;
    s.V = j.V;
    s.tiles = p.tiles;
    const dim3 grid(p.tiles, j.N);
    for (int shift = 0; shift < bits; shift += 8) {
      s.tokens = shift ? nullptr : j.tokens;
      s.wide = j.wide;
      s.key_in = key[cur];
      s.pos_in = pos[cur];
      cur = shift ? 1 - cur : 0;
      s.key_out = key[cur];
      s.pos_out = pos[cur];
      s.shift = shift;
      hipLaunchKernelGGL(sort_hist_kernel, grid, dim3(kSortThreads), 0, ctx->stream, s);
      if ((st = check_launch("sort_hist_kernel")) != GIFT_OK) return st;
      hipLaunchKernelGGL(sort_scan_kernel, dim3(j.N), dim3(1024), 0, ctx->stream, s.hist, p.tiles);
      if ((st = check_launch("sort_scan_kernel")) != GIFT_OK) return st;
      hipLaunchKernelGGL(sort_scatter_kernel, grid, dim3(kSortThreads), 0, ctx->stream, s);
      if ((st = check_launch("sort_scatter_kernel")) != GIFT_OK) return st;
    }
  }
  const int vec = lane_columns(j.d);
  SumArgs a{};
  a.key = key[cur];
  a.pos = pos[cur];
  a.dout = j.dout;
  a.grads = j.grads;
  a.part = reinterpret_cast<float *>(ws + p.part);
  a.T = j.T;
  a.V = j.V;
  a.d = j.d;
  a.d4 = p.d4;
  a.runs = p.runs;
  a.chunks = column_chunks(j.d);
  a.run_waves = (int64_t)j.N * p.runs * a.chunks;
  a.zero_groups = (j.V + kZeroRows - 1) / kZeroRows;
  a.scale = j.scale;
  a.accumulate = j.accumulate;
  a.zero_ranks = j.accumulate ? 0 : j.N;
  const int64_t zero_waves = a.zero_ranks * a.zero_groups;
  return j.bf16 ? sum_launch<uint16_t>(ctx, a, zero_waves, vec) : sum_launch<float>(ctx, a, zero_waves, vec);
}

}  // namespace gift
