// Embedding lookup and its gradient.
//
// Lookup: out[t] = scale * table[tokens[t]].  Gradient, for every rank j:
//
//   grads[j][v] (+)= scale * sum over t with tokens[j][t] = v of dout[j][t]
//
// The gradient first orders each rank's positions by token (stable radix sort),
// so that a row's terms are neighbours and stand in position order.  The
// ordered list is cut into runs of 8 to 32 entries, one wave each, whatever
// tokens they are of.  A wave adds its entries' rows in float32 and stores every
// row that begins and ends in its run; the parts of rows that cross a border go
// to scratch and a second kernel adds them in a fixed order, all parts of a row
// in one workgroup a column chunk: its time grows with the most frequent
// token's count.  No atomics on values: the same inputs give the same bits.
// Rows without a token are zeroed by further workgroups of the same launch.
//
// Ids outside [0, V) (padding) get the sort key V, the largest: they end up
// behind all others and nothing reads them.

#include "bf16.h"
#include "gift_internal.h"
#include "xcd_map.h"

namespace gift {

namespace {

// Rows of any length and address: 16-byte accesses at the element's own
// alignment (gfx950's vector memory takes any address).
typedef float floatx4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t uintx4_u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t uintx2_u __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t uintx1_u __attribute__((aligned(2)));

template <bool STREAM, typename W>
__device__ __forceinline__ W fetch(const W *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}

// VEC neighbouring elements of a row as loaded: converted only where they are
// used, so that several rows' loads are in flight together.
template <typename T, int VEC>
struct RowBits;

template <int VEC>
struct RowBits<float, VEC> {
  float x[VEC];
  // STREAM: past the caches
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const float *p) {
    if constexpr (VEC >= 4) {
#pragma unroll
      for (int i = 0; i < VEC; i += 4) {
        const floatx4_u w = fetch<STREAM>(reinterpret_cast<const floatx4_u *>(p + i));
#pragma unroll
        for (int k = 0; k < 4; ++k) x[i + k] = w[k];
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = p[i];
    }
  }
  __device__ __forceinline__ float operator[](int k) const { return x[k]; }
};

template <int VEC>
struct RowBits<uint16_t, VEC> {
  uint32_t w[(VEC + 1) / 2];
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const uint16_t *p) {
    if constexpr (VEC == 8) {
      const uintx4_u x = fetch<STREAM>(reinterpret_cast<const uintx4_u *>(p));
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = x[k];
    } else if constexpr (VEC == 4) {
      const uintx2_u x = fetch<STREAM>(reinterpret_cast<const uintx2_u *>(p));
#pragma unroll
      for (int k = 0; k < 2; ++k) w[k] = x[k];
    } else if constexpr (VEC == 2) {
      w[0] = *reinterpret_cast<const uintx1_u *>(p);
    } else {
      w[0] = p[0];
    }
  }
  __device__ __forceinline__ float operator[](int k) const { return k & 1 ? bf16_hi(w[k / 2]) : bf16_lo(w[k / 2]); }
};

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
  if constexpr (VEC == 4) {
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

// Columns of a lane: VEC from `first` on, always inside the row.  The row's last
// lane holds fewer: it loads the VEC columns that end the row, and the first
// `skip` of them belong to the lane before; lanes behind it load the same ones
// and own none (skip >= VEC).
template <int VEC>
struct Columns {
  int64_t first, skip;
  __device__ __forceinline__ Columns(int64_t chunk, int64_t d) {
    const int64_t c = (chunk * 64 + (threadIdx.x & 63)) * VEC, last = d - VEC;
    first = c <= last ? c : last;
    skip = c - first;
  }
  __device__ __forceinline__ bool any() const { return skip < VEC; }
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
    if (!c.any()) continue;
    RowBits<TIn, VEC> x[kLookupRows];
    bool in[kLookupRows];
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
      const int64_t id = read_token(tokens, wide, t0 + r < T ? t0 + r : T - 1);
      in[r] = id >= 0 && id < V;
      x[r].load(table + (in[r] ? id : 0) * d + c.first);
    }
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
      if (t0 + r >= T) break;
      float v[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[k] = in[r] ? x[r][k] * scale : 0.f;
      // (a row's last lane rewrites columns of the one before with the same values)
      stream_row<VEC>(out + (t0 + r) * d + c.first, v);
    }
  }
}

// ---------------------------------------------------------------------------
// Sort of each rank's positions by token
// ---------------------------------------------------------------------------
// Ranks of up to kLdsKeys positions are sorted by one workgroup each in LDS, all
// radix passes in one launch; longer ones through memory, a counting and a
// scattering launch a pass.
constexpr int kDigits = 256;
constexpr int kSmallKeys = 2048, kLdsKeys = 8192;

// lanes of the wave that are `in` and hold the same digit (8 bits) as this one
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool in) {
  const uint64_t all = __ballot(in);
  uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const uint64_t ones = __ballot((digit >> b) & 1u);
    const uint32_t own = (uint32_t)__builtin_amdgcn_sbfe((int)digit, b, 1);   // all ones where the bit is set
    lo &= ~((uint32_t)ones ^ own);
    hi &= ~((uint32_t)(ones >> 32) ^ own);
  }
  return (uint64_t)hi << 32 | lo;
}

struct LdsSortArgs {
  const void *tokens;      // [N, T]
  bool wide;
  uint32_t *key, *pos;     // [N, T], ordered
  uint32_t *present;       // null, or [N][words]: bit v % 32 of word v / 32 set where token v occurs
  int64_t T, V, words;
  int bits;                // of a key
};

// One workgroup of WAVES waves sorts one rank; a wave holds up to ITEMS x 64
// neighbouring keys.  Per pass a wave walks its keys in order: a key's place is
// the keys before it (in lower digits, earlier waves, earlier steps and lower
// lanes).  Bound by the chain of counter updates and the vector instructions of
// one CU; 8 x 2048 keys of 15 bits: 4 waves 14 us, 8 waves 10, 16 waves 9.
template <int WAVES, int ITEMS>
__global__ __launch_bounds__(WAVES * 64) void sort_lds_kernel(LdsSortArgs a) {
  constexpr int kThreads = WAVES * 64, kKeys = kThreads * ITEMS;
  __shared__ uint32_t keys[kKeys];
  __shared__ uint16_t places[kKeys];
  __shared__ uint32_t next[WAVES][kDigits];
  __shared__ uint32_t digit_sum[4];
  const int64_t rank = blockIdx.x;
  const int n = (int)a.T;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int steps = (n + kThreads - 1) / kThreads, lo = wave * steps * 64;
  for (int shift = 0; shift < a.bits; shift += 8) {
    for (int i = threadIdx.x; i < WAVES * kDigits; i += kThreads) next[0][i] = 0;
    __syncthreads();
    uint32_t key[ITEMS], where[ITEMS], order[ITEMS];
    constexpr uint32_t mask = kDigits - 1;
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      if (it >= steps) break;
      const int i = lo + it * 64 + lane;
      const bool in = i < n;
      key[it] = 0;
      where[it] = 0;
      if (in) {
        if (shift == 0) {
          const int64_t id = read_token(a.tokens, a.wide, rank * a.T + i);
          key[it] = (uint32_t)(id >= 0 && id < a.V ? id : a.V);
          where[it] = i;
        } else {
          key[it] = keys[i];
          where[it] = places[i];
        }
      }
    }
    // the digits' groups first (independent of each other), then the counters' chain
    uint64_t same[ITEMS];
#pragma unroll
    for (int it = 0; it < ITEMS; ++it)
      if (it < steps) same[it] = same_digit((key[it] >> shift) & mask, lo + it * 64 + lane < n);
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      if (it >= steps) break;
      const bool in = lo + it * 64 + lane < n;
      const uint32_t digit = (key[it] >> shift) & mask;
      const int before = __popcll(same[it] & ((1ull << lane) - 1ull));
      uint32_t seen = 0;
      if (in) seen = next[wave][digit];
      __builtin_amdgcn_wave_barrier();
      if (in && before == 0) next[wave][digit] = seen + (uint32_t)__popcll(same[it]);
      __builtin_amdgcn_wave_barrier();
      order[it] = seen + before;
    }
    __syncthreads();
    uint32_t sum = 0, upto = 0;
    if (threadIdx.x < kDigits) {
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const uint32_t c = next[w][threadIdx.x];
        next[w][threadIdx.x] = sum;
        sum += c;
      }
      upto = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = (uint32_t)__shfl_up((int)upto, o);
        if (lane >= o) upto += t;
      }
      if (lane == 63) digit_sum[wave] = upto;
    }
    __syncthreads();
    if (threadIdx.x < kDigits) {
      uint32_t base = upto - sum;
      for (int w = 0; w < wave; ++w) base += digit_sum[w];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) next[w][threadIdx.x] += base;
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < ITEMS; ++it) {
      if (it >= steps) break;
      if (lo + it * 64 + lane >= n) continue;
      const uint32_t at = next[wave][(key[it] >> shift) & mask] + order[it];
      keys[at] = key[it];
      places[at] = (uint16_t)where[it];
    }
    __syncthreads();
  }
  uint32_t *key_out = a.key + rank * a.T, *pos_out = a.pos + rank * a.T;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    key_out[i] = keys[i];
    pos_out[i] = places[i];
  }
  if (!a.present) return;
  // the rows that occur, a window of table rows at a time
  uint32_t *bits = &next[0][0];
  uint32_t *out = a.present + rank * a.words;
  for (int64_t word0 = 0; word0 < a.words; word0 += WAVES * kDigits) {
    for (int i = threadIdx.x; i < WAVES * kDigits; i += kThreads) bits[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint32_t k = keys[i];
      const int64_t w = (int64_t)(k / 32) - word0;
      if ((int64_t)k < a.V && w >= 0 && w < WAVES * kDigits && (i == 0 || keys[i - 1] != k)) atomicOr(&bits[w], 1u << (k % 32));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < WAVES * kDigits && word0 + i < a.words; i += kThreads) out[word0 + i] = bits[i];
    __syncthreads();
  }
}

constexpr int kSortWaves = 8, kSortThreads = kSortWaves * 64;
constexpr int kSortPerWave = 256;                      // keys of a wave, in order
constexpr int kSortTile = kSortWaves * kSortPerWave;   // keys of a workgroup
constexpr int kSortItems = kSortTile / kSortThreads;
// Up to this many tiles a scattering workgroup sums their counts itself (65536
// positions: a launch between the two took 8.6 us a pass, this adds 1).
constexpr int kScanTiles = 64;

struct SortArgs {
  const void *tokens;      // first pass: [N, T] ids; else null
  bool wide, scanned;      // scanned: hist holds first places
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t *hist;          // [N][tiles][256] counts, then first places
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
  if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * kSortTile + threadIdx.x;
  uint32_t key[kSortItems];
#pragma unroll
  for (int it = 0; it < kSortItems; ++it)
    key[it] = lo + it * kSortThreads < a.T ? sort_key(a, rank, lo + it * kSortThreads) : 0xffffffffu;
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    if (lo + it * kSortThreads < a.T) atomicAdd(&count[(key[it] >> a.shift) & 255u], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kDigits) a.hist[(rank * a.tiles + blockIdx.x) * kDigits + threadIdx.x] = count[threadIdx.x];
}

// exclusive prefix sums over 256 digits, one a thread of the first four waves
__device__ __forceinline__ uint32_t digits_before(uint32_t count, uint32_t wave_sum[4]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  uint32_t s = count;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t t = (uint32_t)__shfl_up((int)s, o);
    if (lane >= o) s += t;
  }
  if (lane == 63 && wave < 4) wave_sum[wave] = s;
  __syncthreads();
  for (int w = 0; w < wave && w < 4; ++w) s += wave_sum[w];
  return s - count;
}

// one rank's [tiles][256] counts become first places, in place (many tiles): a
// digit's tiles in four quarters, eight loads in flight
__global__ __launch_bounds__(4 * kDigits) void sort_scan_kernel(uint32_t *hist, int tiles) {
  __shared__ uint32_t quarter_sum[4][kDigits];
  __shared__ uint32_t first[kDigits];
  __shared__ uint32_t wave_sum[4];
  const int digit = threadIdx.x % kDigits, quarter = threadIdx.x / kDigits, share = (tiles + 3) / 4;
  const int from = quarter * share, to = from + share < tiles ? from + share : tiles;
  uint32_t *h = hist + (int64_t)blockIdx.x * tiles * kDigits + digit;
  uint32_t sum = 0;
#pragma unroll 8
  for (int t = from; t < to; ++t) sum += h[(int64_t)t * kDigits];
  quarter_sum[quarter][digit] = sum;
  __syncthreads();
  uint32_t before = 0, total = 0;
  for (int q = 0; q < 4; ++q) {
    if (q < quarter) before += quarter_sum[q][digit];
    total += quarter_sum[q][digit];
  }
  // (the first quarter's threads are the first four waves)
  const uint32_t digit_first = digits_before(total, wave_sum);
  if (quarter == 0) first[digit] = digit_first;
  __syncthreads();
  uint32_t at = first[digit] + before;
  for (int t0 = from; t0 < to; t0 += 8) {
    uint32_t c[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) c[u] = t0 + u < to ? h[(int64_t)(t0 + u) * kDigits] : 0u;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (t0 + u < to) h[(int64_t)(t0 + u) * kDigits] = at;
      at += c[u];
    }
  }
}

// Stable scatter: a wave walks its keys in order, 64 at a time; a key's
// place is its digit's next free place plus the equal digits in lower lanes.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortArgs a) {
  __shared__ uint32_t next[kSortWaves][kDigits];
  __shared__ uint32_t wave_sum[4];
  const int64_t rank = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, digit_of = threadIdx.x % kDigits;
  for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) next[0][i] = 0;
  const int64_t lo = (int64_t)blockIdx.x * kSortTile + wave * kSortPerWave;
  uint32_t key[kSortItems], pos[kSortItems];
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    const int64_t i = lo + it * 64 + lane;
    key[it] = i < a.T ? sort_key(a, rank, i) : 0u;
    pos[it] = a.tokens || i >= a.T ? (uint32_t)i : a.pos_in[rank * a.T + i];
  }
  // the tile's first place of digit digit_of (its second half of the threads does the same and keeps nothing)
  const uint32_t *h = a.hist + rank * a.tiles * kDigits + digit_of;
  uint32_t first;
  if (a.scanned) {
    first = h[(int64_t)blockIdx.x * kDigits];
  } else {
    uint32_t total = 0;
    first = 0;
    for (int t0 = 0; t0 < a.tiles; t0 += 16) {
      uint32_t c[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) c[u] = t0 + u < a.tiles ? h[(int64_t)(t0 + u) * kDigits] : 0u;
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        if (t0 + u < (int)blockIdx.x) first += c[u];
        total += c[u];
      }
    }
    first += digits_before(total, wave_sum);
  }
  __syncthreads();
  uint64_t same[kSortItems];
  uint32_t order[kSortItems];
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) same[it] = same_digit((key[it] >> a.shift) & 255u, lo + it * 64 + lane < a.T);
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    const bool in = lo + it * 64 + lane < a.T;
    const uint32_t digit = (key[it] >> a.shift) & 255u;
    const int before = __popcll(same[it] & ((1ull << lane) - 1ull));
    uint32_t seen = 0;
    if (in) seen = next[wave][digit];
    __builtin_amdgcn_wave_barrier();
    if (in && before == 0) next[wave][digit] = seen + (uint32_t)__popcll(same[it]);
    __builtin_amdgcn_wave_barrier();
    order[it] = seen + before;
  }
  __syncthreads();
  if (threadIdx.x < kDigits) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = next[w][digit_of];
      next[w][digit_of] = first;
      first += c;
    }
  }
  __syncthreads();
  uint32_t *key_out = a.key_out + rank * a.T, *pos_out = a.pos_out + rank * a.T;
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    if (lo + it * 64 + lane >= a.T) continue;
    const uint32_t place = next[wave][(key[it] >> a.shift) & 255u] + order[it];
    key_out[place] = key[it];
    pos_out[place] = pos[it];
  }
}

// ---------------------------------------------------------------------------
// Sums over the ordered positions
// ---------------------------------------------------------------------------
struct SumArgs {
  const uint32_t *key, *pos;   // [N][T], ordered by (key, pos)
  const void *dout;            // [N][T][d]
  float *grads;                // [N][V][d]
  float *part;                 // [N][runs][2][d4]: a run's first row, where it began before; its last, where it goes on
  const uint32_t *present;     // null, or [N][words] (LdsSortArgs)
  int64_t T, V, d, d4, words;
  int64_t runs, chunks, run_waves;
  int64_t zero_groups, zero_ranks;   // groups of zero_rows table rows of a rank; ranks to look over
  int64_t run_blocks;                // workgroups of the runs, a multiple of 8; one a zero group follows
  int run;                           // ordered entries of one wave, 8 to 32
  int zero_rows;                     // table rows looked over by one workgroup, a power of two up to 32
  float scale;
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

// n consecutive floats set to zero by one workgroup: whole 128-byte lines past
// the caches, what is left at either end through them (streamed parts of lines
// cost their whole line)
__device__ __forceinline__ void zero_span(float *p, int64_t n) {
  const int64_t lead = (-(int64_t)(reinterpret_cast<uintptr_t>(p) / 4)) & 31, skip = lead < n ? lead : n;
  if (threadIdx.x < skip) p[threadIdx.x] = 0.f;       // up to a line of 128 bytes
  p += skip;
  n -= skip;
  const int64_t whole = n & ~31ll;
  for (int64_t i = threadIdx.x * 4; i < whole; i += 1024)
    __builtin_nontemporal_store(floatx4_u{0.f, 0.f, 0.f, 0.f}, reinterpret_cast<floatx4_u *>(p + i));
  if (threadIdx.x < n - whole) p[whole + threadIdx.x] = 0.f;
}

// Bits of the neighbouring rows from row0 on that occur among a rank's T ordered
// keys, by a bisection a lane (a search by the whole wave, 64 keys at a time,
// starts again behind every frequent token: 131072 positions 62 -> 116 us).
__device__ __forceinline__ uint64_t rows_there(const uint32_t *key, int64_t T, int64_t row0) {
  const int64_t row = row0 + (threadIdx.x & 63);
  int64_t lo = 0, hi = T;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if ((int64_t)key[mid] < row) lo = mid + 1;
    else hi = mid;
  }
  return __ballot(lo < T && (int64_t)key[lo] == row);
}

// Rows without a token among zero_rows neighbours, from the sort's bits or else
// by bisection (every wave of the workgroup for itself); neighbouring empty rows
// are cleared as one span.
__device__ __forceinline__ void zero_rows(const SumArgs &a, int64_t rank, int64_t group) {
  const int64_t row0 = group * a.zero_rows;
  const int rows = (int)(a.V - row0 < a.zero_rows ? a.V - row0 : a.zero_rows);
  const uint64_t there = a.present ? a.present[rank * a.words + row0 / 32] >> (row0 % 32)
                                   : rows_there(a.key + rank * a.T, a.T, row0);
  float *base = a.grads + (rank * a.V + row0) * a.d;
  uint64_t left = ~there & ((1ull << rows) - 1ull);
  while (left) {
    const int s = __ffsll((unsigned long long)left) - 1;
    const int len = __ffsll((unsigned long long)~(left >> s)) - 1;
    zero_span(base + (int64_t)s * a.d, (int64_t)len * a.d);
    left &= ~0ull << (s + len);
  }
}

// ACC: what grads holds of a row is loaded with the row's first entry.
template <typename TIn, int VEC, bool ACC>
__global__ __launch_bounds__(256) void embgrad_sum_kernel(SumArgs a) {
  constexpr int kInFlight = ACC ? 4 : 8;      // rows loaded ahead
  const int lane = threadIdx.x & 63;
  if ((int64_t)blockIdx.x >= a.run_blocks) {
    const int64_t g = xcd_tile((int64_t)blockIdx.x - a.run_blocks, a.zero_ranks * a.zero_groups), rank = g / a.zero_groups;
    zero_rows(a, rank, g - rank * a.zero_groups);
    return;
  }
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (w >= a.run_waves) return;
  const int64_t chunk = w % a.chunks, r = w / a.chunks, rank = r / a.runs, run = r - rank * a.runs;
  const uint32_t *key = a.key + rank * a.T, *pos = a.pos + rank * a.T;
  const int64_t lo = run * a.run, hi = lo + a.run < a.T ? lo + a.run : a.T;
  const int64_t mine = lo + lane < hi ? lo + lane : hi - 1;
  const uint32_t my_key = key[mine], my_pos = pos[mine];
  const uint32_t key_before = lo > 0 ? key[lo - 1] : 0xffffffffu, key_behind = hi < a.T ? key[hi] : 0xffffffffu;
  // entries of ids inside the table come first
  const int count = __popcll(__ballot(lo + lane < hi && (int64_t)my_key < a.V));
  if (count == 0) return;
  const Columns<VEC> c(chunk, a.d);
  const TIn *dout = static_cast<const TIn *>(a.dout) + rank * a.T * a.d + c.first;
  float *grads = a.grads + rank * a.V * a.d + c.first;
  float *part = a.part + ((rank * a.runs + run) * 2) * a.d4 + c.first;
  uint32_t row = __builtin_amdgcn_readlane(my_key, 0);
  bool head = key_before == row;
  // the run's last row goes on behind it (key V never does: an id outside the table is not counted)
  const bool goes_on = count == hi - lo && key_behind == (uint32_t)__builtin_amdgcn_readlane(my_key, count - 1);
  float sum[VEC], old[VEC];
  auto flush = [&](bool tail) {
    if (head || tail) {
      keep_row<VEC>(part + (head ? 0 : a.d4), c, sum);
      return;
    }
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = ACC ? old[e] + sum[e] * a.scale : sum[e] * a.scale;
    keep_row<VEC>(grads + (int64_t)row * a.d, c, v);
  };
  for (int i0 = 0; i0 < count; i0 += kInFlight) {
    RowBits<TIn, VEC> x[kInFlight];
    RowBits<float, VEC> was[ACC ? kInFlight : 1];
    uint32_t k[kInFlight];
    bool starts[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int i = i0 + u < count ? i0 + u : count - 1;
      k[u] = (uint32_t)__builtin_amdgcn_readlane(my_key, i);
      starts[u] = i0 + u < count && (i == 0 || k[u] != (uint32_t)__builtin_amdgcn_readlane(my_key, i > 0 ? i - 1 : 0));
      const uint32_t p = (uint32_t)__builtin_amdgcn_readlane(my_pos, i);
      x[u].template load<true>(dout + (int64_t)p * a.d);
      if constexpr (ACC)
        if (starts[u]) was[u].load(grads + (int64_t)k[u] * a.d);
    }
    __builtin_amdgcn_sched_barrier(0);      // all of them in flight before the first is added
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (i0 + u >= count) break;
      if (starts[u]) {
        if (i0 + u > 0) {
          flush(false);
          head = false;
        }
        row = k[u];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          sum[e] = 0.f;
          if constexpr (ACC) old[e] = was[u][e];
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += x[u][e];
    }
  }
  flush(goes_on);
}

// Rows that cross a run's border: the run where such a row begins adds the
// parts of the following runs.  A wave looks after one run; up to kJoinAlone
// parts it adds itself, in order, longer rows are left to the whole workgroup,
// a share of the parts a wave and then the shares' sums in order.  (A workgroup
// for each run spent most of its 13 us at 65536 x 1536 on being launched.)
// A row's parts are looked up 64 runs at a time and added eight at a time, one
// after the other: 65536 bfloat16 rows of 1536, tokens by Zipf's law, every other
// one the same, all the same: 101, 118, 144 us written and 97, 110, 114 added.
constexpr int kJoinAlone = 8, kJoinWaves = 4;

template <int VEC>
__device__ __forceinline__ void load_sum(const float *p, float sum[VEC]) {
  RowBits<float, VEC> x;
  x.load(p);
#pragma unroll
  for (int k = 0; k < VEC; ++k) sum[k] = x[k];
}

// parts from .. to (exclusive) of a row, the p-th at part + p * stride, added to sum in order
template <int VEC>
__device__ __forceinline__ void add_parts(const float *part, int64_t stride, int64_t from, int64_t to, float sum[VEC]) {
  constexpr int kInFlight = 8;
  for (int64_t u0 = from; u0 < to; u0 += kInFlight) {
    RowBits<float, VEC> x[kInFlight];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) x[u].load(part + (u0 + u < to ? u0 + u : to - 1) * stride);
    __builtin_amdgcn_sched_barrier(0);      // all of them in flight before the first is added
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (u0 + u >= to) break;
#pragma unroll
      for (int k = 0; k < VEC; ++k) sum[k] += x[u][k];
    }
  }
}

template <int VEC, bool ACC>
__device__ __forceinline__ void finish_row(const SumArgs &a, int64_t rank, uint32_t row, const Columns<VEC> &c,
                                           const float sum[VEC]) {
  float *p = a.grads + (rank * a.V + row) * a.d + c.first;
  float v[VEC];
  RowBits<float, VEC> old;
  if constexpr (ACC) old.load(p);
#pragma unroll
  for (int k = 0; k < VEC; ++k) v[k] = ACC ? old[k] + sum[k] * a.scale : sum[k] * a.scale;
  keep_row<VEC>(p, c, v);
}

template <int VEC, bool ACC>
__global__ __launch_bounds__(kJoinWaves * 64) void embgrad_join_kernel(SumArgs a) {
  __shared__ float shares[kJoinWaves][64][VEC];
  __shared__ int64_t parts[kJoinWaves];      // 0, or the parts of a row that is left to the workgroup
  __shared__ uint32_t rows[kJoinWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  // workgroup: kJoinWaves runs of one rank and one chunk of columns
  const int64_t groups = (a.runs + kJoinWaves - 1) / kJoinWaves;
  const int64_t chunk = blockIdx.x % a.chunks, r = blockIdx.x / a.chunks, rank = r / groups;
  const int64_t run0 = (r - rank * groups) * kJoinWaves, run = run0 + wave;
  const uint32_t *key = a.key + rank * a.T;
  const int64_t lo = run * a.run, hi = lo + a.run;
  const Columns<VEC> c(chunk, a.d);
  const float *part = a.part + (rank * a.runs + run) * 2 * a.d4 + c.first;
  int64_t n = 0;
  uint32_t row = 0;
  if (hi < a.T) {
    row = key[hi - 1];
    const bool begun = key[lo] == row && lo > 0 && key[lo - 1] == row;
    if ((int64_t)row < a.V && !begun) {
      // the runs behind this one that begin with the row, 64 looked at together
      for (bool more = true; more;) {
        const int64_t i = (run + 1 + n + lane) * a.run;
        const uint64_t there = __ballot(i < a.T && key[i < a.T ? i : 0] == row);
        more = there == ~0ull;
        n += more ? 64 : __ffsll((unsigned long long)~there) - 1;
      }
    }
  }
  if (lane == 0) {
    parts[wave] = n > kJoinAlone ? n : 0;
    rows[wave] = row;
  }
  if (n > 0 && n <= kJoinAlone) {
    float sum[VEC];
    load_sum<VEC>(part + a.d4, sum);
    add_parts<VEC>(part, 2 * a.d4, 1, n + 1, sum);
    finish_row<VEC, ACC>(a, rank, row, c, sum);
  }
  __syncthreads();
  for (int q = 0; q < kJoinWaves; ++q) {
    const int64_t long_n = parts[q];
    if (long_n == 0) continue;
    const float *first = a.part + (rank * a.runs + run0 + q) * 2 * a.d4 + c.first;
    const int64_t share = (long_n + kJoinWaves - 1) / kJoinWaves;
    const int64_t from = 1 + wave * share, to = from + share < long_n + 1 ? from + share : long_n + 1;
    float sum[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) sum[k] = 0.f;
    if (wave == 0) load_sum<VEC>(first + a.d4, sum);
    add_parts<VEC>(first, 2 * a.d4, from, to, sum);
#pragma unroll
    for (int k = 0; k < VEC; ++k) shares[wave][lane][k] = sum[k];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int s = 1; s < kJoinWaves; ++s)
#pragma unroll
        for (int k = 0; k < VEC; ++k) sum[k] += shares[s][lane][k];
      finish_row<VEC, ACC>(a, rank, rows[q], c, sum);
    }
    __syncthreads();
  }
}

unsigned blocks_for(int64_t waves) { return (unsigned)((waves + 3) / 4); }

// Elements of a lane: enough lanes of a wave at work on narrow rows, 16-byte
// loads of bfloat16 on wide ones.
int lane_columns(int64_t d) { return d > 256 ? 8 : d > 128 ? 4 : d > 64 ? 2 : 1; }

// A sum takes at most four: 65536 rows of 1536 written, float32 136 us (eight:
// 161), bfloat16 101 (111); added 129 (146) and 97 (102).
int sum_columns(int64_t d) {
  const int vec = lane_columns(d);
  return vec > 4 ? 4 : vec;
}

int64_t column_chunks(int64_t d, int vec) { return (d + 64 * vec - 1) / (64 * vec); }

size_t a256(size_t b) { return (b + 255) & ~(size_t)255; }

// Ordered entries of a wave: 32 where that still makes two waves a SIMD, down
// to 8 for short ranks, whose time is the longest chain of additions.
int run_length(int64_t N, int64_t T, int64_t d) {
  int run = 32;
  while (run > 8 && N * ((T + run - 1) / run) * column_chunks(d, sum_columns(d)) < 2048) run /= 2;
  return run;
}

// Table rows that a workgroup looks over for empty ones: 16 to 32 KB of widths
// from 128 to 1024; 32 narrower rows, four wider ones.
int zero_rows_of(int64_t d) {
  int rows = 4;
  while (rows < 32 && rows * d < 4096) rows *= 2;
  return rows;
}

struct GradPlan {
  size_t key[2], pos[2], hist, part, present, bytes;
  int64_t runs, d4, words;      // words: of a rank's row bits, 0 without
  int run, tiles;               // tiles: 0 for the sort in LDS
};

GradPlan grad_plan(int64_t N, int64_t T, int64_t V, int64_t d) {
  GradPlan p{};
  p.run = run_length(N, T, d);
  p.runs = (T + p.run - 1) / p.run;
  p.d4 = (d + 3) / 4 * 4;
  p.tiles = T <= kLdsKeys ? 0 : (int)((T + kSortTile - 1) / kSortTile);
  // row bits from the sort in LDS (past 2^20 rows its windows would take longer
  // than the bisections; the sort through memory leaves none: set there by
  // atomics, frequent tokens' words took 180 us at 65536 positions)
  p.words = p.tiles == 0 && V <= 1 << 20 ? (V + 31) / 32 : 0;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += a256(bytes);
    return o;
  };
  for (int i = 0; i < (p.tiles ? 2 : 1); ++i) {
    p.key[i] = take((size_t)N * T * 4);
    p.pos[i] = take((size_t)N * T * 4);
  }
  p.hist = take((size_t)N * kDigits * p.tiles * 4);
  p.present = take((size_t)N * p.words * 4);
  p.part = take((size_t)N * p.runs * 2 * p.d4 * 4);
  p.bytes = at;
  return p;
}

template <typename TIn, typename TOut, int VEC>
void lookup_launch(gift_ctx *ctx, const LookupJob &j) {
  constexpr int rows = lookup_rows<TIn, VEC>();
  const int chunks = (int)column_chunks(j.d, VEC);
  const int64_t waves = (j.T + rows - 1) / rows * chunks;
  hipLaunchKernelGGL((lookup_kernel<TIn, TOut, VEC>), dim3(blocks_for(waves < 65536 * 4 ? waves : 65536 * 4)),
                     dim3(256), 0, ctx->stream, static_cast<const TIn *>(j.table), j.tokens, j.wide, j.T, j.V, j.d,
                     chunks, j.scale, static_cast<TOut *>(j.out));
}

// A float32 row is stored 16 bytes a lane, so that an instruction writes one
// span; past the caches wherever rows start (65536 x 771 from a float32 table:
// through them 73 us, past them 52; x 259 from bfloat16 30 and 17).
template <typename TIn>
void lookup_launch(gift_ctx *ctx, const LookupJob &j) {
  const int vec = lane_columns(j.d);
  if (j.out_bf16) {
    if (vec == 8) lookup_launch<TIn, uint16_t, 8>(ctx, j);
    else if (vec == 4) lookup_launch<TIn, uint16_t, 4>(ctx, j);
    else if (vec == 2) lookup_launch<TIn, uint16_t, 2>(ctx, j);
    else lookup_launch<TIn, uint16_t, 1>(ctx, j);
  } else if (vec >= 4) {
    lookup_launch<TIn, float, 4>(ctx, j);
  } else if (vec == 2) {
    lookup_launch<TIn, float, 2>(ctx, j);
  } else {
    lookup_launch<TIn, float, 1>(ctx, j);
  }
}

template <typename TIn, int VEC, bool ACC>
gift_status sum_launch(gift_ctx *ctx, const SumArgs &a) {
  // How fast memory takes the zeros hangs on how much of it is written at the
  // same time: 8 x 32000 x 1024 by waves of 16 KB each 206 us, by workgroups of
  // 16 KB whose neighbours run on one XCD 197, and with three of them a CU, which
  // this much LDS makes it, 172.  Sums with few rows to clear do not lose by it:
  // 8 ranks of 8192 positions with 8000, 4000 and 1000 rows 98, 81 and 65 us
  // without, 92, 74 and 62 with; one rank with 1000 rows of 1536 31.1 and 30.9.
  // (The search for empty rows wants more waves.)
  const unsigned lds = a.zero_ranks > 0 && a.present ? 52 * 1024 : 0;
  hipLaunchKernelGGL((embgrad_sum_kernel<TIn, VEC, ACC>),
                     dim3((unsigned)(a.run_blocks + a.zero_ranks * a.zero_groups)), dim3(256), lds, ctx->stream, a);
  gift_status st = check_launch("embgrad_sum_kernel");
  if (st != GIFT_OK || a.runs < 2) return st;
  const int64_t ranks = a.run_waves / (a.runs * a.chunks), groups = (a.runs + kJoinWaves - 1) / kJoinWaves;
  hipLaunchKernelGGL((embgrad_join_kernel<VEC, ACC>), dim3((unsigned)(ranks * groups * a.chunks)),
                     dim3(kJoinWaves * 64), 0, ctx->stream, a);
  return check_launch("embgrad_join_kernel");
}

template <typename TIn, bool ACC>
gift_status sum_launch(gift_ctx *ctx, const SumArgs &a) {
  const int vec = sum_columns(a.d);
  if (vec == 4) return sum_launch<TIn, 4, ACC>(ctx, a);
  if (vec == 2) return sum_launch<TIn, 2, ACC>(ctx, a);
  return sum_launch<TIn, 1, ACC>(ctx, a);
}

// Orders every rank's positions; `cur` receives the buffers (0 or 1) with the result.
gift_status sort_launch(gift_ctx *ctx, const EmbGradJob &j, const GradPlan &p, uint32_t *const key[2],
                        uint32_t *const pos[2], char *ws, int *cur) {
  int bits = 0;
  while ((j.V >> bits) != 0) ++bits;   // the keys are 0 .. V
  gift_status st;
  *cur = 0;
  if (p.tiles == 0) {
    LdsSortArgs a{};
    a.tokens = j.tokens;
    a.wide = j.wide;
    a.key = key[0];
    a.pos = pos[0];
    a.present = p.words && !j.accumulate ? reinterpret_cast<uint32_t *>(ws + p.present) : nullptr;
    a.T = j.T;
    a.V = j.V;
    a.words = p.words;
    a.bits = bits;
    if (j.T <= kSmallKeys)
      hipLaunchKernelGGL((sort_lds_kernel<16, kSmallKeys / 1024>), dim3(j.N), dim3(1024), 0, ctx->stream, a);
    else
      hipLaunchKernelGGL((sort_lds_kernel<16, kLdsKeys / 1024>), dim3(j.N), dim3(1024), 0, ctx->stream, a);
    return check_launch("sort_lds_kernel");
  }
  SortArgs s{};
  s.hist = reinterpret_cast<uint32_t *>(ws + p.hist);
  s.T = j.T;
  s.V = j.V;
  s.tiles = p.tiles;
  s.scanned = p.tiles > kScanTiles;
  const dim3 grid(p.tiles, j.N);
  for (int shift = 0; shift < bits; shift += 8) {
    s.tokens = shift ? nullptr : j.tokens;
    s.wide = j.wide;
    s.key_in = key[*cur];
    s.pos_in = pos[*cur];
    *cur = shift ? 1 - *cur : 0;
    s.key_out = key[*cur];
    s.pos_out = pos[*cur];
    s.shift = shift;
    hipLaunchKernelGGL(sort_hist_kernel, grid, dim3(kSortThreads), 0, ctx->stream, s);
    if ((st = check_launch("sort_hist_kernel")) != GIFT_OK) return st;
    if (s.scanned) {
      hipLaunchKernelGGL(sort_scan_kernel, dim3(j.N), dim3(4 * kDigits), 0, ctx->stream, s.hist, p.tiles);
      if ((st = check_launch("sort_scan_kernel")) != GIFT_OK) return st;
    }
    hipLaunchKernelGGL(sort_scatter_kernel, grid, dim3(kSortThreads), 0, ctx->stream, s);
    if ((st = check_launch("sort_scatter_kernel")) != GIFT_OK) return st;
  }
  return GIFT_OK;
}

}  // namespace

gift_status launch_lookup(gift_ctx *ctx, const LookupJob &j) {
  ProfileScope prof(ctx, GIFT_KERNEL_EMBED);
  if (j.table_bf16) lookup_launch<uint16_t>(ctx, j);
  else lookup_launch<float>(ctx, j);
  return check_launch("lookup_kernel");
}

size_t embgrad_scratch(int64_t N, int64_t T, int64_t V, int64_t d) {
  return T > 0 ? grad_plan(N, T, V, d).bytes : 0;
}

int64_t embgrad_blocks(const EmbGradJob &j) {
  const int run = run_length(j.N, j.T, j.d);
  const int64_t runs = (j.T + run - 1) / run;
  return (int64_t)j.N * ((runs + 3) / 4 + 1) * column_chunks(j.d, sum_columns(j.d)) + 8 +
         (j.accumulate ? 0 : (int64_t)j.N * ((j.V + zero_rows_of(j.d) - 1) / zero_rows_of(j.d)));
}

gift_status launch_embgrad(gift_ctx *ctx, const EmbGradJob &j, char *ws) {
  const GradPlan p = j.T > 0 ? grad_plan(j.N, j.T, j.V, j.d) : GradPlan{};
  uint32_t *key[2], *pos[2];
  for (int i = 0; i < 2; ++i) {
    key[i] = reinterpret_cast<uint32_t *>(ws + p.key[i]);
    pos[i] = reinterpret_cast<uint32_t *>(ws + p.pos[i]);
  }
  ProfileScope prof(ctx, GIFT_KERNEL_EMBED_GRAD);
  int cur = 0;
  if (j.T > 0) {
    gift_status st = sort_launch(ctx, j, p, key, pos, ws, &cur);
    if (st != GIFT_OK) return st;
  }
  SumArgs a{};
  a.key = key[cur];
  a.pos = pos[cur];
  a.dout = j.dout;
  a.grads = j.grads;
  a.part = reinterpret_cast<float *>(ws + p.part);
  a.present = p.words ? reinterpret_cast<const uint32_t *>(ws + p.present) : nullptr;
  a.T = j.T;
  a.V = j.V;
  a.d = j.d;
  a.d4 = p.d4;
  a.words = p.words;
  a.run = p.run;
  a.runs = p.runs;
  a.chunks = column_chunks(j.d, sum_columns(j.d));
  a.run_waves = (int64_t)j.N * p.runs * a.chunks;
  a.zero_rows = zero_rows_of(j.d);
  a.zero_groups = (j.V + a.zero_rows - 1) / a.zero_rows;
  a.zero_ranks = j.accumulate ? 0 : j.N;
  a.run_blocks = ((int64_t)blocks_for(a.run_waves) + 7) / 8 * 8;
  a.scale = j.scale;
  if (j.accumulate) return j.bf16 ? sum_launch<uint16_t, true>(ctx, a) : sum_launch<float, true>(ctx, a);
  return j.bf16 ? sum_launch<uint16_t, false>(ctx, a) : sum_launch<float, false>(ctx, a);
}

}  // namespace gift
