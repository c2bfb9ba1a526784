// Token tables (embeddings): lookup, per-example gradient norms, clipped sum.
//
//   lookup    out[n, :]  = scale * W[id_n, :]
//   norms     n2_i      += scale^2 sum_v || sum_{t: id_it = v} G[i, t, :] ||^2
//   sum       grad[v, :] = scale * sum_i c_i sum_{t: id_it = v} G[i, t, :]
//
// An id outside [0, V) is an empty position: a row of zeros out, and a row of G
// that is never read.
//
// The gradient is formed by sorted tokens, without floating-point atomics. For the
// sum, a counting sort gives the positions of every token in ascending order
// (order, and offsets into it); a wave takes kChunk consecutive entries of that
// list and a block of columns and adds rows until the token changes, so that
// the work is even whatever the frequencies of the tokens are. A token whose
// entries lie in several chunks leaves partial rows that a last pass joins in
// order; rows without a token are filled by waves of their own in the same
// launch. For the norms every example's tokens are sorted in LDS, and equal
// tokens, then neighbours, are added before they are squared.
//
// All of it is bound by memory traffic where it is large, by launches and the
// sorts' latency where it is small. 128 x 256 tokens, a 50257 x 768 table, bf16 G
// (50 MB): lookup (float32 to bf16) 17 us, 104 MB, 6.0 TB/s; norms 23 us;
// sort and part of the zeros 18 us; sum 22 us; join 5 us: the two calls 69 us, where
// reading G twice and writing the table once takes 42.
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

// Inclusive sum over the lanes of a wave: shifts within rows of 16 lanes, then
// the rows' last lanes to the rows after them (six adds, no LDS).
__device__ __forceinline__ int32_t wave_scan(int32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast 31
  return x;
}

// What one lane has written to LDS, the others of its wave read after this (a
// wave's LDS accesses are done in order: this holds the compiler to it).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------- sorting

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortBuckets = 256;    // one workgroup a bucket, one round on the chip
constexpr int kMaxKeysPerWg = 512;   // LDS: kSortWaves counters a key
constexpr int kSortList = 384;       // matches that a wave keeps in LDS
constexpr int kSortBatch = 8;        // loads that a lane has in flight

// Order of the keys [0, n) in a sorted list: by the low bits first (the bucket),
// then by the others. Frequent words have small ids, so neighbouring ids go to
// different buckets. slot() is a key's place among all, and the index of its
// first entry in `offsets`.
struct Buckets {
  uint32_t n, R;   // keys, keys of a bucket
  int32_t log;     // log2 of the number of buckets
  __host__ __device__ uint32_t slot(uint32_t key) const {
    return (key & ((1u << log) - 1u)) * R + (key >> log);
  }
  int64_t slots() const { return (int64_t)R << log; }
};

Buckets buckets_of(int64_t n_keys) {
  Buckets b{(uint32_t)n_keys, 1, 0};
  while ((INT64_C(1) << b.log) < n_keys &&
         ((1 << b.log) < kSortBuckets || n_keys > (int64_t)kMaxKeysPerWg << b.log))
    ++b.log;
  b.R = (uint32_t)ceil_div(n_keys, INT64_C(1) << b.log);
  return b;
}

// Keys of the list to sort; a key of n or more is left out. key(k) is for any
// k < count().
template <class Id>
struct TokenKey {   // key of position p: its token
  const Id* ids;
  int32_t n;
  __device__ int32_t count() const { return n; }
  __device__ __forceinline__ uint32_t key(int32_t k) const {
    if constexpr (sizeof(Id) == 8) {
      const uint2 v = reinterpret_cast<const uint2*>(ids)[k];
      return v.y ? 0xFFFFFFFFu : v.x;
    } else {
      return (uint32_t)ids[k];
    }
  }
  __device__ __forceinline__ int32_t value(int32_t k) const { return k; }
};

struct ExampleKey {   // key of entry k of a list of positions: its example
  const int32_t* order;
  const int32_t* end;   // entries of the list
  uint32_t magic;       // division by T
  int32_t shift;
  __device__ int32_t count() const { return *end; }
  __device__ __forceinline__ uint32_t key(int32_t k) const {
    return magic_divide((uint32_t)order[k], magic, shift);
  }
  __device__ __forceinline__ int32_t value(int32_t k) const { return order[k]; }
};

// Stable counting sort in one launch: workgroup w owns bucket w and reads the
// whole list. Its waves have one contiguous range of the list each. They count
// the entries of the smaller buckets, and keep their own bucket's in LDS, in
// list order (kSortList of them; a wave that finds more reads the rest of its
// range again). Key by key counts of those and a prefix over keys and waves
// give every wave its places. No entry's place depends on the order of an
// atomic (the counts are integers).
//
// The sort is bound by its instructions and leaves the memory idle: workgroups
// after the buckets' may fill `zeros` with zeros meanwhile.
template <class Key>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(Key keys, Buckets bk, int32_t* order,
                                                            int32_t* offsets, float* zeros,
                                                            int64_t n_zeros) {
  if (blockIdx.x >> bk.log) {
    const int64_t step = (int64_t)(gridDim.x - (1u << bk.log)) * kSortThreads;
    const int64_t first = (int64_t)(blockIdx.x - (1u << bk.log)) * kSortThreads + threadIdx.x;
    for (int64_t k = first; k < n_zeros >> 2; k += step)
      reinterpret_cast<f32x4_t*>(zeros)[k] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (first < (n_zeros & 3)) zeros[(n_zeros & ~INT64_C(3)) + first] = 0.0f;
    return;
  }
  extern __shared__ __align__(16) int32_t lds[];
  __shared__ uint2 kept_of[kSortWaves][kSortList];   // value, key within the bucket
  __shared__ int32_t less_of[kSortWaves];
  const uint32_t R = bk.R, w = blockIdx.x, mask = (1u << bk.log) - 1u;
  int32_t* table = lds;                       // [kSortWaves][R]
  int32_t* total = lds + kSortWaves * R;      // [R]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const uint64_t below = (UINT64_C(1) << lane) - 1;
  const int32_t N = keys.count();
  const int32_t groups = (N >> 6) + ((N & 63) != 0), per = (groups + kSortWaves - 1) / kSortWaves;
  // Groups of 64 entries of this wave, and the end of its entries.
  const int32_t first = per * wave < groups ? per * wave : groups;
  const int32_t last = first + per < groups ? first + per : groups;
  const int32_t end = last == groups ? N : last << 6;

  for (uint32_t k = threadIdx.x; k < kSortWaves * R; k += kSortThreads) table[k] = 0;
  uint2* list = kept_of[wave];
  int32_t less = 0, kept = 0;
  int32_t again = last;   // first group whose matches were not kept
  for (int32_t g = first; g < last; g += kSortBatch) {
    const int32_t k0 = (g << 6) + lane;
    uint32_t key[kSortBatch];
    if (g + kSortBatch <= last && (g + kSortBatch) << 6 <= end) {   // every entry is there
#pragma unroll
      for (int u = 0; u < kSortBatch; ++u) key[u] = keys.key(k0 + u * 64);
    } else {
#pragma unroll
      for (int u = 0; u < kSortBatch; ++u) {
        const int32_t k = k0 + u * 64;
        key[u] = keys.key(k < end ? k : end - 1);
        if (k >= end) key[u] = 0xFFFFFFFFu;
      }
    }
#pragma unroll
    for (int u = 0; u < kSortBatch; ++u) {
      const uint32_t b = key[u] < bk.n ? key[u] & mask : 0xFFFFFFFFu;
      less += b < w;
      const uint64_t hits = __ballot(b == w);
      if (hits && again == last) {
        const int32_t more = __popcll(hits);
        if (kept + more <= kSortList) {
          if (b == w) list[kept + __popcll(hits & below)] = make_uint2((uint32_t)keys.value(k0 + u * 64),
                                                                       key[u] >> bk.log);
          kept += more;
        } else {
          again = g + u;
        }
      }
    }
  }
  less = wave_scan(less);
  if (lane == 63) less_of[wave] = less;
  __syncthreads();
  for (int32_t k = lane; k < kept; k += 64) atomicAdd(&table[wave * R + list[k].y], 1);
  for (int32_t g = again; g < last; ++g) {
    const int32_t k = (g << 6) + lane;
    const uint32_t key = k < end ? keys.key(k) : 0xFFFFFFFFu;
    if (key < bk.n && (key & mask) == w) atomicAdd(&table[wave * R + (key >> bk.log)], 1);
  }
  __syncthreads();
  int32_t count[kSortWaves];   // of key threadIdx.x, wave by wave
  if (threadIdx.x < R) {
    int32_t t = 0;
#pragma unroll
    for (int v = 0; v < kSortWaves; ++v) t += count[v] = table[v * R + threadIdx.x];
    total[threadIdx.x] = t;
  }
  __syncthreads();
  if (wave == 0) {   // exclusive prefix of total[], 64 keys at a time
    int32_t run = __builtin_amdgcn_readlane(wave_scan(lane < kSortWaves ? less_of[lane] : 0), 63);
    for (uint32_t base = 0; base < R; base += 64) {
      const int32_t t = base + lane < R ? total[base + lane] : 0;
      const int32_t s = wave_scan(t);
      if (base + lane < R) total[base + lane] = run + s - t;
      run += __builtin_amdgcn_readlane(s, 63);
    }
    if (lane == 0 && w == mask) offsets[bk.R << bk.log] = run;
  }
  __syncthreads();
  if (threadIdx.x < R) {
    int32_t at = total[threadIdx.x];
    offsets[w * R + threadIdx.x] = at;
#pragma unroll
    for (int v = 0; v < kSortWaves; ++v) {
      table[v * R + threadIdx.x] = at;
      at += count[v];
    }
  }
  __syncthreads();
  // Places: lanes with the same key find each other bit by bit; the first of
  // them moves the wave's place of that key on.
  int32_t* place = table + wave * R;
  const auto put = [&](bool here, uint32_t m, int32_t value) {
    uint64_t same = __ballot(here);
    for (uint32_t bit = 1; bit < R; bit <<= 1) {
      const bool set = (m & bit) != 0;
      const uint64_t ones = __ballot(set);
      same &= set ? ones : ~ones;
    }
    if (here) {
      const int32_t at = place[m];
      order[at + __popcll(same & below)] = value;
      if ((same & below) == 0) place[m] = at + __popcll(same);
    }
    wave_fence();
  };
  for (int32_t base = 0; base < kept; base += 64) {
    const bool here = base + lane < kept;
    const uint2 e = list[here ? base + lane : 0];
    put(here, e.y, (int32_t)e.x);
  }
  for (int32_t g = again; g < last; ++g) {
    const int32_t k = (g << 6) + lane;
    const uint32_t key = k < end ? keys.key(k) : 0xFFFFFFFFu;
    const bool match = key < bk.n && (key & mask) == w;
    put(match, match ? key >> bk.log : 0, match ? keys.value(k) : 0);
  }
}

// Workgroups: the buckets', and those of the zeros (64 bytes a thread, at most a round).
int64_t sort_wgs(const Buckets& bk, int64_t n_zeros = 0) {
  const int64_t fill = ceil_div(n_zeros, 16 * kSortThreads);
  return (INT64_C(1) << bk.log) + (fill < kSortBuckets ? fill : kSortBuckets);
}

template <class Key>
int launch_sort(const Key& keys, const Buckets& bk, int32_t* order, int32_t* offsets,
                hipStream_t stream, float* zeros = nullptr, int64_t n_zeros = 0) {
  const size_t lds = (size_t)(kSortWaves + 1) * bk.R * sizeof(int32_t);
  hipLaunchKernelGGL(sort_kernel<Key>, dim3((uint32_t)sort_wgs(bk, n_zeros)), dim3(kSortThreads), lds,
                     stream, keys, bk, order, offsets, zeros, n_zeros);
  return check_launch();
}

// -------------------------------------------------------------------- lookup

struct LookupArgs {
  const void* ids;
  const void* table;
  void* out;
  int64_t N;
  int64_t V;
  int32_t d;
  int32_t wide;
  float scale;
};

__device__ __forceinline__ int64_t read_id(const void* ids, int wide, int64_t n) {
  return wide ? static_cast<const int64_t*>(ids)[n] : static_cast<const int32_t*>(ids)[n];
}

template <class TI, class TO, int V>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs a) {
  const int units = a.d / V;
  const int lane = threadIdx.x & 63;
  // Rows of fewer than 64 units share a wave.
  const int rows = units < 64 ? 64 / units : 1;
  const int sub = units < 64 ? lane / units : 0;
  const int u0 = units < 64 ? lane - sub * units : lane;
  if (sub >= rows) return;
  const int64_t waves = (int64_t)gridDim.x * (kThreads / 64);
  for (int64_t n = ((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * rows + sub; n < a.N;
       n += waves * rows) {
    const int64_t id = read_id(a.ids, a.wide, n);
    const bool there = (uint64_t)id < (uint64_t)a.V;
    const TI* src = static_cast<const TI*>(a.table) + (there ? id : 0) * a.d;
    TO* dst = static_cast<TO*>(a.out) + n * a.d;
    for (int u = u0; u < units; u += 64) {
      float x[V] = {};
      if (there) load_vec<V>(src + (int64_t)u * V, x);
#pragma unroll
      for (int k = 0; k < V; ++k) x[k] *= a.scale;
      store_vec<V>(dst + (int64_t)u * V, x);
    }
  }
}

template <class TI, class TO>
int launch_lookup_of(const LookupArgs& a, hipStream_t stream) {
  const int v = vec_width(a.d, 8);
  const int64_t units = a.d / v, rows = units < 64 ? 64 / units : 1;
  const int64_t wgs = ceil_div(ceil_div(a.N, rows), kThreads / 64);
  const dim3 grid((uint32_t)(wgs < 8192 ? wgs : 8192));
  switch (v) {
    case 8: hipLaunchKernelGGL((lookup_kernel<TI, TO, 8>), grid, dim3(kThreads), 0, stream, a); break;
    case 4: hipLaunchKernelGGL((lookup_kernel<TI, TO, 4>), grid, dim3(kThreads), 0, stream, a); break;
    case 2: hipLaunchKernelGGL((lookup_kernel<TI, TO, 2>), grid, dim3(kThreads), 0, stream, a); break;
    default: hipLaunchKernelGGL((lookup_kernel<TI, TO, 1>), grid, dim3(kThreads), 0, stream, a); break;
  }
  return check_launch();
}

// --------------------------------------------------------------------- norms

constexpr int kNormThreads = 1024;
constexpr int kNormWaves = kNormThreads / 64;
constexpr int kSortedInLds = 4096;   // longest example whose tokens are sorted in LDS
constexpr int kLdsGroups = kSortedInLds / kNormThreads;   // groups of 64 tokens of a wave
constexpr int kMostParts = 16;
constexpr int kRowBatch = 8;         // rows of G that a thread has in flight

struct NormArgs {
  const void* ids;
  const void* G;
  const int32_t* order;     // T > kSortedInLds: positions by example, token, position
  const int32_t* offsets;   // by example slot
  Buckets examples, tokens;
  float* partials;          // [B][wgs * blocks], or norms_sq itself where that is 1
  int32_t T, n_rows, d;
  int32_t wide, accumulate;
  int32_t wgs, blocks;      // workgroups and column blocks of an example
  int32_t units, parts;     // column vectors of a block, parts of a workgroup's entries
  int32_t digits;           // of 8 bits, of a token
  float scale;
};

// An example's entries by token, in LDS ...
struct LdsList {
  const uint32_t* id;
  const uint16_t* t;
  __device__ __forceinline__ uint32_t group(int32_t k) const { return id[k]; }
  __device__ __forceinline__ uint32_t row(int32_t k) const { return t[k]; }
};

// ... or its part of the list of all positions, groups in slot order.
struct GlobalList {
  const int32_t* order;
  const void* ids;
  Buckets tokens;
  int32_t first;   // position of the example's first token
  int32_t wide;
  __device__ uint32_t group(int32_t k) const {
    return tokens.slot((uint32_t)read_id(ids, wide, order[k]));
  }
  __device__ uint32_t row(int32_t k) const { return (uint32_t)(order[k] - first); }
};

// LDS of the sort: two buffers of tokens and of their places t, and the counters
// of the digits.
struct SortLds {
  uint32_t* id;      // [2][padded]
  uint16_t* t;       // [2][padded]
  uint32_t* count;   // [kNormWaves][256]
  uint32_t* sums;    // [4]
  int padded;
};

// Sorts the tokens of one example by (token, t), digit by digit, and returns how
// many there are (empty positions are dropped); they end up in buffer
// digits & 1. Every wave has a contiguous range of the list. Lanes with the same
// digit find each other with eight ballots; the first of them adds their number
// to the wave's counter, so a pass is stable and needs no atomics.
__device__ __forceinline__ int32_t sort_example(const NormArgs& a, int64_t first, const SortLds& l) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const uint64_t below = (UINT64_C(1) << lane) - 1;
  int32_t n = a.T;
  for (int digit = 0; digit < a.digits; ++digit) {
    const int from = digit & 1 ? l.padded : 0, to = l.padded - from;
    for (int k = threadIdx.x; k < kNormWaves * 256; k += kNormThreads) l.count[k] = 0;
    __syncthreads();
    const int32_t groups = (n + 63) >> 6, per = (groups + kNormWaves - 1) / kNormWaves;
    uint32_t id[kLdsGroups], at[kLdsGroups], t[kLdsGroups];   // at: digit | rank << 8, ~0: none
    uint32_t* mine = l.count + wave * 256;
#pragma unroll
    for (int u = 0; u < kLdsGroups; ++u) {
      at[u] = ~0u;
      if (u >= per) continue;
      const int32_t k = ((wave * per + u) << 6) + lane;
      bool there = k < n;
      id[u] = 0;
      if (there) {
        if (digit == 0) {
          const int64_t v = read_id(a.ids, a.wide, first + k);
          there = (uint64_t)v < (uint64_t)a.n_rows;
          id[u] = (uint32_t)v;
          t[u] = (uint32_t)k;
        } else {
          id[u] = l.id[from + k];
          t[u] = l.t[from + k];
        }
      }
      const uint32_t d = (id[u] >> (8 * digit)) & 255u;
      uint64_t same = __ballot(there);
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const bool set = d >> b & 1;
        const uint64_t ones = __ballot(set);
        same &= set ? ones : ~ones;
      }
      if (there) {
        const uint32_t before = mine[d];
        at[u] = d | (before + (uint32_t)__popcll(same & below)) << 8;
        if ((same & below) == 0) mine[d] = before + (uint32_t)__popcll(same);
      }
      wave_fence();
    }
    __syncthreads();
    uint32_t count[kNormWaves], total = 0, scan = 0;   // of digit threadIdx.x, wave by wave
    if (threadIdx.x < 256) {
#pragma unroll
      for (int w = 0; w < kNormWaves; ++w) total += count[w] = l.count[w * 256 + threadIdx.x];
      scan = (uint32_t)wave_scan((int32_t)total);
      if (lane == 63) l.sums[wave] = scan;
    }
    __syncthreads();
    if (threadIdx.x < 256) {
      uint32_t place = scan - total;
      for (int w = 0; w < wave; ++w) place += l.sums[w];
#pragma unroll
      for (int w = 0; w < kNormWaves; ++w) {
        l.count[w * 256 + threadIdx.x] = place;
        place += count[w];
      }
    }
    n = (int32_t)(l.sums[0] + l.sums[1] + l.sums[2] + l.sums[3]);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kLdsGroups; ++u) {
      if (at[u] == ~0u) continue;
      const uint32_t place = l.count[wave * 256 + (at[u] & 255u)] + (at[u] >> 8);
      l.id[to + place] = id[u];
      l.t[to + place] = (uint16_t)t[u];
    }
    __syncthreads();
  }
  return n;
}

// First entry at or after s (of n) that begins a group.
template <class List>
__device__ __forceinline__ int32_t group_start(const List& list, int32_t n, int32_t s) {
  if (s <= 0 || s >= n) return s <= 0 ? 0 : n;
  const uint32_t g = list.group(s - 1);
  if (list.group(s) != g) return s;
  int32_t lo = s, hi = n;   // lo is of group g, hi is not
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (list.group(mid) == g) lo = mid; else hi = mid;
  }
  return hi;
}

// Sum of squares of the group sums of the groups that start in one workgroup's
// share of an example's list. A thread owns V columns and one part of the
// share; parts are cut without regard to groups (one token may be most of an
// example), so a part hands on the sum of its first and of its last group, and
// part 0's threads join those in order.
template <class T, int V, class List>
__device__ __forceinline__ float group_squares(const NormArgs& a, const List& list, int32_t n,
                                               int wg, int blk, const T* G, float* edges) {
  const int part = threadIdx.x / a.units, u = threadIdx.x - part * a.units;
  const int col = (blk * a.units + u) * V;
  const bool mine = part < a.parts && col < a.d;
  const int32_t of_wg = (n + a.wgs - 1) / a.wgs;
  const int32_t S = a.wgs == 1 ? 0 : group_start(list, n, of_wg * wg < n ? of_wg * wg : n);
  const int32_t E = a.wgs == 1 || n - of_wg * wg <= of_wg ? n : group_start(list, n, of_wg * (wg + 1));
  const int32_t of_part = (E - S + a.parts - 1) / a.parts;
  const auto cut = [&](int q) { return E - S - q * of_part < 0 ? E : S + q * of_part; };
  float ss = 0.0f;
  if (mine) {
    const int32_t s = cut(part), e = cut(part + 1);
    float acc[V] = {};
    float* head = edges + (part * a.units + u) * V;
    float* tail = head + a.parts * a.units * V;
    bool first = true;
    uint32_t last = s < e ? list.group(s) : 0;
    // Two batches in turn: one is loaded while the other is added.
    constexpr int kHalf = kRowBatch / 2;
    Raw<T, V> raw[2][kHalf];
    uint32_t g[2][kHalf];
    const auto load = [&](int b, int32_t k0) {
#pragma unroll
      for (int k = 0; k < kHalf; ++k) {
        const int32_t at = k0 + k < e ? k0 + k : e - 1;
        g[b][k] = list.group(at);
        raw[b][k].load(G + (int64_t)list.row(at) * a.d + col);
      }
    };
    const auto add = [&](int b, int32_t k0) {
#pragma unroll
      for (int k = 0; k < kHalf; ++k) {
        if (k0 + k >= e) break;
        float x[V];
        raw[b][k].widen(x);
        if (g[b][k] != last) {
          if (first) {
            store_vec<V>(head, acc);
            first = false;
          } else {
#pragma unroll
            for (int c = 0; c < V; ++c) ss = fmaf(acc[c], acc[c], ss);
          }
#pragma unroll
          for (int c = 0; c < V; ++c) acc[c] = x[c];
          last = g[b][k];
        } else {
#pragma unroll
          for (int c = 0; c < V; ++c) acc[c] += x[c];
        }
      }
    };
    if (s < e) load(0, s);
    for (int32_t k0 = s; k0 < e; k0 += kRowBatch) {
      if (k0 + kHalf < e) load(1, k0 + kHalf);
      add(0, k0);
      if (k0 + kRowBatch < e) load(0, k0 + kRowBatch);
      add(1, k0 + kHalf);
    }
    store_vec<V>(first ? head : tail, acc);
  }
  __syncthreads();
  if (threadIdx.x / 64 * 64 >= a.units) return ss;   // waves without a thread of part 0
  // Bit q: part q has entries; its first group began in the part before; all of
  // its entries are of one group.
  const int q = threadIdx.x & 63;
  const int32_t qs = cut(q < a.parts ? q : 0), qe = cut(q < a.parts ? q + 1 : 1);
  const bool any = q < a.parts && qs < qe;
  const uint64_t there = __ballot(any);
  const uint64_t goes_on = __ballot(any && qs > S && list.group(qs) == list.group(qs - 1));
  const uint64_t single = __ballot(any && list.group(qs) == list.group(qe - 1));
  if (mine && part == 0 && there) {
    float acc[V] = {};
    const int n_parts = 64 - __clzll((long long)there);   // parts with entries come first
#pragma unroll 4
    for (int p = 0; p < n_parts; ++p) {
      float x[V], y[V];   // y is not written where the part is of one group
      load_vec<V>(edges + (p * a.units + u) * V, x);
      load_vec<V>(edges + ((a.parts + p) * a.units + u) * V, y);
      if (!(goes_on >> p & 1)) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          ss = fmaf(acc[c], acc[c], ss);
          acc[c] = 0.0f;
        }
      }
#pragma unroll
      for (int c = 0; c < V; ++c) acc[c] += x[c];
      if (!(single >> p & 1)) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          ss = fmaf(acc[c], acc[c], ss);
          acc[c] = y[c];
        }
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) ss = fmaf(acc[c], acc[c], ss);
  }
  return ss;
}

// Bytes of LDS for the sort of an example of T tokens.
__host__ __device__ inline int sort_lds_bytes(int T) {
  const int padded = (T + 7) & ~7;
  return padded * 12 + kNormWaves * 256 * 4 + 16;
}

template <class T, int V, bool IN_LDS>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(NormArgs a) {
  extern __shared__ __align__(16) char norm_lds[];
  __shared__ float red[kNormWaves];
  const uint32_t per = (uint32_t)(a.wgs * a.blocks);
  const uint32_t i = blockIdx.x / per, rest = blockIdx.x - i * per;
  const int wg = (int)(rest / (uint32_t)a.blocks), blk = (int)rest - wg * a.blocks;
  const T* G = static_cast<const T*>(a.G) + (int64_t)i * a.T * a.d;
  float ss;
  if constexpr (IN_LDS) {
    SortLds l;
    l.padded = (a.T + 7) & ~7;
    l.count = reinterpret_cast<uint32_t*>(norm_lds);
    l.sums = l.count + kNormWaves * 256;
    l.id = l.sums + 4;
    l.t = reinterpret_cast<uint16_t*>(l.id + 2 * l.padded);
    const int32_t n = sort_example(a, (int64_t)i * a.T, l);
    const int at = a.digits & 1 ? l.padded : 0;
    ss = group_squares<T, V>(a, LdsList{l.id + at, l.t + at}, n, wg, blk, G,
                             reinterpret_cast<float*>(norm_lds + sort_lds_bytes(a.T)));
  } else {
    const uint32_t slot = a.examples.slot(i);
    const int32_t s = a.offsets[slot], n = a.offsets[slot + 1] - s;
    ss = group_squares<T, V>(a, GlobalList{a.order + s, a.ids, a.tokens, (int32_t)i * a.T, a.wide}, n, wg,
                             blk, G, reinterpret_cast<float*>(norm_lds));
  }
  ss = wave_sum(ss);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0) {
    float t = 0.0f;
    for (int k = 0; k < kNormWaves; ++k) t += red[k];
    // The square of the scale may be outside float32 where the norm is not.
    t = (float)((double)t * ((double)a.scale * (double)a.scale));
    a.partials[blockIdx.x] = a.accumulate ? a.partials[blockIdx.x] + t : t;
  }
}

// --------------------------------------------------------------- clipped sum

constexpr int kChunk = 32;         // entries of a chunk (one a lane, and one on each side)
constexpr int kRowsPerWave = 16;   // table rows that a wave looks through for empty ones
constexpr int kJoinThreads = 512;

struct SumArgs {
  const void* ids;
  const void* G;
  const int32_t* order;     // positions by token, position
  const int32_t* offsets;   // by token slot
  const float* norms_sq;    // [B], NULL: all factors 1
  float* grad;
  float* partials;          // [chunks][2][d]
  float* factors_out;
  uint8_t* mask_out;
  Buckets tokens;
  int64_t rows, B;   // rows that this launch fills where they have no token
  // Workgroups of the chunks, then of the empty rows, then of the factors.
  uint32_t chunk_wgs, row_wgs;
  int32_t chunks, blocks;   // chunks of the sorted list, column blocks of a row
  int32_t d, accumulate, wide;
  uint32_t magic;           // division by T
  int32_t shift;
  float scale, C;
};

template <int V>
__device__ __forceinline__ void write_row(const SumArgs& a, int64_t v, int col, float (&acc)[V]) {
  float* out = a.grad + v * a.d + col;
  if (a.accumulate) {
    float old[V];
    load_vec<V>(out, old);
#pragma unroll
    for (int c = 0; c < V; ++c) acc[c] = fmaf(a.scale, acc[c], old[c]);
  } else {
#pragma unroll
    for (int c = 0; c < V; ++c) acc[c] *= a.scale;
  }
  store_vec<V>(out, acc);
}

// One chunk of the sorted list and one block of 64 V columns. Lane l holds entry
// s - 1 + l: its position, token and factor. A token's sum goes to its row of
// grad if all of its entries are in the chunk, to partial row 0 of the chunk if
// entries of it come before, and to partial row 1 otherwise.
template <class T, int V>
__device__ __forceinline__ void sum_chunk(const SumArgs& a, int32_t q, int blk) {
  const int lane = threadIdx.x & 63;
  const int32_t total = a.offsets[a.tokens.R << a.tokens.log];
  const int32_t s = q * kChunk;
  if (s >= total) return;
  const int32_t n = total - s < kChunk ? total - s : kChunk;
  const int32_t k = s - 1 + lane;
  int32_t p = 0, token = -1;
  float f = 0.0f;
  if (lane <= n + 1 && k >= 0 && k < total) {
    p = a.order[k];
    token = (int32_t)read_id(a.ids, a.wide, p);
    f = 1.0f;
    if (a.norms_sq) f = clip_factor(a.norms_sq[magic_divide((uint32_t)p, a.magic, a.shift)], a.C);
  }
  const int32_t before = __shfl_up(token, 1, 64);
  const uint64_t starts = __ballot(lane == 0 || token != before);
  const int col = (blk * 64 + lane) * V;
  const bool mine = col < a.d;
  const T* G = static_cast<const T*>(a.G) + col;
  float acc[V] = {};
  bool open = !(starts >> 1 & 1);   // the sum at hand began in an earlier chunk
  const auto flush = [&](int last, bool more) {   // `last`: lane of its last entry
    const int32_t v = __builtin_amdgcn_readlane(token, last);
    if (mine) {
      if (!open && !more)
        write_row<V>(a, v, col, acc);
      else
        store_vec<V>(a.partials + ((int64_t)q * 2 + (open ? 0 : 1)) * a.d + col, acc);
    }
    open = false;
#pragma unroll
    for (int c = 0; c < V; ++c) acc[c] = 0.0f;
  };
  for (int j0 = 1; j0 <= n; j0 += kRowBatch) {
    Raw<T, V> raw[kRowBatch];
    float fj[kRowBatch];
#pragma unroll
    for (int j = 0; j < kRowBatch; ++j) {
      // An example of factor 0 is not read.
      fj[j] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), j0 + j));
      const int32_t pj = __builtin_amdgcn_readlane(p, j0 + j);
      raw[j].zero();
      if (mine && j0 + j <= n && fj[j] != 0.0f) raw[j].load(G + (int64_t)pj * a.d);
    }
#pragma unroll
    for (int j = 0; j < kRowBatch; ++j) {
      if (j0 + j > n) break;
      if (j0 + j > 1 && (starts >> (j0 + j) & 1)) flush(j0 + j - 1, false);
      float x[V];
      raw[j].widen(x);
#pragma unroll
      for (int c = 0; c < V; ++c) acc[c] = fmaf(fj[j], x[c], acc[c]);
    }
  }
  flush(n, !(starts >> (n + 1) & 1));
}

template <class T, int V>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t wg = blockIdx.x;
  if (wg < a.chunk_wgs) {
    const uint32_t job = wg * (kThreads / 64) + wave, q = job / (uint32_t)a.blocks;
    if (q < (uint32_t)a.chunks) sum_chunk<T, V>(a, (int32_t)q, (int)(job - q * a.blocks));
    return;
  }
  wg -= a.chunk_wgs;
  if (wg >= a.row_wgs) {   // the factors and the mask, where they are asked for
    const int64_t i = (int64_t)(wg - a.row_wgs) * kThreads + threadIdx.x;
    if (i < a.B) write_factor(a.norms_sq[i], a.C, i, nullptr, a.factors_out, a.mask_out);
    return;
  }
  // Rows without a token.
  const int64_t v0 = ((int64_t)wg * (kThreads / 64) + wave) * kRowsPerWave;
  bool empty = false;
  if (lane < kRowsPerWave && v0 + lane < a.rows) {
    const uint32_t slot = a.tokens.slot((uint32_t)(v0 + lane));
    empty = a.offsets[slot] == a.offsets[slot + 1];
  }
  float zero[V] = {};
  for (uint64_t left = __ballot(empty); left; left &= left - 1) {
    float* row = a.grad + (v0 + __ffsll((unsigned long long)left) - 1) * a.d;
    for (int col = lane * V; col < a.d; col += 64 * V) store_vec<V>(row + col, zero);
  }
}

// Joins the partial rows of the token that begins in chunk q and goes on after
// it, if there is one: row 1 of chunk q, rows 0 of the chunks after it. Each wave
// adds a range of them in order, then wave 0 the waves' sums.
template <int V>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(SumArgs a) {
  __shared__ float sums[kJoinThreads / 64][64 * V];
  const int32_t q = blockIdx.x;
  const int32_t total = a.offsets[a.tokens.R << a.tokens.log];
  const int32_t s = q * kChunk;
  if (total - s <= kChunk) return;   // nothing comes after this chunk
  const int32_t token = (int32_t)read_id(a.ids, a.wide, a.order[s + kChunk - 1]);
  const uint32_t slot = a.tokens.slot((uint32_t)token);
  const int32_t begin = a.offsets[slot], end = a.offsets[slot + 1];
  if (begin < s || end <= s + kChunk) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = ((int)blockIdx.y * 64 + lane) * V;
  const int32_t n = (end - 1) / kChunk - q + 1;   // partial rows
  const int32_t per = (n + kJoinThreads / 64 - 1) / (kJoinThreads / 64);
  const int32_t from = wave * per, to = from + per < n ? from + per : n;
  float acc[V] = {};
  if (col < a.d) {
#pragma unroll 4
    for (int32_t k = from; k < to; ++k) {
      float x[V];
      load_vec<V>(a.partials + ((int64_t)(q + k) * 2 + (k == 0 ? 1 : 0)) * a.d + col, x);
#pragma unroll
      for (int c = 0; c < V; ++c) acc[c] += x[c];
    }
  }
#pragma unroll
  for (int c = 0; c < V; ++c) sums[wave][c * 64 + lane] = acc[c];
  __syncthreads();
  if (wave == 0 && col < a.d) {
    for (int w = 1; w < kJoinThreads / 64 && w * per < n; ++w)
#pragma unroll
      for (int c = 0; c < V; ++c) acc[c] += sums[w][c * 64 + lane];
    write_row<V>(a, token, col, acc);
  }
}

// Chunks of the sorted list.
int64_t chunk_count(int64_t N) { return ceil_div(N, kChunk); }

// Split of the norms' work: column vectors over the threads of `blocks` blocks,
// what is left of a workgroup over `parts` parts of its entries (at least 8
// each), and, for few examples, several workgroups an example, so that about 256
// run. From 96 examples on one workgroup each, and no launch to add up partial
// sums: at 128 examples two workgroups each and that launch took no less time.
// Up to 160 CUs are idle then (128 x 256 tokens at 768 in bf16, 50 MB: 16.7 us
// with clean caches, 3.0 TB/s).
struct NormPlan {
  int vec, blocks, units, parts, wgs;
  bool in_lds;
};

NormPlan norm_plan(const dpsgd_embedding& e, int32_t dtype) {
  NormPlan p;
  p.vec = vec_width(e.d, dtype == DPSGD_BF16 ? 8 : 4);
  const int64_t units = e.d / p.vec;
  p.blocks = (int)ceil_div(units, kNormThreads);
  p.units = (int)ceil_div(units, p.blocks);
  int64_t parts = kNormThreads / p.units;
  if (parts > kMostParts) parts = kMostParts;
  if (parts > ceil_div(e.T, 8)) parts = ceil_div(e.T, 8);
  p.parts = (int)parts;
  int64_t wgs = e.B * p.blocks >= 96 ? 1 : ceil_div(256, e.B * p.blocks);
  const int64_t most = ceil_div(e.T, 8 * parts);
  p.wgs = (int)(wgs < most ? wgs : most);
  p.in_lds = e.T <= kSortedInLds;
  return p;
}

size_t order_bytes(int64_t N) { return round_up((size_t)N * sizeof(int32_t), 256); }
size_t list_bytes(int64_t N, const Buckets& b) {
  return order_bytes(N) + round_up((size_t)(b.slots() + 1) * sizeof(int32_t), 256);
}

int sort_tokens(const dpsgd_embedding& e, const Buckets& b, int32_t* order, int32_t* offsets,
                hipStream_t stream, float* zeros = nullptr, int64_t n_zeros = 0) {
  if (e.index_dtype == DPSGD_I64)
    return launch_sort(TokenKey<int64_t>{static_cast<const int64_t*>(e.ids), (int32_t)(e.B * e.T)}, b, order, offsets,
                       stream, zeros, n_zeros);
  return launch_sort(TokenKey<int32_t>{static_cast<const int32_t*>(e.ids), (int32_t)(e.B * e.T)}, b, order, offsets,
                     stream, zeros, n_zeros);
}

template <class T, int V>
void launch_norm_kernel(const NormPlan& p, const NormArgs& a, uint32_t wgs, hipStream_t stream) {
  const size_t edges = 2 * (size_t)p.parts * p.units * V * sizeof(float);
  if (p.in_lds)
    hipLaunchKernelGGL((norm_kernel<T, V, true>), dim3(wgs), dim3(kNormThreads),
                       (size_t)sort_lds_bytes(a.T) + edges, stream, a);
  else
    hipLaunchKernelGGL((norm_kernel<T, V, false>), dim3(wgs), dim3(kNormThreads), edges, stream, a);
}

}  // namespace

// Workspace: the list by token (order, offsets); then, for the norms, the list by
// example (T > kSortedInLds) and the partial sums, or, for the sum, the chunks'
// partial rows.
size_t embedding_workspace_bytes(const dpsgd_embedding& e) {
  const int64_t N = e.B * e.T;
  size_t partials = 0;
  for (int32_t dtype : {DPSGD_F32, DPSGD_BF16}) {
    const NormPlan p = norm_plan(e, dtype);
    const size_t n = (size_t)(e.B * p.wgs * p.blocks) * sizeof(float);
    partials = n > partials ? n : partials;
  }
  const size_t norms = (e.T > kSortedInLds ? list_bytes(N, buckets_of(e.B)) : 0) + partials;
  const size_t sum = (size_t)chunk_count(N) * 2 * (size_t)e.d * sizeof(float);
  return list_bytes(N, buckets_of(e.n_rows)) + (norms > sum ? norms : sum);
}

int launch_embedding_lookup(const dpsgd_embedding& e, const void* table, int32_t table_dtype,
                            void* out, int32_t out_dtype, hipStream_t stream) {
  const LookupArgs a{e.ids, table, out, e.B * e.T, e.n_rows, (int32_t)e.d,
                     e.index_dtype == DPSGD_I64, e.scale};
  const bool bi = table_dtype == DPSGD_BF16, bo = out_dtype == DPSGD_BF16;
  if (bi) return bo ? launch_lookup_of<uint16_t, uint16_t>(a, stream) : launch_lookup_of<uint16_t, float>(a, stream);
  return bo ? launch_lookup_of<float, uint16_t>(a, stream) : launch_lookup_of<float, float>(a, stream);
}

int launch_embedding_norms(const dpsgd_embedding& e, const void* G, int32_t dtype, float* norms_sq,
                           int accumulate, void* workspace, hipStream_t stream) {
  const int64_t N = e.B * e.T;
  const NormPlan p = norm_plan(e, dtype);
  const int64_t wgs = e.B * p.wgs * p.blocks;
  // Launches that cannot be made are refused before the first.
  if (!launchable(wgs, kNormThreads)) return DPSGD_ERR_INVALID_ARG;
  if (!p.in_lds && !(launchable(sort_wgs(buckets_of(e.n_rows)), kSortThreads) &&
                     launchable(sort_wgs(buckets_of(e.B)), kSortThreads)))
    return DPSGD_ERR_INVALID_ARG;
  NormArgs a{};
  a.ids = e.ids;
  a.G = G;
  a.T = (int32_t)e.T;
  a.n_rows = (int32_t)e.n_rows;
  a.digits = 1;
  while (a.digits < 4 && (e.n_rows - 1) >> (8 * a.digits)) ++a.digits;
  a.d = (int32_t)e.d;
  a.wide = e.index_dtype == DPSGD_I64;
  a.wgs = p.wgs;
  a.blocks = p.blocks;
  a.units = p.units;
  a.parts = p.parts;
  a.scale = e.scale;
  a.tokens = buckets_of(e.n_rows);
  char* ws = static_cast<char*>(workspace);
  char* partials = ws + list_bytes(N, a.tokens);
  int st = DPSGD_OK;
  if (!p.in_lds) {
    int32_t* order = reinterpret_cast<int32_t*>(ws);
    int32_t* offsets = reinterpret_cast<int32_t*>(ws + order_bytes(N));
    a.examples = buckets_of(e.B);
    int32_t* by_example = reinterpret_cast<int32_t*>(partials);
    int32_t* starts = reinterpret_cast<int32_t*>(partials + order_bytes(N));
    partials += list_bytes(N, a.examples);
    st = sort_tokens(e, a.tokens, order, offsets, stream);
    if (st != DPSGD_OK) return st;
    ExampleKey ex{order, offsets + a.tokens.slots(), 0, 0};
    divide_magic(e.T, &ex.magic, &ex.shift);
    st = launch_sort(ex, a.examples, by_example, starts, stream);
    if (st != DPSGD_OK) return st;
    a.order = by_example;
    a.offsets = starts;
  }
  const bool whole = p.wgs * p.blocks == 1;   // one workgroup an example: no partial sums
  a.partials = whole ? norms_sq : reinterpret_cast<float*>(partials);
  a.accumulate = whole && accumulate;
  const uint32_t w = (uint32_t)wgs;
  if (dtype == DPSGD_BF16) {
    switch (p.vec) {
      case 8: launch_norm_kernel<uint16_t, 8>(p, a, w, stream); break;
      case 4: launch_norm_kernel<uint16_t, 4>(p, a, w, stream); break;
      case 2: launch_norm_kernel<uint16_t, 2>(p, a, w, stream); break;
      default: launch_norm_kernel<uint16_t, 1>(p, a, w, stream); break;
    }
  } else {
    switch (p.vec) {
      case 4: launch_norm_kernel<float, 4>(p, a, w, stream); break;
      case 2: launch_norm_kernel<float, 2>(p, a, w, stream); break;
      default: launch_norm_kernel<float, 1>(p, a, w, stream); break;
    }
  }
  st = check_launch();
  if (st != DPSGD_OK || whole) return st;
  return launch_norms_reduce(a.partials, (int64_t)p.wgs * p.blocks, e.B, norms_sq, accumulate, stream);
}

int launch_embedding_sum(const dpsgd_embedding& e, const void* G, int32_t dtype,
                         const float* norms_sq, float C, float* grad, int accumulate,
                         float* factors_out, uint8_t* mask_out, void* workspace,
                         hipStream_t stream) {
  const int64_t N = e.B * e.T;
  char* ws = static_cast<char*>(workspace);
  SumArgs a{};
  a.tokens = buckets_of(e.n_rows);
  int32_t* order = reinterpret_cast<int32_t*>(ws);
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + order_bytes(N));
  // Rows from `filled` on are zeroed beside the sort, about as many as the memory
  // takes meanwhile (at 6 TB/s; the sort takes 5 us and 0.3 ns an entry), and
  // those with a token are written again. They are the last ones, as frequent
  // words have small ids. (50257 x 768, 32768 tokens: norms and sum 68.7 us, 73.7
  // with every empty row filled by the sum.)
  const int64_t fill_rows = accumulate ? 0 : ((INT64_C(30) << 20) + 1800 * N) / (e.d * (int64_t)sizeof(float));
  const int64_t filled = fill_rows < e.n_rows ? round_up((size_t)(e.n_rows - fill_rows), 4) : 0;
  const bool fill = !accumulate && filled < e.n_rows;
  a.ids = e.ids;
  a.G = G;
  a.order = order;
  a.offsets = offsets;
  a.norms_sq = norms_sq;
  a.grad = grad;
  a.partials = reinterpret_cast<float*>(ws + list_bytes(N, a.tokens));
  a.factors_out = factors_out;
  a.mask_out = mask_out;
  a.rows = accumulate ? 0 : fill ? filled : e.n_rows;
  a.B = e.B;
  a.d = (int32_t)e.d;
  a.accumulate = accumulate;
  a.wide = e.index_dtype == DPSGD_I64;
  a.scale = e.scale;
  a.C = C;
  divide_magic(e.T, &a.magic, &a.shift);
  const int vec = vec_width(e.d, 4);
  a.chunks = (int32_t)chunk_count(N);
  a.blocks = (int32_t)ceil_div(e.d, 64 * vec);
  const int64_t chunk_wgs = ceil_div((int64_t)a.chunks * a.blocks, kThreads / 64);
  const int64_t row_wgs = ceil_div(a.rows, kThreads / 64 * kRowsPerWave);
  const int64_t wgs = chunk_wgs + row_wgs + (factors_out || mask_out ? ceil_div(e.B, kThreads) : 0);
  a.chunk_wgs = (uint32_t)chunk_wgs;
  a.row_wgs = (uint32_t)row_wgs;
  const int64_t n_zeros = fill ? (e.n_rows - filled) * e.d : 0;
  // Launches that cannot be made are refused before the first.
  if (!launchable(sort_wgs(a.tokens, n_zeros), kSortThreads) || !launchable(wgs, kThreads) ||
      !launchable(a.chunks, kJoinThreads))
    return DPSGD_ERR_INVALID_ARG;
  const int st = sort_tokens(e, a.tokens, order, offsets, stream, fill ? grad + filled * e.d : nullptr, n_zeros);
  if (st != DPSGD_OK) return st;
  const dim3 grid((uint32_t)wgs), block(kThreads), jgrid((uint32_t)a.chunks, (uint32_t)a.blocks);
#define DPSGD_SUM(V)                                                                                \
  if (dtype == DPSGD_BF16) {                                                                        \
    hipLaunchKernelGGL((sum_kernel<uint16_t, V>), grid, block, 0, stream, a);                       \
  } else {                                                                                          \
    hipLaunchKernelGGL((sum_kernel<float, V>), grid, block, 0, stream, a);                          \
  }                                                                                                 \
  if (a.chunks > 1) hipLaunchKernelGGL(join_kernel<V>, jgrid, dim3(kJoinThreads), 0, stream, a);
  switch (vec) {
    case 4: DPSGD_SUM(4) break;
    case 2: DPSGD_SUM(2) break;
    default: DPSGD_SUM(1) break;
  }
#undef DPSGD_SUM
  return check_launch();
}

}  // namespace dpsgd
