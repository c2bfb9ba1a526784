// Token tables (embeddings): lookup, per-example gradient norms, clipped sum.
//
//   lookup    out[n, :]  = scale * W[id_n, :]
//   norms     n2_i      += scale^2 sum_v || sum_{t: id_it = v} G[i, t, :] ||^2
//   sum       grad[v, :] = scale * sum_i c_i sum_{t: id_it = v} G[i, t, :]
//
// An id outside [0, V) is an empty position: a row of zeros out, and a row of G
// that is never read.
//
// The gradient is formed by sorted tokens, without floating-point atomics: a
// counting sort gives the positions of every token in ascending order
// (order, and offsets[v] into it), one wave sums the rows of one table row in
// that order, and rows with more than `chunk` positions are summed in chunks of
// the sorted list that a last pass joins in order. For the norms the list is
// sorted once more by example, so that equal tokens of an example are
// neighbours: a lane adds rows until the token changes, then adds the square of
// its sum, and the cross-lane sum is taken once at the end.
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

// ------------------------------------------------------------------- sorting

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxKeysPerWg = 512;   // LDS: kSortWaves counters a key

// Keys of the list to sort; a key outside [0, n_keys) is left out.
struct TokenKey {   // key of position p: its token
  const void* ids;
  int32_t wide;     // int64 ids
  uint32_t n_keys;
  int64_t n;
  __device__ int64_t count() const { return n; }
  __device__ uint32_t key(int64_t k) const {
    if (wide) {
      const uint64_t v = static_cast<const uint64_t*>(ids)[k];
      return v < n_keys ? (uint32_t)v : 0xFFFFFFFFu;
    }
    return static_cast<const uint32_t*>(ids)[k];
  }
  __device__ int32_t value(int64_t k) const { return (int32_t)k; }
};

struct ExampleKey {   // key of entry k of a list of positions: its example
  const int32_t* order;
  const int32_t* end;   // entries of the list
  uint32_t magic;       // division by T
  int32_t shift;
  uint32_t n_keys;
  __device__ int64_t count() const { return *end; }
  __device__ uint32_t key(int64_t k) const { return magic_divide((uint32_t)order[k], magic, shift); }
  __device__ int32_t value(int64_t k) const { return order[k]; }
};

// Stable counting sort in one launch: workgroup w owns the keys [w R, (w + 1) R)
// and reads the whole list twice. The first pass counts, wave by wave (each wave
// has one contiguous range of the list), its own keys and the entries with a
// smaller key; a prefix over keys and waves then gives every wave its place, and
// the second pass writes the entries there in list order. No entry depends on
// the order of an atomic (the counts are integers).
template <class Key>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(Key keys, uint32_t R,
                                                            int32_t* order, int32_t* offsets) {
  extern __shared__ int32_t lds[];
  int32_t* table = lds;                       // [kSortWaves][R]
  int32_t* total = lds + kSortWaves * R;      // [R]
  int32_t* less_of = total + R;               // [kSortWaves]
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t lo = blockIdx.x * R;
  const uint32_t n_here = keys.n_keys - lo < R ? keys.n_keys - lo : R;
  const int64_t N = keys.count();
  const int64_t per = ((N + kSortThreads - 1) / kSortThreads) * 64;   // entries of a wave
  const int64_t begin = per * wave < N ? per * wave : N;
  const int64_t end = begin + per < N ? begin + per : N;

  for (uint32_t k = threadIdx.x; k < kSortWaves * R; k += kSortThreads) table[k] = 0;
  __syncthreads();
  int32_t less = 0;
  for (int64_t k = begin + lane; k < end; k += 64) {
    const uint32_t key = keys.key(k);
    if (key < lo) ++less;
    const uint32_t m = key - lo;
    if (key >= lo && m < n_here) atomicAdd(&table[wave * R + m], 1);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) less += __shfl_xor(less, off, 64);
  if (lane == 0) less_of[wave] = less;
  __syncthreads();
  if (threadIdx.x < R) {
    int32_t t = 0;
    for (int w = 0; w < kSortWaves; ++w) t += table[w * R + threadIdx.x];
    total[threadIdx.x] = t;
  }
  __syncthreads();
  if (threadIdx.x < 64) {   // exclusive prefix of total[], 64 keys at a time
    int32_t run = 0;
    for (int w = 0; w < kSortWaves; ++w) run += less_of[w];
    for (uint32_t base = 0; base < R; base += 64) {
      const int32_t t = base + lane < R ? total[base + lane] : 0;
      int32_t s = t;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int32_t u = __shfl_up(s, off, 64);
        if (lane >= off) s += u;
      }
      if (base + lane < R) total[base + lane] = run + s - t;
      run += __shfl(s, 63, 64);
    }
    if (lane == 0 && lo + n_here == keys.n_keys) offsets[keys.n_keys] = run;
  }
  __syncthreads();
  if (threadIdx.x < n_here) {
    int32_t at = total[threadIdx.x];
    offsets[lo + threadIdx.x] = at;
    for (int w = 0; w < kSortWaves; ++w) {
      const int32_t t = table[w * R + threadIdx.x];
      table[w * R + threadIdx.x] = at;
      at += t;
    }
  }
  __syncthreads();
  volatile int32_t* place = table + wave * R;   // written by one lane, read by the others of its wave
  for (int64_t base = begin; base < end; base += 64) {
    const int64_t k = base + lane;
    const uint32_t key = k < end ? keys.key(k) : 0xFFFFFFFFu;
    const uint32_t m = key - lo;
    uint64_t left = __ballot(key >= lo && m < n_here);
    while (left) {   // one round for each distinct key among the 64 entries
      const int first = __ffsll((unsigned long long)left) - 1;
      const uint32_t m0 = (uint32_t)__builtin_amdgcn_readlane((int)m, first);
      const uint64_t same = __ballot(m == m0) & left;
      const int32_t at = place[m0];
      if (same >> lane & 1) {
        const int rank = __popcll(same & ((UINT64_C(1) << lane) - 1));
        order[at + rank] = keys.value(k);
      }
      if (lane == first) place[m0] = at + __popcll(same);
      left &= ~same;
    }
  }
}

uint32_t keys_per_wg(int64_t n_keys) {
  const int64_t r = ceil_div(n_keys, 256);
  return (uint32_t)(r < kMaxKeysPerWg ? r : kMaxKeysPerWg);
}

template <class Key>
int launch_sort(const Key& keys, int32_t* order, int32_t* offsets, hipStream_t stream) {
  const uint32_t R = keys_per_wg(keys.n_keys);
  const size_t lds = ((size_t)(kSortWaves + 1) * R + kSortWaves) * sizeof(int32_t);
  hipLaunchKernelGGL(sort_kernel<Key>, dim3((uint32_t)ceil_div(keys.n_keys, R)), dim3(kSortThreads),
                     lds, stream, keys, R, order, offsets);
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

struct NormArgs {
  const void* ids;
  const void* G;
  const int32_t* order;     // positions by example, token, position
  const int32_t* offsets;   // [B + 1]
  float* partials;          // [B][parts * blocks]
  int64_t jobs;             // B * parts * blocks
  int32_t d, wide, parts, blocks;
  float scale;
};

// First entry at or after s (of n) whose token differs from the entry before it.
__device__ __forceinline__ int32_t group_start(const NormArgs& a, const int32_t* list, int32_t n,
                                               int32_t s) {
  const int lane = threadIdx.x & 63;
  if (s <= 0) return 0;
  for (; s < n; s += 64) {
    const int32_t k = s + lane;
    const bool starts = k < n && read_id(a.ids, a.wide, list[k]) != read_id(a.ids, a.wide, list[k - 1]);
    const uint64_t b = __ballot(starts);
    if (b) return s + __ffsll((unsigned long long)b) - 1;
  }
  return n;
}

// One wave: the column block `blk` of the groups that start in part `part` of
// example i's list.
template <class T, int V>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  const int64_t job = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (job >= a.jobs) return;
  const int lane = threadIdx.x & 63;
  const int64_t i = job / (a.parts * a.blocks);
  const int rest = (int)(job - i * (a.parts * a.blocks));
  const int part = rest / a.blocks, blk = rest - part * a.blocks;
  const int32_t* list = a.order + a.offsets[i];
  const int32_t n = a.offsets[i + 1] - a.offsets[i];
  const int32_t s = group_start(a, list, n, (int32_t)((int64_t)n * part / a.parts));
  const int32_t e = group_start(a, list, n, (int32_t)((int64_t)n * (part + 1) / a.parts));
  const int col = (blk * 64 + lane) * V;
  float ss = 0.0f;
  if (col < a.d) {
    float acc[V] = {};
    int64_t last = -1;
    for (int32_t k = s; k < e; ++k) {
      const int32_t p = list[k];
      const int64_t id = read_id(a.ids, a.wide, p);
      float x[V];
      load_vec<V>(static_cast<const T*>(a.G) + (int64_t)p * a.d + col, x);
      if (id != last) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          ss = fmaf(acc[c], acc[c], ss);
          acc[c] = x[c];
        }
        last = id;
      } else {
#pragma unroll
        for (int c = 0; c < V; ++c) acc[c] += x[c];
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) ss = fmaf(acc[c], acc[c], ss);
  }
  ss = wave_sum(ss);
  if (lane == 0) a.partials[job] = ss * a.scale * a.scale;
}

// --------------------------------------------------------------- clipped sum

struct SumArgs {
  const void* G;
  const int32_t* order;     // positions by token, position
  const int32_t* offsets;   // [V + 1]
  const float* factors;     // [B], NULL: all 1
  float* grad;
  float* partials;          // [chunks][2][d]
  int64_t V;
  int64_t chunk_wgs;        // workgroups of the chunks, before those of the rows
  int32_t chunks, chunk;    // chunks of the sorted list, entries of one
  int32_t d, accumulate;
  uint32_t magic;           // division by T
  int32_t shift;
  float scale;
};

// Sum of factor * G over the entries [s, e) of the sorted list, V columns a lane.
template <class T, int V>
__device__ __forceinline__ void sum_rows(const SumArgs& a, int32_t s, int32_t e, int col,
                                         float (&acc)[V]) {
#pragma unroll
  for (int c = 0; c < V; ++c) acc[c] = 0.0f;
  for (int32_t k = s; k < e; ++k) {
    const int32_t p = a.order[k];
    const float f = a.factors ? a.factors[magic_divide((uint32_t)p, a.magic, a.shift)] : 1.0f;
    if (f == 0.0f) continue;   // factor 0: the example's rows are not read
    float x[V];
    load_vec<V>(static_cast<const T*>(a.G) + (int64_t)p * a.d + col, x);
#pragma unroll
    for (int c = 0; c < V; ++c) acc[c] = fmaf(f, x[c], acc[c]);
  }
}

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

// Token whose entries hold list position k: the last v with offsets[v] <= k.
__device__ __forceinline__ int64_t token_at(const SumArgs& a, int32_t k) {
  int64_t lo = 0, hi = a.V - 1;
  while (lo < hi) {
    const int64_t mid = (lo + hi + 1) >> 1;
    if (a.offsets[mid] <= k) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// A wave per row of the table; rows with more than `chunk` entries are left to
// the waves of the chunks, each of which sums the entries of its chunk that
// belong to such a row: at most two of them, one that began before or at the
// chunk's start (slot 0) and one that begins inside it (slot 1).
template <class T, int V>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a) {
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  if (blockIdx.x < a.chunk_wgs) {
    const int64_t q = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (q >= a.chunks) return;
    const int32_t total = a.offsets[a.V];
    const int32_t s = (int32_t)q * a.chunk;
    if (s >= total) return;
    const int32_t e = s + a.chunk < total ? s + a.chunk : total;
    const int64_t v0 = token_at(a, s), v1 = token_at(a, e - 1);
    for (int slot = 0; slot < 2; ++slot) {
      const int64_t v = slot == 0 ? v0 : v1;
      if (slot == 1 && v1 == v0) break;
      const int32_t vs = a.offsets[v], ve = a.offsets[v + 1];
      if (ve - vs <= a.chunk) continue;
      float* out = a.partials + (q * 2 + slot) * a.d;
      for (int col = lane * V; col < a.d; col += 64 * V) {
        float acc[V];
        sum_rows<T, V>(a, vs > s ? vs : s, ve < e ? ve : e, col, acc);
        store_vec<V>(out + col, acc);
      }
    }
    return;
  }
  const int64_t v = ((int64_t)blockIdx.x - a.chunk_wgs) * (kThreads / 64) + wave;
  if (v >= a.V) return;
  const int32_t s = a.offsets[v], e = a.offsets[v + 1];
  if ((s == e && a.accumulate) || (a.chunks > 0 && e - s > a.chunk)) return;
  for (int col = lane * V; col < a.d; col += 64 * V) {
    float acc[V];
    sum_rows<T, V>(a, s, e, col, acc);
    write_row<V>(a, v, col, acc);
  }
}

// Joins the partial sums of each row with more than `chunk` entries: the
// workgroups of the chunk in which the row begins add them in order.
template <int V>
__global__ __launch_bounds__(kThreads) void join_kernel(SumArgs a) {
  const int32_t q = blockIdx.x;
  const int32_t total = a.offsets[a.V];
  const int32_t s = q * a.chunk;
  if (s >= total) return;
  const int32_t e = s + a.chunk < total ? s + a.chunk : total;
  for (int slot = 0; slot < 2; ++slot) {
    const int64_t v = token_at(a, slot == 0 ? s : e - 1);
    const int32_t vs = a.offsets[v], ve = a.offsets[v + 1];
    if (vs < s || ve - vs <= a.chunk) continue;
    if (slot == 1 && vs == s) break;   // the row of slot 0
    const int32_t last = (ve - 1) / a.chunk;
    for (int col = ((int)blockIdx.y * kThreads + (int)threadIdx.x) * V; col < a.d;
         col += (int)gridDim.y * kThreads * V) {
      float acc[V];
      load_vec<V>(a.partials + ((int64_t)q * 2 + slot) * a.d + col, acc);
      for (int32_t k = q + 1; k <= last; ++k) {
        float x[V];
        load_vec<V>(a.partials + (int64_t)k * 2 * a.d + col, x);
#pragma unroll
        for (int c = 0; c < V; ++c) acc[c] += x[c];
      }
      write_row<V>(a, v, col, acc);
    }
  }
}

// Entries of one chunk of the sorted list: at least 64, at most about 1024 chunks.
int32_t chunk_entries(int64_t N) {
  const int64_t c = ceil_div(N, 1024);
  return (int32_t)(c < 64 ? 64 : c);
}

// Chunks of the sorted list; none where no row can have more than one.
int32_t chunk_count(int64_t N) {
  const int64_t c = chunk_entries(N);
  return N <= c ? 0 : (int32_t)ceil_div(N, c);
}

// Column blocks (of one wave) and parts of an example's list.
void norm_jobs(int64_t B, int64_t T, int64_t d, int* vec, int* blocks, int* parts) {
  *vec = vec_width(d, 4);
  *blocks = (int)ceil_div(d, 64 * *vec);
  int64_t p = ceil_div(8192, B * *blocks);
  const int64_t most = ceil_div(T, 8);
  *parts = (int)(p < most ? p : most);
}

size_t list_bytes(int64_t N, int64_t keys) {
  return round_up((size_t)N * sizeof(int32_t), 256) + round_up((size_t)(keys + 1) * sizeof(int32_t), 256);
}

TokenKey token_key(const dpsgd_embedding& e) {
  return TokenKey{e.ids, e.index_dtype == DPSGD_I64, (uint32_t)e.n_rows, e.B * e.T};
}

}  // namespace

size_t embedding_workspace_bytes(const dpsgd_embedding& e) {
  const int64_t N = e.B * e.T;
  int vec, blocks, parts;
  norm_jobs(e.B, e.T, e.d, &vec, &blocks, &parts);
  const size_t norms = list_bytes(N, e.B) + (size_t)(e.B * blocks * parts) * sizeof(float);
  const size_t sum = round_up((size_t)e.B * sizeof(float), 256) +
                     (size_t)chunk_count(N) * 2 * (size_t)e.d * sizeof(float);
  return list_bytes(N, e.n_rows) + (norms > sum ? norms : sum);
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
  char* ws = static_cast<char*>(workspace);
  int32_t* order = reinterpret_cast<int32_t*>(ws);
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + round_up((size_t)N * sizeof(int32_t), 256));
  ws += list_bytes(N, e.n_rows);
  int32_t* by_example = reinterpret_cast<int32_t*>(ws);
  int32_t* starts = reinterpret_cast<int32_t*>(ws + round_up((size_t)N * sizeof(int32_t), 256));
  float* partials = reinterpret_cast<float*>(ws + list_bytes(N, e.B));
  int st = launch_sort(token_key(e), order, offsets, stream);
  if (st != DPSGD_OK) return st;
  ExampleKey ex{order, offsets + e.n_rows, 0, 0, (uint32_t)e.B};
  divide_magic(e.T, &ex.magic, &ex.shift);
  st = launch_sort(ex, by_example, starts, stream);
  if (st != DPSGD_OK) return st;
  NormArgs a{};
  a.ids = e.ids;
  a.G = G;
  a.order = by_example;
  a.offsets = starts;
  a.partials = partials;
  a.d = (int32_t)e.d;
  a.wide = e.index_dtype == DPSGD_I64;
  a.scale = e.scale;
  int vec;
  norm_jobs(e.B, e.T, e.d, &vec, &a.blocks, &a.parts);
  a.jobs = e.B * a.parts * a.blocks;
  const int64_t wgs = ceil_div(a.jobs, kThreads / 64);
  if (wgs > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
  const dim3 grid((uint32_t)wgs), block(kThreads);
#define DPSGD_NORMS(T)                                                                              \
  switch (vec) {                                                                                    \
    case 4: hipLaunchKernelGGL((norm_kernel<T, 4>), grid, block, 0, stream, a); break;              \
    case 2: hipLaunchKernelGGL((norm_kernel<T, 2>), grid, block, 0, stream, a); break;              \
    default: hipLaunchKernelGGL((norm_kernel<T, 1>), grid, block, 0, stream, a); break;             \
  }
  if (dtype == DPSGD_BF16) {
    DPSGD_NORMS(uint16_t)
  } else {
    DPSGD_NORMS(float)
  }
#undef DPSGD_NORMS
  st = check_launch();
  if (st != DPSGD_OK) return st;
  return launch_norms_reduce(partials, (int64_t)a.parts * a.blocks, e.B, norms_sq, accumulate, stream);
}

int launch_embedding_sum(const dpsgd_embedding& e, const void* G, int32_t dtype,
                         const float* norms_sq, float C, float* grad, int accumulate,
                         float* factors_out, uint8_t* mask_out, void* workspace,
                         hipStream_t stream) {
  const int64_t N = e.B * e.T;
  char* ws = static_cast<char*>(workspace);
  int32_t* order = reinterpret_cast<int32_t*>(ws);
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + round_up((size_t)N * sizeof(int32_t), 256));
  ws += list_bytes(N, e.n_rows);
  float* factors = reinterpret_cast<float*>(ws);
  int st = DPSGD_OK;
  if (norms_sq) {
    st = launch_clip_factors(norms_sq, e.B, C, factors, factors_out, mask_out, stream);
    if (st != DPSGD_OK) return st;
  }
  st = launch_sort(token_key(e), order, offsets, stream);
  if (st != DPSGD_OK) return st;
  SumArgs a{};
  a.G = G;
  a.order = order;
  a.offsets = offsets;
  a.factors = norms_sq ? factors : nullptr;
  a.grad = grad;
  a.partials = reinterpret_cast<float*>(ws + round_up((size_t)e.B * sizeof(float), 256));
  a.V = e.n_rows;
  a.chunk = chunk_entries(N);
  a.chunks = chunk_count(N);
  a.chunk_wgs = ceil_div(a.chunks, kThreads / 64);
  a.d = (int32_t)e.d;
  a.accumulate = accumulate;
  a.scale = e.scale;
  divide_magic(e.T, &a.magic, &a.shift);
  const int64_t wgs = a.chunk_wgs + ceil_div(a.V, kThreads / 64);
  if (wgs > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
  const int vec = vec_width(e.d, 4);
  const dim3 grid((uint32_t)wgs), block(kThreads);
  const dim3 jgrid((uint32_t)a.chunks, (uint32_t)ceil_div(e.d, (int64_t)kThreads * vec));
#define DPSGD_SUM(V)                                                                                \
  if (dtype == DPSGD_BF16) {                                                                        \
    hipLaunchKernelGGL((sum_kernel<uint16_t, V>), grid, block, 0, stream, a);                       \
  } else {                                                                                          \
    hipLaunchKernelGGL((sum_kernel<float, V>), grid, block, 0, stream, a);                          \
  }                                                                                                 \
  if (a.chunks > 0) hipLaunchKernelGGL(join_kernel<V>, jgrid, block, 0, stream, a);
  switch (vec) {
    case 4: DPSGD_SUM(4) break;
    case 2: DPSGD_SUM(2) break;
    default: DPSGD_SUM(1) break;
  }
#undef DPSGD_SUM
  return check_launch();
}

}  // namespace dpsgd
