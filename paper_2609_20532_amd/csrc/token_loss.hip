// Log probabilities of tokens, entropy, the most likely tokens, and the loss with its
// gradient, over rows of V logits:
//
//   z = scale x;  m = max z;  d = z - m;  S = sum e^d;  E = sum e^d d
//   lse = m + ln S;  logp = d_target - ln S;  entropy = ln S - E / S
//   dx_v = scale (p_v (g_lse - g_logp - g_H (ln p_v + H)) + g_logp [v = target])
//
// Bound by memory traffic: each logit is read once, and written once in a gradient. About
// 16 operations an entry (the exponential counts four) are half of what the card does in
// the time of its four bytes in bf16. Rows lie at any alignment (an odd V): vectors of 16
// bytes between the 16-byte boundaries, single entries before and after them.
//  - Loss: a row is held in the registers of a workgroup (of a wave for small V), its
//    maximum and sum are two passes over them, and the gradient is written from them: a
//    workgroup of 512 threads has 64 registers of a row, and two share a CU, so that one
//    loads while the other computes and stores. 8192 rows of 50257 in bf16: 313 us for
//    1.65 GB (5.3 TB/s; with three reads of a row 1453 us; with more registers a thread,
//    one workgroup a CU, 375 us). 6 x 509 rows of 32003 in float32: 132 us.
//  - Sums alone (no alternatives): one pass with a running maximum a thread, nothing held,
//    loads of four vectors in flight. 2048 rows of 32003 in float32: 40 us for 262 MB, of
//    which the last-level cache holds a part (held rows took 116).
//  - Alternatives: rows held, candidates by a bound (top_entries): 54 us for 5 of the same
//    rows' entries, 64 us for 64 (reading the row once for each took 1616 us for 20).
//  - Rows that no workgroup holds, or few long ones: in parts, joined by a second launch
//    (loss of 1024 rows of 128256 in float32: 302 us, its logits read twice).
//  - The gradient of log probabilities: parts of rows, p from lse, 290 us for 8192 rows of
//    50257 in bf16 (5.7 TB/s); rows whose lse is far from 0 by one workgroup each.
#include <math.h>

#include "vec.h"

// z - m is formed from the rounded product z: contracted, it could be above 0 by a
// rounding of z, which is any number for logits far from 0.
#pragma clang fp contract(off)

namespace dpsgd {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int64_t kMostWgs = 1 << 20;
constexpr int64_t kFewRows = 64;

struct TokenArgs {
  const void* logits;
  const void* targets;        // may be null
  void* dlogits;
  const float* weights;       // null: 1
  const float* lse;           // backward
  const float* entropy;
  const float* g_logp;
  const float* g_lse;
  const float* g_entropy;
  float* losses;              // [rows], of examples of one position
  float* logp_out;            // the outputs may be null
  float* lse_out;
  float* entropy_out;
  int64_t* top_ids;
  float* top_logprobs;
  int64_t rows, stride, grad_stride;
  int32_t V, k, wide_ids;
  float scale;
};

// e^d for d <= 0: exactly 0 for -inf, else within (2 |d| + 2) 2^-24 of itself (the rounding of
// d log2 e, and the instruction's).
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// The target of a row, -1 for an empty position; *empty: there is none.
__device__ __forceinline__ int32_t target_of(const TokenArgs& a, int64_t row, bool* empty) {
  *empty = false;
  if (!a.targets) return -1;
  const int64_t t = a.wide_ids ? static_cast<const int64_t*>(a.targets)[row]
                               : (int64_t)static_cast<const int32_t*>(a.targets)[row];
  *empty = t < 0 || t >= a.V;
  return *empty ? -1 : (int32_t)t;
}

template <class T>
__device__ __forceinline__ float entry(const T* x, int32_t v) {
  float f[1];
  load_vec<1>(x + v, f);
  return f[0];
}

template <class T>
__device__ __forceinline__ void put(T* x, int32_t v, float value) {
  const float f[1] = {value};
  store_vec<1>(x + v, f);
}

// An order of logits (the larger first, of equal ones the lower token) as whole
// numbers; 0 is below every logit.
__device__ __forceinline__ uint64_t order_of(float x, int32_t v) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // -0 as 0
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (uint32_t)~v;
}

// Largest value of the wave in every lane (a NaN is passed over).
__device__ __forceinline__ float wave_max(float v) {
#define DPSGD_DPP_MAX(ctrl, rows)                                                                 \
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v),   \
                                                          ctrl, rows, 0xf, false)))
  DPSGD_DPP_MAX(0x111, 0xf);   // row_shr 1, 2, 4, 8
  DPSGD_DPP_MAX(0x112, 0xf);
  DPSGD_DPP_MAX(0x114, 0xf);
  DPSGD_DPP_MAX(0x118, 0xf);
  DPSGD_DPP_MAX(0x142, 0xa);   // row_bcast 15, 31
  DPSGD_DPP_MAX(0x143, 0xc);
#undef DPSGD_DPP_MAX
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)v, off, 64);
    v = o > v ? o : v;
  }
  return v;
}

// Vectors are worked on one after the other: interleaved, their intermediate values do
// not fit the registers beside the row, and there are waves enough to fill the pauses.
__device__ __forceinline__ void one_by_one() { __builtin_amdgcn_sched_barrier(0); }

// n entries in a row from an address of any alignment, in the registers of NT
// threads: vectors of 16 bytes between the first and the last 16-byte boundary, and
// the entries before and after them, one a thread. Places without an entry hold -inf.
template <class T, int NT, int NVEC>
struct Held {
  static constexpr int VE = 16 / (int)sizeof(T);
  static constexpr int kMost = NT * NVEC * VE;   // entries that always fit
  Raw<T, VE> raw[NVEC];
  float edge;
  int32_t edge_at;   // -1: none
  int32_t head, vecs;

  __device__ __forceinline__ void load(const T* x, int32_t n, int32_t tid) {
    head = (int32_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int32_t)sizeof(T);
    head = head < n ? head : n;
    vecs = (n - head) / VE;
    const int32_t tail = n - head - vecs * VE;
    edge_at = tid < head ? tid : (tid - head < tail ? n - tail + tid - head : -1);
#pragma unroll
    for (int j = 0; j < NVEC; ++j) {
#pragma unroll
      for (uint32_t& w : raw[j].w) w = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
      if (tid < vecs - j * NT) raw[j].load(x + head + j * NT * VE + (uint32_t)(tid * VE));
    }
    edge = edge_at >= 0 ? entry(x, edge_at) : -INFINITY;
  }

  // f(x) for every entry of the thread, and for places without one.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < NVEC; ++j) {
      if (j * NT < vecs) {
        float x[VE];
        raw[j].widen(x);
#pragma unroll
        for (int c = 0; c < VE; ++c) f(x[c]);
      }
      one_by_one();
    }
    f(edge);
  }

  // The largest entry of the thread in each quarter of its vectors; the one beside the
  // vectors counts to the first.
  __device__ __forceinline__ void quarter_maxima(float (&g)[4]) const {
    static_assert(NVEC % 4 == 0, "");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      g[q] = q == 0 ? edge : -INFINITY;
#pragma unroll
      for (int j = q * NVEC / 4; j < (q + 1) * NVEC / 4; ++j) {
        float x[VE];
        raw[j].widen(x);
#pragma unroll
        for (int c = 0; c < VE; ++c) g[q] = fmaxf(g[q], x[c]);
      }
    }
  }

  // f(x, place in the row) for the entries x >= least, which are few.
  template <class F>
  __device__ __forceinline__ void each_from(float least, int32_t tid, F f) const {
#pragma unroll
    for (int j = 0; j < NVEC; ++j) {
      if (j * NT + tid < vecs) {
        float x[VE];
        raw[j].widen(x);
        uint32_t which = 0;
#pragma unroll
        for (int c = 0; c < VE; ++c) which |= x[c] >= least ? 1u << c : 0u;
        while (which) {
          const int32_t at = __builtin_ctz(which);
          which &= which - 1;
          float v = x[0];
#pragma unroll
          for (int c = 1; c < VE; ++c) v = c == at ? x[c] : v;
          f(v, head + (j * NT + tid) * VE + at);
        }
      }
      one_by_one();
    }
    if (edge >= least && edge_at >= 0) f(edge, edge_at);
  }

  // Nothing that was formed from the entries before is held on to: the next pass forms
  // it again, and only the entries stay in registers.
  __device__ __forceinline__ void entries_alone() {
#pragma unroll
    for (int j = 0; j < NVEC; ++j) {
#pragma unroll
      for (uint32_t& w : raw[j].w) asm volatile("" : "+v"(w));
    }
  }
};

// Reductions over the NT threads of a row (a wave of its own, or a workgroup). With a
// workgroup every thread has to call them, and `slot` goes from call to call between
// two places, so that one barrier a call is enough.
template <int NT>
struct Team {
  float (*red)[NT / 64][2];   // [2]
  int slot;

  __device__ __forceinline__ float max(float v) {
    v = wave_max(v);
    if constexpr (NT == 64) return v;
    if ((threadIdx.x & 63) == 0) red[slot][threadIdx.x >> 6][0] = v;
    __syncthreads();
    float r = red[slot][0][0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r = fmaxf(r, red[slot][w][0]);
    slot ^= 1;
    return r;
  }

  __device__ __forceinline__ void sum(float& a, float& b) {
    a = wave_total(a);
    b = wave_total(b);
    if constexpr (NT == 64) return;
    if ((threadIdx.x & 63) == 0) {
      red[slot][threadIdx.x >> 6][0] = a;
      red[slot][threadIdx.x >> 6][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      a += red[slot][w][0];
      b += red[slot][w][1];
    }
    slot ^= 1;
  }

  __device__ __forceinline__ void barrier() {
    if constexpr (NT == 64) {   // LDS accesses of one wave stay in order; so has the compiler to
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      __syncthreads();
    }
  }
};

// The exponents (base 2) of a row's entries relative to its largest one, top. Near 0
// they are one multiply-add, x c - top c: the product's rounding, `off`, is the same
// for all entries, at most 2^-4, and is taken back where it matters. For |top c| above
// 2^20 that would not do, and z - m is formed from the rounded products.
struct Exponents {
  float scale, m, c, top_c, off;
  bool near;

  __device__ __forceinline__ Exponents(float scale_, float top) {
    scale = scale_;
    m = scale * top;
    if (m == -INFINITY) m = 0.0f;
    c = scale * kLog2e;
    top_c = top * c;
    near = fabsf(top_c) <= 1048576.0f;
    off = near ? fmaf(top, c, -top_c) : 0.0f;
  }
  template <bool NEAR>
  __device__ __forceinline__ float at(float x) const {
    return NEAR ? fmaf(x, c, -top_c) : (scale * x - m) * kLog2e;
  }
};

// S and E of the entries, both relative to the exact largest one: S = sum 2^t, E =
// sum 2^t t.
template <bool NEAR, bool ENTROPY, class H>
__device__ __forceinline__ void sums_of(const H& held, const Exponents& ex, float& S, float& E) {
  S = E = 0.0f;
  held.each([&](float x) {
    const float t = ex.at<NEAR>(x), p = __builtin_amdgcn_exp2f(t);
    S += p;
    if constexpr (ENTROPY) E = fmaf(p, fmaxf(t, -256.0f), E);   // 0 for -inf; a NaN is in p
  });
}

// What a row's (or a part's) sums say.
struct RowStats {
  float top, m, S, E, log_S;   // largest logit and scale times it
  bool nan, none;

  __device__ __forceinline__ RowStats(float scale, float top_, float S_, float E_) {
    top = top_;
    m = scale * top;
    S = S_;
    E = E_;
    nan = !(S == S) || m == INFINITY;
    none = !nan && m == -INFINITY;
    log_S = logf(S);
  }
  __device__ __forceinline__ float lse() const { return nan ? NAN : (none ? -INFINITY : m + log_S); }
  __device__ __forceinline__ float entropy() const {
    return nan ? NAN : (none ? 0.0f : log_S - kLn2 * (E / S));
  }
  __device__ __forceinline__ float logp(float z) const {
    return nan ? NAN : (none ? -INFINITY : (z - m) - log_S);
  }
};

// What a position adds to its example's loss.
__device__ __forceinline__ float loss_of(float w, float logp) { return w != 0.0f ? -w * logp : 0.0f; }

template <class Tm, class H>
__device__ __forceinline__ void reduce_row(Tm& team, H& held, float scale, bool entropy,
                                           float& top, float& S, float& E, float& mine) {
  mine = -INFINITY;
  held.each([&](float x) { mine = fmaxf(mine, x); });
  top = team.max(mine);
  held.entries_alone();
  const Exponents ex(scale, top);
  if (ex.near) {
    if (entropy) sums_of<true, true>(held, ex, S, E); else sums_of<true, false>(held, ex, S, E);
  } else {
    if (entropy) sums_of<false, true>(held, ex, S, E); else sums_of<false, false>(held, ex, S, E);
  }
  team.sum(S, E);
  held.entries_alone();
  E = fmaf(-ex.off, S, E);
  const float back = __builtin_amdgcn_exp2f(-ex.off);
  S *= back;
  E *= back;
}

// S and E as sums_of's for a row of any length in one pass over memory, no entry held:
// every thread has a running reference R (base 2, at least what makes its largest
// exponent so far 0) and sums relative to it, rescaled once a batch of vectors. R is
// kept within 2^20: entries below are 0 beside any row's largest that is not; where the
// largest is outside, *near is false and the sums say nothing.
template <class T, int NT>
struct Running {
  static constexpr int VE = 16 / (int)sizeof(T);
  static constexpr int kBatch = 4;
  float top = -INFINITY, R = -1048576.0f, S = 0.0f, E = 0.0f;

  template <bool ENTROPY, int N>
  __device__ __forceinline__ void add(const float (&x)[N], float c) {
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);
    const float R1 = fminf(fmaxf(top * c, -1048576.0f), 1048576.0f), d = R - R1;
    const float w = __builtin_amdgcn_exp2f(d);
    if constexpr (ENTROPY) E = w * fmaf(d, S, E);
    S *= w;
    R = R1;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float t = fmaf(x[k], c, -R), p = __builtin_amdgcn_exp2f(t);
      S += p;
      if constexpr (ENTROPY) E = fmaf(p, fmaxf(t, -256.0f), E);
    }
  }

  template <bool ENTROPY>
  __device__ __forceinline__ void row(const T* x, int32_t n, int32_t tid, float c) {
    int32_t head = (int32_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int32_t)sizeof(T);
    head = head < n ? head : n;
    const int32_t vecs = (n - head) / VE, tail = n - head - vecs * VE;
    const int32_t edge_at = tid < head ? tid : (tid - head < tail ? n - tail + tid - head : -1);
    const float edge[1] = {edge_at >= 0 ? entry(x, edge_at) : -INFINITY};
    const T* body = x + head;
    int32_t j = tid;
    for (; j + (kBatch - 1) * NT < vecs; j += kBatch * NT) {
      Raw<T, VE> raw[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) raw[b].load(body + (int64_t)(j + b * NT) * VE);
      float f[kBatch * VE];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        float g[VE];
        raw[b].widen(g);
#pragma unroll
        for (int k = 0; k < VE; ++k) f[b * VE + k] = g[k];
      }
      add<ENTROPY>(f, c);
    }
    for (; j < vecs; j += NT) {
      float f[VE];
      load_vec<VE>(body + (int64_t)j * VE, f);
      add<ENTROPY>(f, c);
    }
    if (edge_at >= 0) add<ENTROPY>(edge, c);
  }

  // The row's, in every thread: relative to the exact largest entry.
  __device__ __forceinline__ bool join(Team<NT>& team, float c) {
    top = team.max(top);
    const float top_c = top * c, Rf = fminf(fmaxf(top_c, -1048576.0f), 1048576.0f);
    const bool near = fabsf(top_c) <= 1048576.0f;
    const float off = near ? fmaf(top, c, -top_c) : 0.0f, d = (R - Rf) - off;
    const float w = __builtin_amdgcn_exp2f(d);
    E = w == 0.0f ? 0.0f : w * fmaf(d, S, E);
    S = w == 0.0f && S == S ? 0.0f : w * S;
    team.sum(S, E);
    return near;
  }
};

// The same sums where the largest entry is far from 0 (or there is none), by exponents
// of the rounded products.
template <class T, int NT>
__device__ __forceinline__ void far_sums(Team<NT>& team, const T* x, int32_t n, int32_t tid, float scale,
                                         float top, float& S, float& E) {
  const Exponents ex(scale, top);
  S = E = 0.0f;
  for (int32_t v = tid; v < n; v += NT) {
    const float t = ex.template at<false>(entry(x, v)), p = __builtin_amdgcn_exp2f(t);
    S += p;
    E = fmaf(p, fmaxf(t, -256.0f), E);
  }
  team.sum(S, E);
}

// One row a team (as below), nothing but sums asked for.
template <class T, int NT, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void token_sums_kernel(TokenArgs a) {
  constexpr int kTeams = kThreads / NT;
  __shared__ float red[2][NT / 64][2];
  const int32_t team_at = NT == 64 ? __builtin_amdgcn_readfirstlane((int32_t)(threadIdx.x >> 6)) : 0;
  const int32_t tid = NT == 64 ? (int32_t)(threadIdx.x & 63) : (int32_t)threadIdx.x;
  Team<NT> team{red, 0};
  for (int64_t row = (int64_t)blockIdx.x * kTeams + team_at; row < a.rows; row += (int64_t)gridDim.x * kTeams) {
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    Running<T, NT> run;
    float at_target = 0.0f;
    run.S = empty ? 1.0f : 0.0f;
    if (!empty) {
      if (target >= 0) at_target = entry(x, target);
      run.template row<ENTROPY>(x, a.V, tid, a.scale * kLog2e);
      if (!run.join(team, a.scale * kLog2e)) far_sums(team, x, a.V, tid, a.scale, run.top, run.S, run.E);
    }
    if (tid == 0) {
      const RowStats st(a.scale, run.top, run.S, run.E);
      if (a.logp_out) a.logp_out[row] = empty ? 0.0f : st.logp(a.scale * at_target);
      if (a.lse_out) a.lse_out[row] = empty ? 0.0f : st.lse();
      if (a.entropy_out) a.entropy_out[row] = empty ? 0.0f : st.entropy();
    }
  }
}

constexpr int kListed = 2048;       // candidates that a workgroup's list holds
constexpr int kListedWave = 512;    // that a wave's list holds

// Where the most likely entries of a row are collected.
template <int NT>
struct TopLds {
  static constexpr int kMost = NT == 64 ? kListedWave : kListed;
  uint64_t key[kMost];
  alignas(16) uint32_t group[256];
  uint32_t least;
  int32_t count;
};

__device__ __forceinline__ uint32_t order_bits(float x) { return (uint32_t)(order_of(x, 0) >> 32); }
__device__ __forceinline__ float logit_of(uint64_t order) {
  const uint32_t o = (uint32_t)(order >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

// put(i, order) for the k largest of n different keys in LDS, in order; returns their
// number. Every key finds its place by counting the larger ones.
template <int NT, class P>
__device__ __forceinline__ int32_t put_in_order(const uint64_t* keys, int32_t n, int32_t k, int32_t tid, P put) {
  for (int32_t i = tid; i < n; i += NT) {
    const uint64_t own = keys[i];
    int32_t rank = 0;
#pragma unroll 4
    for (int32_t j = 0; j < n; ++j) rank += keys[j] > own ? 1 : 0;
    if (rank < k) put(rank, own);
  }
  return n < k ? n : k;
}

// A bound on the k-th largest of 256 group maxima, by one wave: its upper 16 bits, from the
// highest down, which is all of a bf16 logit. Of float32 ones, whose 7 bits of fraction may be
// too coarse for the row (all logits at 1000 and more, say), the lower bits as well where more
// than twice the groups that are needed reach the bound: with 16 bits the list of candidates
// overflows there (2048 rows of 32003, k = 64: 66 us centred on 0; at 3000 68, with 16 bits
// 5770).
template <class T>
__device__ __forceinline__ void bound_of_groups(const uint32_t* group, int32_t k, int32_t lane, uint32_t* to) {
  const uint4 g = reinterpret_cast<const uint4*>(group)[lane];
  uint32_t least = 0;
  int32_t reach = 256;   // groups from `least` on
  const auto take = [&](int bit) {
    const uint32_t t = least | 1u << bit;
    const int n = __popcll(__ballot(g.x >= t)) + __popcll(__ballot(g.y >= t)) +
                  __popcll(__ballot(g.z >= t)) + __popcll(__ballot(g.w >= t));
    if (n >= k) least = t, reach = n;
  };
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) take(bit);
  if (sizeof(T) == 4 && reach > 2 * k)
    for (int bit = 15; bit >= 0; --bit) take(bit);
  if (lane == 0) *to = least;
}

// The k largest entries in order: put(i, order) for i < the number that there are.
// The entries are in 256 groups (a vector's places of one lane, the places of one, two
// or four neighbouring lanes); at least k of the groups' largest ones are not below the
// k-th largest of them, so entries below it are none of the k. Of V unordered entries
// about 256 ln(256 / (256 - k)) are left, 21 for k = 20 and 74 for k = 64 (41 and 178 where
// twice as many groups reach the bound): they are listed and put in order. `first` is added to the entries' places. Where the list is too
// short (many equal or sorted logits) the n_row entries at x are searched once for each
// alternative.
template <int NT, class T, class H, class P>
__device__ __forceinline__ int32_t top_entries(Team<NT>& team, const H& held, const T* x, int32_t n_row,
                                               float mine, int32_t k, int32_t first, TopLds<NT>& lds,
                                               uint64_t* red64, P put) {
  const int32_t tid = NT == 64 ? (int32_t)(threadIdx.x & 63) : (int32_t)threadIdx.x;
  if constexpr (NT == 64) {
    float g[4];
    held.quarter_maxima(g);
#pragma unroll
    for (int j = 0; j < 4; ++j) lds.group[tid * 4 + j] = order_bits(g[j]);
  } else {
    constexpr int kLanes = NT / 256;   // threads of a group
    uint32_t g = order_bits(mine);
#pragma unroll
    for (int off = 1; off < kLanes; off <<= 1) {
      const uint32_t o = (uint32_t)__shfl_xor((int)g, off, 64);
      g = o > g ? o : g;
    }
    if (tid % kLanes == 0) lds.group[tid / kLanes] = g;
  }
  if (tid == 0) lds.count = 0;
  team.barrier();
  if (tid < 64) bound_of_groups<T>(lds.group, k, tid, &lds.least);
  team.barrier();
  // Entries of -inf are none.
  const uint32_t none = order_bits(-INFINITY);
  const uint32_t least = lds.least > none ? lds.least : none + 1;
  if (order_bits(mine) >= least) {
    held.each_from(logit_of((uint64_t)least << 32), tid, [&](float f, int32_t v) {
      const int32_t at = atomicAdd(&lds.count, 1);
      if (at < TopLds<NT>::kMost) lds.key[at] = order_of(f, first + v);
    });
  }
  team.barrier();
  const int32_t n = lds.count;
  int32_t found;
  if (n <= TopLds<NT>::kMost) {
    found = put_in_order<NT>(lds.key, n, k, tid, put);
  } else {
    uint64_t last = ~(uint64_t)0;
    for (found = 0; found < k; ++found) {
      uint64_t best = 0;
      for (int32_t v = tid; v < n_row; v += NT) {
        const float f = entry(x, v);
        const uint64_t o = order_of(f, first + v);
        if (f != -INFINITY && o < last && o > best) best = o;
      }
      best = wave_max_u64(best);
      if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) red64[threadIdx.x >> 6] = best;
        __syncthreads();
        for (int w = 0; w < NT / 64; ++w) best = red64[w] > best ? red64[w] : best;
        __syncthreads();
      }
      if (best == 0) break;
      if (tid == 0) put(found, best);
      last = best;
    }
  }
  team.barrier();   // the lists may be written again
  return found;
}

// Alternatives from place `from` on that there are none of.
__device__ __forceinline__ void fill_top(const TokenArgs& a, int64_t row, int32_t from, int32_t step,
                                         bool nan) {
  for (int32_t i = from; i < a.k; i += step) {
    if (a.top_ids) a.top_ids[row * a.k + i] = -1;
    if (a.top_logprobs) a.top_logprobs[row * a.k + i] = nan ? NAN : -INFINITY;
  }
}

template <class T>
__device__ __forceinline__ void write_zeros(T* g, int32_t n, int32_t tid, int32_t threads) {
  constexpr int VE = 16 / (int)sizeof(T);
  int32_t head = (int32_t)((16 - (reinterpret_cast<uintptr_t>(g) & 15)) & 15) / (int32_t)sizeof(T);
  head = head < n ? head : n;
  const int32_t vecs = (n - head) / VE, tail = n - head - vecs * VE;
  const float zero[VE] = {};
  for (int32_t j = tid; j < vecs; j += threads) store_vec<VE>(g + head + j * VE, zero);
  if (tid < head) put(g, tid, 0.0f);
  if (tid >= head && tid - head < tail) put(g, n - tail + tid - head, 0.0f);
}

// value(x) of entries in registers to g, `add` added at the target (a place among them,
// or any other number: it is not there).
template <class T, int NT, int NVEC, class F>
__device__ __forceinline__ void write_entries(const Held<T, NT, NVEC>& held, const T* x, T* g, int32_t tid,
                                              int32_t target, float add, F value) {
  constexpr int VE = Held<T, NT, NVEC>::VE;
  const int32_t rel = target - held.head, vec = rel >= 0 && rel < held.vecs * VE ? rel / VE : -1;
  const int32_t at_j = vec >= 0 && vec % NT == tid ? vec / NT : -1;   // where this thread has the target
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
#pragma unroll
  for (int j = 0; j < NVEC; ++j) {
    if (j * NT + tid < held.vecs) {
      float v[VE];
      held.raw[j].widen(v);
#pragma unroll
      for (int c = 0; c < VE; ++c) v[c] = value(v[c]);
      if (j == at_j) {
#pragma unroll
        for (int c = 0; c < VE; ++c) v[c] += c == rel % VE ? add : 0.0f;
      }
      T* to = g + held.head + j * NT * VE + (uint32_t)(tid * VE);
      if (same) {
        store_vec<VE>(to, v);
      } else {
#pragma unroll
        for (int c = 0; c < VE; ++c) put(to, c, v[c]);
      }
    }
    one_by_one();
  }
  if (held.edge_at >= 0) put(g, held.edge_at, value(held.edge) + (held.edge_at == target ? add : 0.0f));
}

// scale w (p_v - [v = target]) of n entries in registers, of a row with these sums.
template <class T, int NT, int NVEC>
__device__ __forceinline__ void write_gradient(const Held<T, NT, NVEC>& held, const T* x, T* g, int32_t n,
                                               int32_t tid, int32_t target, float w, float scale,
                                               const RowStats& st) {
  if (w == 0.0f || st.none) return write_zeros(g, n, tid, NT);
  const Exponents ex(scale, st.top);
  const float f = scale * w, fp = f * (__builtin_amdgcn_exp2f(-ex.off) / st.S);
  if (ex.near)
    write_entries(held, x, g, tid, target, -f,
                  [&](float v) { return fp * __builtin_amdgcn_exp2f(ex.template at<true>(v)); });
  else
    write_entries(held, x, g, tid, target, -f,
                  [&](float v) { return fp * __builtin_amdgcn_exp2f(ex.template at<false>(v)); });
}

// Waves a SIMD that the registers are divided among: the fastest of those tried (4096 rows
// of 32000 in bf16, loss: 98 us with 5, 105 with 8, 102 with 6).
constexpr int waves_of(int nvec, bool loss) {
  return loss ? (nvec > 8 ? 4 : (nvec > 4 ? 5 : 8)) : (nvec > 4 ? 4 : 6);
}

// One row a team: a wave of its own (NT = 64, four of them a workgroup), or a
// workgroup. LOSS: the gradient from the same registers; else the log probabilities,
// entropy and alternatives.
template <class T, int NT, int NVEC, bool LOSS>
__global__ __launch_bounds__(NT == 64 ? kThreads : NT, waves_of(NVEC, LOSS)) void token_row_kernel(TokenArgs a) {
  constexpr int kTeams = NT == 64 ? kThreads / 64 : 1;
  __shared__ float red[2][NT / 64][2];
  __shared__ uint64_t red64[NT / 64];
  __shared__ TopLds<NT> top_lds[LOSS ? 1 : kTeams];
  const int32_t team_at = NT == 64 ? __builtin_amdgcn_readfirstlane((int32_t)(threadIdx.x >> 6)) : 0;
  const int32_t tid = NT == 64 ? (int32_t)(threadIdx.x & 63) : (int32_t)threadIdx.x;
  Team<NT> team{red, 0};
  for (int64_t row = (int64_t)blockIdx.x * kTeams + team_at; row < a.rows;
       row += (int64_t)gridDim.x * kTeams) {
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    Held<T, NT, NVEC> held;
    float top = -INFINITY, S = 1.0f, E = 0.0f, mine = -INFINITY, at_target = 0.0f;
    if (!empty) {
      held.load(x, a.V, tid);
      if (target >= 0) at_target = entry(x, target);   // before a gradient is written there
      reduce_row(team, held, a.scale, !LOSS && a.entropy_out, top, S, E, mine);
    }
    const RowStats st(a.scale, top, S, E);
    if (tid == 0) {
      if (a.logp_out) a.logp_out[row] = empty ? 0.0f : st.logp(a.scale * at_target);
      if (a.lse_out) a.lse_out[row] = empty ? 0.0f : st.lse();
      if (a.entropy_out) a.entropy_out[row] = empty ? 0.0f : st.entropy();
    }
    if constexpr (LOSS) {
      T* g = static_cast<T*>(a.dlogits) + row * a.grad_stride;
      const float w = empty ? 0.0f : (a.weights ? a.weights[row] : 1.0f);
      if (a.losses && tid == 0) a.losses[row] = loss_of(w, st.logp(a.scale * at_target));
      write_gradient<T, NT, NVEC>(held, x, g, a.V, tid, target, w, a.scale, st);
    } else if (a.k > 0) {
      int32_t found = 0;
      if (!empty && !st.nan && !st.none)
        found = top_entries<NT>(team, held, x, a.V, mine, a.k, 0, top_lds[team_at], red64,
                                [&](int32_t i, uint64_t o) {
                                  if (a.top_ids) a.top_ids[row * a.k + i] = (int32_t)~(uint32_t)o;
                                  if (a.top_logprobs)
                                    a.top_logprobs[row * a.k + i] = st.logp(a.scale * logit_of(o));
                                });
      fill_top(a, row, found + tid, NT, !empty && st.nan);
    }
  }
}

// Rows in parts, where one workgroup's registers do not hold a row, or where there are
// few rows: every part leaves its sums (relative to its own largest logit), the logit of
// the target if it has it, and its most likely entries; a second launch joins them.
constexpr int kPartVecs = 4;
template <class T>
using PartHeld = Held<T, kThreads, kPartVecs>;

struct Parts {
  float4* sums;      // [rows][parts]: largest logit, S, E, logit of the target
  uint64_t* keys;    // [rows][parts][k], the largest first, 0 behind them
  int32_t n;         // of a row
  int32_t size;      // entries of a part (the last one of a row may have fewer)
};

template <class T>
__global__ __launch_bounds__(kThreads) void token_part_kernel(TokenArgs a, Parts parts) {
  __shared__ float red[2][kThreads / 64][2];
  __shared__ uint64_t red64[kThreads / 64];
  __shared__ TopLds<kThreads> top_lds;
  Team<kThreads> team{red, 0};
  const int32_t tid = threadIdx.x;
  for (int64_t at = blockIdx.x; at < a.rows * parts.n; at += gridDim.x) {
    const int64_t row = at / parts.n;
    const int32_t part = (int32_t)(at - row * parts.n), first = part * parts.size;
    const int32_t n = a.V - first < parts.size ? a.V - first : parts.size;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    if (empty) continue;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride + first;
    PartHeld<T> held;
    held.load(x, n, tid);
    float top, S, E, mine;
    reduce_row(team, held, a.scale, a.entropy_out != nullptr, top, S, E, mine);
    if (tid == 0)
      parts.sums[at] = make_float4(top, S, E, target >= first && target < first + n ? entry(x, target - first) : 0.0f);
    if (a.k > 0) {
      uint64_t* keys = parts.keys + at * a.k;
      int32_t found = 0;
      if (S == S && top != INFINITY && top != -INFINITY)   // what the row is, the join says
        found = top_entries<kThreads>(team, held, x, n, mine, a.k, first, top_lds, red64,
                                      [&](int32_t i, uint64_t o) { keys[i] = o; });
      if (found + tid < a.k) keys[found + tid] = 0;
    }
  }
}

// The sums of a row from those of its parts; *z: the logit of the target, where there is one.
template <class T>
__device__ __forceinline__ RowStats join_parts(const TokenArgs& a, const Parts& parts, int64_t row,
                                               int32_t target, Team<kThreads>& team, float* z) {
  const float4* sums = parts.sums + row * parts.n;
  float top = -INFINITY;
  for (int32_t p = threadIdx.x; p < parts.n; p += kThreads) top = fmaxf(top, sums[p].x);
  top = team.max(top);
  // Exponents as within a part: from rounded products the parts' shares would be off by the
  // products' rounding, and p would not sum to 1.
  const Exponents ex(a.scale, top);
  float S = 0.0f, E = 0.0f;
  for (int32_t p = threadIdx.x; p < parts.n; p += kThreads) {
    const float4 q = sums[p];
    if (q.y != 0.0f) {   // 0: all of the part is -inf; NaN counts
      const float t = (ex.near ? ex.at<true>(q.x) : ex.at<false>(q.x)) - ex.off, w = __builtin_amdgcn_exp2f(t);
      S = fmaf(w, q.y, S);
      E += w * fmaf(q.y, fmaxf(t, -256.0f), q.z);
    }
  }
  team.sum(S, E);
  *z = target >= 0 ? a.scale * sums[target / parts.size].w : 0.0f;
  return RowStats(a.scale, top, S, E);
}

template <class T>
__global__ __launch_bounds__(kThreads) void token_join_kernel(TokenArgs a, Parts parts) {
  __shared__ float red[2][kThreads / 64][2];
  __shared__ uint64_t red64[kThreads / 64];
  __shared__ TopLds<kThreads> lists;
  Team<kThreads> team{red, 0};
  const int32_t tid = threadIdx.x;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    float z = 0.0f;
    RowStats st(a.scale, 0.0f, 1.0f, 0.0f);
    if (!empty) st = join_parts<T>(a, parts, row, target, team, &z);
    if (tid == 0) {
      if (a.logp_out) a.logp_out[row] = empty ? 0.0f : st.logp(z);
      if (a.lse_out) a.lse_out[row] = empty ? 0.0f : st.lse();
      if (a.entropy_out) a.entropy_out[row] = empty ? 0.0f : st.entropy();
    }
    if (a.k == 0) continue;
    int32_t found = 0;
    if (!empty && !st.nan && !st.none) {
      const uint64_t* keys = parts.keys + row * parts.n * a.k;
      const int64_t all = (int64_t)parts.n * a.k;
      const auto put = [&](int32_t i, uint64_t o) {
        if (a.top_ids) a.top_ids[row * a.k + i] = (int32_t)~(uint32_t)o;
        if (a.top_logprobs) a.top_logprobs[row * a.k + i] = st.logp(a.scale * logit_of(o));
      };
      const auto largest = [&](uint64_t v) {
        v = wave_max_u64(v);
        if ((tid & 63) == 0) red64[tid >> 6] = v;
        __syncthreads();
        for (int w = 0; w < kThreads / 64; ++w) v = red64[w] > v ? red64[w] : v;
        __syncthreads();
        return v;
      };
      // The bound again, with the parts' best entries, second best ones and so on each in a
      // group of its own.
      const auto key = [&](int64_t i) {
        const int64_t r = i / parts.n;
        return keys[(i - r * parts.n) * a.k + r];
      };
      uint32_t g = 0;
      for (int64_t i = tid; i < all; i += kThreads) {
        const uint32_t o = (uint32_t)(key(i) >> 32);
        g = o > g ? o : g;
      }
      lists.group[tid] = g;
      if (tid == 0) lists.count = 0;
      __syncthreads();
      if (tid < 64) bound_of_groups<T>(lists.group, a.k, tid, &lists.least);
      __syncthreads();
      const uint64_t least = lists.least ? (uint64_t)lists.least << 32 : 1;
      for (int64_t i = tid; i < all; i += kThreads) {
        const uint64_t o = key(i);
        if (o >= least) {
          const int32_t at = atomicAdd(&lists.count, 1);
          if (at < kListed) lists.key[at] = o;
        }
      }
      __syncthreads();
      const int32_t n = lists.count;
      if (n <= kListed) {
        found = put_in_order<kThreads>(lists.key, n, a.k, tid, put);
      } else {
        uint64_t last = ~(uint64_t)0;
        for (found = 0; found < a.k; ++found) {
          uint64_t best = 0;
          for (int64_t i = tid; i < all; i += kThreads) best = keys[i] < last && keys[i] > best ? keys[i] : best;
          best = largest(best);
          if (best == 0) break;
          if (tid == 0) put(found, best);
          last = best;
        }
      }
      __syncthreads();
    }
    fill_top(a, row, found + tid, kThreads, !empty && st.nan);
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void token_part_loss_kernel(TokenArgs a, Parts parts) {
  __shared__ float red[2][kThreads / 64][2];
  Team<kThreads> team{red, 0};
  const int32_t tid = threadIdx.x;
  for (int64_t at = blockIdx.x; at < a.rows * parts.n; at += gridDim.x) {
    const int64_t row = at / parts.n;
    const int32_t part = (int32_t)(at - row * parts.n), first = part * parts.size;
    const int32_t n = a.V - first < parts.size ? a.V - first : parts.size;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    const T* x = static_cast<const T*>(a.logits) + row * a.stride + first;
    T* g = static_cast<T*>(a.dlogits) + row * a.grad_stride + first;
    const float w = empty ? 0.0f : (a.weights ? a.weights[row] : 1.0f);
    PartHeld<T> held;
    float z = 0.0f;
    RowStats st(a.scale, 0.0f, 1.0f, 0.0f);
    if (!empty) {
      held.load(x, n, tid);
      st = join_parts<T>(a, parts, row, target, team, &z);
    }
    if (part == 0 && tid == 0 && a.logp_out) a.logp_out[row] = empty ? 0.0f : st.logp(z);
    if (part == 0 && tid == 0 && a.losses) a.losses[row] = loss_of(w, st.logp(z));
    write_gradient(held, x, g, n, tid, target - first, w, a.scale, st);
  }
}

// A row's upstream gradients, and its entropy (with ge).
struct Upstream {
  float gp, q, ge, H;   // q: g_lse - g_logp
};

// scale (p_v (q - ge (ln p_v + H)) + gp [v = target]) of entries in registers; p and ln p
// from the sums of their row.
template <class T, int NT, int NVEC>
__device__ __forceinline__ void write_backward(const Held<T, NT, NVEC>& held, const T* x, T* g, int32_t tid,
                                               int32_t target, float scale, const Upstream& u,
                                               const RowStats& st) {
  const Exponents ex(scale, st.top);
  const float f = __builtin_amdgcn_exp2f(-ex.off) / st.S;
  write_entries(held, x, g, tid, target, scale * u.gp, [&](float v) {
    const float t = ex.near ? ex.template at<true>(v) : ex.template at<false>(v);
    const float p = f * __builtin_amdgcn_exp2f(t);
    if (u.ge == 0.0f) return scale * (p * u.q);
    const float l = fmaxf((t - ex.off) * kLn2, -256.0f) - st.log_S;   // 0 for -inf; a NaN is in p
    return scale * (p * (u.q - u.ge * (l + u.H)));
  });
}

// Rows whose p is formed from lse as it is stored: its rounding, half a step of lse, is then
// at most 2^-20 of p (2^-15, a 64th of the gradient's own rounding, in bf16), and the same for
// all p of the row. Beyond, where it would grow with the logits' common offset (to 3% of p at
// 10^6), the row's sums are formed again, relative to its largest entry.
template <class T>
constexpr float kNearLse = sizeof(T) == 2 ? 1024.0f : 32.0f;

// The part whose workgroup has all of a row, spread by a multiplicative hash: workgroups go to
// the XCDs and their CUs in turn, and with the same part of every row few of them have work
// (512 rows of 262144 in bf16 1930 us with part 0, 254 spread).
__device__ __forceinline__ int32_t owner_of(int64_t row, int32_t parts) {
  return (int32_t)(((uint32_t)row * 0x9E3779B1u >> 16) % (uint32_t)parts);
}

// dx_v = scale (p_v (g_lse - g_logp - g_H (ln p_v + H)) + g_logp [v = target]): rows, or
// parts of them, one after the other. A row in parts with its lse far from 0 is one
// workgroup's, which reads it twice (8192 rows of 50257 in bf16: 290 us, 419 far from 0; every
// row held in registers as in the loss: 306 and 313).
template <class T, int NT>
__global__ __launch_bounds__(kThreads) void token_backward_kernel(TokenArgs a, int32_t parts) {
  constexpr int kTeams = kThreads / NT;
  __shared__ float red[2][NT / 64][2];
  const int32_t tid = NT == 64 ? (int32_t)(threadIdx.x & 63) : (int32_t)threadIdx.x;
  const int32_t team_at = NT == 64 ? __builtin_amdgcn_readfirstlane((int32_t)(threadIdx.x >> 6)) : 0;
  Team<NT> team{red, 0};
  using H = Held<T, NT, kPartVecs>;
  for (int64_t at = (int64_t)blockIdx.x * kTeams + team_at; at < a.rows * parts; at += (int64_t)gridDim.x * kTeams) {
    const int64_t row = at / parts;
    const int32_t part = (int32_t)(at - row * parts), first = part * H::kMost;
    const int32_t n = a.V - first < H::kMost ? a.V - first : H::kMost;
    const T* x_row = static_cast<const T*>(a.logits) + row * a.stride;
    T* g_row = static_cast<T*>(a.dlogits) + row * a.grad_stride;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    const float gp = empty || !a.g_logp ? 0.0f : a.g_logp[row];
    const float gl = empty || !a.g_lse ? 0.0f : a.g_lse[row];
    const float ge = empty || !a.g_entropy ? 0.0f : a.g_entropy[row];
    const bool zero = gp == 0.0f && gl == 0.0f && ge == 0.0f;
    const float lse = zero ? 0.0f : a.lse[row], H_row = ge != 0.0f ? a.entropy[row] : 0.0f;
    if (zero || lse == -INFINITY) {
      write_zeros(g_row + first, n, tid, NT);
      continue;
    }
    const float q = gl - gp;
    H held;
    if (fabsf(lse) > kNearLse<T>) {   // not a NaN
      const Upstream up{gp, q, ge, H_row};
      float top, S, E, mine;
      if (NT == 64 || parts == 1) {
        held.load(x_row, n, tid);
        reduce_row(team, held, a.scale, false, top, S, E, mine);
        write_backward(held, x_row, g_row, tid, target, a.scale, up, RowStats(a.scale, top, S, E));
      } else if (part == owner_of(row, parts)) {
        Running<T, NT> run;
        run.template row<false>(x_row, a.V, tid, a.scale * kLog2e);
        if (!run.join(team, a.scale * kLog2e)) far_sums(team, x_row, a.V, tid, a.scale, run.top, run.S, run.E);
        const RowStats st(a.scale, run.top, run.S, run.E);
        for (int32_t v = 0; v < a.V; v += H::kMost) {
          held.load(x_row + v, a.V - v < H::kMost ? a.V - v : H::kMost, tid);
          write_backward(held, x_row + v, g_row + v, tid, target - v, a.scale, up, st);
        }
      }
      continue;
    }
    const T* x = x_row + first;
    T* g = g_row + first;
    held.load(x, n, tid);
    if (ge == 0.0f) {
      write_entries(held, x, g, tid, target - first, a.scale * gp,
                    [&](float v) { return a.scale * (exp_of(fmaf(a.scale, v, -lse)) * q); });
    } else {
      write_entries(held, x, g, tid, target - first, a.scale * gp, [&](float v) {
        const float l = fmaf(a.scale, v, -lse), p = exp_of(l);
        return a.scale * (p * (q - ge * (fmaxf(l, -256.0f) + H_row)));   // 0 for -inf; a NaN is in p
      });
    }
  }
}

// losses[i] = -sum_t w logp, a team an example (T = 1: the rows' kernels write them).
template <int NT>
__global__ __launch_bounds__(kThreads) void token_losses_kernel(TokenArgs a, const float* logp,
                                                                float* losses, int64_t B, int64_t T) {
  constexpr int kTeams = kThreads / NT;
  __shared__ float red[2][NT / 64][2];
  Team<NT> team{red, 0};
  const int32_t tid = NT == 64 ? (int32_t)(threadIdx.x & 63) : (int32_t)threadIdx.x;
  const int32_t team_at = NT == 64 ? (int32_t)(threadIdx.x >> 6) : 0;
  for (int64_t i = (int64_t)blockIdx.x * kTeams + team_at; i < B; i += (int64_t)gridDim.x * kTeams) {
    float s = 0.0f, none = 0.0f;
#pragma unroll 4
    for (int64_t t = tid; t < T; t += NT) {
      const int64_t row = i * T + t;
      bool empty;
      target_of(a, row, &empty);
      const float w = a.weights ? a.weights[row] : 1.0f, lp = logp[row];
      if (!empty && w != 0.0f) s = fmaf(-w, lp, s);
    }
    team.sum(s, none);
    if (tid == 0) losses[i] = s;
  }
}

TokenArgs common_args(const dpsgd_logits& d, const void* logits) {
  TokenArgs a{};
  a.logits = logits;
  a.targets = d.targets;
  a.rows = d.B * d.T;
  a.stride = d.stride;
  a.V = (int32_t)d.V;
  a.wide_ids = d.index_dtype == DPSGD_I64;
  a.scale = d.scale;
  return a;
}

uint32_t grid_of(int64_t n) { return (uint32_t)(n < kMostWgs ? n : kMostWgs); }

template <class T>
int launch_sums_of(const TokenArgs& a, hipStream_t stream) {
  const bool wave = a.V <= Held<T, 64, 4>::kMost;
  const uint32_t grid = grid_of(wave ? ceil_div(a.rows, 4) : a.rows);
  if (wave && a.entropy_out)
    hipLaunchKernelGGL((token_sums_kernel<T, 64, true>), dim3(grid), dim3(kThreads), 0, stream, a);
  else if (wave)
    hipLaunchKernelGGL((token_sums_kernel<T, 64, false>), dim3(grid), dim3(kThreads), 0, stream, a);
  else if (a.entropy_out)
    hipLaunchKernelGGL((token_sums_kernel<T, kThreads, true>), dim3(grid), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((token_sums_kernel<T, kThreads, false>), dim3(grid), dim3(kThreads), 0, stream, a);
  return check_launch();
}

// The smallest team that holds a row: larger ones wait longer for each other (8192 rows in
// bf16, loss: of 1000 by waves 9 us, by 256 threads 17; of 8192 by 256 threads 44 us, by 512 61;
// with five alternatives 11 and 25, 37 and 80).
template <class T, bool LOSS>
int launch_rows_of(const TokenArgs& a, hipStream_t stream) {
  const int64_t wave4 = Held<T, 64, 4>::kMost;
  if (!LOSS && a.k == 0) return launch_sums_of<T>(a, stream);
  if (a.V <= wave4)
    hipLaunchKernelGGL((token_row_kernel<T, 64, 4, LOSS>), dim3(grid_of(ceil_div(a.rows, 4))), dim3(kThreads), 0, stream, a);
  else if (a.V <= 4 * wave4)
    hipLaunchKernelGGL((token_row_kernel<T, 256, 4, LOSS>), dim3(grid_of(a.rows)), dim3(256), 0, stream, a);
  else if (a.V <= 16 * wave4)
    hipLaunchKernelGGL((token_row_kernel<T, 512, 8, LOSS>), dim3(grid_of(a.rows)), dim3(512), 0, stream, a);
  else if (!LOSS || a.V <= 32 * wave4)
    hipLaunchKernelGGL((token_row_kernel<T, 512, 16, LOSS>), dim3(grid_of(a.rows)), dim3(512), 0, stream, a);
  else if constexpr (LOSS)
    hipLaunchKernelGGL((token_row_kernel<T, 1024, 16, true>), dim3(grid_of(a.rows)), dim3(1024), 0, stream, a);
  return check_launch();
}

int64_t part_entries(int32_t dtype) {
  return dtype == DPSGD_BF16 ? PartHeld<uint16_t>::kMost : PartHeld<float>::kMost;
}

// Whether rows are taken in parts: where no workgroup holds a row (sums alone need none
// to), and for few rows of more than 512 threads hold, for which a workgroup a row would
// leave the card idle. Below that a second launch costs what it saves (8 rows of 32003 in
// float32, calls in a row: 6.0 us without alternatives, 8.5 in parts; k = 5 9.1 and 10.8;
// loss 7.1 and 8.6; of 50257 in bf16: 6.4 and 8.7, 12.7 and 11.5, 8.9 and 8.6). Alternatives
// take parts where a row would be 1024 threads and one workgroup a CU (2048 rows of 131072
// in bf16, k = 5: 145 us, 187 by whole rows); a loss, which would read its logits twice, does
// not (289 and 233).
bool in_parts(const dpsgd_logits& d, int32_t k, bool loss) {
  const bool bf16 = d.dtype == DPSGD_BF16;
  if (d.B * d.T <= kFewRows && d.V > 8 * part_entries(d.dtype)) return true;
  if (loss) return d.V > (bf16 ? Held<uint16_t, 1024, 16>::kMost : Held<float, 1024, 16>::kMost);
  return k > 0 && d.V > (bf16 ? Held<uint16_t, 512, 16>::kMost : Held<float, 512, 16>::kMost);
}

// The workspace: log probabilities of the rows, then the parts' sums and keys.
struct Plan {
  size_t sums, keys, bytes;   // offsets
  int32_t parts, size;        // parts of a row (0: whole rows) and their entries
};

Plan plan_of(const dpsgd_logits& d, int32_t k, bool loss) {
  Plan p{};
  const size_t rows = (size_t)(d.B * d.T);
  p.sums = p.keys = p.bytes = round_up(rows * sizeof(float), 16);
  if (in_parts(d, k, loss)) {
    // Equal parts, of whole vectors.
    const int64_t n = ceil_div(d.V, part_entries(d.dtype));
    p.size = (int32_t)round_up((size_t)ceil_div(d.V, n), 64);
    p.parts = (int32_t)ceil_div(d.V, p.size);
    p.keys = p.sums + rows * (size_t)p.parts * sizeof(float4);
    p.bytes = p.keys + rows * (size_t)p.parts * (size_t)k * sizeof(uint64_t);
  }
  return p;
}

template <class T>
int launch_parts_of(const TokenArgs& a, const Parts& parts, hipStream_t stream) {
  const uint32_t grid = grid_of(a.rows * parts.n);
  hipLaunchKernelGGL(token_part_kernel<T>, dim3(grid), dim3(kThreads), 0, stream, a, parts);
  if (check_launch() != DPSGD_OK) return DPSGD_ERR_HIP;
  if (a.dlogits)
    hipLaunchKernelGGL(token_part_loss_kernel<T>, dim3(grid), dim3(kThreads), 0, stream, a, parts);
  else
    hipLaunchKernelGGL(token_join_kernel<T>, dim3(grid_of(a.rows)), dim3(kThreads), 0, stream, a, parts);
  return check_launch();
}

int launch_rows(const TokenArgs& a, const dpsgd_logits& d, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(d, a.k, a.dlogits != nullptr);
  const bool bf16 = d.dtype == DPSGD_BF16;
  if (p.parts) {
    char* ws = static_cast<char*>(workspace);
    const Parts parts{reinterpret_cast<float4*>(ws + p.sums), reinterpret_cast<uint64_t*>(ws + p.keys), p.parts, p.size};
    return bf16 ? launch_parts_of<uint16_t>(a, parts, stream) : launch_parts_of<float>(a, parts, stream);
  }
  if (a.dlogits)
    return bf16 ? launch_rows_of<uint16_t, true>(a, stream) : launch_rows_of<float, true>(a, stream);
  return bf16 ? launch_rows_of<uint16_t, false>(a, stream) : launch_rows_of<float, false>(a, stream);
}

template <class T>
int launch_backward_of(const TokenArgs& a, hipStream_t stream) {
  const int64_t wave = Held<T, 64, kPartVecs>::kMost, part = PartHeld<T>::kMost;
  if (a.V <= wave) {
    hipLaunchKernelGGL((token_backward_kernel<T, 64>), dim3(grid_of(ceil_div(a.rows, 4))), dim3(kThreads), 0, stream, a, 1);
  } else {
    const int64_t parts = ceil_div(a.V, part);
    hipLaunchKernelGGL((token_backward_kernel<T, kThreads>), dim3(grid_of(a.rows * parts)), dim3(kThreads), 0, stream,
                       a, (int32_t)parts);
  }
  return check_launch();
}

}  // namespace

size_t token_workspace_bytes(const dpsgd_logits& d, int32_t k) {
  const size_t bytes = plan_of(d, k, false).bytes, loss = k == 0 ? plan_of(d, 0, true).bytes : 0;
  return bytes > loss ? bytes : loss;
}

int launch_token_logprobs(const dpsgd_logits& d, const void* logits, float* logprobs, float* lse,
                          float* entropy, int32_t k, int64_t* top_ids, float* top_logprobs,
                          void* workspace, hipStream_t stream) {
  TokenArgs a = common_args(d, logits);
  a.logp_out = logprobs;
  a.lse_out = lse;
  a.entropy_out = entropy;
  a.k = k;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  return launch_rows(a, d, workspace, stream);
}

int launch_token_backward(const dpsgd_logits& d, const void* logits, const float* lse,
                          const float* entropy, const float* g_logp, const float* g_lse,
                          const float* g_entropy, void* dlogits, int64_t dlogits_stride,
                          hipStream_t stream) {
  TokenArgs a = common_args(d, logits);
  a.lse = lse;
  a.entropy = entropy;
  a.g_logp = g_logp;
  a.g_lse = g_lse;
  a.g_entropy = g_entropy;
  a.dlogits = dlogits;
  a.grad_stride = dlogits_stride;
  return d.dtype == DPSGD_BF16 ? launch_backward_of<uint16_t>(a, stream) : launch_backward_of<float>(a, stream);
}

int launch_token_loss(const dpsgd_logits& d, const void* logits, const float* weights,
                      float* losses, float* logprobs, void* dlogits, int64_t dlogits_stride,
                      void* workspace, hipStream_t stream) {
  TokenArgs a = common_args(d, logits);
  a.weights = weights;
  a.dlogits = dlogits;
  a.grad_stride = dlogits_stride;
  a.losses = d.T == 1 ? losses : nullptr;
  a.logp_out = logprobs || !losses || d.T == 1 ? logprobs : static_cast<float*>(workspace);
  const int st = launch_rows(a, d, workspace, stream);
  if (st != DPSGD_OK || !losses || d.T == 1) return st;
  // A wave an example up to two rows a lane (this launch's share of the call, by waves and by
  // workgroups: 4096 x 8 2.8 and 4.9 us, 256 x 128 2.3 and 2.3, 6 x 509 6.5 and 2.5).
  if (d.T <= 128)
    hipLaunchKernelGGL(token_losses_kernel<64>, dim3(grid_of(ceil_div(d.B, 4))), dim3(kThreads), 0,
                       stream, a, a.logp_out, losses, d.B, d.T);
  else
    hipLaunchKernelGGL(token_losses_kernel<kThreads>, dim3(grid_of(d.B)), dim3(kThreads), 0, stream,
                       a, a.logp_out, losses, d.B, d.T);
  return check_launch();
}

}  // namespace dpsgd
