// Log-probabilities of given tokens with entropy and top alternatives, the gradient back to the logits, and the
// gradient of the clipped objective: the learner's row-wise operators on a [R][V] matrix of logits.
//
// With s_v = (z_v - zmax) / T, l = sum_v e^{s_v}:
//   log p_y = s_y - log l,   H = log l - (1/l) sum_v e^{s_v} s_v,
//   dL/dz_v = (1/T) [ a (1[v = y] - p_v) - b p_v (log p_v + H) ]   for upstream gradients a of log p_y and b of H.
// An exponent is one FMA, z c - K with c = log2(e) / T and K the rounded product of c and the reference, with z floored
// in its own format; rows whose maximum is too large or too low for that are summed a second time with the difference
// formed before it is scaled.  So a row may sit at any offset, and a row whose every entry is the type's lowest value is
// an ordinary (uniform) row.  All sums are fp32.

#include <cmath>
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "objective.cuh"
#include "ptx.cuh"

namespace echo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFarBelow = -512.0f;         // stands for exponents whose power of 2 is 0, where 0 * -inf would be formed

// ---- element formats: 0 bf16, 1 IEEE half, 2 fp32 ----------------------------------------------
template <int FMT> struct Fmt { static constexpr int kBytes = FMT == 2 ? 4 : 2, kPerVec = 16 / kBytes; };

template <int FMT> __device__ __forceinline__ float load_elem(const void *p, size_t i) {
  if (FMT == 2) return static_cast<const float *>(p)[i];
  return widen16(static_cast<const uint16_t *>(p)[i], FMT == 1);
}
template <int FMT> __device__ __forceinline__ void store_elem(void *p, size_t i, float v) {
  if (FMT == 2) static_cast<float *>(p)[i] = v;
  else static_cast<uint16_t *>(p)[i] = cvt16(v, FMT == 1);
}
// -inf in every lane of a vector: the filling of loads past the end of a row
template <int FMT> __device__ __forceinline__ uint4 neg_inf_vec() {
  const uint32_t w = FMT == 2 ? 0xff800000u : FMT == 0 ? 0xff80ff80u : 0xfc00fc00u;
  return make_uint4(w, w, w, w);
}
__device__ __forceinline__ uint4 load_stream(const uint4 *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
// for memory that this launch also writes (in place): not through the read-only path
__device__ __forceinline__ uint4 load_once(const uint4 *p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}
using ptx::add2;
using ptx::ex2;
using ptx::fma2;
using ptx::mul2;
// elements 2i and 2i+1 of a vector as fp32
template <int FMT> __device__ __forceinline__ float2 pair_of(const uint4 &v, int i) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (FMT == 2) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  return widen16x2(w[i], FMT == 1);
}
template <int FMT> __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
  if (FMT == 0) {
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&m);
  }
  const __half2 m = __hmax2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&m);
}
// A value far below every logit that can matter (checked at the row's end), as a word of the format and as a float.
template <int FMT> struct Floor;
template <> struct Floor<0> { static constexpr uint32_t kWord = 0xf149f149u; static constexpr float kValue = -9.95e29f; };
template <> struct Floor<1> { static constexpr uint32_t kWord = 0xfbfffbffu; static constexpr float kValue = -65504.f; };
template <> struct Floor<2> { static constexpr uint32_t kWord = 0xf149f2cau; static constexpr float kValue = -1e30f; };
// a vector with its elements raised to at least that (NaN stays)
template <int FMT> __device__ __forceinline__ uint4 floored(const uint4 &v) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo = Floor<FMT>::kWord;
    if constexpr (FMT == 2) {
      asm("max.NaN.f32 %0, %1, %2;" : "=f"(reinterpret_cast<float &>(w[i])) : "f"(__uint_as_float(w[i])), "f"(__uint_as_float(lo)));
    } else if constexpr (FMT == 0) {
      const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<__nv_bfloat162 *>(&w[i]), *reinterpret_cast<__nv_bfloat162 *>(&lo));
      w[i] = *reinterpret_cast<const uint32_t *>(&m);
    } else {
      const __half2 m = __hmax2_nan(*reinterpret_cast<__half2 *>(&w[i]), *reinterpret_cast<__half2 *>(&lo));
      w[i] = *reinterpret_cast<const uint32_t *>(&m);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// largest element of N vectors (NaN is passed over)
template <int FMT, int N> __device__ __forceinline__ float max_of(const uint4 (&v)[N]) {
  if (FMT == 2) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i)
      m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(v[i].x), __uint_as_float(v[i].y))),
                fmaxf(__uint_as_float(v[i].z), __uint_as_float(v[i].w)));
    return m;
  }
  uint32_t m = neg_inf_vec<FMT>().x;
#pragma unroll
  for (int i = 0; i < N; ++i)
    m = max_word<FMT>(m, max_word<FMT>(max_word<FMT>(v[i].x, v[i].y), max_word<FMT>(v[i].z, v[i].w)));
  const float2 f = widen16x2(m, FMT == 1);
  return fmaxf(f.x, f.y);
}

// ---- running statistics of a row --------------------------------------------------------------
// m: largest logit so far; l = sum 2^x, t = sum 2^x x over x = z c - K, c = log2(e) / T, K = max(fp32(m c), k_min).
// One FMA an element: the reference is K itself, so that K's rounding is no error; m c - K enters once, at the end.
// z is raised to the floor first, so that -inf makes no 0 * -inf.  k_min is at least -2^23 (below it K's rounding alone
// would be more than 1: x could be large; such a maximum counts for nothing beside an ordinary one) and so far above
// the floor's x that a floored element counts as 0.  A row whose own maximum is not ordinary (nothing left, everything
// at some huge negative value, infinities, extreme temperatures) is found at its end and summed again by sum_plainly.
struct RowStats {
  float m, l, t;
};
struct Scale {
  float c, k_min;
};
__device__ __forceinline__ float reference(float m, const Scale &s) { return fmaxf(__fmul_rn(m, s.c), s.k_min); }
__device__ __forceinline__ bool ordinary(float m, const Scale &s) {
  const float k = __fmul_rn(m, s.c);
  return k >= s.k_min && k <= 8388608.0f;
}
__device__ __forceinline__ void merge(RowStats &a, const RowStats &b, const Scale &s) {
  const float m = fmaxf(a.m, b.m), k = reference(m, s);
  const float da = reference(a.m, s) - k, db = reference(b.m, s) - k, fa = ex2(da), fb = ex2(db);
  a.t = fa * fmaf(da, a.l, a.t) + fb * fmaf(db, b.l, b.t);
  a.l = fa * a.l + fb * b.l;
  a.m = m;
}
// moves the reference to a larger maximum
__device__ __forceinline__ void raise(RowStats &a, float m, const Scale &s) {
  const float d = reference(a.m, s) - reference(m, s), f = ex2(d);
  a.t = f * fmaf(d, a.l, a.t);
  a.l *= f;
  a.m = m;
}
__device__ __forceinline__ RowStats shfl_stats(const RowStats &a, int o) {
  return RowStats{__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.l, o),
                  __shfl_xor_sync(0xffffffffu, a.t, o)};
}

// ---- order of the alternatives ----------------------------------------------------------------
// One 64-bit number per entry: larger logit first, equal ones by the lower id.  0: no entry (-inf and NaN are none).
__device__ __forceinline__ uint64_t entry_key(float z, uint32_t id) {
  return (static_cast<uint64_t>(order_key(z + 0.0f)) << 32) | (0xffffffffu - id);      // + 0: -0 equals 0
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t u = static_cast<uint32_t>(key >> 32);
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}
__device__ __forceinline__ bool listable(float z) { return z > -INFINITY; }           // false for NaN

constexpr int kTopMax = 32;        // alternatives per row
constexpr int kCandidates = 1024;  // candidates gathered per CTA before the exact selection takes over
constexpr int kHotPieces = 512;
constexpr int kRescan = 2;         // vectors per thread and turn there
constexpr int kUnroll = 4;         // 16-byte vectors per thread and step
template <int NT> constexpr int kPieces = 1024 / NT;       // parts of a thread's elements whose maxima are kept
constexpr uint32_t kNoEntry = 0x007fffffu;         // order_key(-inf)
constexpr int kMaxSplit = 8;       // CTAs per row (one cluster)
constexpr int kMaxVocab = 1 << 24; // (find_alternatives divides places of a row in fp32)

struct TopShared {
  uint32_t piece[1024];                      // order keys of the pieces' maxima
  uint32_t sorted[8][32];                    // the threads' maxima, each warp's in descending order
  uint32_t bound;
  alignas(16) uint64_t cand[kCandidates + 2];
  uint64_t best[kTopMax];                    // this CTA's alternatives, sorted
  alignas(16) uint64_t gathered[kMaxSplit * kTopMax + 2];      // first CTA of a cluster: everybody's
  int hot[kHotPieces];
  uint32_t hist[256];
  int n_cand, n_hot, need, warp_count[16];
  uint32_t prefix;
};
struct NoTop {};

// What a row of the launch scores and where its results go.  Plain calls: row r of the logits, token tokens[r],
// outputs at r.  Scoring whole trajectories (T > 0): the row's place in [sequences][T] is flat = tok_idx[r] + 1, or
// r * T without tok_idx, rows_per_logit_row of them share a logits row, and places after a sequence's first end token
// hold log-probability 0, entropy 0 and no alternatives.
struct LogprobArgs {
  const void *logits;
  int64_t row_stride;
  int R, V;
  const int32_t *tokens;
  float c, inv_temperature;
  float k_min;                 // lowest reference (set by logprobs_launch)
  int top_k;
  float *out_logprobs, *out_entropy;
  float2 *out_stats;
  int32_t *out_top_ids;
  float *out_top_logprobs;
  int T, rows_per_logit_row;
  const int32_t *tok_idx, *first_end;
  int *status;
};

// Exact selection of the k first entries of elements [begin, end) of a row, whatever their distribution: radix
// selection of the k-th largest value, then everything above it and the lowest ids that equal it.  Reached when more
// candidates than the buffer holds tie with, or sit above, the bound of the one-pass filter (constant rows, sorted rows,
// rows whose masked ids share a finite value with fewer than k ids above it).  It reads the elements five times out of
// L2 (four digits, then the entries), one element a thread and turn, and is slow: eight ids above the type's lowest
// value and 20 alternatives, 256 x 151936 bf16 in 1094 us and 2048 rows in 6580, against 31 and 123 with -inf instead.
template <int FMT, int NT>
__device__ __noinline__ void select_exact(const void *row, int begin, int end, int k, TopShared &sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    sh.n_cand = 0;
    sh.prefix = 0;
    sh.need = k;
  }
  __syncthreads();
  bool all = false;                          // fewer than k entries: list them all
  for (int shift = 24; shift >= 0 && !all; shift -= 8) {
    for (int i = tid; i < 256; i += NT) sh.hist[i] = 0;
    __syncthreads();
    const uint32_t prefix = sh.prefix;
    for (int base = begin; base < end; base += NT) {          // same trip count in every thread
      const int i = base + tid;
      const float z = i < end ? load_elem<FMT>(row, i) : -INFINITY;
      const uint32_t key = order_key(z + 0.0f);
      const bool in = listable(z) && (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)));
      const int bin = in ? static_cast<int>((key >> shift) & 255u) : -1;
      const int bin0 = __shfl_sync(0xffffffffu, bin, 0);
      if (__all_sync(0xffffffffu, bin == bin0)) {             // equal values: one addition for the warp
        if (lane == 0 && bin0 >= 0) atomicAdd(&sh.hist[bin0], 32u);
      } else if (bin >= 0) {
        atomicAdd(&sh.hist[bin], 1u);
      }
    }
    __syncthreads();
    if (tid == 0) {
      int need = sh.need, b = 255;
      while (b >= 0 && static_cast<int>(sh.hist[b]) < need) need -= static_cast<int>(sh.hist[b--]);
      if (b < 0) sh.need = 0;                                  // only possible in the first pass
      else {
        sh.need = need;
        sh.prefix = prefix | (static_cast<uint32_t>(b) << shift);
      }
    }
    __syncthreads();
    all = sh.need == 0;
  }
  // sh.prefix is the k-th largest key, sh.need how many of the entries equal to it belong to the first k
  const uint32_t cut = all ? 0u : sh.prefix;
  const int need = sh.need;
  int taken = 0;
  for (int base = begin; base < end; base += NT) {
    const int i = base + tid;
    const float z = i < end ? load_elem<FMT>(row, i) : -INFINITY;
    const uint32_t key = order_key(z + 0.0f);
    if (listable(z) && key > cut) sh.cand[atomicAdd(&sh.n_cand, 1)] = entry_key(z, i);       // fewer than k <= 32
    if (taken < need) {                                        // uniform: ids ascend with the thread index
      const bool eq = listable(z) && key == cut;
      const unsigned votes = __ballot_sync(0xffffffffu, eq);
      if (lane == 0) sh.warp_count[warp] = __popc(votes);
      __syncthreads();
      int before = taken, total = 0;
      for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) before += sh.warp_count[w];
        total += sh.warp_count[w];
      }
      before += __popc(votes & ((1u << lane) - 1u));
      if (eq && before < need) sh.cand[atomicAdd(&sh.n_cand, 1)] = entry_key(z, i);
      taken += total;
      __syncthreads();
    }
  }
  __syncthreads();
}

// The sums of a whole row about its maximum m with x = (z - m) c, which holds for any m and c: l and t in every thread.
template <int FMT, int NT>
__device__ __noinline__ float2 sum_plainly(const void *row, int V, float m, float c, float *scratch) {
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, t = 0.f;
  for (int i = threadIdx.x; i < V; i += NT) {
    const float x = (load_elem<FMT>(row, i) - ref) * c, e = ex2(x);
    l += e;
    t = fmaf(e, fmaxf(x, kFarBelow), t);                       // (-inf would make 0 * -inf)
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    l += __shfl_xor_sync(0xffffffffu, l, o);
    t += __shfl_xor_sync(0xffffffffu, t, o);
  }
  if ((threadIdx.x & 31) == 0) {
    scratch[threadIdx.x >> 5] = l;
    scratch[NT / 32 + (threadIdx.x >> 5)] = t;
  }
  __syncthreads();
  l = t = 0.f;
  for (int w = 0; w < NT / 32; ++w) {
    l += scratch[w];
    t += scratch[NT / 32 + w];
  }
  return make_float2(l, t);
}

// sorts n entries by counting how many precede each; the first kTopMax go to dst.  src[n] is 0 where n is odd.
__device__ __forceinline__ void rank_entries(const uint64_t *src, int n, uint64_t *dst, int nt) {
  const ulonglong2 *pairs = reinterpret_cast<const ulonglong2 *>(src);
  for (int i = threadIdx.x; i < n; i += nt) {
    const uint64_t mine = src[i];
    if (!mine) continue;
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < (n + 1) / 2; ++j) {
      const ulonglong2 q = pairs[j];
      rank += (q.x > mine ? 1 : 0) + (q.y > mine ? 1 : 0);
    }
    if (rank < kTopMax) dst[rank] = mine;
  }
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_first(const void *p) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(ptx::smem_u32(p)));
  return a;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// The CTA's alternatives, sorted, into sh.best.  (Not inlined: the registers of the streaming loop are worth more than
// the call: 112 against 116 us for 8 alternatives at 2048 x 151936 bf16, where scoring alone takes 101.)
template <int FMT, int NT>
__device__ __noinline__ void find_alternatives(const void *row, const uint4 *vec, int begin, int end, int head, int n_vec,
                                               int per, int k, TopShared &sh) {
  constexpr int kPerVec = Fmt<FMT>::kPerVec, kWarps = NT / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tail0 = begin + head + n_vec * kPerVec;          // elements behind the whole vectors
  // Lower bound of the k-th largest entry: the k-th largest of the threads' maxima (k entries reach it; not many more
  // than k do).  Every warp sorts its 32, and an element of one list finds its place among all by bisecting the others.
  uint32_t most = sh.piece[tid];
#pragma unroll
  for (int i = 1; i < kPieces<NT>; ++i) most = max(most, sh.piece[i * NT + tid]);
#pragma unroll
  for (int span = 2; span <= 32; span <<= 1)
#pragma unroll
    for (int o = span >> 1; o > 0; o >>= 1) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, most, o);
      most = ((lane & o) == 0) == ((lane & span) == 0 || span == 32) ? max(most, other) : min(most, other);
    }
  sh.sorted[warp][lane] = most;
  if (tid == 0) sh.n_cand = sh.n_hot = 0;
  if (tid < kTopMax) sh.best[tid] = 0;
  __syncthreads();
  if (lane < k) {
    int before[kWarps];                                      // entries of each list that precede this one
#pragma unroll
    for (int w = 0; w < kWarps; ++w) before[w] = 0;
#pragma unroll
    for (int half = 16; half > 0; half >>= 1)
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const uint32_t other = sh.sorted[w][before[w] + half - 1];
        if (other > most || (other == most && w < warp)) before[w] += half;
      }
    int rank = lane;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
      if (w != warp) {
        const uint32_t other = sh.sorted[w][before[w]];      // (at most 31 so far: one more may precede)
        rank += before[w] + (other > most || (other == most && w < warp) ? 1 : 0);
      }
    if (rank == k - 1) sh.bound = most;
  }
  __syncthreads();
  const uint32_t bound_key = sh.bound;
  const float bound = key_value(static_cast<uint64_t>(bound_key) << 32);
#pragma unroll
  for (int i = 0; i < kPieces<NT>; ++i) {
    const uint32_t key = sh.piece[i * NT + tid];
    if (key >= bound_key && key > kNoEntry) {
      const int at = atomicAdd(&sh.n_hot, 1);
      if (at < kHotPieces) sh.hot[at] = i * NT + tid;
    }
  }
  __syncthreads();
  const int n_hot = sh.n_hot;
  if (n_hot <= kHotPieces) {
    auto offer = [&](float z, int id) {
      if (z >= bound && listable(z)) {
        const int at = atomicAdd(&sh.n_cand, 1);
        if (at < kCandidates) sh.cand[at] = entry_key(z, static_cast<uint32_t>(id));
      }
    };
    if (tid < head) offer(load_elem<FMT>(row, begin + tid), begin + tid);
    if (tail0 + tid < end) offer(load_elem<FMT>(row, tail0 + tid), tail0 + tid);
    // a few vectors of the hot pieces per thread and turn, requested together
    const float pieces_per_vec = 1.0f / static_cast<float>(per);
    // at most 512 pieces of kMaxVocab / 4 / 1024 + 8 vectors: w + 1/2 is exact in fp32, and the quotient is off by less
    // than 512 * 2^-23, half a vector's share of a piece being 1.2e-4
    const int total = n_hot * per;
    for (int w0 = tid; w0 < total; w0 += kRescan * NT) {
      uint4 q[kRescan];
      int at[kRescan];
#pragma unroll
      for (int b = 0; b < kRescan; ++b) {
        const int w = w0 + b * NT;
        at[b] = n_vec;
        if (w < total) {
          const int p = static_cast<int>((static_cast<float>(w) + 0.5f) * pieces_per_vec), which = sh.hot[p];
          at[b] = ((which / NT) * per + (w - p * per)) * NT + which % NT;
        }
        q[b] = at[b] < n_vec ? load_stream(vec + at[b]) : neg_inf_vec<FMT>();
      }
      // bit j: element j of the thread's vectors is an entry at or above the bound (few are)
      uint32_t found = 0;
#pragma unroll
      for (int b = 0; b < kRescan; ++b)
#pragma unroll
        for (int e = 0; e < kPerVec / 2; ++e) {
          const float2 z = pair_of<FMT>(q[b], e);
          if (z.x >= bound && listable(z.x)) found |= 1u << (b * kPerVec + 2 * e);
          if (z.y >= bound && listable(z.y)) found |= 2u << (b * kPerVec + 2 * e);
        }
      for (; found; found &= found - 1) {
        const int which = __ffs(found) - 1;
        float z = 0.f;
        int id = 0;
#pragma unroll
        for (int b = 0; b < kRescan; ++b)
#pragma unroll
          for (int e = 0; e < kPerVec / 2; ++e)
            if (which / 2 == (b * kPerVec + 2 * e) / 2) {
              const float2 pair = pair_of<FMT>(q[b], e);
              z = (which & 1) ? pair.y : pair.x;
              id = begin + head + at[b] * kPerVec + 2 * e + (which & 1);
            }
        offer(z, id);
      }
    }
    __syncthreads();
  }
  if (n_hot > kHotPieces || sh.n_cand > kCandidates) {
    __syncthreads();
    select_exact<FMT, NT>(row, begin, end, k, sh);
  }
  const int n_cand = sh.n_cand;
  if (tid == 0) sh.cand[n_cand] = 0;
  __syncthreads();
  rank_entries(sh.cand, n_cand, sh.best, NT);
  __syncthreads();
}

// One cluster of `split` CTAs per row (split = 1: one CTA), each with a contiguous share of the row, one pass.
// Bound by HBM and, for 16-bit logits, almost as much by the exponentials (16 a cycle and SM): 2048 x 151936 bf16 in
// 112 to 115 us under sustained load, 5.4 to 5.6 TB/s, where power holds the SM clock at 1.62 GHz; 100 us, 6.2 TB/s, in
// short bursts (exponential unit 71 % busy at 1024 such rows).
// A thread keeps (m, l, t) of its own elements and moves the reference only when a step of its vectors exceeds it.
// Alternatives cost no second pass: the threads also keep the maxima of 1024 parts of the CTA's elements ("pieces");
// from these comes a lower bound of the k-th largest logit, and only the pieces that reach it, little more than k,
// are looked at again for entries that reach it.
template <int FMT, int NT, bool TOP>
__global__ void __launch_bounds__(NT, 1024 / NT)
token_logprobs_kernel(const __grid_constant__ LogprobArgs a, int split) {
  constexpr int kPerVec = Fmt<FMT>::kPerVec, kBytes = Fmt<FMT>::kBytes, kWarps = NT / 32;
  __shared__ RowStats warp_stats[kWarps];
  __shared__ RowStats cta_stats[kMaxSplit];
  __shared__ typename std::conditional<TOP, TopShared, NoTop>::type top_mem;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = static_cast<int>(blockIdx.x) / split;
  const int rank = split > 1 ? static_cast<int>(cluster_rank()) : 0;
  // ---- which token, where to
  size_t flat = static_cast<size_t>(r);
  if (a.T > 0) {
    flat = a.tok_idx ? static_cast<size_t>(a.tok_idx[r]) + 1 : static_cast<size_t>(r) * a.T;
    if (a.first_end && static_cast<int>(flat % a.T) > a.first_end[flat / a.T]) {
      if (rank == 0) {                        // the whole cluster leaves here
        if (tid == 0) {
          if (a.out_logprobs) a.out_logprobs[flat] = 0.f;
          if (a.out_entropy) a.out_entropy[flat] = 0.f;
        }
        if (TOP && tid < a.top_k) {
          a.out_top_ids[flat * a.top_k + tid] = -1;
          a.out_top_logprobs[flat * a.top_k + tid] = -INFINITY;
        }
      }
      return;
    }
  }
  const int token = a.tokens ? a.tokens[flat] : -1;
  if (!TOP && !a.out_entropy && !a.out_stats && token < 0 && a.T == 0) {      // (a trajectory has no places without a token)
    if (rank == 0 && tid == 0 && a.out_logprobs) a.out_logprobs[flat] = 0.f;
    return;
  }
  if (split > 1) cluster_arrive();            // (waited for below: the first CTA's memory is written by the others)
  const int zr = a.T > 0 ? r / a.rows_per_logit_row : r;
  const char *row = static_cast<const char *>(a.logits) + static_cast<size_t>(zr) * a.row_stride * kBytes;
  // ---- this CTA's share of the row
  const int share = split > 1 ? ((a.V + split - 1) / split + 63) / 64 * 64 : a.V;
  const int begin = min(rank * share, a.V), end = min(begin + share, a.V);
  // elements before the first 16-byte boundary, whole vectors, the rest
  const int lead = static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row + static_cast<size_t>(begin) * kBytes) & 15)) & 15) / kBytes;
  const int head = min(lead, end - begin);
  const int n_vec = (end - begin - head) / kPerVec;
  const int tail0 = begin + head + n_vec * kPerVec;
  const uint4 *vec = reinterpret_cast<const uint4 *>(row + static_cast<size_t>(begin + head) * kBytes);
  const float c = a.c;
  const Scale scale{a.c, a.k_min};
  RowStats st{-INFINITY, 0.f, 0.f};

  auto absorb = [&](const uint4 (&v)[kUnroll]) -> float {
    const float bm = max_of<FMT>(v);
    if (bm > st.m) raise(st, bm, scale);
    const float k = -reference(st.m, scale);
    const float2 kk = make_float2(k, k), cc = make_float2(c, c);
    float2 l0 = make_float2(st.l, 0.f), t0 = make_float2(st.t, 0.f);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint4 q = floored<FMT>(v[u]);
#pragma unroll
      for (int i = 0; i < kPerVec / 2; ++i) {
        const float2 x = fma2(pair_of<FMT>(q, i), cc, kk);
        const float2 e = make_float2(ex2(x.x), ex2(x.y));
        l0 = add2(l0, e);
        t0 = fma2(e, x, t0);
      }
    }
    st.l = l0.x + l0.y;
    st.t = t0.x + t0.y;
    return bm;
  };
  auto fetch = [&](uint4 (&v)[kUnroll], int step) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = (step * kUnroll + u) * NT + tid;
      v[u] = i < n_vec ? load_stream(vec + i) : neg_inf_vec<FMT>();
    }
  };
  auto absorb_one = [&](float z) {
    if (z > st.m) raise(st, z, scale);
    const float raised = z < Floor<FMT>::kValue ? Floor<FMT>::kValue : z;      // (NaN stays)
    const float x = fmaf(raised, c, -reference(st.m, scale)), e = ex2(x);
    st.l += e;
    st.t = fmaf(e, x, st.t);
  };

  const int steps = (n_vec + NT * kUnroll - 1) / (NT * kUnroll);
  const int piece_steps = (steps + 2 * kPieces<NT> - 1) / (2 * kPieces<NT>) * 2;      // (whole turns of the loop below)
  {
    uint4 va[kUnroll], vb[kUnroll];
    fetch(va, 0);
    // the few elements outside whole vectors, under the first loads' latency
    if (tid < head) absorb_one(load_elem<FMT>(row, begin + tid));
    if (tail0 + tid < end) absorb_one(load_elem<FMT>(row, tail0 + tid));
    int s = 0;
    if constexpr (TOP) {
#pragma unroll 1
      for (int h = 0; h < kPieces<NT>; ++h) {
        float most = -INFINITY;
        for (const int until = min((h + 1) * piece_steps, steps); s < until; s += 2) {
          fetch(vb, s + 1);
          most = fmaxf(most, absorb(va));
          fetch(va, s + 2);
          if (s + 1 < steps) most = fmaxf(most, absorb(vb));
        }
        top_mem.piece[h * NT + tid] = order_key(most + 0.0f);          // (+ 0: -0 equals 0)
      }
    } else {
      for (; s < steps; s += 2) {
        fetch(vb, s + 1);
        absorb(va);
        fetch(va, s + 2);
        if (s + 1 < steps) absorb(vb);
      }
    }
  }
  // ---- join the threads' statistics
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) merge(st, shfl_stats(st, o), scale);
  if (lane == 0) warp_stats[warp] = st;
  // the token's own logit, wanted at the end: requested here, under the joins
  const float taken = tid == 0 && rank == 0 && token >= 0 && token < a.V ? load_elem<FMT>(row, token) : 0.f;
  __syncthreads();
  if (warp == 0) {
    st = lane < kWarps ? warp_stats[lane] : RowStats{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) merge(st, shfl_stats(st, o), scale);
  }
  if constexpr (TOP) find_alternatives<FMT, NT>(row, vec, begin, end, head, n_vec, piece_steps * kUnroll, a.top_k, top_mem);
  // ---- join the CTAs of the row
  if (split > 1) {
    cluster_wait();                          // every CTA of the cluster runs: its shared memory may be written
    if (tid == 0) {
      const uint32_t dst = map_to_first(&cta_stats[rank]);
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(st.m) : "memory");
      asm volatile("st.shared::cluster.f32 [%0 + 4], %1;" ::"r"(dst), "f"(st.l) : "memory");
      asm volatile("st.shared::cluster.f32 [%0 + 8], %1;" ::"r"(dst), "f"(st.t) : "memory");
    }
    if constexpr (TOP) {
      if (tid < a.top_k)
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(map_to_first(&top_mem.gathered[rank * a.top_k + tid])),
                     "l"(top_mem.best[tid])
                     : "memory");
    }
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    if constexpr (TOP) {
      TopShared &sh = top_mem;
      if (tid < kTopMax) sh.best[tid] = 0;
      if (tid == kTopMax) sh.gathered[split * a.top_k] = 0;
      __syncthreads();
      rank_entries(sh.gathered, split * a.top_k, sh.best, NT);
      __syncthreads();
    }
    if (warp == 0) {
      st = lane < split ? cta_stats[lane] : RowStats{-INFINITY, 0.f, 0.f};
#pragma unroll
      for (int o = kMaxSplit / 2; o > 0; o >>= 1) merge(st, shfl_stats(st, o), scale);
    }
  }
  // ---- rows without an ordinary maximum (the CTA that holds the joined statistics decides)
  if (tid == 0) cta_stats[0] = st;
  __syncthreads();
  st = cta_stats[0];
  float log_l = logf(st.l);
  if (ordinary(st.m, scale)) {
    log_l -= kLn2 * fmaf(st.m, c, -reference(st.m, scale));
  } else if (!(st.m == -INFINITY && st.l == 0.f)) {           // (nothing left: the sums are 0 already)
    const float2 sums = sum_plainly<FMT, NT>(row, a.V, st.m, c, &warp_stats[0].m);
    st.l = sums.x;
    st.t = sums.y;
    log_l = logf(st.l);
  }
  if (warp != 0) return;
  const bool empty = st.l == 0.f;                             // nothing left in the row (all -inf)
  if (lane == 0) {
    if (a.out_logprobs) {
      float lp = 0.f;
      if (token >= a.V || (a.T > 0 && token < 0)) {
        lp = NAN;
        if (a.status) atomicExch(a.status, STATUS_BAD_TOKEN);
      } else if (token >= 0) {
        lp = empty ? -INFINITY : (taken - st.m) * a.inv_temperature - log_l;
      }
      a.out_logprobs[flat] = lp;
    }
    if (a.out_entropy) a.out_entropy[flat] = empty ? 0.f : logf(st.l) - kLn2 * (st.t / st.l);
    if (a.out_stats) a.out_stats[flat] = make_float2(st.m, log_l);
  }
  if constexpr (TOP) {
    if (lane < a.top_k) {
      const uint64_t key = top_mem.best[lane];
      const size_t o = flat * a.top_k + lane;
      a.out_top_ids[o] = key ? static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(key)) : -1;
      a.out_top_logprobs[o] = key ? (key_value(key) - st.m) * a.inv_temperature - log_l : -INFINITY;
    }
  }
}

template <int FMT, int NT>
cudaError_t launch_logprobs(const LogprobArgs &a, int split, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.R) * split);
  cfg.blockDim = dim3(NT);
  cfg.stream = s;
  // (Not started early behind the kernel before it: the CTAs of a launch that fits in one round would be dealt to
  // whatever SMs have room at that moment, and unevenly: 400 rows of 151936 bf16 values in 31.7 us, not 26.5.)
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 1 : 0;
  return a.top_k > 0 ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<FMT, NT, true>, a, split)
                     : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<FMT, NT, false>, a, split);
}
template <int FMT>
cudaError_t launch_logprobs_fmt(const LogprobArgs &a, int split, bool wide, cudaStream_t s) {
  return wide ? launch_logprobs<FMT, 256>(a, split, s) : launch_logprobs<FMT, 128>(a, split, s);
}

// Half values reach down to -65504 only: their lowest reference lies halfway.  Where the floor's x would not vanish
// beside it, or z c may overflow, no maximum is ordinary.
float lowest_reference(int format, float c) {
  const float floor = format == 1 ? Floor<1>::kValue : Floor<2>::kValue * 0.99f;
  const float k_min = format == 1 ? fmaxf(-8388608.0f, -32000.0f * c) : -8388608.0f;
  return c < 1e7f && floor * c < k_min - 200.0f ? k_min : INFINITY;
}

cudaError_t logprobs_launch(LogprobArgs a, int format, cudaStream_t s) {
  a.k_min = lowest_reference(format, a.c);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int64_t row_vecs = static_cast<int64_t>(a.V) * (format == 2 ? 4 : 2) / 16;
  // Few rows are cut over the CTAs of a cluster until the launch has two CTAs per SM.  With alternatives, which cost more
  // to join, one and a half will do unless the parts stay long: 200 rows of 151936 fp32 values with 5 alternatives take
  // 23.9 us in two parts and 28.3 in one, 256 rows 30.2 and 32.0, but bf16 24.2 and 21.4; 64 rows fp32 12.3 us in four and
  // 14.0 in eight.  (Parts of 9496 vectors stay whole and parts of 18992 are cut there; the border of 16384 lies between
  // and was not measured at other vocabularies.)
  int split = 1;
  auto more = [&] {
    const int64_t ctas = a.R * static_cast<int64_t>(split), part = row_vecs / (2 * split);
    return split < kMaxSplit && part >= 512 && (ctas < 3 * sms / 2 || (ctas < 2 * sms && (a.top_k == 0 || part >= 16384)));
  };
  while (more()) split *= 2;
  // Four CTAs of 256 threads or eight of 128 fit an SM.  While the launch fits in one round the larger ones finish sooner
  // (592 rows of 151936 half values: 33.0 against 37.5 us); in a launch of several rounds the smaller ones leave less
  // idle at the end and overlap their beginnings and ends better (3000 x 20000 bf16: 26.0 against 33.4 us; 777 x 50263
  // fp32: 22.8 against 29.2; 2048 x 151936 bf16: 101.0 against 101.8).
  const bool wide = row_vecs > 1024 && static_cast<int64_t>(a.R) * split <= 4 * sms;
  switch (format) {
    case 0: return launch_logprobs_fmt<0>(a, split, wide, s);
    case 1: return launch_logprobs_fmt<1>(a, split, wide, s);
    default: return launch_logprobs_fmt<2>(a, split, wide, s);
  }
}

// ---- gradient -----------------------------------------------------------------------------------
struct BackwardArgs {
  const void *logits;
  int64_t row_stride;
  int R, V;
  const int32_t *tokens;
  float c, inv_temperature;
  const float *entropy;
  const float2 *stats;
  const float *grad_logprobs, *grad_entropy;
  void *out;
  int64_t out_stride;
};
// dz_v = -p_v (A + B log2 p_v) + [v = y] a / T, with A = (a + b H) / T, B = b ln 2 / T, log2 p = (z - m) c - log2 l.
struct RowGrad {
  float m, log2_l, A, B, hot;
  int token;
};
template <bool ENT> __device__ __forceinline__ float2 grad_pair(float2 z, const RowGrad &g, float c) {
  float2 x = mul2(add2(z, make_float2(-g.m, -g.m)), make_float2(c, c));
  x = add2(x, make_float2(-g.log2_l, -g.log2_l));
  const float2 p = make_float2(ex2(x.x), ex2(x.y));
  if (!ENT) return mul2(p, make_float2(-g.A, -g.A));
  x.x = fmaxf(x.x, kFarBelow);
  x.y = fmaxf(x.y, kFarBelow);
  return mul2(p, fma2(x, make_float2(-g.B, -g.B), make_float2(-g.A, -g.A)));
}
template <int FMT> __device__ __forceinline__ uint4 pack_vec(const float (&f)[Fmt<FMT>::kPerVec]) {
  if constexpr (FMT == 2) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  } else {
    return make_uint4(cvt16x2(f[0], f[1], FMT == 1), cvt16x2(f[2], f[3], FMT == 1), cvt16x2(f[4], f[5], FMT == 1),
                      cvt16x2(f[6], f[7], FMT == 1));
  }
}
// 16 bytes that start `bytes` (a multiple of 2) into the 32 bytes lo, hi
__device__ __forceinline__ uint4 bytes_from(const uint4 &lo, const uint4 &hi, int bytes) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (bytes & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (bytes & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const int bits = (bytes & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

constexpr int kBackThreads = 256, kBackUnroll = 2;

// One CTA per slice of a row.  The first vectors are requested before the row's scalars, whose latency would otherwise
// stand in front of every slice, and from then on a step's loads run under the step before it.  Bound by HBM, as many
// bytes written as read: 2048 x 151936 bf16 in 198 us, 6.3 TB/s (205 under sustained load, 6.1 TB/s).  Logits on another
// 16-byte boundary than the output cost a second load a vector: 1024 x 151936 bf16 in 123 us, not 107.  Two vectors a step and six
// CTAs an SM against four and four: 219 against 226 us; ordinary stores against evict-first ones: 213 against 219; eight
// rounds of CTAs against four: 207 against 211; ordinary loads against L1::no_allocate: 198 against 205.
template <int FMT, bool ENT>
__global__ void __launch_bounds__(kBackThreads, 6)
token_logprobs_backward_kernel(const __grid_constant__ BackwardArgs a, int slices, int slice_elems) {
  constexpr int kPerVec = Fmt<FMT>::kPerVec, kBytes = Fmt<FMT>::kBytes;
  early_start_sync();
  const int tid = threadIdx.x;
  const int r = static_cast<int>(blockIdx.x / slices), slice = static_cast<int>(blockIdx.x % slices);
  const int begin = slice * slice_elems, end = min(begin + slice_elems, a.V);
  const char *zrow = static_cast<const char *>(a.logits) + static_cast<size_t>(r) * a.row_stride * kBytes;
  char *orow = static_cast<char *>(a.out) + static_cast<size_t>(r) * a.out_stride * kBytes;
  // whole 16-byte vectors of the output; where the logits lie differently on 16-byte boundaries (a padded or offset
  // row beside a dense output) a vector is cut out of the two aligned ones around it, both inside the row
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(orow + static_cast<size_t>(begin) * kBytes) & 15);
  int head = min(((16 - off) & 15) / kBytes, end - begin);
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(zrow + static_cast<size_t>(begin + head) * kBytes) & 15);
  if (skew && begin + head - skew / kBytes < 0) head = min(head + kPerVec, end - begin);       // would begin before the row
  int n_vec = (end - begin - head) / kPerVec;
  if (skew && n_vec > 0 && begin + head + n_vec * kPerVec + kPerVec - skew / kBytes > a.V) --n_vec;   // would end behind it
  const int tail0 = begin + head + n_vec * kPerVec;
  const uint4 *zv = reinterpret_cast<const uint4 *>(zrow + static_cast<size_t>(begin + head) * kBytes - skew);
  uint4 *ov = reinterpret_cast<uint4 *>(orow + static_cast<size_t>(begin + head) * kBytes);
  auto fetch = [&](uint4 (&q)[kBackUnroll], int step) {
#pragma unroll
    for (int u = 0; u < kBackUnroll; ++u) {
      const int i = (step * kBackUnroll + u) * kBackThreads + tid;
      if (i < n_vec) {
        q[u] = load_once(zv + i);
        if (skew) q[u] = bytes_from(q[u], load_once(zv + i + 1), skew);
      }
    }
  };
  uint4 qa[kBackUnroll], qb[kBackUnroll];
  fetch(qa, 0);
  RowGrad g;
  g.token = a.tokens ? a.tokens[r] : -1;
  const float2 st = a.stats[r];
  const float gl = a.grad_logprobs ? a.grad_logprobs[r] : 0.f;
  const float gb = ENT ? a.grad_entropy[r] : 0.f, H = ENT ? a.entropy[r] : 0.f;
  const bool unknown = g.token >= a.V && gl != 0.f;          // the forward call scored NaN: so is the row's gradient
  const float ga = unknown ? NAN : g.token >= 0 ? gl : 0.f;
  // no gradient arrives, or nothing is left in the row: zeros, whatever the logits hold
  const bool zero = (ga == 0.f && gb == 0.f) || (st.y == -INFINITY && !unknown);
  g.m = st.x;
  g.log2_l = st.y * kLog2e;
  g.hot = ga * a.inv_temperature;
  g.A = (gb != 0.f ? fmaf(gb, H, ga) : ga) * a.inv_temperature;
  g.B = gb * kLn2 * a.inv_temperature;
  const float c = a.c;
  auto one = [&](int i) {
    float d = 0.f;
    if (!zero) {
      const float z = load_elem<FMT>(zrow, i);
      d = grad_pair<ENT>(make_float2(z, z), g, c).x;
      if (i == g.token) d += g.hot;
    }
    store_elem<FMT>(orow, i, d);
  };
  for (int i = begin + tid; i < begin + head; i += kBackThreads) one(i);
  for (int i = tail0 + tid; i < end; i += kBackThreads) one(i);
  if (zero) {
    for (int i = tid; i < n_vec; i += kBackThreads) __stcs(ov + i, make_uint4(0u, 0u, 0u, 0u));
    return;
  }
  auto finish = [&](const uint4 (&q)[kBackUnroll], int step) {
#pragma unroll
    for (int u = 0; u < kBackUnroll; ++u) {
      const int i = (step * kBackUnroll + u) * kBackThreads + tid;
      if (i >= n_vec) continue;
      float f[kPerVec];
#pragma unroll
      for (int e = 0; e < kPerVec / 2; ++e) {
        const float2 d = grad_pair<ENT>(pair_of<FMT>(q[u], e), g, c);
        f[2 * e] = d.x;
        f[2 * e + 1] = d.y;
      }
      const int at = g.token - (begin + head + i * kPerVec);
      if (at >= 0 && at < kPerVec) {
#pragma unroll
        for (int e = 0; e < kPerVec; ++e)
          if (e == at) f[e] += g.hot;
      }
      ov[i] = pack_vec<FMT>(f);
    }
  };
  const int steps = (n_vec + kBackThreads * kBackUnroll - 1) / (kBackThreads * kBackUnroll);
  for (int s = 0; s < steps; s += 2) {
    fetch(qb, s + 1);
    finish(qa, s);
    fetch(qa, s + 2);
    finish(qb, s + 1);
  }
}

template <int FMT> cudaError_t launch_backward(const BackwardArgs &a, int slices, int slice_elems, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>(a.R) * slices;
  const auto kernel = a.grad_entropy ? token_logprobs_backward_kernel<FMT, true> : token_logprobs_backward_kernel<FMT, false>;
  return launch_early(kernel, dim3(grid), dim3(kBackThreads), 0, s, a, slices, slice_elems);
}

// ---- gradient of the clipped objective ----------------------------------------------------------
struct GrpoGradArgs {
  const float *ln, *lo, *ls, *lr, *adv;
  const uint8_t *mask;
  const float *grad_out;
  int n, T;
  GrpoRule rule;
  float *out, *grad;
};
// sum over the NT threads that share a sequence (a warp, or the whole block)
template <int NT> __device__ __forceinline__ float team_sum(float v, float *scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (NT == 32) return v;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) v += scratch[w];
  return v;
}
// NT threads per sequence: a warp (several sequences a block) or a block.  VEC: rows are read as float4 / uchar4.
// Latency: the mask is counted before the first gradient can be written (256 x 2048 tokens: 4.4 us, 16 x 32: 2.1 us).
template <int NT, bool VEC>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT)
grpo_gradient_kernel(const __grid_constant__ GrpoGradArgs a) {
  __shared__ float scratch[32];
  early_start_sync();
  const int i = NT == 32 ? static_cast<int>(blockIdx.x) * 4 + (threadIdx.x >> 5) : static_cast<int>(blockIdx.x);
  if (i >= a.n) return;
  const int t0 = NT == 32 ? (threadIdx.x & 31) : threadIdx.x;
  const size_t base = static_cast<size_t>(i) * a.T;
  const float A = a.adv[i], up = a.grad_out ? a.grad_out[i] : 1.0f;
  float count = static_cast<float>(a.T);
  if (a.mask) {
    int c = 0;
    if (VEC) {
      const uint32_t *m4 = reinterpret_cast<const uint32_t *>(a.mask + base);
      for (int t = t0; t < a.T / 4; t += NT) c += __popc(__vcmpne4(m4[t], 0u)) >> 3;
    } else {
      for (int t = t0; t < a.T; t += NT) c += a.mask[base + t] ? 1 : 0;
    }
    count = team_sum<NT>(static_cast<float>(c), scratch);
  }
  const float share = count > 0.f ? 1.0f / count : 0.f, scale = up * share;
  float value = 0.f;
  if (VEC) {
    for (int t = t0; t < a.T / 4; t += NT) {
      const size_t q = base / 4 + t;
      const uint32_t m = a.mask ? reinterpret_cast<const uint32_t *>(a.mask)[q] : 0x01010101u;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      if (m) {
        const float4 ln = reinterpret_cast<const float4 *>(a.ln)[q], lo = reinterpret_cast<const float4 *>(a.lo)[q],
                     ls = reinterpret_cast<const float4 *>(a.ls)[q];
        const float4 lr = a.lr ? reinterpret_cast<const float4 *>(a.lr)[q] : ln;
        const float *pn = &ln.x, *po = &lo.x, *ps = &ls.x, *pr = &lr.x;
        float *pg = &o.x;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((m >> (8 * e)) & 0xffu) {
            const GrpoToken k = grpo_token(a.rule, A, pn[e], po[e], ps[e], pr[e]);
            value += k.w * k.term;
            pg[e] = k.w * k.slope * scale;
          }
      }
      reinterpret_cast<float4 *>(a.grad)[q] = o;
    }
  } else {
    for (int t = t0; t < a.T; t += NT) {
      float o = 0.f;
      if (!a.mask || a.mask[base + t]) {
        const float ln = a.ln[base + t];
        const GrpoToken k = grpo_token(a.rule, A, ln, a.lo[base + t], a.ls[base + t], a.lr ? a.lr[base + t] : ln);
        value += k.w * k.term;
        o = k.w * k.slope * scale;
      }
      a.grad[base + t] = o;
    }
  }
  if (a.out) {
    value = team_sum<NT>(value, scratch);
    if (t0 == 0) a.out[i] = value * share;
  }
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

cudaError_t score_detail_launch(const float *logits, int rows, int V, int rows_per_logit_row, float temperature,
                                const int32_t *tokens, const int32_t *tok_idx, int T, const int32_t *first_end,
                                float *out, float *out_entropy, int top_k, int32_t *out_ids, float *out_top, int *status,
                                cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  LogprobArgs a{};
  a.logits = logits;
  a.row_stride = V;
  a.R = rows;
  a.V = V;
  a.tokens = tokens;
  a.c = static_cast<float>(1.4426950408889634 / temperature);
  a.inv_temperature = static_cast<float>(1.0 / temperature);
  a.top_k = top_k;
  a.out_logprobs = out;
  a.out_entropy = out_entropy;
  a.out_top_ids = out_ids;
  a.out_top_logprobs = out_top;
  a.T = T;
  a.rows_per_logit_row = rows_per_logit_row;
  a.tok_idx = tok_idx;
  a.first_end = first_end;
  a.status = status;
  return logprobs_launch(a, 2, s);
}

}  // namespace echo

// ============================================================================
// C ABI
// ============================================================================
using namespace echo;

namespace {
int elem_bytes(int32_t format) { return format == 2 ? 4 : 2; }
// logits shapes and temperature of both directions
bool logits_ok(const void *logits, int32_t format, int64_t row_stride, int32_t R, int32_t V, float temperature) {
  if (!logits || format < 0 || format > 2 || R < 0 || V < 1 || row_stride < V) return false;
  if (reinterpret_cast<uintptr_t>(logits) % elem_bytes(format)) return false;
  return temperature > 0.f && std::isfinite(temperature) && std::isfinite(static_cast<float>(1.4426950408889634 / temperature));
}
}  // namespace

extern "C" {

int echo_token_logprobs(const void *logits, int32_t logits_format, int64_t row_stride, int32_t R, int32_t V,
                        const int32_t *tokens, float temperature, int32_t top_k, float *out_logprobs,
                        float *out_entropy, float *out_stats, int32_t *out_top_ids, float *out_top_logprobs,
                        void *cuda_stream) {
  if (R == 0) return ECHO_OK;
  if (!logits_ok(logits, logits_format, row_stride, R, V, temperature)) return ECHO_ERR_INVALID;
  if ((tokens == nullptr) != (out_logprobs == nullptr)) return ECHO_ERR_INVALID;
  if (top_k < 0 || (top_k > 0 && (!out_top_ids || !out_top_logprobs))) return ECHO_ERR_INVALID;
  if (!out_logprobs && !out_entropy && !out_stats && top_k == 0) return ECHO_ERR_INVALID;
  if (!aligned(out_stats, 8)) return ECHO_ERR_INVALID;
  if (top_k > kTopMax || V > kMaxVocab || static_cast<int64_t>(R) * kMaxSplit > 0x7fffffffLL) return ECHO_ERR_UNSUPPORTED;
  LogprobArgs a{};
  a.logits = logits;
  a.row_stride = row_stride;
  a.R = R;
  a.V = V;
  a.tokens = tokens;
  a.c = static_cast<float>(1.4426950408889634 / temperature);
  a.inv_temperature = static_cast<float>(1.0 / temperature);
  a.top_k = top_k;
  a.out_logprobs = out_logprobs;
  a.out_entropy = out_entropy;
  a.out_stats = reinterpret_cast<float2 *>(out_stats);
  a.out_top_ids = out_top_ids;
  a.out_top_logprobs = out_top_logprobs;
  return logprobs_launch(a, logits_format, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? ECHO_OK : ECHO_ERR_CUDA;
}

int echo_token_logprobs_backward(const void *logits, int32_t logits_format, int64_t row_stride, int32_t R, int32_t V,
                                 const int32_t *tokens, float temperature, const float *entropy, const float *stats,
                                 const float *grad_logprobs, const float *grad_entropy, void *out_grad,
                                 int64_t grad_stride, void *cuda_stream) {
  if (R == 0) return ECHO_OK;
  if (!logits_ok(logits, logits_format, row_stride, R, V, temperature)) return ECHO_ERR_INVALID;
  if (!out_grad || !stats || !aligned(stats, 8) || grad_stride < V) return ECHO_ERR_INVALID;
  if (!grad_logprobs && !grad_entropy) return ECHO_ERR_INVALID;
  if ((grad_logprobs && !tokens) || (grad_entropy && !entropy)) return ECHO_ERR_INVALID;
  const size_t eb = elem_bytes(logits_format);
  if (reinterpret_cast<uintptr_t>(out_grad) % eb) return ECHO_ERR_INVALID;
  // in place (the same rows), or apart
  const uintptr_t z0 = reinterpret_cast<uintptr_t>(logits), o0 = reinterpret_cast<uintptr_t>(out_grad);
  const uintptr_t z1 = z0 + (static_cast<size_t>(R - 1) * row_stride + V) * eb, o1 = o0 + (static_cast<size_t>(R - 1) * grad_stride + V) * eb;
  if (z0 < o1 && o0 < z1 && !(z0 == o0 && (row_stride == grad_stride || R == 1))) return ECHO_ERR_INVALID;
  if (V > kMaxVocab) return ECHO_ERR_UNSUPPORTED;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return ECHO_ERR_CUDA;
  // slices of whole steps: as long as a row allows while the launch still has about eight rounds of CTAs (few rows are
  // cut finely, many rows into long runs whose start-up counts for little)
  const int64_t step = kBackThreads * kBackUnroll * (16 / static_cast<int64_t>(eb)), steps = (V + step - 1) / step;
  const int64_t wanted = std::min(steps, (48 * static_cast<int64_t>(sms) + R - 1) / R);
  const int64_t per_slice = (steps + wanted - 1) / wanted, slices = (steps + per_slice - 1) / per_slice;
  const int slice = static_cast<int>(per_slice * step);
  if (static_cast<int64_t>(R) * slices > 0x7fffffffLL) return ECHO_ERR_UNSUPPORTED;
  BackwardArgs a{};
  a.logits = logits;
  a.row_stride = row_stride;
  a.R = R;
  a.V = V;
  a.tokens = tokens;
  a.c = static_cast<float>(1.4426950408889634 / temperature);
  a.inv_temperature = static_cast<float>(1.0 / temperature);
  a.entropy = entropy;
  a.stats = reinterpret_cast<const float2 *>(stats);
  a.grad_logprobs = grad_logprobs;
  a.grad_entropy = grad_entropy;
  a.out = out_grad;
  a.out_stride = grad_stride;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = logits_format == 0   ? launch_backward<0>(a, static_cast<int>(slices), slice, s)
                  : logits_format == 1 ? launch_backward<1>(a, static_cast<int>(slices), slice, s)
                                       : launch_backward<2>(a, static_cast<int>(slices), slice, s);
  return e == cudaSuccess ? ECHO_OK : ECHO_ERR_CUDA;
}

int echo_grpo_gradient(const float *logp_new, const float *logp_old, const float *logp_sampler, const float *logp_ref,
                       const float *adv, const uint8_t *mask, const float *grad_out, int32_t n, int32_t T,
                       float eps_clip, float C, float beta, float *out, float *out_grad, void *cuda_stream) {
  if (n < 0 || T < 1 || !(eps_clip >= 0.f) || !(C > 0.f) || !(beta >= 0.f)) return ECHO_ERR_INVALID;
  if (n == 0) return ECHO_OK;
  if (!logp_new || !logp_old || !logp_sampler || !adv || !out_grad) return ECHO_ERR_INVALID;
  if (T > (1 << 30)) return ECHO_ERR_UNSUPPORTED;             // (32-bit places within a sequence)
  GrpoGradArgs a{};
  a.ln = logp_new;
  a.lo = logp_old;
  a.ls = logp_sampler;
  a.lr = beta > 0.f ? logp_ref : nullptr;      // (no KL term, so that an estimate that overflows makes no 0 * inf)
  a.adv = adv;
  a.mask = mask;
  a.grad_out = grad_out;
  a.n = n;
  a.T = T;
  a.rule = {eps_clip, C, a.lr ? beta : 0.f, std::log1p(static_cast<double>(eps_clip)),
            eps_clip < 1.f ? std::log1p(-static_cast<double>(eps_clip)) : -INFINITY};
  a.out = out;
  a.grad = out_grad;
  const bool vec = T % 4 == 0 && aligned(logp_new, 16) && aligned(logp_old, 16) && aligned(logp_sampler, 16) &&
                   aligned(logp_ref, 16) && aligned(out_grad, 16) && aligned(mask, 4);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  // short responses: a warp each, four to a CTA; longer ones: 512 threads each
  const bool warps = T <= 256;
  const auto kernel = warps ? (vec ? grpo_gradient_kernel<32, true> : grpo_gradient_kernel<32, false>)
                            : (vec ? grpo_gradient_kernel<512, true> : grpo_gradient_kernel<512, false>);
  const cudaError_t e = launch_early(kernel, dim3(warps ? (static_cast<unsigned>(n) + 3) / 4 : n), dim3(warps ? 128 : 512), 0, s, a);
  return e == cudaSuccess ? ECHO_OK : ECHO_ERR_CUDA;
}

}  // extern "C"
