// New tokens into a caller's paged cache: queries and keys rotated by their positions, keys and values to their pages.
//
// Position of row i of a chunk of n rows in a cache of L keys (the chunk included): t = L - n + i.  Pairs (j, j + hd/2)
// turn by t theta^(-2j/hd).  The angle is formed in turns, t times a 64-bit rate, and its whole turns are taken off in 64
// bits: what is left is exact to 2^-23 of a turn at t = 2^30, where a 32-bit angle would be off by many turns.
//
// Bound: HBM for many rows (each element is read once and written once in 16 bits), latency for few: the loads of a
// row's elements are under way while its sequence, position and page are looked up.

#include <cmath>

#include "chunks.cuh"

namespace echo {
namespace {

// What hides HBM's latency is the number of warps: one item in a thread's registers, 40 registers, and CTAs of 128 threads
// where there are many rows (16 x 1024 rows at 64/8 heads, bf16: 119 us, 0.86 of the copy rate; two items a thread 144).  Where
// there are few, a row's items at once (384 threads are the 48 heads of 128 of one row).
constexpr int kAppThreads = 128, kAppFewThreads = 384;
constexpr int kAppRows = 2;                     // most rows of a CTA

struct AppendArgs {
  const void *q, *k, *v;                        // q may be null
  int64_t q_stride, k_stride, v_stride;         // elements
  uint16_t *pool, *out_q;
  int Hq, Hkv, hd, n_pages, half_out, rows_per_cta;
  ChunkArgs c;
  double rate[64];                              // turns per position of pair j
};

// eight consecutive elements as fp32.  VEC: the address is a multiple of 16 bytes.
template <int IN, bool VEC> __device__ __forceinline__ void load8(const void *base, int64_t i, float (&f)[8]) {
  if (IN == 2) {
    const float *p = static_cast<const float *>(base) + i;
    if (VEC) {
      const float4 a = *reinterpret_cast<const float4 *>(p), b = *(reinterpret_cast<const float4 *>(p) + 1);
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
      f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = p[e];
    }
  } else {
    const uint16_t *p = static_cast<const uint16_t *>(base) + i;
    if (VEC) {
      const uint4 a = *reinterpret_cast<const uint4 *>(p);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 t = widen16x2(w[e], IN == 1);
        f[2 * e] = t.x;
        f[2 * e + 1] = t.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = widen16(p[e], IN == 1);
    }
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8], bool half) {
  return make_uint4(cvt16x2(f[0], f[1], half), cvt16x2(f[2], f[3], half), cvt16x2(f[4], f[5], half), cvt16x2(f[6], f[7], half));
}

// The sequence that holds `row`: the last one that starts at or before it, by 32 probes a step.  -1: none.
__device__ __forceinline__ int find_sequence(const ChunkArgs &c, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = c.S;
  while (true) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const unsigned before = __ballot_sync(0xffffffffu, at < hi && c.row_starts[at] <= row);
    if (!before) return -1;
    lo += (31 - __clz(before)) * step;
    hi = min(hi, lo + step);
    if (hi - lo <= 1) return lo;
  }
}

template <int IN, bool VEC>
__global__ void __launch_bounds__(kAppFewThreads, 4)
append_kv_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ int s_pos[kAppRows];
  __shared__ long long s_slot[kAppRows];            // element of the pool where head 0's key goes; -1: nowhere
  __shared__ float2 s_turn[kAppRows][64];           // (cos, sin)
  early_start_sync();
  const int half = a.hd / 2, per_unit = half / 8, units = a.Hq + 2 * a.Hkv;      // a work item: eight pairs of a head
  const int row0 = static_cast<int>(blockIdx.x) * a.rows_per_cta, rows = min(a.rows_per_cta, a.c.n_rows - row0);
  const int items = rows * units * per_unit;
  const int warp = threadIdx.x >> 5;
  const int threads = blockDim.x;
  for (int item = threadIdx.x, begin = 0; begin < items; item += threads, begin += threads) {
    const int u = item / per_unit, at = (item % per_unit) * 8, row = u / units, unit = item < items ? u % units : -1;
    const bool value = unit >= a.Hq + a.Hkv;
    float x[8], y[8];
    if (unit >= 0) {
      const int64_t r = row0 + row;
      const void *src = value ? a.v : unit < a.Hq ? a.q : a.k;
      const int64_t off = value           ? r * a.v_stride + (unit - a.Hq - a.Hkv) * a.hd
                          : unit < a.Hq ? r * a.q_stride + unit * a.hd
                                          : r * a.k_stride + (unit - a.Hq) * a.hd;
      load8<IN, VEC>(src, off + at, x);
      load8<IN, VEC>(src, off + at + half, y);
    }
    if (begin == 0) {
      // every sequence's lengths are looked at once, by the first CTA
      if (blockIdx.x == 0)
        for (int s = threadIdx.x; s < a.c.S; s += threads) {
          const SeqSpan p = seq_span(a.c, s);
          if (!p.ok || p.kv < p.n) atomicMax(a.c.status, STATUS_BAD_CHUNK);
        }
      if (warp < rows) {
        const int r = row0 + warp, s = find_sequence(a.c, r);
        int pos = -1;
        long long slot = -1;
        if (s >= 0) {
          const SeqSpan p = seq_span(a.c, s);
          if (p.ok && p.kv >= p.n && r >= p.row0 && r < p.row0 + p.n) {
            pos = p.kv - p.n + (r - p.row0);
            const int page = a.c.page_table[static_cast<int64_t>(s) * a.c.pt_width + pos / kChunkPage];
            if (page < 0 || page >= a.n_pages) {
              if ((threadIdx.x & 31) == 0) atomicMax(a.c.status, STATUS_BAD_PAGE);
            } else {
              slot = (static_cast<long long>(page) * a.Hkv * 2 * kChunkPage + pos % kChunkPage) * a.hd;
            }
          }
        }
        if ((threadIdx.x & 31) == 0) {
          s_pos[warp] = pos;
          s_slot[warp] = slot;
        }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < rows * half; i += threads) {
        const int r = i / half, j = i % half;
        const double turns = static_cast<double>(s_pos[r]) * a.rate[j];
        float sn, cs;
        sincospif(2.0f * static_cast<float>(turns - rint(turns)), &sn, &cs);
        s_turn[r][j] = make_float2(cs, sn);
      }
      __syncthreads();
    }
    if (unit < 0 || s_pos[row] < 0) continue;
    if (!value) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 t = s_turn[row][at + e];
        const float lo = x[e] * t.x - y[e] * t.y, hi = y[e] * t.x + x[e] * t.y;
        x[e] = lo;
        y[e] = hi;
      }
    }
    uint16_t *dst;
    if (unit < a.Hq) {
      dst = a.out_q + (static_cast<int64_t>(row0 + row) * a.Hq + unit) * a.hd + at;
    } else {
      const long long slot = s_slot[row];
      if (slot < 0) continue;
      const int head = unit - a.Hq - (value ? a.Hkv : 0);
      dst = a.pool + slot + static_cast<long long>(head * 2 + (value ? 1 : 0)) * kChunkPage * a.hd + at;
    }
    *reinterpret_cast<uint4 *>(dst) = pack8(x, a.half_out);
    *reinterpret_cast<uint4 *>(dst + half) = pack8(y, a.half_out);
  }
}

}  // namespace
}  // namespace echo

using namespace echo;

extern "C" int echo_append_kv(const void *q, const void *k, const void *v, int32_t in_format, int64_t q_stride,
                              int64_t k_stride, int64_t v_stride, const echo_kv_chunks *chunks, int32_t Hq, int32_t Hkv,
                              int32_t hd, float rope_theta, void *kv_pool, int32_t n_pages, int32_t kv_format, void *out_q,
                              void *cuda_stream) {
  AppendArgs a{};
  if ((q == nullptr) != (out_q == nullptr) || (q && Hq < 1)) return ECHO_ERR_INVALID;
  if (!q) Hq = 0;
  const int rc = chunk_args(chunks, Hq, Hkv, hd, kv_pool, n_pages, kv_format, &a.c);
  if (rc != ECHO_OK) return rc;
  const bool none = a.c.S == 0 || a.c.n_rows == 0;
  if ((!none && (!k || !v)) || in_format < 0 || in_format > 2 || !(rope_theta > 0.f) || !std::isfinite(rope_theta)) return ECHO_ERR_INVALID;
  if ((q && q_stride < static_cast<int64_t>(Hq) * hd) || k_stride < static_cast<int64_t>(Hkv) * hd ||
      v_stride < static_cast<int64_t>(Hkv) * hd)
    return ECHO_ERR_INVALID;
  const uint64_t eb = in_format == 2 ? 4 : 2;
  const void *given[3] = {q, k, v};
  const int64_t strides[3] = {q_stride, k_stride, v_stride};
  const int64_t widths[3] = {static_cast<int64_t>(Hq) * hd, static_cast<int64_t>(Hkv) * hd, static_cast<int64_t>(Hkv) * hd};
  if (reinterpret_cast<uintptr_t>(out_q) & 15) return ECHO_ERR_INVALID;
  if (none) return ECHO_OK;
  bool vec = true;
  const uint64_t pool = pool_bytes(n_pages, Hkv, hd), outs = static_cast<uint64_t>(a.c.n_rows) * Hq * hd * 2;
  if (ranges_meet(kv_pool, pool, out_q, outs) || meets_tables(a.c, kv_pool, pool) || meets_tables(a.c, out_q, outs) || status_in_tables(a.c))
    return ECHO_ERR_INVALID;
  for (int i = 0; i < 3; ++i) {
    if (!given[i]) continue;
    const uintptr_t p = reinterpret_cast<uintptr_t>(given[i]);
    if (p % eb || strides[i] > (int64_t(1) << 30)) return ECHO_ERR_INVALID;
    const uint64_t bytes = (static_cast<uint64_t>(a.c.n_rows - 1) * strides[i] + widths[i]) * eb;
    if (ranges_meet(given[i], bytes, kv_pool, pool) || ranges_meet(given[i], bytes, a.c.status, 4)) return ECHO_ERR_INVALID;
    // the rotated queries may replace the given ones, element for element
    const bool same = i == 0 && q == out_q && in_format == kv_format && (q_stride == widths[0] || a.c.n_rows == 1);
    if (!same && ranges_meet(given[i], bytes, out_q, outs)) return ECHO_ERR_INVALID;
    vec = vec && p % 16 == 0 && (strides[i] * eb % 16 == 0 || a.c.n_rows == 1);
  }
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.pool = static_cast<uint16_t *>(kv_pool);
  a.out_q = static_cast<uint16_t *>(out_q);
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.hd = hd;
  a.n_pages = n_pages;
  a.half_out = kv_format == 1;
  for (int j = 0; j < hd / 2; ++j)
    a.rate[j] = std::pow(static_cast<double>(rope_theta), -2.0 * j / hd) / 6.283185307179586476925286766559;
  // few rows (fewer than eight CTAs an SM): a row to a CTA; otherwise two rows share the look-ups' latency
  const bool few = a.c.n_rows < 8 * 148;
  const int rows = few ? 1 : kAppRows;
  a.rows_per_cta = rows;
  const auto kernel = in_format == 0   ? (vec ? append_kv_kernel<0, true> : append_kv_kernel<0, false>)
                      : in_format == 1 ? (vec ? append_kv_kernel<1, true> : append_kv_kernel<1, false>)
                                       : (vec ? append_kv_kernel<2, true> : append_kv_kernel<2, false>);
  const cudaError_t e = launch_early(kernel, dim3((static_cast<unsigned>(a.c.n_rows) + rows - 1) / rows), dim3(few ? kAppFewThreads : kAppThreads), 0,
                                     static_cast<cudaStream_t>(cuda_stream), a);
  return e == cudaSuccess ? ECHO_OK : ECHO_ERR_CUDA;
}
