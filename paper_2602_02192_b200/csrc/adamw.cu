// One AdamW step over many tensors in one launch, with moments in fp32 or in 8 bits.
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments: 256 consecutive elements of a tensor share two fp32 scales, the largest |m| (M) and the largest v (V)
// of the block.  A code stands for M (c/127) |c/127| (first moment) and V (c/255)^4 (second moment): quadratic and
// quartic companding put the steps where small values are, so that a block may span five decades of |m| and nine of v.
//   first moment   nearest code on the companded axis, rint(127 sqrt(|m| / M)): it turns over by 1 - b1 a step, far
//                  more than a code's width;
//   second moment  one of the two codes around v, the upper with the probability that keeps the mean (v moves by
//                  1 - b2 a step, less than a code's width: rounding to the nearest would never let it fall), and never
//                  0 for a v above 0, since a lost v beside a kept m would make a huge update.
// Codes and scales are those of the 64-bit arithmetic: fp32 decides, and where fp32's own error could move a value
// across a border between two codes the element is decided again in 64 bits (about one in ten thousand).  A scale is
// the fp32 rounding of the 64-bit maximum.
#include <cmath>
#include <new>
#include <algorithm>

#include "common.cuh"
#include "ptx.cuh"

namespace echo {
namespace {

constexpr int kBlock = 256;                  // elements that share the 8-bit scales; one warp, eight per lane
constexpr int kThreads = 256;

struct Entry {
  float *p;
  const void *g;
  void *m, *v;
  float *m_scale, *v_scale;
  __nv_bfloat16 *copy;
  int64_t n;
  float decay;                               // 1 - lr wd
  uint32_t first;                            // blocks of the launch before this tensor's
  uint32_t id;                               // place in the caller's list (keys the random numbers)
  uint32_t vec;                              // every array starts on a boundary of its 8-element pieces
};
struct Scalars {
  const float *grad_scale;
  float b1, b1c, b2, b2c, root_corr, eps, rate;      // rate = lr / (1 - b1^t), root_corr = 1 / sqrt(1 - b2^t)
  double b1_d, b1c_d, b2_d, b2c_d;
  uint32_t key0, key1, step;
  uint32_t n_tensors, n_blocks;
};
template <int N> struct Table {
  Scalars s;
  Entry e[N];
};
constexpr int kSmallTable = 32, kLargeTable = 400;   // kernel parameters may hold 32764 bytes
static_assert(sizeof(Table<kLargeTable>) <= 32764, "table of tensors exceeds the kernel parameters");

// eight consecutive floats, 32-byte aligned
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
  asm volatile("ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
  asm volatile("st.global.L1::no_allocate.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]),
               "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
               : "memory");
}
// the eight elements of a lane: whole, or the first `left` of them one by one (the others read as 0)
template <bool WHOLE> __device__ __forceinline__ void get_f32(const float *p, int left, float (&x)[8]) {
  if (WHOLE) return load8(p, x);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = j < left ? p[j] : 0.f;
}
template <bool WHOLE> __device__ __forceinline__ void put_f32(float *p, int left, const float (&x)[8]) {
  if (WHOLE) return store8(p, x);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) p[j] = x[j];
}
template <int FMT, bool WHOLE> __device__ __forceinline__ void get_grad(const void *g, size_t at, int left, float (&x)[8]) {
  if constexpr (FMT == 2) {
    get_f32<WHOLE>(static_cast<const float *>(g) + at, left, x);
  } else {
    const uint16_t *h = static_cast<const uint16_t *>(g) + at;
    if (WHOLE) {
      const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(h));
      const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = widen16x2(a[j], FMT == 1);
        x[2 * j] = f.x;
        x[2 * j + 1] = f.y;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = j < left ? widen16(h[j], FMT == 1) : 0.f;
    }
  }
}
template <bool WHOLE> __device__ __forceinline__ void put_copy(__nv_bfloat16 *c, int left, const float (&x)[8]) {
  if (WHOLE) {
    *reinterpret_cast<uint4 *>(c) = make_uint4(cvt16x2(x[0], x[1], false), cvt16x2(x[2], x[3], false),
                                               cvt16x2(x[4], x[5], false), cvt16x2(x[6], x[7], false));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) c[j] = __float2bfloat16(x[j]);
  }
}
template <bool WHOLE> __device__ __forceinline__ uint2 get_codes(const void *c, size_t at, int left) {
  const uint8_t *b = static_cast<const uint8_t *>(c) + at;
  if (WHOLE) return __ldcs(reinterpret_cast<const uint2 *>(b));
  uint2 w = make_uint2(0u, 0u);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) (j < 4 ? w.x : w.y) |= static_cast<uint32_t>(b[j]) << (8 * (j & 3));
  return w;
}
template <bool WHOLE> __device__ __forceinline__ void put_codes(void *c, size_t at, int left, uint2 w) {
  uint8_t *b = static_cast<uint8_t *>(c) + at;
  if (WHOLE) {
    *reinterpret_cast<uint2 *>(b) = w;
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) b[j] = static_cast<uint8_t>((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
}
__device__ __forceinline__ uint32_t byte_of(uint2 w, int j) { return ((j < 4 ? w.x : w.y) >> (8 * (j & 3))) & 0xffu; }
__device__ __forceinline__ int signed_byte(uint2 w, int j) { return static_cast<int>(static_cast<int8_t>(byte_of(w, j))); }
__device__ __forceinline__ float sqrt_fast(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Philox4x32-10 (Salmon et al., SC'11), as in the sampler
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c.x, b = static_cast<uint64_t>(0xCD9E8D57u) * c.z;
    c = make_uint4(static_cast<uint32_t>(b >> 32) ^ c.y ^ k0, static_cast<uint32_t>(b),
                   static_cast<uint32_t>(a >> 32) ^ c.w ^ k1, static_cast<uint32_t>(a));
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// the moments in 64 bits
__device__ __forceinline__ double exact_avg(const Scalars &s, int code, float scale, float g, float gs) {
  const double q = code / 127.0;
  return s.b1_d * (q * fabs(q) * scale) + s.b1c_d * (static_cast<double>(g) * gs);
}
__device__ __forceinline__ double exact_sq(const Scalars &s, uint32_t code, float scale, float g, float gs) {
  const double q = code / 255.0, h = static_cast<double>(g) * gs;
  return s.b2_d * (q * q * (q * q) * scale) + s.b2c_d * h * h;
}
// Largest of non-negative values by their bits, which order like the values; NaN is above infinity, so that it shows.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(fabsf(v)); }
__device__ __forceinline__ float warp_max(uint32_t bits) { return __uint_as_float(__reduce_max_sync(0xffffffffu, bits)); }

// relative error of the fp32 moments, generously: a handful of roundings of 2^-24 each
constexpr float kMomentErr = 1e-6f;

template <int FMT, bool EIGHT, bool WHOLE>
__device__ __forceinline__ void step_block(const Scalars &s, const Entry &e, int64_t block, int lane, float gs) {
  const int64_t at = block * kBlock + lane * 8;
  const int left = WHOLE ? 8 : static_cast<int>(min(static_cast<int64_t>(8), max(static_cast<int64_t>(0), e.n - at)));
  float p[8], g[8];
  get_grad<FMT, WHOLE>(e.g, at, left, g);
  get_f32<WHOLE>(e.p + at, left, p);
  if constexpr (!EIGHT) {
    float m[8], v[8];
    get_f32<WHOLE>(static_cast<float *>(e.m) + at, left, m);
    get_f32<WHOLE>(static_cast<float *>(e.v) + at, left, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float h = g[j] * gs;
      m[j] = fmaf(s.b1, m[j], s.b1c * h);
      v[j] = fmaf(s.b2, v[j], s.b2c * h * h);
      const float denom = fmaf(sqrt_fast(v[j]), s.root_corr, s.eps);
      p[j] = fmaf(p[j], e.decay, -s.rate * __fdividef(m[j], denom));
    }
    put_f32<WHOLE>(static_cast<float *>(e.m) + at, left, m);
    put_f32<WHOLE>(static_cast<float *>(e.v) + at, left, v);
  } else {
    const uint2 mc = get_codes<WHOLE>(e.m, at, left), vc = get_codes<WHOLE>(e.v, at, left);
    const float M0 = e.m_scale[block], V0 = e.v_scale[block];
    float m[8], v[8], err[8];                  // err: how far m may be off
    uint32_t top_m = 0, top_v = 0;
    float sure_m = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float h = g[j] * gs;
      const float q = static_cast<float>(signed_byte(mc, j)) * (1.0f / 127.0f);
      const float a = s.b1 * (q * fabsf(q) * M0), b = s.b1c * h;
      m[j] = a + b;
      err[j] = kMomentErr * (fabsf(a) + fabsf(b));
      float r = static_cast<float>(byte_of(vc, j)) * (1.0f / 255.0f);
      r *= r;
      v[j] = fmaf(s.b2, r * r * V0, s.b2c * h * h);
      top_m = max(top_m, magnitude(m[j]));
      sure_m = fmaxf(sure_m, fabsf(m[j]) - err[j]);
      top_v = max(top_v, magnitude(v[j]));
      const float denom = fmaf(sqrt_fast(v[j]), s.root_corr, s.eps);
      p[j] = fmaf(p[j], e.decay, -s.rate * __fdividef(m[j], denom));
    }
    // scales: the 64-bit maximum as fp32, found among the elements that fp32 cannot tell from it
    const float big_m = warp_max(top_m), big_v = warp_max(top_v);
    sure_m = warp_max(magnitude(sure_m));
    float M = 0.f, V = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (fabsf(m[j]) + err[j] >= sure_m && err[j] > 0.f)
        M = fmaxf(M, static_cast<float>(fabs(exact_avg(s, signed_byte(mc, j), M0, g[j], gs))));
      if (v[j] >= big_v * (1.0f - 2.0f * kMomentErr) && v[j] != 0.f)
        V = fmaxf(V, static_cast<float>(exact_sq(s, byte_of(vc, j), V0, g[j], gs)));
    }
    M = isfinite(big_m) ? warp_max(magnitude(M)) : big_m;
    V = isfinite(big_v) ? warp_max(magnitude(V)) : big_v;
    if (M < 1.17549435e-38f) M = 0.f;          // below the normal numbers: counts as 0
    if (V < 1.17549435e-38f) V = 0.f;
    const float inv_m = M > 0.f ? 16129.0f / M : 0.f, inv_v = V > 0.f ? 4228250625.0f / V : 0.f;     // 127^2, 255^4
    const uint64_t octet = static_cast<uint64_t>(block) * (kBlock / 8) + lane;
    const uint4 rnd = philox(make_uint4(static_cast<uint32_t>(octet), static_cast<uint32_t>(octet >> 32), e.id, s.step),
                             s.key0, s.key1);
    const uint32_t words[4] = {rnd.x, rnd.y, rnd.z, rnd.w};
    uint2 mo = make_uint2(0u, 0u), vo = make_uint2(0u, 0u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // ---- first moment: y = 127^2 |m| / M lies between the borders (c - 1/2)^2 and (c + 1/2)^2
      const float y = fabsf(m[j]) * inv_m;
      float c = rintf(sqrt_fast(y));
      const float mid = fmaf(c, c, 0.25f);
      const float up = (mid + c) - y, down = c > 0.f ? y - (mid - c) : 1e30f;
      if (fminf(up, down) <= fmaf(err[j], inv_m, y * kMomentErr))
        c = M > 0.f ? static_cast<float>(rint(sqrt(fabs(exact_avg(s, signed_byte(mc, j), M0, g[j], gs)) * 16129.0 / M))) : 0.f;
      int code = static_cast<int>(c);
      code = m[j] < 0.f ? -code : code;
      (j < 4 ? mo.x : mo.y) |= (static_cast<uint32_t>(code) & 0xffu) << (8 * (j & 3));
      // ---- second moment: w = 255^4 v / V lies between c^4 and (c + 1)^4
      const float w = v[j] * inv_v;
      float d = fminf(floorf(sqrt_fast(sqrt_fast(w))), 254.0f);
      const float d2 = d * d, above = w - d2 * d2, width = fmaf(fmaf(fmaf(4.0f, d, 6.0f), d, 4.0f), d, 1.0f);
      const uint32_t half16 = (words[j >> 1] >> (16 * (j & 1))) & 0xffffu;
      const float u = static_cast<float>(half16) * 1.52587890625e-05f;
      const float diff = above - u * width, err_w = w * (1.2f * kMomentErr);
      uint32_t vcode = static_cast<uint32_t>(d) + (diff > 0.f ? 1u : 0u);
      if (v[j] == big_v) {
        vcode = 255u;                          // the block's largest
      } else if (fminf(fminf(fabsf(diff), above), width - above) <= err_w) {
        const double we = V > 0.f ? exact_sq(s, byte_of(vc, j), V0, g[j], gs) * (4228250625.0 / V) : 0.0;
        const double dd = fmin(floor(sqrt(sqrt(we))), 254.0);
        const double lo = dd * dd * (dd * dd), hi = (dd + 1.0) * (dd + 1.0) * ((dd + 1.0) * (dd + 1.0));
        vcode = static_cast<uint32_t>(dd) + (half16 * 1.52587890625e-05 * (hi - lo) < we - lo ? 1u : 0u);
      }
      if (vcode == 0u) vcode = 1u;
      if (!(w > 0.f)) vcode = 0u;
      (j < 4 ? vo.x : vo.y) |= vcode << (8 * (j & 3));
    }
    put_codes<WHOLE>(e.m, at, left, mo);
    put_codes<WHOLE>(e.v, at, left, vo);
    if (lane == 0) {
      e.m_scale[block] = M;
      e.v_scale[block] = V;
    }
  }
  put_f32<WHOLE>(e.p + at, left, p);
  if (e.copy) put_copy<WHOLE>(e.copy + at, left, p);
}

// A grid that fills the GPU; a warp takes every n-th block of 256 elements of the whole list.
template <int N, typename F> __device__ __forceinline__ void for_blocks(const Table<N> &t, F f) {
  const uint32_t warps = gridDim.x * (kThreads / 32);
  uint32_t cur = 0, from = 0, to = 0;
  for (uint32_t b = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); b < t.s.n_blocks; b += warps) {
    if (b < from || b >= to) {
      uint32_t lo = 0, hi = t.s.n_tensors;               // last tensor whose first block is at most b
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (t.e[mid].first <= b) lo = mid;
        else hi = mid;
      }
      cur = lo;
      from = t.e[lo].first;
      to = lo + 1 < t.s.n_tensors ? t.e[lo + 1].first : t.s.n_blocks;
    }
    f(t.e[cur], static_cast<int64_t>(b - from), cur);
  }
}

template <int N, int FMT, bool EIGHT>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<N> t) {
  const float gs = t.s.grad_scale ? *t.s.grad_scale : 1.0f;
  if (!isfinite(gs)) return;                              // an overflowed step changes nothing
  const int lane = threadIdx.x & 31;
  for_blocks(t, [&](const Entry &e, int64_t block, uint32_t) {
    if (e.vec && (block + 1) * kBlock <= e.n) step_block<FMT, EIGHT, true>(t.s, e, block, lane, gs);
    else step_block<FMT, EIGHT, false>(t.s, e, block, lane, gs);
  });
}

// The values that 8-bit moments stand for: p and copy of an entry hold the two outputs.
template <int N> __global__ void __launch_bounds__(kThreads) adamw_unpack_kernel(const __grid_constant__ Table<N> t) {
  const int lane = threadIdx.x & 31;
  for_blocks(t, [&](const Entry &e, int64_t block, uint32_t) {
    const int64_t at = block * kBlock + lane * 8;
    const int left = static_cast<int>(min(static_cast<int64_t>(8), max(static_cast<int64_t>(0), e.n - at)));
    const bool whole = e.vec && left == 8;
    const uint2 mc = whole ? get_codes<true>(e.m, at, left) : get_codes<false>(e.m, at, left);
    const uint2 vc = whole ? get_codes<true>(e.v, at, left) : get_codes<false>(e.v, at, left);
    const float M = e.m_scale[block], V = e.v_scale[block];
    float m[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float q = static_cast<float>(signed_byte(mc, j)) * (1.0f / 127.0f);
      m[j] = q * fabsf(q) * M;
      float r = static_cast<float>(byte_of(vc, j)) * (1.0f / 255.0f);
      r *= r;
      v[j] = r * r * V;
    }
    float *om = e.p + at, *ov = reinterpret_cast<float *>(e.copy) + at;
    if (whole) {
      put_f32<true>(om, left, m);
      put_f32<true>(ov, left, v);
    } else {
      put_f32<false>(om, left, m);
      put_f32<false>(ov, left, v);
    }
  });
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <int N, int FMT, bool EIGHT> cudaError_t launch_step(const Table<N> &t, int grid, cudaStream_t s) {
  adamw_kernel<N, FMT, EIGHT><<<grid, kThreads, 0, s>>>(t);
  return cudaGetLastError();
}
template <int N> cudaError_t launch_any(const Table<N> &t, int grad_format, int state_bits, int grid, cudaStream_t s) {
  if (state_bits == 0) {
    adamw_unpack_kernel<N><<<grid, kThreads, 0, s>>>(t);
    return cudaGetLastError();
  }
  if (state_bits == 32)
    return grad_format == 0   ? launch_step<N, 0, false>(t, grid, s)
           : grad_format == 1 ? launch_step<N, 1, false>(t, grid, s)
                              : launch_step<N, 2, false>(t, grid, s);
  return grad_format == 0   ? launch_step<N, 0, true>(t, grid, s)
         : grad_format == 1 ? launch_step<N, 1, true>(t, grid, s)
                            : launch_step<N, 2, true>(t, grid, s);
}

// Launches over the entries that make(i, entry) fills (false: nothing to do for tensor i), as many per launch as the
// kernel parameters hold.  state_bits 0: unpack.
template <typename Make>
cudaError_t launch_list(int n_tensors, const Scalars &base, int grad_format, int state_bits, Make make, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (err != cudaSuccess) return err;
  int i = 0;
  while (i < n_tensors) {
    Table<kLargeTable> t;
    t.s = base;
    uint32_t n = 0;
    uint64_t blocks = 0;
    while (i < n_tensors && n < kLargeTable) {
      Entry e{};
      if (make(i, e)) {
        const uint64_t more = (static_cast<uint64_t>(e.n) + kBlock - 1) / kBlock;
        if (n > 0 && blocks + more > 0x7fffffffu) break;
        e.first = static_cast<uint32_t>(blocks);
        blocks += more;
        t.e[n++] = e;
      }
      ++i;
    }
    if (n == 0) continue;
    t.s.n_tensors = n;
    t.s.n_blocks = static_cast<uint32_t>(blocks);
    const uint64_t need = (blocks + kThreads / 32 - 1) / (kThreads / 32);
    const int grid = static_cast<int>(std::min<uint64_t>(need, static_cast<uint64_t>(sms) * 8));
    if (n <= kSmallTable) {
      Table<kSmallTable> small;
      small.s = t.s;
      std::copy(t.e, t.e + n, small.e);
      err = launch_any(small, grad_format, state_bits, grid, s);
    } else {
      err = launch_any(t, grad_format, state_bits, grid, s);
    }
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

struct Range {
  uintptr_t from, to;
  bool written;
};
// false: two arrays overlap of which one is written (the same tensor twice, a gradient inside a weight)
bool apart(Range *r, size_t n) {
  std::sort(r, r + n, [](const Range &a, const Range &b) { return a.from < b.from; });
  uintptr_t end_written = 0, end_any = 0;
  for (size_t i = 0; i < n; ++i) {
    if (r[i].from < (r[i].written ? end_any : end_written)) return false;
    end_any = std::max(end_any, r[i].to);
    if (r[i].written) end_written = std::max(end_written, r[i].to);
  }
  return true;
}
int elem_bytes(int format) { return format == 2 ? 4 : 2; }
bool list_ok(const echo_adamw_tensor *t, int32_t n_tensors, int32_t state_bits, int32_t grad_format, bool step) {
  for (int i = 0; i < n_tensors; ++i) {
    const echo_adamw_tensor &x = t[i];
    if (x.n < 0 || x.n > (1LL << 38)) return false;
    if (x.n == 0) continue;
    if (!x.exp_avg || !x.exp_avg_sq) return false;
    if (step && (!x.param || !x.grad || !aligned(x.param, 4) || !aligned(x.grad, elem_bytes(grad_format)) ||
                 !aligned(x.param_copy, 2)))
      return false;
    if (state_bits == 8 && (!x.avg_scales || !x.sq_scales || !aligned(x.avg_scales, 4) || !aligned(x.sq_scales, 4)))
      return false;
    if (state_bits == 32 && (!aligned(x.exp_avg, 4) || !aligned(x.exp_avg_sq, 4))) return false;
  }
  return true;
}

}  // namespace
}  // namespace echo

using namespace echo;

extern "C" {

int echo_adamw_step(const echo_adamw_tensor *tensors, int32_t n_tensors, const echo_adamw_options *opt, void *cuda_stream) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !opt) return ECHO_ERR_INVALID;
  const auto fraction = [](double x) { return x >= 0.0 && x < 1.0; };       // false for NaN
  if (!fraction(opt->beta1) || !fraction(opt->beta2) || !(opt->lr >= 0.0) || !std::isfinite(opt->lr)) return ECHO_ERR_INVALID;
  if (!(static_cast<float>(opt->eps) > 0.f) || !std::isfinite(static_cast<float>(opt->eps))) return ECHO_ERR_INVALID;
  if (opt->step < 1 || opt->step > 0xffffffffLL || !aligned(opt->grad_scale, 4)) return ECHO_ERR_INVALID;
  if (opt->grad_format < 0 || opt->grad_format > 2 || (opt->state_bits != 8 && opt->state_bits != 32)) return ECHO_ERR_INVALID;
  const int bits = opt->state_bits, gb = elem_bytes(opt->grad_format);
  if (!list_ok(tensors, n_tensors, bits, opt->grad_format, true)) return ECHO_ERR_INVALID;
  for (int i = 0; i < n_tensors; ++i)
    if (!(tensors[i].weight_decay >= 0.0) || !std::isfinite(tensors[i].weight_decay)) return ECHO_ERR_INVALID;
  if (n_tensors == 0) return ECHO_OK;
  Range *r = new (std::nothrow) Range[static_cast<size_t>(n_tensors) * 7 + 1];
  if (!r) return ECHO_ERR_ARENA;
  size_t n_ranges = 0;
  auto range = [&](const void *p, int64_t bytes, bool written) {
    if (p && bytes > 0) {
      const uintptr_t from = reinterpret_cast<uintptr_t>(p);
      r[n_ranges++] = Range{from, from + static_cast<size_t>(bytes), written};
    }
  };
  for (int i = 0; i < n_tensors; ++i) {
    const echo_adamw_tensor &x = tensors[i];
    if (x.n == 0) continue;
    const int64_t blocks = (x.n + kBlock - 1) / kBlock;
    range(x.param, x.n * 4, true);
    range(x.exp_avg, x.n * (bits / 8), true);
    range(x.exp_avg_sq, x.n * (bits / 8), true);
    range(x.param_copy, x.n * 2, true);
    range(x.grad, x.n * gb, false);
    if (bits == 8) {
      range(x.avg_scales, blocks * 4, true);
      range(x.sq_scales, blocks * 4, true);
    }
  }
  range(opt->grad_scale, 4, false);
  const bool ok = apart(r, n_ranges);
  delete[] r;
  if (!ok) return ECHO_ERR_INVALID;
  Scalars s{};
  const double t = static_cast<double>(opt->step);
  s.grad_scale = opt->grad_scale;
  s.b1_d = opt->beta1;
  s.b1c_d = 1.0 - opt->beta1;
  s.b2_d = opt->beta2;
  s.b2c_d = 1.0 - opt->beta2;
  s.b1 = static_cast<float>(s.b1_d);
  s.b1c = static_cast<float>(s.b1c_d);
  s.b2 = static_cast<float>(s.b2_d);
  s.b2c = static_cast<float>(s.b2c_d);
  s.root_corr = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(opt->beta2, t)));
  s.rate = static_cast<float>(opt->lr / (1.0 - std::pow(opt->beta1, t)));
  s.eps = static_cast<float>(opt->eps);
  s.key0 = static_cast<uint32_t>(opt->seed);
  s.key1 = static_cast<uint32_t>(opt->seed >> 32);
  s.step = static_cast<uint32_t>(opt->step);
  auto make = [&](int i, Entry &e) {
    const echo_adamw_tensor &x = tensors[i];
    if (x.n == 0) return false;
    e.p = x.param;
    e.g = x.grad;
    e.m = x.exp_avg;
    e.v = x.exp_avg_sq;
    e.m_scale = x.avg_scales;
    e.v_scale = x.sq_scales;
    e.copy = static_cast<__nv_bfloat16 *>(x.param_copy);
    e.n = x.n;
    e.decay = static_cast<float>(1.0 - opt->lr * x.weight_decay);
    e.id = static_cast<uint32_t>(i);
    e.vec = aligned(x.param, 32) && aligned(x.grad, 8 * gb) && aligned(x.exp_avg, bits) && aligned(x.exp_avg_sq, bits) &&
            aligned(x.param_copy, 16);
    return true;
  };
  return launch_list(n_tensors, s, opt->grad_format, bits, make, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
             ? ECHO_OK
             : ECHO_ERR_CUDA;
}

int echo_adamw_unpack(const echo_adamw_tensor *tensors, int32_t n_tensors, float *const *out_avg,
                      float *const *out_avg_sq, void *cuda_stream) {
  if (n_tensors < 0 || (n_tensors > 0 && (!tensors || !out_avg || !out_avg_sq))) return ECHO_ERR_INVALID;
  if (!list_ok(tensors, n_tensors, 8, 2, false)) return ECHO_ERR_INVALID;
  for (int i = 0; i < n_tensors; ++i)
    if (tensors[i].n > 0 && (!out_avg[i] || !out_avg_sq[i] || !aligned(out_avg[i], 4) || !aligned(out_avg_sq[i], 4)))
      return ECHO_ERR_INVALID;
  if (n_tensors == 0) return ECHO_OK;
  auto make = [&](int i, Entry &e) {
    const echo_adamw_tensor &x = tensors[i];
    if (x.n == 0) return false;
    e.p = out_avg[i];
    e.copy = reinterpret_cast<__nv_bfloat16 *>(out_avg_sq[i]);
    e.m = x.exp_avg;
    e.v = x.exp_avg_sq;
    e.m_scale = x.avg_scales;
    e.v_scale = x.sq_scales;
    e.n = x.n;
    e.vec = aligned(out_avg[i], 32) && aligned(out_avg_sq[i], 32) && aligned(x.exp_avg, 8) && aligned(x.exp_avg_sq, 8);
    return true;
  };
  return launch_list(n_tensors, Scalars{}, 2, 0, make, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? ECHO_OK
                                                                                                              : ECHO_ERR_CUDA;
}

}  // extern "C"
