// One AdamW step over many tensors in one launch, with moments in fp32 or in 8 bits.
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,
//   p <- p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments: 256 consecutive elements of a tensor share two fp32 scales, the largest |m| (M) and the largest v (V)
// of the block.  A code stands for M (c/127) |c/127| (first moment) and V (c/255)^4 (second moment): quadratic and
// quartic companding put the steps where small values are, so that a block may span five decades of |m| and nine of v.
//   first moment   the nearest code on the companded axis, rint(127 sqrt(|m| / M)), or (RANDOM) one of the two codes
//                  around |m| with the mean kept.  Without a gradient a step multiplies a code by sqrt(b1), and the
//                  nearest to sqrt(0.9) c is c itself up to c = 9: such an element keeps its m while the block's largest
//                  stays, and as v falls beside it the update grows.  Rounding at random lets it fall as it should (one
//                  element in 16 without a gradient after step 50, b2 = 0.95: after 2000 steps exact AdamW has moved
//                  it by 7 lr, the nearest code by 8400 lr, random rounding by 7.5 lr);
//   second moment  one of the two codes around v, the upper with the probability that keeps the mean (v moves by
//                  1 - b2 a step, less than a code's width: rounding to the nearest would never let it fall), and never
//                  0 for a v above 0, since a lost v beside a kept m would make a huge update.
// Codes and scales are those of the 64-bit arithmetic: fp32 decides, and where fp32's own error could move a value
// across a border between two codes the element is decided again in 64 bits.  A scale is
// the fp32 rounding of the 64-bit maximum.
//
// The weight's update is formed in fp32 from the moments before they are rounded, with approximate roots and reciprocals
// (2^-23 each): some fifteen roundings of an update that is itself a small part of the weight, which is rounded once.
//
// A warp takes a block of 256 elements, eight consecutive ones a lane, moved with 32-byte accesses.  fp32 moments: bound
// by HBM (193 M elements with bf16 gradients and copies: 893 to 902 us, 6.0 TB/s).  8-bit moments, the same step against
// 471 us of traffic at the copy rate: 776 us with nearest codes, about 100 instructions an element, and 934 us with
// random first moments, 120 (a second Philox and the squares' rule); instructions issue in 69 % of the slots.  Unpacking
// them: 322 us, 6.0 TB/s.  Tensors off the 8-element boundaries go element by element: 40 M elements with fp32 moments in
// 287 us instead of 176, with 8-bit random ones in 255 instead of 196.  Bytes and whole numbers become floats, and back, through a float's low
// bits, not the conversion unit.  Fetching the next 8-bit block into L2 ahead of time: 1134 against 1086 us for step and
// unpack, so it is not done.
#include <cmath>
#include <new>
#include <algorithm>

#include "common.cuh"
#include "ptx.cuh"

namespace echo {
namespace {

constexpr int kBlock = 256;                  // elements that share the 8-bit scales; one warp, eight per lane
constexpr int kThreads = 256, kResident = 4;        // threads per CTA, CTAs per SM

struct Entry {
  float *p;
  const void *g;
  void *m, *v;
  float *m_scale, *v_scale;
  __nv_bfloat16 *copy;
  int64_t n;
  // 1 - lr wd in two parts, the larger rounded towards zero: fp32's nearest number alone is off by up to 2^-25, which is
  // 0.7 % of a decay of 3e-6 and all of one of 1e-8.  (Both have one sign and, where there is a weight left, neither is
  // 0, so that an infinite weight stays what it is without a branch: 1 is 1 - 2^-24 and 2^-24.)
  float decay, decay_rest;
  uint32_t first;                            // blocks of the launch before this tensor's
  uint32_t id_vec;                           // place in the caller's list (keys the random numbers); bit 31: every array
                                             // starts on a boundary of its 8-element pieces
  __device__ uint32_t id() const { return id_vec & 0x7fffffffu; }
  __device__ bool vec() const { return (id_vec >> 31) != 0; }
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
  if constexpr (WHOLE) {
    load8(p, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? p[j] : 0.f;
  }
}
template <bool WHOLE> __device__ __forceinline__ void put_f32(float *p, int left, const float (&x)[8]) {
  if constexpr (WHOLE) {
    store8(p, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = x[j];
  }
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
// the eight codes of a lane, element j in byte j
template <bool WHOLE> __device__ __forceinline__ uint64_t get_codes(const void *c, size_t at, int left) {
  const uint8_t *b = static_cast<const uint8_t *>(c) + at;
  if constexpr (WHOLE) {
    const uint2 w = __ldcs(reinterpret_cast<const uint2 *>(b));
    return static_cast<uint64_t>(w.y) << 32 | w.x;
  } else {
    uint64_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) w |= static_cast<uint64_t>(b[j]) << (8 * j);
    return w;
  }
}
template <bool WHOLE> __device__ __forceinline__ void put_codes(void *c, size_t at, int left, uint64_t w) {
  uint8_t *b = static_cast<uint8_t *>(c) + at;
  if constexpr (WHOLE) {
    *reinterpret_cast<uint2 *>(b) = make_uint2(static_cast<uint32_t>(w), static_cast<uint32_t>(w >> 32));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) b[j] = static_cast<uint8_t>(w >> (8 * j));
  }
}
__device__ __forceinline__ uint32_t byte_of(uint64_t w, int j) { return static_cast<uint32_t>(w >> (8 * j)) & 0xffu; }
__device__ __forceinline__ int signed_byte(uint64_t w, int j) { return static_cast<int>(static_cast<int8_t>(byte_of(w, j))); }
__device__ __forceinline__ void set_byte(uint64_t &w, int j, int code) {
  w = (w & ~(0xffull << (8 * j))) | static_cast<uint64_t>(code & 0xff) << (8 * j);
}
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
  const double q = code * (1.0 / 127.0);
  return s.b1_d * (q * fabs(q) * scale) + s.b1c_d * (static_cast<double>(g) * gs);
}
__device__ __forceinline__ double exact_sq(const Scalars &s, uint32_t code, float scale, float g, float gs) {
  const double q = code * (1.0 / 255.0), h = static_cast<double>(g) * gs;
  return s.b2_d * (q * q * (q * q) * scale) + s.b2c_d * h * h;
}
// Largest magnitude of three; NaN wins, so that it shows.  Across a warp by the bits of the (non-negative) values, which
// order like the values, NaN above infinity.
__device__ __forceinline__ float max_or_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
  return d;
}
__device__ __forceinline__ float warp_max(float v) {
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fabsf(v))));
}
// Whole numbers and floats without the conversion unit: a float 2^23 + n holds n in its low bits.
constexpr float kTwo23 = 8388608.0f, kRound = 12582912.0f;      // 2^23, 1.5 * 2^23
__device__ __forceinline__ float byte_plus_two23(uint32_t word, int byte) {
  return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440u | byte));
}
__device__ __forceinline__ float half_plus_two23(uint32_t word, int half) {
  return __uint_as_float(__byte_perm(word, 0x4B000000u, half ? 0x7432u : 0x7410u));
}
__device__ __forceinline__ bool has_zero_byte(uint32_t x) { return ((x - 0x01010101u) & ~x & 0x80808080u) != 0; }
// low bytes of eight registers
__device__ __forceinline__ uint64_t low_bytes(const uint32_t (&r)[8]) {
  const uint32_t lo = __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
  const uint32_t hi = __byte_perm(__byte_perm(r[4], r[5], 0x0040), __byte_perm(r[6], r[7], 0x0040), 0x5410);
  return static_cast<uint64_t>(hi) << 32 | lo;
}
__device__ __forceinline__ float sqrt_ftz(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_ftz(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rsqrt_ftz(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
using ptx::add2;
using ptx::fma2;
using ptx::mul2;
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// relative error of the fp32 moments, generously: a handful of roundings of 2^-24 each
constexpr float kMomentErr = 1e-6f;

// Below these a block's products of codes and scales may leave fp32's normal numbers (M / 127^2, V / 255^4).
constexpr float kTinyAvg = 1e-32f, kTinySq = 1e-27f;
// a largest value below the normal numbers counts as 0
__device__ __forceinline__ float kept_scale(float largest) { return largest < 1.17549435e-38f ? 0.f : largest; }

// a lane's elements, by number (each lane reads its own only)
struct Stash {
  float4 g[2][32];
  uint64_t m[32], v[32];
  __device__ float old_g(int lane, int j) const { return reinterpret_cast<const float *>(&g[j >> 2][lane])[j & 3]; }
  __device__ int old_m(int lane, int j) const { return reinterpret_cast<const int8_t *>(&m[lane])[j]; }
  __device__ uint32_t old_v(int lane, int j) const { return reinterpret_cast<const uint8_t *>(&v[lane])[j]; }
};

// the random numbers of eight elements for the second (moment 0) or the first moment (1), and the one of element j in
// [0, 1).  (An octet's number stays below 2^35: the counter's bit 63 is free.)
__device__ __forceinline__ uint4 random_words(const Scalars &s, const Entry &e, uint64_t octet, uint32_t moment = 0) {
  return philox(make_uint4(static_cast<uint32_t>(octet), static_cast<uint32_t>(octet >> 32) | moment << 31, e.id(), s.step),
                s.key0, s.key1);
}
__device__ __forceinline__ double random_of(const uint4 &w, int j) {
  const uint64_t half = j < 4 ? static_cast<uint64_t>(w.y) << 32 | w.x : static_cast<uint64_t>(w.w) << 32 | w.z;
  return static_cast<double>(static_cast<uint32_t>(half >> (16 * (j & 3))) & 0xffffu) * 1.52587890625e-05;
}

// The first-moment code below or above y = 127^2 |m| / M, the upper one where u + 2^-17 is below y's place between the two
// (u has 16 bits; half a step more keeps the mean, and a code whose own value returns with another last bit).
__device__ __forceinline__ int random_avg_code(double y, double u) {
  const double d = fmin(floor(sqrt(y)), 126.0);
  return static_cast<int>(d) + ((u + 7.62939453125e-06) * (2.0 * d + 1.0) < y - d * d ? 1 : 0);
}

// A block so small that fp32 products of its codes and scales leave the normal numbers: all of it in 64 bits.
template <bool RANDOM>
__device__ __noinline__ void quantise_tiny(const Scalars &s, const Entry &e, int64_t block, int lane, int left, float gs,
                                           float M0, float V0, const Stash &stash) {
  const uint64_t octet = static_cast<uint64_t>(block) * (kBlock / 8) + lane;
  const uint4 words = random_words(s, e, octet), avg_words = RANDOM ? random_words(s, e, octet, 1) : words;
  float M = 0.f, V = 0.f;
  for (int j = 0; j < left; ++j) {
    M = max_or_nan(M, static_cast<float>(exact_avg(s, stash.old_m(lane, j), M0, stash.old_g(lane, j), gs)), 0.f);
    V = max_or_nan(V, static_cast<float>(exact_sq(s, stash.old_v(lane, j), V0, stash.old_g(lane, j), gs)), 0.f);
  }
  M = kept_scale(warp_max(M));
  V = kept_scale(warp_max(V));
  uint64_t mo = 0, vo = 0;
  for (int j = 0; j < left; ++j) {
    const double x = exact_avg(s, stash.old_m(lane, j), M0, stash.old_g(lane, j), gs);
    const double y = exact_sq(s, stash.old_v(lane, j), V0, stash.old_g(lane, j), gs);
    const int c = !(M > 0.f) ? 0
                  : RANDOM   ? random_avg_code(fabs(x) / M * 16129.0, random_of(avg_words, j))
                             : static_cast<int>(rint(127.0 * sqrt(fabs(x) / M)));
    set_byte(mo, j, x < 0.0 ? -c : c);
    if (V > 0.f && y > 0.0) {
      const double w = y / V * 4228250625.0, d = fmin(floor(sqrt(sqrt(w))), 254.0), lo = d * d * (d * d);
      const double hi = (d + 1.0) * (d + 1.0) * ((d + 1.0) * (d + 1.0));
      set_byte(vo, j, max(static_cast<int>(d) + (random_of(words, j) * (hi - lo) < w - lo ? 1 : 0), 1));
    }
  }
  put_codes<false>(e.m, block * kBlock + lane * 8, left, mo);
  put_codes<false>(e.v, block * kBlock + lane * 8, left, vo);
  if (lane == 0) {
    e.m_scale[block] = M;
    e.v_scale[block] = V;
  }
}

template <int FMT, bool EIGHT, bool RANDOM, bool WHOLE>
__device__ __forceinline__ void step_block(const Scalars &s, const Entry &e, int64_t block, int lane, float gs, Stash &stash) {
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
      p[j] = fmaf(p[j], e.decay, fmaf(p[j], e.decay_rest, -s.rate * __fdividef(m[j], denom)));
    }
    put_f32<WHOLE>(static_cast<float *>(e.m) + at, left, m);
    put_f32<WHOLE>(static_cast<float *>(e.v) + at, left, v);
    put_f32<WHOLE>(e.p + at, left, p);
    if (e.copy) put_copy<WHOLE>(e.copy + at, left, p);
  } else {
    const uint64_t mc = get_codes<WHOLE>(e.m, at, left), vc = get_codes<WHOLE>(e.v, at, left);
    const float M0 = e.m_scale[block], V0 = e.v_scale[block];
    // (what the 64-bit parts below want of single elements by number is kept in shared memory, not in registers)
    stash.g[0][lane] = make_float4(g[0], g[1], g[2], g[3]);
    stash.g[1][lane] = make_float4(g[4], g[5], g[6], g[7]);
    stash.m[lane] = mc;
    stash.v[lane] = vc;
    auto old_g = [&](int j) { return stash.old_g(lane, j); };
    auto old_m = [&](int j) { return stash.old_m(lane, j); };
    auto old_v = [&](int j) { return stash.old_v(lane, j); };
    float m[8], v[8];
    float big_m = 0.f, big_b = 0.f, big_v = 0.f;
    const uint64_t mb = mc ^ 0x8080808080808080ull;            // c + 128
    const float km = s.b1 * M0 * (1.0f / 16129.0f), kv = s.b2 * V0 * (1.0f / 4228250625.0f);      // 127^2, 255^4
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint32_t mw = static_cast<uint32_t>(i < 4 ? mb : mb >> 32), vw = static_cast<uint32_t>(i < 4 ? vc : vc >> 32);
      const float2 c = add2(make_float2(byte_plus_two23(mw, i & 3), byte_plus_two23(mw, (i & 3) + 1)), both(-kTwo23 - 128.0f));
      const float2 d = add2(make_float2(byte_plus_two23(vw, i & 3), byte_plus_two23(vw, (i & 3) + 1)), both(-kTwo23));
      const float2 h = mul2(make_float2(g[i], g[i + 1]), both(gs)), b = mul2(h, both(s.b1c));
      const float2 cc = make_float2(c.x * fabsf(c.x), c.y * fabsf(c.y));
      const float2 mm = fma2(cc, both(km), b);
      const float2 d2 = mul2(d, d), vv = fma2(mul2(d2, d2), both(kv), mul2(mul2(h, both(s.b2c)), h));
      m[i] = mm.x;
      m[i + 1] = mm.y;
      v[i] = vv.x;
      v[i + 1] = vv.y;
      big_m = max_or_nan(big_m, mm.x, mm.y);
      big_v = max_or_nan(big_v, vv.x, vv.y);
      big_b = max_or_nan(big_b, b.x, b.y);
      const float2 denom = fma2(make_float2(sqrt_ftz(vv.x), sqrt_ftz(vv.y)), both(s.root_corr), both(s.eps));
      const float2 up = mul2(mm, make_float2(rcp_ftz(denom.x), rcp_ftz(denom.y)));        // (denom is at least eps)
      const float2 old = make_float2(p[i], p[i + 1]);
      const float2 pp = fma2(old, both(e.decay), fma2(old, both(e.decay_rest), mul2(up, both(-s.rate))));
      p[i] = pp.x;
      p[i + 1] = pp.y;
    }
    put_f32<WHOLE>(e.p + at, left, p);
    if (e.copy) put_copy<WHOLE>(e.copy + at, left, p);
    // scales: the 64-bit maximum as fp32, found among the elements that fp32 cannot tell from it.  (The 64-bit parts
    // are loops over bit masks: unrolled, their code would not fit the instruction cache.)
    big_m = warp_max(big_m);
    big_v = warp_max(big_v);
    const bool tiny = (big_v > 0.f && big_v < kTinySq) || (V0 > 0.f && V0 < kTinySq) || (big_m > 0.f && big_m < kTinyAvg) ||
                      (M0 > 0.f && M0 < kTinyAvg);
    // b1 |m| is at most b1 M0 and (1 - b1) |g| at most its largest: their sum's kMomentErr-th part bounds the error of
    // every m of the block
    const float err_m = kMomentErr * fmaf(s.b1, M0, warp_max(big_b));
    uint32_t near_m = 0, near_v = 0;
    const float from_m = err_m > 0.f ? fmaf(err_m, -2.0f, big_m) : INFINITY;
    const float from_v = big_v > 0.f ? big_v * (1.0f - 2.0f * kMomentErr) : INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (fabsf(m[j]) >= from_m) near_m |= 1u << j;
      if (v[j] >= from_v) near_v |= 1u << j;
    }
    float M = 0.f, V = 0.f;
#pragma unroll 1
    for (; near_m; near_m &= near_m - 1) {
      const int j = __ffs(near_m) - 1;
      M = fmaxf(M, static_cast<float>(fabs(exact_avg(s, old_m(j), M0, old_g(j), gs))));
    }
#pragma unroll 1
    for (; near_v; near_v &= near_v - 1) {
      const int j = __ffs(near_v) - 1;
      V = fmaxf(V, static_cast<float>(exact_sq(s, old_v(j), V0, old_g(j), gs)));
    }
    M = isfinite(big_m) ? kept_scale(warp_max(M)) : big_m;
    V = isfinite(big_v) ? kept_scale(warp_max(V)) : big_v;
    const float inv_m = M > 0.f ? 16129.0f / M : 0.f, inv_v = V > 0.f ? 4228250625.0f / V : 0.f;
    const uint64_t octet = static_cast<uint64_t>(block) * (kBlock / 8) + lane;
    const uint4 words4 = random_words(s, e, octet);
    const uint32_t words[4] = {words4.x, words4.y, words4.z, words4.w};
    uint4 avg_words4 = make_uint4(0u, 0u, 0u, 0u);
    if (RANDOM) avg_words4 = random_words(s, e, octet, 1);
    const uint32_t avg_words[4] = {avg_words4.x, avg_words4.y, avg_words4.z, avg_words4.w};
    uint32_t mr[8], vr[8];                     // codes in the low bytes
    uint32_t unsure_m = 0, unsure_v = 0;
    const float err_y = 0.5f * err_m * inv_m;
    const float of_g = 2.0f * kMomentErr * s.b1c * fabsf(gs) * inv_m;
    const float4 ga = RANDOM ? stash.g[0][lane] : float4{}, gb = RANDOM ? stash.g[1][lane] : float4{};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 ym = mul2(make_float2(m[i], m[i + 1]), both(inv_m)), w = mul2(make_float2(v[i], v[i + 1]), both(inv_v));
      if constexpr (!RANDOM) {
        // first moment: x = sqrt(y), y = 127^2 |m| / M, is off by (error of y) / (2 x) and, x being at most 127, less than
        // 1e-4 of its own rounding.  (Below y = 1/1000 every code is 0, and so stands for the smaller ones.)
        const float2 y = make_float2(fmaxf(fabsf(ym.x), 1e-3f), fmaxf(fabsf(ym.y), 1e-3f));
        const float2 rs = make_float2(rsqrt_ftz(y.x), rsqrt_ftz(y.y)), x = mul2(y, rs);
        const float2 xs = make_float2(copysignf(x.x, ym.x), copysignf(x.y, ym.y));
        const float2 r = add2(xs, both(kRound)), dist = fma2(add2(r, both(-kRound)), both(-1.0f), xs);
        const float2 clear = fma2(rs, both(-err_y), both(0.4999f));
        mr[i] = __float_as_uint(r.x);
        mr[i + 1] = __float_as_uint(r.y);
        if (fabsf(dist.x) > clear.x) unsure_m |= 1u << i;
        if (fabsf(dist.y) > clear.y) unsure_m |= 2u << i;
      } else {
        // first moment: y = 127^2 |m| / M lies between d^2 and (d + 1)^2 (d at most 126; 126.5 stands for all above it),
        // the second moment's rule with squares.  m is off by kMomentErr of its terms, |b1 m0| + |(1 - b1) g|, at most
        // |m| + 2 |(1 - b1) g|: `near` in y.  The root's error may name the neighbouring interval where y's place is
        // within near / width + 1.5e-5 of 0 or 1: that matters only for random numbers as near to them.
        const float2 y = make_float2(fabsf(ym.x), fabsf(ym.y));
        const float2 z = make_float2(fminf(sqrt_ftz(y.x), 126.5f), fminf(sqrt_ftz(y.y), 126.5f));
        const float2 zr = make_float2(__fadd_rd(z.x, kTwo23), __fadd_rd(z.y, kTwo23)), d = add2(zr, both(-kTwo23));
        const float2 above = fma2(mul2(d, both(-1.0f)), d, y), width = fma2(d, both(2.0f), both(1.0f));
        const float2 u = fma2(make_float2(half_plus_two23(avg_words[i >> 1], 0), half_plus_two23(avg_words[i >> 1], 1)),
                              both(-1.52587890625e-05f), both(128.0f - 7.62939453125e-06f));   // minus the random number
        const float2 diff = fma2(u, width, above), mid = add2(u, both(0.5f));
        const float2 h = i < 4 ? (i & 2 ? make_float2(ga.z, ga.w) : make_float2(ga.x, ga.y))
                               : (i & 2 ? make_float2(gb.z, gb.w) : make_float2(gb.x, gb.y));
        const float2 near = fma2(make_float2(fabsf(h.x), fabsf(h.y)), both(of_g), mul2(y, both(1.2f * kMomentErr)));
        const float2 edge = fma2(make_float2(fabsf(mid.x), fabsf(mid.y)), width, near), from = mul2(width, both(0.4999f));
        const uint32_t cx = __float_as_uint(zr.x) + (diff.x > 0.f ? 1u : 0u), cy = __float_as_uint(zr.y) + (diff.y > 0.f ? 1u : 0u);
        mr[i] = ym.x < 0.f ? 0u - cx : cx;
        mr[i + 1] = ym.y < 0.f ? 0u - cy : cy;
        if (fabsf(diff.x) <= near.x || edge.x > from.x) unsure_m |= 1u << i;
        if (fabsf(diff.y) <= near.y || edge.y > from.y) unsure_m |= 2u << i;
      }
      // second moment: w = 255^4 v / V lies between d^4 and (d + 1)^4 (d at most 254; 254.5 stands for all above it).
      // Next to d^4 the rounded root may name the neighbouring interval, which gives the same code unless the random
      // number u is within (error of the place in the interval) < 2.4e-4 of 0 or 1.  (A v that just decays with its
      // block sits there step after step: only these u may cost anything.)
      const bool some_x = w.x > 0.f, some_y = w.y > 0.f;
      const float2 z = make_float2(fminf(sqrt_ftz(sqrt_ftz(w.x)), 254.5f), fminf(sqrt_ftz(sqrt_ftz(w.y)), 254.5f));
      const float2 zr = make_float2(__fadd_rd(z.x, kTwo23), __fadd_rd(z.y, kTwo23)), d = add2(zr, both(-kTwo23));
      const float2 d2 = mul2(d, d), above = fma2(mul2(d2, both(-1.0f)), d2, w);
      const float2 width = fma2(fma2(fma2(d, both(4.0f), both(6.0f)), d, both(4.0f)), d, both(1.0f));
      const float2 u = fma2(make_float2(half_plus_two23(words[i >> 1], 0), half_plus_two23(words[i >> 1], 1)),
                            both(-1.52587890625e-05f), both(128.0f));          // minus the random number
      const float2 diff = fma2(u, width, above), near = mul2(w, both(1.2f * kMomentErr)), mid = add2(u, both(0.5f));
      vr[i] = max(__float_as_uint(zr.x) + (diff.x > 0.f ? 1u : 0u), some_x ? 0x4B000001u : 0x4B000000u);
      vr[i + 1] = max(__float_as_uint(zr.y) + (diff.y > 0.f ? 1u : 0u), some_y ? 0x4B000001u : 0x4B000000u);
      if (fabsf(diff.x) <= near.x || fabsf(mid.x) > 0.49976f) unsure_v |= 1u << i;
      if (fabsf(diff.y) <= near.y || fabsf(mid.y) > 0.49976f) unsure_v |= 2u << i;
    }
    uint64_t mo = low_bytes(mr), vo = low_bytes(vr);
    // A gradient (or an old v) so far below its block's that fp32 does not hold its v still makes one above 0: 64 bits
    // decide on codes 0 beside either.
    if (has_zero_byte(static_cast<uint32_t>(vo)) || has_zero_byte(static_cast<uint32_t>(vo >> 32))) {
#pragma unroll 1
      for (int j = 0; j < 8; ++j)
        if (byte_of(vo, j) == 0 && (old_g(j) != 0.f || old_v(j) != 0)) unsure_v |= 1u << j;
    }
    if (!(M > 0.f)) unsure_m = 0;
    if (!(V > 0.f)) unsure_v = 0;
    // A code from the 64-bit moment, rounded to fp32 only for the root, is right or next to it: it is compared with the
    // borders around it in 64 bits.  (Of a second moment, a sum without cancellation, that holds for fp32's own code.)
#pragma unroll 1
    for (; unsure_m; unsure_m &= unsure_m - 1) {
      const int j = __ffs(unsure_m) - 1;
      const double x = exact_avg(s, old_m(j), M0, old_g(j), gs), y = fabs(x) * 16129.0;
      int c;
      if (RANDOM) {
        c = random_avg_code(y / M, random_of(avg_words4, j));
      } else {
        c = static_cast<int>(rintf(sqrt_ftz(static_cast<float>(fabs(x)) * inv_m)));
        const double up = (c + 0.5) * (c + 0.5) * M, down = (c - 0.5) * (c - 0.5) * M;
        const bool odd = (c & 1) != 0;                          // (y on the border: the even code, as rint has it)
        if (odd ? y >= up : y > up) ++c;
        else if (c > 0 && (odd ? y <= down : y < down)) --c;
      }
      set_byte(mo, j, x < 0.0 ? -c : c);
    }
#pragma unroll 1
    for (; unsure_v; unsure_v &= unsure_v - 1) {
      const int j = __ffs(unsure_v) - 1;
      const double y = exact_sq(s, old_v(j), V0, old_g(j), gs) * 4228250625.0;
      double d = min(static_cast<int>(byte_of(vo, j)), 254), lo = d * d * (d * d) * V;
      if (y < lo) {                            // the code is the upper one of its interval
        d -= 1.0;
        lo = d * d * (d * d) * V;
      }
      const double hi = (d + 1.0) * (d + 1.0) * ((d + 1.0) * (d + 1.0)) * V;
      if (y > 0.0) set_byte(vo, j, max(static_cast<int>(d) + (random_of(words4, j) * (hi - lo) < y - lo ? 1 : 0), 1));
    }
    if (tiny) {                                // (here few registers are live; the codes above mean nothing)
      quantise_tiny<RANDOM>(s, e, block, lane, left, gs, M0, V0, stash);
      return;
    }
    put_codes<WHOLE>(e.m, at, left, mo);
    put_codes<WHOLE>(e.v, at, left, vo);
    if (lane == 0) {
      e.m_scale[block] = M;
      e.v_scale[block] = V;
    }
  }
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

template <int N, int FMT, bool EIGHT, bool RANDOM>
__global__ void __launch_bounds__(kThreads, kResident) adamw_kernel(const __grid_constant__ Table<N> t) {
  const float gs = t.s.grad_scale ? *t.s.grad_scale : 1.0f;
  if (!isfinite(gs)) return;                              // an overflowed step changes nothing
  const int lane = threadIdx.x & 31;
  __shared__ Stash stashes[EIGHT ? kThreads / 32 : 1];
  Stash &stash = stashes[EIGHT ? threadIdx.x >> 5 : 0];
  for_blocks(t, [&](const Entry &e, int64_t block, uint32_t) {
    if (e.vec() && (block + 1) * kBlock <= e.n) step_block<FMT, EIGHT, RANDOM, true>(t.s, e, block, lane, gs, stash);
    else step_block<FMT, EIGHT, RANDOM, false>(t.s, e, block, lane, gs, stash);
  });
}

// The values that 8-bit moments stand for: p and copy of an entry hold the two outputs.
template <int N> __global__ void __launch_bounds__(kThreads) adamw_unpack_kernel(const __grid_constant__ Table<N> t) {
  const int lane = threadIdx.x & 31;
  for_blocks(t, [&](const Entry &e, int64_t block, uint32_t) {
    const int64_t at = block * kBlock + lane * 8;
    const int left = static_cast<int>(min(static_cast<int64_t>(8), max(static_cast<int64_t>(0), e.n - at)));
    const bool whole = e.vec() && left == 8;
    const uint64_t mc = whole ? get_codes<true>(e.m, at, left) : get_codes<false>(e.m, at, left);
    const uint64_t vc = whole ? get_codes<true>(e.v, at, left) : get_codes<false>(e.v, at, left);
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

template <int N, int FMT> cudaError_t launch_step(const Table<N> &t, int state_bits, bool random_avg, int grid, cudaStream_t s) {
  if (state_bits == 32) adamw_kernel<N, FMT, false, false><<<grid, kThreads, 0, s>>>(t);
  else if (random_avg) adamw_kernel<N, FMT, true, true><<<grid, kThreads, 0, s>>>(t);
  else adamw_kernel<N, FMT, true, false><<<grid, kThreads, 0, s>>>(t);
  return cudaGetLastError();
}
template <int N>
cudaError_t launch_any(const Table<N> &t, int grad_format, int state_bits, bool random_avg, int grid, cudaStream_t s) {
  if (state_bits == 0) {
    adamw_unpack_kernel<N><<<grid, kThreads, 0, s>>>(t);
    return cudaGetLastError();
  }
  return grad_format == 0   ? launch_step<N, 0>(t, state_bits, random_avg, grid, s)
         : grad_format == 1 ? launch_step<N, 1>(t, state_bits, random_avg, grid, s)
                            : launch_step<N, 2>(t, state_bits, random_avg, grid, s);
}

// Launches over the entries that make(i, entry) fills (false: nothing to do for tensor i), as many per launch as the
// kernel parameters hold.  state_bits 0: unpack.
template <typename Make>
cudaError_t launch_list(int n_tensors, const Scalars &base, int grad_format, int state_bits, bool random_avg, Make make,
                        cudaStream_t s) {
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
    const int grid = static_cast<int>(std::min<uint64_t>(need, static_cast<uint64_t>(sms) * kResident));
    if (n <= kSmallTable) {
      Table<kSmallTable> small;
      small.s = t.s;
      std::copy(t.e, t.e + n, small.e);
      err = launch_any(small, grad_format, state_bits, random_avg, grid, s);
    } else {
      err = launch_any(t, grad_format, state_bits, random_avg, grid, s);
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
  // (the first step's moments come from zeros: nothing is there to fall, and the nearest code is the better one)
  const bool random_avg = opt->state_bits == (8 | ECHO_ADAMW_RANDOM_AVG) && opt->step > 1;
  const int bits = opt->state_bits == (8 | ECHO_ADAMW_RANDOM_AVG) ? 8 : opt->state_bits;
  if (opt->grad_format < 0 || opt->grad_format > 2 || (bits != 8 && bits != 32)) return ECHO_ERR_INVALID;
  // 8-bit moments: roots of denormal numbers count as 0 beside eps
  if (bits == 8 && opt->eps < 1e-12) return ECHO_ERR_UNSUPPORTED;
  const int gb = elem_bytes(opt->grad_format);
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
    const double decay = 1.0 - opt->lr * x.weight_decay;
    e.decay = static_cast<float>(decay);
    if (std::fabs(static_cast<double>(e.decay)) >= std::fabs(decay)) e.decay = std::nextafter(e.decay, 0.0f);
    e.decay_rest = static_cast<float>(decay - e.decay);
    const bool vec = aligned(x.param, 32) && aligned(x.grad, 8 * gb) && aligned(x.exp_avg, bits) &&
                     aligned(x.exp_avg_sq, bits) && aligned(x.param_copy, 16);
    e.id_vec = static_cast<uint32_t>(i) | static_cast<uint32_t>(vec) << 31;
    return true;
  };
  return launch_list(n_tensors, s, opt->grad_format, bits, random_avg, make, static_cast<cudaStream_t>(cuda_stream)) ==
                 cudaSuccess
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
  Range *r = new (std::nothrow) Range[static_cast<size_t>(n_tensors) * 6];
  if (!r) return ECHO_ERR_ARENA;
  size_t n_ranges = 0;
  auto range = [&](const void *p, int64_t bytes, bool written) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    r[n_ranges++] = Range{from, from + static_cast<size_t>(bytes), written};
  };
  for (int i = 0; i < n_tensors; ++i) {
    const echo_adamw_tensor &x = tensors[i];
    if (x.n == 0) continue;
    const int64_t blocks = (x.n + kBlock - 1) / kBlock;
    range(out_avg[i], x.n * 4, true);
    range(out_avg_sq[i], x.n * 4, true);
    range(x.exp_avg, x.n, false);
    range(x.exp_avg_sq, x.n, false);
    range(x.avg_scales, blocks * 4, false);
    range(x.sq_scales, blocks * 4, false);
  }
  const bool ok = apart(r, n_ranges);
  delete[] r;
  if (!ok) return ECHO_ERR_INVALID;
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
    const bool vec = aligned(out_avg[i], 32) && aligned(out_avg_sq[i], 32) && aligned(x.exp_avg, 8) && aligned(x.exp_avg_sq, 8);
    e.id_vec = static_cast<uint32_t>(i) | static_cast<uint32_t>(vec) << 31;
    return true;
  };
  return launch_list(n_tensors, Scalars{}, 2, 0, false, make, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
             ? ECHO_OK
             : ECHO_ERR_CUDA;
}

}  // extern "C"
