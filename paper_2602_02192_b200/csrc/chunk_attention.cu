// Attention of a ragged batch of new tokens over a caller's paged caches.
//
//   o_i = sum_{u <= t_i} exp(q_i . k_u / sqrt(hd)) v_u / sum_{u <= t_i} exp(q_i . k_u / sqrt(hd)),   t_i = L - n + i
//
// Tiles.  The query heads of a kv head read the same keys, so a row of a tile is a (token, query head) pair: 128 rows are
// 128 / (Hq / Hkv) tokens.  Keys come in tiles of 128 (eight pages).  S = Q K^T and O += P V run on the tcgen05 tensor
// cores: Q, K, V in shared memory as TMA leaves them (128-byte swizzle; K is the K-major operand, V the same bytes read as an
// MN-major one), S, P and O in tensor memory, P over the columns that held S.
//
// Two streams of tiles are in flight in a CTA, each with its own warps, S and O, so that the tensor cores work on one while
// the other's probabilities are formed:
//   paired items   two row tiles share each K and V tile (long chunks: keys are read once per 256 rows)
//   single items   one row tile; the streams take 64 keys each of every tile, and their two results are joined at the end
//                  (few rows: what counts is to keep the copies running)
// Either way both streams take every key tile in order, so that a barrier's phase is never more than one away from what is
// waited for.  A step of a stream is 64 keys, and its S has room for two: of pairs, S of the next step is formed while this
// one's probabilities are.
//
// Work.  An item is (sequence, kv head, pair of row tiles or last single one) with its keys.  Items have very different
// lengths and the lengths are in device memory, so every CTA (one to an SM) adds up all items' costs, takes its equal share
// of the total, and walks the items in it; an item that crosses a border is cut between two key tiles.  Cut items leave
// fp32 partial results (unnormalised O, reference, sum) in the workspace, in places that only depend on the CTA, and a second
// launch joins them in key order: no atomics, equal inputs give equal outputs.  Every other item of a head takes its key
// tiles from the last to the first: those are what L2 may still hold.
//
// A row's reference (what its exponents are relative to) is its maximum over the item's first step.  It moves when a
// step's probabilities, relative to it, add up to more than 2^11 (half: 2^15, of 2^6 for the reference) in one of the
// row's four threads, which have sixteen each: the maximum has then grown.  So O is hardly ever rescaled, most steps need no
// maxima, and a probability that is used is at most 2^11 (2^15), which the formats hold.
//
// Probabilities are rounded to the cache's format: the second product wants both operands in it, and V is the caller's.  The
// row's sum is that of the fp32 values.  Measured, the distance to the 64-bit result is 1.1 to 1.7 times that of fp32
// probabilities (of 131001 keys, bf16: 0.0019 to 0.0027 of the result's norm, where rounding the result alone makes 0.0016).
// The sum of the rounded values instead would take 1 to 11 % off that distance, and 2048 tokens over 14336 453 us (422).  A
// second product, of what the rounding leaves, would turn a visible infinite value into NaN (0 times it).
//
// What a row does not see has no part in it: masked scores are replaced, not added to.  A masked probability is 0, but
// 0 times an undefined value would not be: where a step has keys that only some of its rows see, their values are looked
// at, and a step with an infinity or a NaN among them is accumulated by the threads instead (slow, and nothing else).
//
// Roles: warps 0-7 and 8-15 the two streams' softmax, warps 16 and 18 issue their MMAs, warp 17 walks the items and loads.
// A softmax warp has 16 rows, four threads to a row: with 32 rows to a warp and a thread to a row two warps shared a
// scheduler, and what one waited for the other could not fill (2048 tokens over 14336: 447 us, with 16 rows 431).
//
// Measured (32/8 heads of 128, bf16, in bursts; in a run of them the SM clock falls with the power): 256 single tokens over
// 512 to 2559 keys 257 us, 0.96 of the copy rate; 2048 tokens over 14336 422 us, 1.22 PFLOP/s.  Few rows are bound by HBM
// (by power in a run), long chunks of heads of 128 by the issue of MMAs: 12 to a step, about 64 cycles each, where the eight of
// Q K^T with their 64 keys have half the work of the four of P V.  S of 128 keys would halve their number, but with two O
// there is room for one such S a stream, and then its products wait for its softmax (452 us with S of 128, 499 with S of
// 128 whose probabilities go in halves).  Heads of 64 are bound by the softmax warps' chain: wait, load, exponentials, store.

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

#include "chunks.cuh"
#include "ptx.cuh"

namespace echo {

using namespace ptx;

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

namespace {

constexpr int kKeys = 128;                     // keys of a tile
constexpr int kPages = kKeys / kChunkPage;
constexpr int kSoftWarps = 16;
constexpr int kAttThreads = 32 * (kSoftWarps + 4);
constexpr int kMaxCtas = 148;                  // CTAs of a launch: sizes the workspace
constexpr int kItemRing = 4;
constexpr int kDevices = 64;                   // whose properties are remembered
// Probabilities are relative to 2^kShift for a score that equals the reference.  Half precision ends at 2^-24 below: with 1
// for the largest, 100,000 keys whose scores lie 18 below it would lose all that they add up to (bf16 ends at 2^-133).
constexpr int shift_of(bool half) { return half ? 6 : 0; }
// of a thread's sixteen probabilities of a row's step before its reference has to move (half: 65504 ends it)
constexpr float most_sum(bool half) { return half ? 32768.0f : 2048.0f; }

// References beyond this (of q . k) are taken off the scores before these are scaled, which is exact where it counts: relative
// to a rounded product of the two a probability of 1 would be off by 2^(2^-24 times the product), and end in infinity or 0.
constexpr float kFar = 4194304.0f;

// Costs that the shares are cut by: of a key, and of an item's beginning and end.
constexpr int kSingleWeight = 6, kPairWeight = 8, kSingleStart = 2 * 1024, kPairStart = 3 * 1024;
// Measured with heads of 128: with the weights 4 : 8 and half of these starts 40 chunks of 16 to 400 tokens took 437 us instead
// of 356.  Heads of 64 and tiles of 64 rows, whose keys cost less, are cut by the same ratio: shares are then less even.
constexpr int kLeastShare = 1024;              // of a CTA that has work: little work goes to few CTAs

// FEW: no item has more than 64 rows.  MMAs of 64 rows, which take less power (a decode step is bound by HBM in a burst and by
// power in a run), and smaller query tiles, so that the copies get a stage more.
constexpr int kFewRows = 64;
template <int HD, bool FEW> struct AttSmem {
  static constexpr int kQRows = FEW ? kFewRows : 128;
  static constexpr int kRowWarps = kQRows / 16;                       // softmax warps of a stream that can have rows
  static constexpr int kQHalf = kQRows * 128;                         // 64 elements of every row
  static constexpr int kQTile = HD / 64 * kQHalf;
  static constexpr int kStage = kKeys * HD * 2;
  static constexpr int kStages = HD == 128 ? (FEW ? 6 : 5) : (FEW ? 11 : 9);
  static constexpr int kQ = 0, kKV = 2 * kQTile, kBars = kKV + kStages * kStage;
  static constexpr int kBarBytes = 3 * 1024, kTotal = kBars + kBarBytes;
  static_assert(kTotal <= 227 * 1024, "shared memory");
};

struct Item {
  int row0, n_tok, head, pos0;      // first row and tokens of the item, its kv head, position of the first token
  int t0, t1, seen_end, flags;      // key tiles [t0, t1); no row sees key seen_end or a later one
};
constexpr int kPaired = 1, kEnd = 2, kPartLater = 4, kPartFirst = 8;      // parts of a cut item: a later one, the first
constexpr int kBackwards = 16;                                            // the tiles from the last to the first

// What a CTA says of its (at most two) partial results to the joining launch.
struct PartRecord {
  int first, later;                 // partial result present: of the first tiles of an item; of later ones
  int later_ends;                   // the later one reaches the item's last tile
  Item item;                        // of `first`
};
constexpr int kRecordBytes = 64;
static_assert(sizeof(PartRecord) <= kRecordBytes, "record");

struct WaitLimit {
  uint64_t ns;                      // of a wait
  uint32_t look;                    // the clock is read every look + 1 tries (a power of two)
};

struct AttendArgs {
  ChunkArgs c;
  WaitLimit limit;
  uint16_t *out;
  float *part_o;                    // [cta][2][rows_cap][hd]
  float2 *part_ml;                  // [cta][2][rows_cap]: reference in log2 units, sum
  PartRecord *records;
  int Hq, Hkv, group, tile_tok, load_tok /* of a query tile's tokens, those that are loaded */, n_pages, rows_cap;
  float scale_log2;
};

// ---- tensor memory and descriptors -----------------------------------------------------------------
// A warp reads 16 rows (lanes): thread t holds of row t / 4, and of row t / 4 + 8, two neighbouring columns of every eight
// (r[4 b], r[4 b + 1]; r[4 b + 2], r[4 b + 3]).  Loads include their wait.
__device__ __forceinline__ void tc_ld_64cols(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      "\n\ttcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_ld_32cols(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      "\n\ttcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_st_32cols(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
// The same rows with one column of every four to a thread: 16-bit numbers in pairs, as the columns above.
__device__ __forceinline__ void tc_st_64keys(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tc_ld_8keys(uint32_t taddr, uint32_t (&r)[2]) {
  asm volatile("tcgen05.ld.sync.aligned.16x128b.x1.b32 {%0, %1}, [%2];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=r"(r[0]), "=r"(r[1])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// largest of three; NaN wins
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// A whole warp's bounded wait; its lanes go on or give up together.  Votes keep the loop free of divergence, and the clock
// is read now and then only: a wait that has nothing to wait for takes 60 cycles, four times less than with a clock and a
// branch of each lane's own.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag, const WaitLimit &limit) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  uint64_t t0 = 0;
#pragma unroll 1
  for (uint32_t i = 1;; ++i) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((i & limit.look) == 0) {
      const uint64_t now = global_timer_ns();
      if (t0 == 0) t0 = now;
      if (__any_sync(0xffffffffu, *abort_flag != 0 || now - t0 > limit.ns)) break;
    }
  }
  *abort_flag = 1;
  return false;
}
// D += A B with A in tensor memory (16-bit pairs of one row in a 32-bit column)
__device__ __forceinline__ void tc_mma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// shared-memory matrix descriptor, 128-byte swizzle: atoms of 8 rows x 128 bytes.  K-major: sbo between 8-row groups.
// MN-major (a row of 128 bytes holds 64 elements of the MN dimension at one k): lbo between atoms along MN, sbo along K.
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(lbo >> 4) << 16) |
         (static_cast<uint64_t>(sbo >> 4) << 32) | (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
constexpr uint32_t kIdescBMajorMN = 1u << 16;
// M = 128, or 64: rows 16 i .. 16 i + 15 are then the first 16 lanes of warp quarter i
__host__ __device__ constexpr uint32_t idesc_rows(uint32_t idesc, int rows) {
  return (idesc & ~(31u << 24)) | (static_cast<uint32_t>(rows >> 4) << 24);
}
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}

__device__ __forceinline__ void tma_load_3d(const CUtensorMap *map, uint64_t *bar, uint32_t dst, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(const CUtensorMap *map, uint64_t *bar, uint32_t dst, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// ---- costs -------------------------------------------------------------------------------------------
// Items of one kv head of a sequence: n_items of up to 2 tile_tok tokens, the last one single if its tokens fit one tile.
struct SeqCost {
  int n_items, base, n, step;       // base = L - n: keys in front of the chunk (below 0: the first rows see nothing)
  bool last_single;
  // keys that item i's last token sees
  __device__ __forceinline__ int seen(int i) const { return max(0, base + min(n, (i + 1) * step)); }
  __device__ __forceinline__ bool single(int i) const { return i == n_items - 1 && last_single; }
  __device__ __forceinline__ long long cost(int i) const {
    return single(i) ? kSingleStart + static_cast<long long>(kSingleWeight) * seen(i) : kPairStart + static_cast<long long>(kPairWeight) * seen(i);
  }
  // cost of the items before i
  __device__ __forceinline__ long long before(int i) const {
    const int full = min(i, n_items - 1), dead = base < 0 ? min(full, -base / step) : 0;      // items 0 .. dead - 1 see nothing
    const long long m = full - dead;
    long long c = static_cast<long long>(full) * kPairStart +
                  kPairWeight * (m * base + static_cast<long long>(step) * (m * (dead + 1) + m * (m - 1) / 2));
    if (i == n_items) c += cost(n_items - 1);
    return c;
  }
  __device__ __forceinline__ long long head() const { return n_items ? before(n_items) : 0; }
};
__device__ __forceinline__ SeqCost seq_cost(const SeqSpan &p, int tile_tok) {
  SeqCost k;
  k.step = 2 * tile_tok;
  k.n = p.ok ? p.n : 0;
  k.base = p.kv - p.n;
  k.n_items = (k.n + k.step - 1) / k.step;
  const int rest = k.n - (k.n_items - 1) * k.step;
  k.last_single = k.n_items && rest <= tile_tok;
  return k;
}
// key tile at which an item is cut, x into its cost
__device__ __forceinline__ int cut_tile(long long x, bool single, int seen) {
  const int tiles = (seen + kKeys - 1) / kKeys;
  const long long y = x - (single ? kSingleStart : kPairStart), per = (single ? kSingleWeight : kPairWeight) * kKeys;
  return y <= 0 ? 0 : static_cast<int>(min(static_cast<long long>(tiles), (y + per - 1) / per));
}

// ---- the kernel ----------------------------------------------------------------------------------------
template <int HD, bool FEW> struct Shared {
  uint64_t q_full[2], q_empty[2], kv_full[AttSmem<HD, FEW>::kStages], kv_empty[AttSmem<HD, FEW>::kStages];
  uint64_t s_full[2][2], p_ready[2][2], pv_done[2][2],                // [stream][parity of its step]
      item_full[kItemRing], item_empty[kItemRing];
  uint64_t look[2], join[2], turn[2], drain[2];
  Item items[kItemRing];
  int bad_key[kItemRing];           // first key of the item's first page whose id is outside the pool
  int bad_value[2][2];              // [stream][parity of its step]: step + 1 whose P V the threads add themselves
  uint32_t tmem;
  int abort_flag;
  int kv_loads, q_loads[2];         // copies issued: of key and value tiles, into each query tile
  long long x0, x1, start;          // plan: the CTA's share of the cost; cost in front of its first sequence
  int first_seq;
  long long warp_sum[2][kAttThreads / 32];
  float2 ml[2][128];
};

// Four threads of a row hold a word each of four 16-byte units (v[i]: unit i); afterwards thread j of them holds unit j.
__device__ __forceinline__ void units_of_quad(uint32_t (&v)[4], int lane) {
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? v[i] : v[i + 1], 1);
    if (odd) v[i] = got;
    else v[i + 1] = got;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t got = __shfl_xor_sync(0xffffffffu, high ? v[i] : v[i + 2], 2);
    if (high) v[i] = got;
    else v[i + 2] = got;
  }
}
template <bool HALF> __device__ __forceinline__ bool any_undefined(uint4 v) {
  const uint32_t m = HALF ? 0x7c007c00u : 0x7f807f80u;
  return (__vcmpeq2(v.x & m, m) | __vcmpeq2(v.y & m, m) | __vcmpeq2(v.z & m, m) | __vcmpeq2(v.w & m, m)) != 0;
}
// byte of 16-byte unit c of key `key` in a K or V stage: [8-row group][64-element half][row][128 bytes], swizzled
template <int HD> __device__ __forceinline__ uint32_t kv_unit(int key, int c) {
  return (key >> 3) * (HD * 16) + (c >> 3) * 1024 + (key & 7) * 128 + (((c & 7) ^ (key & 7)) << 4);
}

// The CTA's share of the total cost, [x0, x1), and the sequence that it begins in.  Every thread takes a sequence (and one
// of the next kAttThreads ...): prefix sums over the warp, then over the warps.
template <int HD, bool FEW> __device__ __forceinline__ void make_plan(const AttendArgs &a, Shared<HD, FEW> &sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kWarps = kAttThreads / 32;
  auto cost_of = [&](int s, bool report) -> long long {
    if (s >= a.c.S) return 0;
    const SeqSpan p = seq_span(a.c, s);
    if (report && !p.ok) atomicMax(a.c.status, STATUS_BAD_CHUNK);
    return seq_cost(p, a.tile_tok).head() * a.Hkv;
  };
  // costs up to and with this thread's, of this warp
  auto scan = [&](long long run) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    return run;
  };
  const long long first = cost_of(threadIdx.x, blockIdx.x == 0), first_run = scan(first);
  long long rest = 0;
  if (a.c.S > kAttThreads) {
    for (int s = threadIdx.x + kAttThreads; s < a.c.S; s += kAttThreads) rest += cost_of(s, blockIdx.x == 0);
    rest = scan(rest);
  }
  if (lane == 31) {
    sh.warp_sum[0][warp] = first_run;
    sh.warp_sum[1][warp] = rest;
  }
  if (threadIdx.x == 0) sh.first_seq = -1;
  __syncthreads();
  long long before = 0, firsts = 0, rests = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += sh.warp_sum[0][w];
    firsts += sh.warp_sum[0][w];
    rests += sh.warp_sum[1][w];
  }
  const long long total = firsts + rests;
  const unsigned ctas = static_cast<unsigned>(max(1ll, min(static_cast<long long>(gridDim.x), total / kLeastShare)));
  const long long each = total / ctas, more = total - each * ctas;      // (the first `more` CTAs take one more)
  const long long c = min(blockIdx.x, ctas);
  const long long x0 = each * c + min(c, more), x1 = blockIdx.x < ctas ? x0 + each + (c < more) : x0;
  if (threadIdx.x == 0) {
    sh.x0 = x0;
    sh.x1 = x1;
  }
  if (x0 == x1) return;                          // nothing to do (first_seq stays -1)
  before += first_run - first;
  if (first > 0 && x0 >= before && x0 < before + first) {
    sh.first_seq = threadIdx.x;
    sh.start = before;
  }
  if (x0 < firsts) return;
  before = firsts;                               // among the later ones
  for (int s0 = kAttThreads; s0 < a.c.S; s0 += kAttThreads) {
    const long long cost = cost_of(s0 + threadIdx.x, false), run = scan(cost);
    __syncthreads();
    if (lane == 31) sh.warp_sum[0][warp] = run;
    __syncthreads();
    long long mine = before + run - cost;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) mine += sh.warp_sum[0][w];
      before += sh.warp_sum[0][w];
    }
    if (cost > 0 && x0 >= mine && x0 < mine + cost) {
      sh.first_seq = s0 + threadIdx.x;
      sh.start = mine;
    }
    if (x0 < before) break;
  }
}

template <int HD, bool HALF, bool FEW>
__global__ void __launch_bounds__(kAttThreads, 1)
chunk_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kv,
                       const __grid_constant__ AttendArgs a) {
  using M = AttSmem<HD, FEW>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Shared<HD, FEW> &sh = *reinterpret_cast<Shared<HD, FEW> *>(smem + M::kBars);
  static_assert(sizeof(Shared<HD, FEW>) <= M::kBarBytes, "barriers");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kMma0 = kSoftWarps, kLoad = kSoftWarps + 1, kMma1 = kSoftWarps + 2;
  volatile int *abort_flag = &sh.abort_flag;
  if (smem_u32(smem) & 1023) {                 // (swizzled tiles need it; a dynamic array alone begins there)
    if (threadIdx.x == 0) {
      atomicMax(a.c.status, STATUS_WAIT_TIMEOUT);
      a.records[blockIdx.x] = PartRecord{};
    }
    return;
  }

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 1);
      mbar_init(&sh.q_empty[i], 2);
      mbar_init(&sh.drain[i], 1);
      mbar_init(&sh.turn[i], 1);
      for (int b = 0; b < 2; ++b) {
        mbar_init(&sh.s_full[i][b], 1);
        mbar_init(&sh.pv_done[i][b], 1);
        mbar_init(&sh.p_ready[i][b], M::kRowWarps);
        sh.bad_value[i][b] = 0;
      }
      mbar_init(&sh.look[i], M::kRowWarps);
      mbar_init(&sh.join[i], 2 * M::kRowWarps);
    }
    for (int i = 0; i < M::kStages; ++i) {
      mbar_init(&sh.kv_full[i], 1);
      mbar_init(&sh.kv_empty[i], 2);
    }
    for (int i = 0; i < kItemRing; ++i) {
      mbar_init(&sh.item_full[i], 1);
      mbar_init(&sh.item_empty[i], 2 * M::kRowWarps + 2);
    }
    sh.abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == kMma0) tc_alloc(&sh.tmem, 512);
  if (warp == kLoad && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_q)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_kv)) : "memory");
  }
  early_start_sync();
  make_plan<HD, FEW>(a, sh);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;               // S of the streams at columns 0 and 128, O at 256 and 384

  // waits of a whole warp, whose lanes go on or give up together
  auto wait = [&](uint64_t *bar, int parity) { return warp_wait(bar, parity & 1, abort_flag, a.limit); };

  if (warp == kLoad) {
    // ---------------------------------------------------------------- items and copies
    PartRecord rec = {};
    int n_items = 0;                            // published
    int q_uses0 = 0, q_uses1 = 0, next_slot = 0;
    int kv_at = 0, ring = 0, ring_use = 0;      // stages loaded; the next one, and how often it was used
    bool ok = true;
    const uint32_t q_s = smem_u32(smem + M::kQ), kv_s = smem_u32(smem + M::kKV);
    const int q_bytes = 2 * HD * a.group * a.load_tok;
    auto publish = [&](const Item &it) {
      const int slot = n_items % kItemRing;
      if (n_items >= kItemRing) ok = wait(&sh.item_empty[slot], (n_items / kItemRing) - 1);
      if (!ok) return;
      if (lane == 0) {
        sh.items[slot] = it;
        sh.bad_key[slot] = INT_MAX;
        mbar_arrive(&sh.item_full[slot]);
      }
      __syncwarp();
      ++n_items;
    };
    auto load_q = [&](const Item &it, int slot, int tile) {
      const int uses = slot ? q_uses1 : q_uses0;
      if (ok && uses > 0) ok = wait(&sh.q_empty[slot], uses - 1);
      if (!ok) return;
      if (elect_one()) {
        mbar_expect_tx(&sh.q_full[slot], q_bytes);
#pragma unroll
        for (int h = 0; h < HD / 64; ++h)
          tma_load_3d(&tm_q, &sh.q_full[slot], q_s + slot * M::kQTile + h * M::kQHalf, 64 * h, it.head * a.group,
                      it.row0 + tile * a.tile_tok);
      }
      __syncwarp();
      if (slot) ++q_uses1;
      else ++q_uses0;
    };
    if (sh.first_seq >= 0) {
      long long left = sh.x1 - sh.x0, y = sh.x0 - sh.start;        // cost left to do; place within the sequence
      int window = sh.first_seq & ~31;
      SeqSpan span = {};
      int seq = sh.first_seq;
      bool load_window = true;
      while (left > 0 && seq < a.c.S && ok) {
        if (load_window || seq >= window + 32) {
          window = seq & ~31;
          span.ok = false;
          if (window + lane < a.c.S) span = seq_span(a.c, window + lane);
          load_window = false;
        }
        SeqSpan p;
        p.row0 = __shfl_sync(0xffffffffu, span.row0, seq - window);
        p.n = __shfl_sync(0xffffffffu, span.n, seq - window);
        p.kv = __shfl_sync(0xffffffffu, span.kv, seq - window);
        p.ok = __shfl_sync(0xffffffffu, span.ok ? 1 : 0, seq - window) != 0;
        const SeqCost k = seq_cost(p, a.tile_tok);
        if (k.n_items == 0) {
          ++seq;
          y = 0;
          continue;
        }
        const long long head_cost = k.head();
        int head = static_cast<int>(y / head_cost);
        y -= head * head_cost;
        // last item that starts at or before y
        int lo = 0, hi = k.n_items;
        while (hi - lo > 1) {
          const int step = (hi - lo + 31) / 32, at = lo + lane * step;
          const unsigned m = __ballot_sync(0xffffffffu, at < hi && k.before(at) <= y);
          lo += (31 - __clz(m)) * step;
          hi = min(hi, lo + step);
        }
        y -= k.before(lo);
        const int32_t *pages = a.c.page_table + static_cast<int64_t>(seq) * a.c.pt_width;
        for (int i = lo; head < a.Hkv && left > 0 && ok;) {
          const bool single = k.single(i);
          const long long cost = k.cost(i), take = min(left, cost - y);
          const int seen = k.seen(i), tiles = (seen + kKeys - 1) / kKeys;
          Item it;
          it.t0 = cut_tile(y, single, seen);
          it.t1 = cut_tile(y + take, single, seen);
          it.row0 = p.row0 + i * k.step;
          it.n_tok = min(k.step, p.n - i * k.step);
          it.head = head;
          it.pos0 = k.base + i * k.step;
          it.seen_end = seen;
          it.flags = (single ? 0 : kPaired) | (i & 1 ? kBackwards : 0);
          if (it.t0 > 0) it.flags |= kPartLater;
          else if (it.t1 < tiles) it.flags |= kPartFirst;
          const bool none = tiles == 0 && y == 0;                    // rows that see nothing: zeros
          if (it.t0 < it.t1 || none) {
            if (it.flags & kPartLater) {
              rec.later = 1;
              rec.later_ends = it.t1 == tiles;
            }
            if (it.flags & kPartFirst) {
              rec.first = 1;
              rec.item = it;
            }
            const int slot = n_items % kItemRing;
            publish(it);
            if (!ok) break;
            if (it.t0 < it.t1) {
              if (single) {
                load_q(it, next_slot, 0);
                next_slot ^= 1;
              } else {
                load_q(it, 0, 0);
                load_q(it, 1, 1);
              }
              const bool back = it.flags & kBackwards;
              int ids = 0, ids_next = 0, block = -1;
              const int n_need = (seen + kChunkPage - 1) / kChunkPage;
              auto fetch = [&](int b) { return b >= 0 && 32 * b + lane < n_need ? pages[32 * b + lane] : -1; };
              for (int n = it.t0; n < it.t1 && ok; ++n) {
                const int t = back ? it.t0 + it.t1 - 1 - n : n;
                if (block != t / 4) {
                  ids = block < 0 ? fetch(t / 4) : ids_next;
                  block = t / 4;
                  ids_next = fetch(back ? block - 1 : block + 1);
                }
                const int id = __shfl_sync(0xffffffffu, ids, (t & 3) * 8 + (lane & 7));
                const bool need = t * kPages + (lane & 7) < n_need, valid = need && id >= 0 && id < a.n_pages;
                const unsigned bad = __ballot_sync(0xffffffffu, need && !valid) & 0xffu;
                if (bad) {
                  if (lane == 0) {
                    sh.bad_key[slot] = min(sh.bad_key[slot], (t * kPages + __ffs(bad) - 1) * kChunkPage);
                    atomicMax(a.c.status, STATUS_BAD_PAGE);
                  }
                  __syncwarp();                  // before the copy that the others wait for is issued
                }
                // a page that nothing sees, or that does not exist, reads as zeros
                const int unit = valid ? (id * a.Hkv + it.head) * 4 : a.n_pages * a.Hkv * 4;
                // one lane issues, from coordinates that all lanes hold: copies from eight lanes' own coordinates take
                // three times as long to issue, and then bound the whole (1900 cycles a tile)
                int units[kPages];
#pragma unroll
                for (int j = 0; j < kPages; ++j) units[j] = __shfl_sync(0xffffffffu, unit, j);
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                  if (ring_use > 0) ok = wait(&sh.kv_empty[ring], ring_use - 1);
                  if (!ok) break;
                  if (elect_one()) {
                    mbar_expect_tx(&sh.kv_full[ring], M::kStage);
#pragma unroll
                    for (int j = 0; j < kPages; ++j)
                      tma_load_4d(&tm_kv, &sh.kv_full[ring], kv_s + ring * M::kStage + j * (M::kStage / kPages), 0, 0, 0, units[j] + 2 * kv);
                  }
                  __syncwarp();
                  ++kv_at;
                  if (++ring == M::kStages) {
                    ring = 0;
                    ++ring_use;
                  }
                }
              }
            }
          }
          left -= take;
          y = 0;
          if (++i == k.n_items) {
            i = 0;
            ++head;
          }
        }
        ++seq;
        y = 0;
      }
    }
    if (ok) {
      Item end = {};
      end.flags = kEnd;
      publish(end);
    }
    if (lane == 0) {
      a.records[blockIdx.x] = rec;
      sh.kv_loads = kv_at;
      sh.q_loads[0] = q_uses0;
      sh.q_loads[1] = q_uses1;
    }
  } else if (warp >= kSoftWarps) {
    // ---------------------------------------------------------------- MMA issue
    // A warp for each stream, so that one's waits and bookkeeping run under the other's products (one warp for both left
    // the tensor cores idle for half of the time).  They issue in turn: two streams whose products mix on the tensor cores
    // finish them at the same time, form their probabilities at the same time, and each pipe idles while the other works.
    // The whole warp takes every step and one elected lane issues: operands that are the same for all lanes are in uniform
    // registers when an MMA needs them there; with one lane walking alone an MMA took 100 to 150 cycles to issue, twice as
    // long as it runs.
    if (warp == kMma0 || warp == kMma1) {
      const int w = warp == kMma0 ? 0 : 1;
      constexpr uint32_t idesc_s = idesc_operands(idesc_rows(instr_desc_bf16(64), M::kQRows), HALF);
      constexpr uint32_t idesc_o = idesc_operands(idesc_rows(instr_desc_bf16(HD), M::kQRows), HALF) | kIdescBMajorMN;
      constexpr int kStages = M::kStages;
      const uint32_t q_s = smem_u32(smem + M::kQ), kv_s = smem_u32(smem + M::kKV);
      const uint32_t t_s = tmem + w * 128, t_o = tmem + 256 + w * 128;
      bool ok = true;
      int next_slot = 0, k_stage = 0, k_phase = 0, v_stage = 1, v_phase = 0, step = 0, batch = 0;
      uint32_t q_uses = 0;                                            // parity of each query tile's use
      // the other stage of the same kind (K, V, K, V, ...)
      auto next = [&](int &stage, int &phase) {
        stage += 2;
        if (stage >= kStages) {
          stage -= kStages;
          phase ^= 1;
        }
      };
      for (int n = 0; ok; ++n) {
        const int slot = n % kItemRing;
        ok = wait(&sh.item_full[slot], n / kItemRing);
        if (!ok) break;
        const int flags = __shfl_sync(0xffffffffu, sh.items[slot].flags, 0);
        if (flags & kEnd) break;
        const int t0 = __shfl_sync(0xffffffffu, sh.items[slot].t0, 0), t1 = __shfl_sync(0xffffffffu, sh.items[slot].t1, 0);
        const int pos0 = __shfl_sync(0xffffffffu, sh.items[slot].pos0, 0);
        const bool paired = !FEW && (flags & kPaired) != 0;
        const int qs = paired ? w : next_slot, steps = paired ? 2 * (t1 - t0) : t1 - t0;
        // of the stream's steps, those that may be added by the threads: with keys behind the first row's position
        const int pos_first = pos0 + (paired ? w * a.tile_tok : 0);
        auto masked = [&](int i) {
          const int tile = paired ? i >> 1 : i, key0 = (flags & kBackwards ? t1 - 1 - tile : t0 + tile) * kKeys + 64 * (paired ? i & 1 : w);
          return key0 + 64 > pos_first + 1;
        };
        const uint64_t dq = smem_desc(q_s + qs * M::kQTile, 16, 1024);
        if (steps > 0) {                                              // (both tiles' uses are seen by both warps)
          if (paired) ok = wait(&sh.q_full[0], q_uses & 1) && wait(&sh.q_full[1], q_uses >> 1);
          else ok = wait(&sh.q_full[qs], q_uses >> qs);
        }
        // batch i: the products P V of step i - ahead, then S = Q K^T of step i.  (Single items wait for memory: a K tile that
        // is needed early would have to be loaded in place of a later one.)
        const int ahead = paired ? 2 : 1;
        for (int i = 0; ok && steps > 0 && i < steps + ahead; ++i) {
          const int half = paired ? i & 1 : w;                        // (of pairs, steps i and i - 2 are the same half)
          const bool open = !paired || half == 0, close = !paired || half == 1;      // first and last use of a tile
          if (i < steps && open) ok = wait(&sh.kv_full[k_stage], k_phase);
          bool by_mma = true;
          if (ok && i >= ahead) {
            if (open) ok = wait(&sh.kv_full[v_stage], v_phase);
            if (ok) ok = wait(&sh.p_ready[w][step & 1], step >> 1);
            if (ok && masked(i - ahead))
              by_mma = __shfl_sync(0xffffffffu, *const_cast<volatile int *>(&sh.bad_value[w][step & 1]), 0) != step + 1;
          }
          if (ok) ok = wait(&sh.turn[w], batch - (w == 0 ? 1 : 0));
          if (!ok) break;
          ++batch;
          tc_fence_after();
          const int q_buf = (i < ahead ? step + i : step + ahead) & 1;
          const uint32_t t_p = t_s + (step & 1) * 64, t_q = t_s + q_buf * 64;
          if (elect_one()) {
            if (i >= ahead) {
              if (by_mma) {
                const uint64_t dv = smem_desc(kv_s + v_stage * M::kStage + half * (64 * HD * 2), 1024, HD * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) tc_mma_ts(t_o, t_p + k * 8, dv + k * (HD * 32 >> 4), idesc_o, k > 0 || i != ahead);
              }
              tc_commit(&sh.pv_done[w][step & 1]);
              if (close) tc_commit(&sh.kv_empty[v_stage]);
            }
            if (i < steps) {
              const uint64_t db = smem_desc(kv_s + k_stage * M::kStage + half * (64 * HD * 2), 16, HD * 16);
#pragma unroll
              for (int k = 0; k < HD / 16; ++k)
                tc_mma_bf16(t_q, dq + (k >> 2) * (M::kQHalf >> 4) + (k & 3) * 2, db + (k >> 2) * (1024 >> 4) + (k & 3) * 2, idesc_s, k > 0);
              tc_commit(&sh.s_full[w][q_buf]);
              if (close) tc_commit(&sh.kv_empty[k_stage]);
              if (i + 1 == steps) {                                   // (both of a pair's tiles wait for both warps, as both see them)
                tc_commit(&sh.q_empty[qs]);
                if (paired) tc_commit(&sh.q_empty[qs ^ 1]);
              }
            }
            mbar_arrive(&sh.turn[w ^ 1]);
          }
          __syncwarp();
          if (i >= ahead) {
            ++step;
            if (close) next(v_stage, v_phase);
          }
          if (i < steps && close) next(k_stage, k_phase);
        }
        if (!ok) break;
        if (steps > 0) {
          q_uses ^= paired ? 3u : 1u << qs;
          if (!paired) next_slot ^= 1;
        }
        if (lane == 0) mbar_arrive(&sh.item_empty[slot]);
      }
    }
  } else {
    // ---------------------------------------------------------------- softmax and results
    // 16 rows: of 128, the first or the second 16 lanes of the warp's quarter of tensor memory; of 64, its first 16 (the
    // other warp of the quarter takes no part)
    const int w = warp >> 3, high = (warp >> 2) & 1, quarter = warp & 3;
    const int lane0 = quarter * 32 + high * 16, row0 = FEW ? quarter * 16 : lane0;
    const int stream_tid = (FEW ? quarter : warp & 7) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(lane0) << 16;
    const uint32_t t_s0 = tmem + lanes + w * 128, t_o = tmem + lanes + 256 + w * 128;
    const float c = a.scale_log2;
    constexpr float kShift = shift_of(HALF), kMost = most_sum(HALF);
    const int row_a = row0 + (lane >> 2), row_b = row_a + 8, col = 2 * (lane & 3);      // of every eight columns: col, col + 1
    const int tok_a = row_a / a.group, tok_b = row_b / a.group;
    int n_item = 0, steps_done = 0, tiles_done = 0, looks = 0, joins = 0;
    bool ok = true;
    // Barriers by the parity of the step, since two steps' products may be under way: a barrier that had both would be a
    // phase before or behind the one that is waited for, and a phase is known by its parity alone.
    auto products_done = [&](int step) { return wait(&sh.pv_done[w][step & 1], step >> 1); };
    while (ok && !(FEW && high)) {
      const int slot = n_item % kItemRing;
      ok = wait(&sh.item_full[slot], n_item / kItemRing);
      if (!ok) break;
      const Item it = sh.items[slot];
      if (it.flags & kEnd) break;
      const bool paired = !FEW && (it.flags & kPaired);
      const int row_tile = paired ? w : 0, steps = (it.t1 - it.t0) * (paired ? 2 : 1);
      const int tok0 = row_tile * a.tile_tok, n_rows = min(a.tile_tok, it.n_tok - tok0) * a.group;
      const int pos_first = it.pos0 + tok0, pos_a = pos_first + tok_a, pos_b = pos_first + tok_b;
      const bool mine_a = row_a < n_rows, mine_b = row_b < n_rows, warp_mine = row0 < n_rows;
      float m_a = -INFINITY, m_b = -INFINITY;                         // references (score units)
      float l_a = 0.f, l_b = 0.f;                                     // sums of this thread's columns
      bool far = false;                                               // a row of the warp has had a far reference
      for (int i = 0; i < steps; ++i) {          // of 64 keys
        const int tile = paired ? i >> 1 : i, key_off = 64 * (paired ? i & 1 : w);
        const int key0 = (it.flags & kBackwards ? it.t1 - 1 - tile : it.t0 + tile) * kKeys + key_off;
        const int buf = steps_done & 1;
        const uint32_t t_s = t_s0 + 64 * buf;
        ok = wait(&sh.s_full[w][buf], steps_done >> 1);
        if (!ok) break;
        tc_fence_after();
        const bool masked = key0 + 64 > pos_first + 1;                // some row does not see all of these keys
        if (warp_mine) {
          uint32_t s[32], p[16];
          float2 sum_a, sum_b;
          tc_ld_64cols(t_s, s);
          if (masked) {
            const int last_a = pos_a - key0 - col, last_b = pos_b - key0 - col;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
              if (8 * b > last_a) s[4 * b] = 0xff800000u;
              if (8 * b + 1 > last_a) s[4 * b + 1] = 0xff800000u;
              if (8 * b > last_b) s[4 * b + 2] = 0xff800000u;
              if (8 * b + 1 > last_b) s[4 * b + 3] = 0xff800000u;
            }
          }
          // With the references as they are, unless a row has none yet or a far one: maxima take a quarter of a step's
          // time, and a reference that is too low shows in the sum.  Where one does, once more with maxima.
          bool careful = __any_sync(0xffffffffu, (mine_a && m_a == -INFINITY) || (mine_b && m_b == -INFINITY)) || far;
          while (true) {
            if (careful) {
              float to_a = m_a, to_b = m_b;
#pragma unroll
              for (int b = 0; b < 8; ++b) {
                to_a = max3_nan(to_a, __uint_as_float(s[4 * b]), __uint_as_float(s[4 * b + 1]));
                to_b = max3_nan(to_b, __uint_as_float(s[4 * b + 2]), __uint_as_float(s[4 * b + 3]));
              }
#pragma unroll
              for (int o = 1; o < 4; o <<= 1) {
                to_a = max_nan(to_a, __shfl_xor_sync(0xffffffffu, to_a, o));
                to_b = max_nan(to_b, __shfl_xor_sync(0xffffffffu, to_b, o));
              }
              const float fix_a = to_a == m_a ? 1.0f : ex2((m_a - to_a) * c);      // (from -inf: 0)
              const float fix_b = to_b == m_b ? 1.0f : ex2((m_b - to_b) * c);
              m_a = to_a;
              m_b = to_b;
              l_a *= fix_a;
              l_b *= fix_b;
              if (i > 0) {
                ok = products_done(steps_done - 1);
                if (!ok) break;
                tc_fence_after();
#pragma unroll 1
                for (int b = 0; b < HD / 32; ++b) {
                  uint32_t o[16];
                  tc_ld_32cols(t_o + b * 32, o);
#pragma unroll
                  for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * ((e & 2) ? fix_b : fix_a));
                  tc_st_32cols(t_o + b * 32, o);
                }
              }
              const bool far_a = mine_a && fabsf(m_a) > kFar && fabsf(m_a) < INFINITY;      // (other rows hold anything)
              const bool far_b = mine_b && fabsf(m_b) > kFar && fabsf(m_b) < INFINITY;
              if (__any_sync(0xffffffffu, far_a || far_b)) {
                // (in place of the block below, which this leaves as fast as it is; every further step comes here too)
                far = true;
                const float off_a = far_a ? m_a : 0.f, off_b = far_b ? m_b : 0.f;
                const float base_a = far_a ? kShift : m_a == -INFINITY ? 0.f : m_a == INFINITY ? NAN : kShift - m_a * c;
                const float base_b = far_b ? kShift : m_b == -INFINITY ? 0.f : m_b == INFINITY ? NAN : kShift - m_b * c;
                sum_a = sum_b = make_float2(0.f, 0.f);
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                  const float ax = ex2(fmaf(__uint_as_float(s[4 * b]) - off_a, c, base_a));
                  const float ay = ex2(fmaf(__uint_as_float(s[4 * b + 1]) - off_a, c, base_a));
                  const float bx = ex2(fmaf(__uint_as_float(s[4 * b + 2]) - off_b, c, base_b));
                  const float by = ex2(fmaf(__uint_as_float(s[4 * b + 3]) - off_b, c, base_b));
                  sum_a.x += ax + ay;
                  sum_b.x += bx + by;
                  p[2 * b] = cvt16x2(ax, ay, HALF);
                  p[2 * b + 1] = cvt16x2(bx, by, HALF);
                }
                break;
              }
            }
            const float base_a = m_a == -INFINITY ? 0.f : m_a == INFINITY ? NAN : kShift - m_a * c;
            const float base_b = m_b == -INFINITY ? 0.f : m_b == INFINITY ? NAN : kShift - m_b * c;
            const float2 c2 = make_float2(c, c), base2_a = make_float2(base_a, base_a), base2_b = make_float2(base_b, base_b);
            sum_a = sum_b = make_float2(0.f, 0.f);
#pragma unroll
            for (int b = 0; b < 8; ++b) {
              const float2 x = fma2(make_float2(__uint_as_float(s[4 * b]), __uint_as_float(s[4 * b + 1])), c2, base2_a);
              const float2 y = fma2(make_float2(__uint_as_float(s[4 * b + 2]), __uint_as_float(s[4 * b + 3])), c2, base2_b);
              const float2 px = make_float2(ex2(x.x), ex2(x.y)), py = make_float2(ex2(y.x), ex2(y.y));
              sum_a = add2(sum_a, px);
              sum_b = add2(sum_b, py);
              p[2 * b] = cvt16x2(px.x, px.y, HALF);
              p[2 * b + 1] = cvt16x2(py.x, py.y, HALF);
            }
            sum_a.x += sum_a.y;
            sum_b.x += sum_b.y;
            if (careful || !__any_sync(0xffffffffu, (mine_a && !(sum_a.x <= kMost)) || (mine_b && !(sum_b.x <= kMost)))) break;
            careful = true;
          }
          if (!ok) break;
          l_a += sum_a.x;
          l_b += sum_b.x;
          tc_st_64keys(t_s, p);
          tc_wait_st();
        }
        // keys that some row of the tile does not see: their values must be finite, or kept out of the products
        if (masked && it.seen_end > key0) {
          const int ks = max(0, pos_first + 1 - key0), ke = min(64, it.seen_end - key0);
          const int ke16 = (ke + 15) & ~15;
          const int at = 2 * (tiles_done + tile) + 1, stage = at % M::kStages;
          ok = wait(&sh.kv_full[stage], at / M::kStages);
          if (!ok) break;
          uint8_t *v = smem + M::kKV + stage * M::kStage;
          const int u0 = min(ks, ke) * (HD / 8), u1 = ke16 * (HD / 8);
          bool bad = false;
          for (int u = u0 + stream_tid; u < u1; u += 32 * M::kRowWarps) {
            uint4 *unit = reinterpret_cast<uint4 *>(v + kv_unit<HD>(key_off + u / (HD / 8), u % (HD / 8)));
            if (u / (HD / 8) < ke) bad |= any_undefined<HALF>(*unit);
            else *unit = make_uint4(0u, 0u, 0u, 0u);                  // no row of the item sees it
          }
          fence_proxy_async();
          bool slow = false;
          if (ks < ke) {
            if (bad) *const_cast<volatile int *>(&sh.bad_value[w][buf]) = steps_done + 1;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.look[w]);
            ok = wait(&sh.look[w], looks);
            if (!ok) break;
            ++looks;
            slow = *const_cast<volatile int *>(&sh.bad_value[w][buf]) == steps_done + 1;
          }
          if (slow && warp_mine) {
            if (i > 0) ok = products_done(steps_done - 1);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int b = 0; b < HD / 32; ++b) {
              uint32_t o[16];
              tc_ld_32cols(t_o + b * 32, o);
              if (i == 0)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0u;
#pragma unroll 1
              for (int key = 0; key < 64; ++key) {
                uint32_t p[2];
                if ((key & 7) == 0) __syncwarp();
                tc_ld_8keys(t_s + (key >> 3) * 4, p);
                const int from = (lane & ~3) | ((key & 7) >> 1);
                const float2 qa = widen16x2(__shfl_sync(0xffffffffu, p[0], from), HALF);
                const float2 qb = widen16x2(__shfl_sync(0xffffffffu, p[1], from), HALF);
                const float pa = (key & 1) ? qa.y : qa.x, pb = (key & 1) ? qb.y : qb.x;
                const bool see_a = key <= pos_a - key0, see_b = key <= pos_b - key0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t vv = *reinterpret_cast<const uint32_t *>(v + kv_unit<HD>(key_off + key, b * 4 + e) + 2 * col);
                  const float2 f = widen16x2(vv, HALF);
                  if (see_a) {
                    o[4 * e] = __float_as_uint(fmaf(pa, f.x, __uint_as_float(o[4 * e])));
                    o[4 * e + 1] = __float_as_uint(fmaf(pa, f.y, __uint_as_float(o[4 * e + 1])));
                  }
                  if (see_b) {
                    o[4 * e + 2] = __float_as_uint(fmaf(pb, f.x, __uint_as_float(o[4 * e + 2])));
                    o[4 * e + 3] = __float_as_uint(fmaf(pb, f.y, __uint_as_float(o[4 * e + 3])));
                  }
                }
                __syncwarp();
              }
              tc_st_32cols(t_o + b * 32, o);
            }
            tc_wait_st();
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_ready[w][buf]);
        ++steps_done;
      }
      if (!ok) break;
      // ---- the item's result: whole rows, or a part for the joining launch
      const bool any = it.t0 < it.t1;
      if (any) {
        ok = products_done(steps_done - 1);
        if (!ok) break;
      }
      tc_fence_after();
      const int bad_key = *const_cast<volatile int *>(&sh.bad_key[slot]);
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        l_a += __shfl_xor_sync(0xffffffffu, l_a, o);
        l_b += __shfl_xor_sync(0xffffffffu, l_b, o);
      }
      float ref_a = m_a * c, ref_b = m_b * c, a0 = 1.f, a1 = 0.f, b0 = 1.f, b1 = 0.f;      // scales of the streams' O
      int col0 = 0, col1 = HD;
      uint32_t o_main = t_o, o_other = t_o;
      if (!paired) {
        // both streams hold a share of the keys: each joins half of the columns
        if ((lane & 3) == 0) {
          sh.ml[w][row_a] = make_float2(ref_a, l_a);
          sh.ml[w][row_b] = make_float2(ref_b, l_b);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.join[0]);
        ok = wait(&sh.join[0], joins);
        if (!ok) break;
        tc_fence_after();
        auto join = [&](int row, float &ref, float &sum, float &x0, float &x1) {
          const float2 m0 = sh.ml[0][row], m1 = sh.ml[1][row];
          ref = max_nan(m0.x, m1.x);
          x0 = m0.x == -INFINITY ? 0.f : ex2(m0.x - ref);
          x1 = m1.x == -INFINITY ? 0.f : ex2(m1.x - ref);
          sum = m0.y * x0 + m1.y * x1;
        };
        join(row_a, ref_a, l_a, a0, a1);
        join(row_b, ref_b, l_b, b0, b1);
        o_main = tmem + lanes + 256;
        o_other = o_main + 128;
        col0 = w * (HD / 2);
        col1 = col0 + HD / 2;
      }
      if (warp_mine) {
        const bool part = it.flags & (kPartFirst | kPartLater);
        const int64_t part_at = (static_cast<int64_t>(blockIdx.x) * 2 + (it.flags & kPartFirst ? 1 : 0)) * a.rows_cap + row_tile * 128;
        if (pos_a >= bad_key) {                  // the row needs the page: whatever else it holds, it is undefined
          l_a = NAN;
          ref_a = 0.f;
        }
        if (pos_b >= bad_key) {
          l_b = NAN;
          ref_b = 0.f;
        }
        if (part && col0 == 0 && (lane & 3) == 0) {
          if (mine_a) a.part_ml[part_at + row_a] = make_float2(ref_a, l_a);
          if (mine_b) a.part_ml[part_at + row_b] = make_float2(ref_b, l_b);
        }
        const float norm_a = 1.0f / l_a, norm_b = 1.0f / l_b;
        const int64_t tok_first = it.row0 + tok0;
        uint16_t *dst_a = a.out + ((tok_first + tok_a) * a.Hq + it.head * a.group + row_a % a.group) * HD + 8 * (lane & 3);
        uint16_t *dst_b = a.out + ((tok_first + tok_b) * a.Hq + it.head * a.group + row_b % a.group) * HD + 8 * (lane & 3);
#pragma unroll 1
        for (int c0 = col0; c0 < col1; c0 += 32) {
          float f[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) f[e] = 0.f;
          if (any) {
            uint32_t o[16];
            tc_ld_32cols(o_main + c0, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) f[e] = __uint_as_float(o[e]) * ((e & 2) ? b0 : a0);
            if (!paired) {
              tc_ld_32cols(o_other + c0, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) f[e] = fmaf(__uint_as_float(o[e]), (e & 2) ? b1 : a1, f[e]);
            }
          }
          if (part) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (mine_a) *reinterpret_cast<float2 *>(a.part_o + (part_at + row_a) * HD + c0 + 8 * e + col) = make_float2(f[4 * e], f[4 * e + 1]);
              if (mine_b) *reinterpret_cast<float2 *>(a.part_o + (part_at + row_b) * HD + c0 + 8 * e + col) = make_float2(f[4 * e + 2], f[4 * e + 3]);
            }
          } else {                               // (rows that see nothing: 0)
            uint32_t va[4], vb[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              va[e] = pos_a < 0 ? 0u : cvt16x2(f[4 * e] * norm_a, f[4 * e + 1] * norm_a, HALF);
              vb[e] = pos_b < 0 ? 0u : cvt16x2(f[4 * e + 2] * norm_b, f[4 * e + 3] * norm_b, HALF);
            }
            units_of_quad(va, lane);
            units_of_quad(vb, lane);
            if (mine_a) *reinterpret_cast<uint4 *>(dst_a + c0) = make_uint4(va[0], va[1], va[2], va[3]);
            if (mine_b) *reinterpret_cast<uint4 *>(dst_b + c0) = make_uint4(vb[0], vb[1], vb[2], vb[3]);
          }
          __syncwarp();
        }
      }
      if (!paired) {
        // the other stream's warps have read this one's O before it is written again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.join[1]);
        ok = wait(&sh.join[1], joins);
        if (!ok) break;
        ++joins;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.item_empty[slot]);
      ++n_item;
      tiles_done += it.t1 - it.t0;
    }
  }
  __syncthreads();
  if (sh.abort_flag) {
    // A wait ran out.  Whichever it was, copies and products may be under way that nobody waited for, since the warps that did
    // not wait in vain have gone on or ended: they land before shared and tensor memory go.
    if (threadIdx.x == 0) atomicMax(a.c.status, STATUS_WAIT_TIMEOUT);
    if (warp == kLoad && lane == 0) {
      for (int i = 0; i < 2; ++i)
        if (sh.q_loads[i] > 0) mbar_drain(&sh.q_full[i], (sh.q_loads[i] - 1) & 1);
      for (int i = max(0, sh.kv_loads - M::kStages); i < sh.kv_loads; ++i)
        mbar_drain(&sh.kv_full[i % M::kStages], (i / M::kStages) & 1);
    }
    if ((warp == kMma0 || warp == kMma1) && elect_one()) {
      uint64_t *bar = &sh.drain[warp == kMma0 ? 0 : 1];
      tc_commit(bar);
      mbar_drain(bar, 0);
    }
    __syncthreads();
  }
  if (warp == kMma0) {
    tc_fence_after();
    tc_dealloc(tmem, 512);
  }
}

// Joins the parts of the items that were cut, in key order: CTA (b, g) the item whose first part CTA b left, rows 16 g ..
// Half a warp to a row; its lanes look up 16 CTAs' records and partial sums at once.
template <int HD, bool HALF>
__global__ void __launch_bounds__(256) join_parts_kernel(const __grid_constant__ AttendArgs a, int n_ctas) {
  early_start_sync();
  const int b = blockIdx.x, lane = threadIdx.x & 15, upper = threadIdx.x & 16;
  // lane i: the part of CTA b + i
  PartRecord mine = {};
  if (b + lane < n_ctas) mine = a.records[b + lane];
  if (!__shfl_sync(0xffffffffu, mine.first, 0)) return;
  const Item it = a.records[b].item;
  const int row = blockIdx.y * 16 + (threadIdx.x >> 4);
  const int tile = row >> 7, r = row & 127, tok = tile * a.tile_tok + r / a.group;
  const bool there = row < a.rows_cap && r < a.tile_tok * a.group && tok < it.n_tok;
  const int64_t stride = 2 * static_cast<int64_t>(a.rows_cap);
  constexpr int kCols = HD / 16;                 // of a lane
  float ref = -INFINITY, l = 0.f, o[kCols];
#pragma unroll
  for (int e = 0; e < kCols; ++e) o[e] = 0.f;
  for (int k0 = b; k0 < n_ctas; k0 += 16) {
    if (k0 > b) mine = k0 + lane < n_ctas ? a.records[k0 + lane] : PartRecord{};
    const unsigned ends = __ballot_sync(0xffffffffu, (k0 > b || lane > 0) && mine.later && mine.later_ends) & 0xffffu;
    const int n = ends ? __ffs(ends) : 16;       // lanes that belong to the item
    const bool part = lane < n && (k0 + lane == b || mine.later);
    const int64_t at = (k0 + lane) * stride + (k0 + lane == b ? a.rows_cap : 0) + row;
    const float2 ml = part && there ? a.part_ml[at] : make_float2(-INFINITY, 0.f);
    float to = fmaxf(ref, ml.x);
#pragma unroll
    for (int d = 8; d; d >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, d));
    const float fix = to == ref ? 1.f : ref == -INFINITY ? 0.f : ex2(ref - to);      // (from -inf: nothing yet)
    l *= fix;
#pragma unroll
    for (int e = 0; e < kCols; ++e) o[e] *= fix;
    ref = to;
    const float scale = ml.x == -INFINITY ? 0.f : ex2(ml.x - ref);
    float sum = ml.y * scale;
#pragma unroll
    for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    l += sum;
    for (unsigned left = __ballot_sync(0xffffffffu, part) & 0xffffu; left; left &= left - 1) {
      const int k = upper + __ffs(left) - 1;
      const float *p = a.part_o + __shfl_sync(0xffffffffu, at, k) * HD + lane * kCols;
      const float s = __shfl_sync(0xffffffffu, scale, k);
      if (!there) continue;
#pragma unroll
      for (int e = 0; e < kCols; e += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(p + e);
        o[e] = fmaf(x.x, s, o[e]);
        o[e + 1] = fmaf(x.y, s, o[e + 1]);
        o[e + 2] = fmaf(x.z, s, o[e + 2]);
        o[e + 3] = fmaf(x.w, s, o[e + 3]);
      }
    }
    if (ends) break;
  }
  if (!there) return;
  const float norm = 1.0f / l;
  uint16_t *dst = a.out + (static_cast<int64_t>(it.row0 + tok) * a.Hq + it.head * a.group + r % a.group) * HD + lane * kCols;
#pragma unroll
  for (int e = 0; e < kCols; e += 4)
    *reinterpret_cast<uint2 *>(dst + e) =
        it.pos0 + tok < 0 ? make_uint2(0u, 0u) : make_uint2(cvt16x2(o[e] * norm, o[e + 1] * norm, HALF), cvt16x2(o[e + 2] * norm, o[e + 3] * norm, HALF));
}

// ---- host ------------------------------------------------------------------------------------------------
EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}
bool make_map(CUtensorMap *out, int rank, const void *base, bool half, const cuuint64_t *dims, const cuuint64_t *strides,
              const cuuint32_t *box) {
  const EncodeTiledFn fn = encode_fn();
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  return fn && fn(out, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(base),
                  dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

std::atomic<uint64_t> g_wait_limit_ns{kWaitLimitNs};

// rows of an item's partial result
int rows_cap(int max_chunk, int group) {
  const int tile_tok = 128 / group;
  return max_chunk > tile_tok ? 256 : (max_chunk * group + 7) / 8 * 8;
}

// SMs of the current device (0: unknown), looked up once.
int sm_count(int dev) {
  static std::atomic<int> known[kDevices];
  int n = dev < kDevices ? known[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && dev < kDevices)
    known[dev].store(n, std::memory_order_relaxed);
  return n;
}

template <int HD, bool HALF, bool FEW>
cudaError_t launch_attend(const CUtensorMap &tm_q, const CUtensorMap &tm_kv, const AttendArgs &a, int dev, int ctas, cudaStream_t s) {
  constexpr int smem = AttSmem<HD, FEW>::kTotal;
  static std::atomic<bool> allowed[kDevices];      // the kernel's shared memory, on a device
  if (dev >= kDevices || !allowed[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(chunk_attention_kernel<HD, HALF, FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (dev < kDevices) allowed[dev].store(true, std::memory_order_release);
  }
  const cudaError_t e = launch_early(chunk_attention_kernel<HD, HALF, FEW>, dim3(ctas), dim3(kAttThreads), smem, s, tm_q, tm_kv, a);
  if (e != cudaSuccess) return e;
  return launch_early(join_parts_kernel<HD, HALF>, dim3(ctas, (a.rows_cap + 15) / 16), dim3(256), 0, s, a, ctas);
}

}  // namespace
}  // namespace echo

using namespace echo;

extern "C" {

size_t echo_chunk_attention_workspace_bytes(int32_t max_chunk, int32_t Hq, int32_t Hkv, int32_t hd) {
  if (max_chunk < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || Hq / Hkv > 128 || (hd != 64 && hd != 128)) return 0;
  const size_t rows = static_cast<size_t>(kMaxCtas) * 2 * rows_cap(max_chunk, Hq / Hkv);
  return kMaxCtas * kRecordBytes + rows * (hd * sizeof(float) + sizeof(float2));
}

int echo_chunk_attention(const void *q, int64_t q_stride, const void *kv_pool, int32_t n_pages, int32_t format,
                         const echo_kv_chunks *chunks, int32_t Hq, int32_t Hkv, int32_t hd, void *workspace,
                         size_t workspace_bytes, void *out, void *cuda_stream) {
  AttendArgs a{};
  const int rc = chunk_args(chunks, Hq, Hkv, hd, kv_pool, n_pages, format, &a.c);
  if (rc != ECHO_OK) return rc;
  const int64_t width = static_cast<int64_t>(Hq) * hd;
  const bool none = a.c.S == 0 || a.c.n_rows == 0;
  if ((!none && (!q || !out)) || Hq < 1 || q_stride < width || q_stride % 8 || q_stride > (1 << 30)) return ECHO_ERR_INVALID;
  for (const void *p : {q, const_cast<const void *>(out), const_cast<const void *>(workspace)})
    if (reinterpret_cast<uintptr_t>(p) & 15) return ECHO_ERR_INVALID;
  if (Hq / Hkv > 128 || static_cast<int64_t>(n_pages) * Hkv > (1 << 26)) return ECHO_ERR_UNSUPPORTED;
  const size_t need = echo_chunk_attention_workspace_bytes(a.c.max_chunk, Hq, Hkv, hd);
  if (none) return ECHO_OK;
  if (!workspace || workspace_bytes < need) return ECHO_ERR_INVALID;
  const uint64_t qs = (static_cast<uint64_t>(a.c.n_rows - 1) * q_stride + width) * 2, outs = a.c.n_rows * static_cast<uint64_t>(width) * 2;
  if (ranges_meet(out, outs, q, qs) || ranges_meet(out, outs, kv_pool, pool_bytes(n_pages, Hkv, hd)) ||
      ranges_meet(out, outs, workspace, need) || ranges_meet(workspace, need, q, qs) ||
      ranges_meet(workspace, need, kv_pool, pool_bytes(n_pages, Hkv, hd)))
    return ECHO_ERR_INVALID;
  if (meets_tables(a.c, out, outs) || meets_tables(a.c, workspace, need) || status_in_tables(a.c) ||
      ranges_meet(a.c.status, 4, q, qs) || ranges_meet(a.c.status, 4, kv_pool, pool_bytes(n_pages, Hkv, hd)))
    return ECHO_ERR_INVALID;
  a.limit.ns = g_wait_limit_ns.load(std::memory_order_relaxed);
  a.limit.look = a.limit.ns < kWaitLimitNs ? 0 : 255;
  a.out = static_cast<uint16_t *>(out);
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.group = Hq / Hkv;
  a.tile_tok = 128 / a.group;
  const bool few = static_cast<int64_t>(a.c.max_chunk) * a.group <= kFewRows;
  a.load_tok = few ? kFewRows / a.group : a.tile_tok;
  a.n_pages = n_pages;
  a.rows_cap = rows_cap(a.c.max_chunk, a.group);
  a.scale_log2 = 1.4426950408889634f / std::sqrt(static_cast<float>(hd));
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  a.records = reinterpret_cast<PartRecord *>(ws);
  ws += kMaxCtas * kRecordBytes;
  a.part_o = reinterpret_cast<float *>(ws);
  a.part_ml = reinterpret_cast<float2 *>(ws + static_cast<size_t>(kMaxCtas) * 2 * a.rows_cap * hd * sizeof(float));
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ECHO_ERR_CUDA;
  const int ctas = std::min(sm_count(dev), kMaxCtas);
  if (ctas < 1) return ECHO_ERR_CUDA;
  const bool half = format == 1;
  CUtensorMap tm_q, tm_kv;
  // queries: 64 elements of a head x the heads of a group x the tokens of a tile
  const cuuint64_t qd[3] = {static_cast<cuuint64_t>(hd), static_cast<cuuint64_t>(Hq), static_cast<cuuint64_t>(a.c.n_rows)};
  const cuuint64_t qst[2] = {static_cast<cuuint64_t>(hd) * 2, static_cast<cuuint64_t>(q_stride) * 2};
  const cuuint32_t qb[3] = {64, static_cast<cuuint32_t>(a.group), static_cast<cuuint32_t>(a.load_tok)};
  // the pool in groups of eight rows, each read as 64-element halves: 64 elements x 8 rows x halves x the two groups of a
  // page's K (or V) lie in shared memory as [group][half][row], so that operands have one stride from group to group
  const cuuint64_t kd[4] = {64, 8, static_cast<cuuint64_t>(hd / 64), static_cast<cuuint64_t>(n_pages) * Hkv * 4};
  const cuuint64_t kst[3] = {static_cast<cuuint64_t>(hd) * 2, 128, static_cast<cuuint64_t>(hd) * 16};
  const cuuint32_t kb[4] = {64, 8, static_cast<cuuint32_t>(hd / 64), 2};
  if (!make_map(&tm_q, 3, q, half, qd, qst, qb) || !make_map(&tm_kv, 4, kv_pool, half, kd, kst, kb)) return ECHO_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const auto launch = hd == 128 ? (half ? (few ? launch_attend<128, true, true> : launch_attend<128, true, false>)
                                        : (few ? launch_attend<128, false, true> : launch_attend<128, false, false>))
                                : (half ? (few ? launch_attend<64, true, true> : launch_attend<64, true, false>)
                                        : (few ? launch_attend<64, false, true> : launch_attend<64, false, false>));
  const cudaError_t e = launch(tm_q, tm_kv, a, dev, ctas, s);
  return e == cudaSuccess ? ECHO_OK : ECHO_ERR_CUDA;
}

int echo_debug_chunk_wait_limit(uint64_t limit_ns) {
  if (limit_ns > kWaitLimitNs) return ECHO_ERR_INVALID;
  g_wait_limit_ns.store(limit_ns ? limit_ns : kWaitLimitNs, std::memory_order_relaxed);
  return ECHO_OK;
}

}  // extern "C"
