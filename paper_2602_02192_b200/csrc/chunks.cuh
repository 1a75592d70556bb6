// A ragged batch of new tokens over a caller's paged caches (echo_kv_chunks), as the kernels see it.
#pragma once

#include "common.cuh"

namespace echo {

constexpr int kChunkPage = 16;                 // tokens of a page
constexpr int STATUS_BAD_CHUNK = 4;            // lengths outside the batch's limits (with common.cuh's codes)

struct ChunkArgs {
  const int32_t *row_starts, *kv_lens, *page_table;
  int *status;
  int S, n_rows, pt_width, max_chunk;
};

// Host checks that both calls share.  heads: Hq may be 0 (no queries in the call).
inline int chunk_args(const echo_kv_chunks *c, int32_t Hq, int32_t Hkv, int32_t hd, const void *pool, int32_t n_pages,
                      int32_t format, ChunkArgs *out) {
  if (!c || c->n_seqs < 0 || c->n_rows < 0 || c->pt_width < 0 || c->max_chunk < 0) return ECHO_ERR_INVALID;
  const bool none = c->n_seqs == 0 || c->n_rows == 0;      // nothing to do, and arrays of nothing may have no address
  if (!none && (c->pt_width < 1 || c->max_chunk < 1 || !c->row_starts || !c->kv_lens || !c->page_table || !c->status))
    return ECHO_ERR_INVALID;
  for (const void *p : {static_cast<const void *>(c->row_starts), static_cast<const void *>(c->kv_lens),
                        static_cast<const void *>(c->page_table), static_cast<const void *>(c->status)})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ECHO_ERR_INVALID;
  if (Hkv < 1 || Hq < 0 || Hq % Hkv || hd < 1 || format < 0 || format > 1) return ECHO_ERR_INVALID;
  if (!pool || n_pages < 1 || (reinterpret_cast<uintptr_t>(pool) & 15)) return ECHO_ERR_INVALID;
  if (hd != 64 && hd != 128) return ECHO_ERR_UNSUPPORTED;
  if (c->pt_width > (1 << 26) || Hkv > 4096 || Hq > 65536) return ECHO_ERR_UNSUPPORTED;      // positions fit 30 bits
  *out = {c->row_starts, c->kv_lens, c->page_table, c->status, c->n_seqs, c->n_rows, c->pt_width, c->max_chunk};
  return ECHO_OK;
}
inline uint64_t pool_bytes(int32_t n_pages, int32_t Hkv, int32_t hd) {
  return static_cast<uint64_t>(n_pages) * Hkv * 2 * kChunkPage * hd * 2;
}
inline bool ranges_meet(const void *a, uint64_t na, const void *b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && x < y + nb && y < x + na;
}
// An array that a call writes, and the batch's tables and status.
inline bool meets_tables(const ChunkArgs &c, const void *p, uint64_t bytes) {
  const uint64_t seqs = static_cast<uint64_t>(c.S);
  return ranges_meet(p, bytes, c.row_starts, (seqs + 1) * 4) || ranges_meet(p, bytes, c.kv_lens, seqs * 4) ||
         ranges_meet(p, bytes, c.page_table, seqs * c.pt_width * 4) || ranges_meet(p, bytes, c.status, 4);
}
// The status, which every call writes, and the tables.
inline bool status_in_tables(const ChunkArgs &c) {
  ChunkArgs tables = c;
  tables.status = nullptr;
  return meets_tables(tables, c.status, 4);
}

#ifdef __CUDACC__
struct SeqSpan {
  int row0, n, kv;         // first row, new tokens, keys once they are appended
  bool ok;
};
// Lengths are the caller's device memory: nothing is read or written by them before they passed these checks.
__device__ __forceinline__ SeqSpan seq_span(const ChunkArgs &c, int s) {
  SeqSpan p;
  const int r0 = c.row_starts[s], r1 = c.row_starts[s + 1];
  p.kv = c.kv_lens[s];
  p.row0 = r0;
  p.n = r1 - r0;
  p.ok = r0 >= 0 && r1 >= r0 && r1 <= c.n_rows && r1 - r0 <= c.max_chunk && p.kv >= 0 && p.kv <= c.pt_width * kChunkPage;
  return p;
}
#endif

}  // namespace echo
