// Attention of a ragged batch of new tokens over a caller's paged caches.
//
// One warp per (row, query head): lanes share the head's elements, keys go by one at a time with a running maximum and
// sum.  Right for every shape; nothing in it is fast.

#include <cmath>

#include "chunks.cuh"

namespace echo {
namespace {

struct AttendArgs {
  const uint16_t *q;
  int64_t q_stride;
  const uint16_t *pool;
  uint16_t *out;
  int Hq, Hkv, hd, n_pages, half_io;
  float scale;
  ChunkArgs c;
};

__global__ void __launch_bounds__(128) attend_rows_kernel(const __grid_constant__ AttendArgs a) {
  early_start_sync();
  const int lane = threadIdx.x & 31, head = blockIdx.y * 4 + (threadIdx.x >> 5), row = blockIdx.x;
  const bool h16 = a.half_io != 0;
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int s = threadIdx.x; s < a.c.S; s += blockDim.x)
      if (!seq_span(a.c, s).ok) atomicMax(a.c.status, STATUS_BAD_CHUNK);
  if (head >= a.Hq) return;
  int seq = -1;
  SeqSpan p;
  for (int s0 = 0; s0 < a.c.S && seq < 0; s0 += 32) {
    const int s = s0 + lane;
    bool mine = false;
    if (s < a.c.S) {
      p = seq_span(a.c, s);
      mine = p.ok && row >= p.row0 && row < p.row0 + p.n;
    }
    const unsigned any = __ballot_sync(0xffffffffu, mine);
    if (any) seq = s0 + __ffs(any) - 1;
  }
  if (seq < 0) return;
  p = seq_span(a.c, seq);
  const int pos = p.kv - p.n + (row - p.row0), per = a.hd / 32, kvh = head / (a.Hq / a.Hkv);
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  bool bad = false;
  for (int e = 0; e < per; ++e) q[e] = widen16(a.q[row * a.q_stride + head * a.hd + lane + 32 * e], h16);
  for (int u = 0; u <= pos; ++u) {
    const int page = a.c.page_table[static_cast<int64_t>(seq) * a.c.pt_width + u / kChunkPage];
    if (page < 0 || page >= a.n_pages) {
      bad = true;
      break;
    }
    const uint16_t *k = a.pool + ((static_cast<int64_t>(page) * a.Hkv + kvh) * 2 * kChunkPage + u % kChunkPage) * a.hd + lane;
    const uint16_t *v = k + kChunkPage * a.hd;
    float s = 0.f;
    for (int e = 0; e < per; ++e) s += q[e] * widen16(k[32 * e], h16);
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s *= a.scale;
    const float top = fmaxf(m, s), fix = m == -INFINITY ? 0.f : expf(m - top), w = top == -INFINITY ? 0.f : expf(s - top);
    l = l * fix + w;
    for (int e = 0; e < per; ++e) o[e] = o[e] * fix + w * widen16(v[32 * e], h16);
    m = top;
  }
  if (bad && lane == 0) atomicMax(a.c.status, STATUS_BAD_PAGE);
  for (int e = 0; e < per; ++e)
    a.out[(static_cast<int64_t>(row) * a.Hq + head) * a.hd + lane + 32 * e] =
        cvt16(bad ? NAN : pos < 0 ? 0.f : o[e] / l, h16);
}

}  // namespace
}  // namespace echo

using namespace echo;

extern "C" {

size_t echo_chunk_attention_workspace_bytes(int32_t max_chunk, int32_t Hq, int32_t Hkv, int32_t hd) {
  if (max_chunk < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || (hd != 64 && hd != 128)) return 0;
  return 16;
}

int echo_chunk_attention(const void *q, int64_t q_stride, const void *kv_pool, int32_t n_pages, int32_t format,
                         const echo_kv_chunks *chunks, int32_t Hq, int32_t Hkv, int32_t hd, void *workspace,
                         size_t workspace_bytes, void *out, void *cuda_stream) {
  AttendArgs a{};
  const int rc = chunk_args(chunks, Hq, Hkv, hd, kv_pool, n_pages, format, &a.c);
  if (rc != ECHO_OK) return rc;
  const int64_t width = static_cast<int64_t>(Hq) * hd;
  if (!q || !out || Hq < 1 || q_stride < width || q_stride % 8 || q_stride > (1 << 30)) return ECHO_ERR_INVALID;
  for (const void *p : {q, const_cast<const void *>(out), const_cast<const void *>(workspace)})
    if (reinterpret_cast<uintptr_t>(p) & 15) return ECHO_ERR_INVALID;
  const size_t need = echo_chunk_attention_workspace_bytes(a.c.max_chunk, Hq, Hkv, hd);
  if (!workspace || workspace_bytes < need) return ECHO_ERR_INVALID;
  if (Hq / Hkv > 128 || static_cast<int64_t>(n_pages) * Hkv > (1 << 26)) return ECHO_ERR_UNSUPPORTED;
  if (a.c.S == 0 || a.c.n_rows == 0) return ECHO_OK;
  const uint64_t qs = (static_cast<uint64_t>(a.c.n_rows - 1) * q_stride + width) * 2, outs = a.c.n_rows * static_cast<uint64_t>(width) * 2;
  if (ranges_meet(out, outs, q, qs) || ranges_meet(out, outs, kv_pool, pool_bytes(n_pages, Hkv, hd)) ||
      ranges_meet(out, outs, workspace, need) || ranges_meet(workspace, need, q, qs) ||
      ranges_meet(workspace, need, kv_pool, pool_bytes(n_pages, Hkv, hd)))
    return ECHO_ERR_INVALID;
  a.q = static_cast<const uint16_t *>(q);
  a.q_stride = q_stride;
  a.pool = static_cast<const uint16_t *>(kv_pool);
  a.out = static_cast<uint16_t *>(out);
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.hd = hd;
  a.n_pages = n_pages;
  a.half_io = format == 1;
  a.scale = 1.0f / std::sqrt(static_cast<float>(hd));
  const cudaError_t e = launch_early(attend_rows_kernel, dim3(a.c.n_rows, (Hq + 3) / 4), dim3(128), 0,
                                     static_cast<cudaStream_t>(cuda_stream), a);
  return e == cudaSuccess ? ECHO_OK : ECHO_ERR_CUDA;
}

}  // extern "C"
