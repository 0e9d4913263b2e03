// Attention of new tokens over a paged KV cache.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

constexpr int kMaxSeqs = 112;  // sequences whose sizes fit in a launch's parameters (4 KB)

struct PagedSeq {
  int q0, n, len, prefix, seq;
};
struct PagedArgs {
  const __nv_bfloat16 *q, *pool;
  const int32_t* table;
  int max_pages, n_pages, page_size, n_heads, n_kv_heads, n_seqs;
  float scale;
  __nv_bfloat16* o;
  float* lse;
  int* status;
  PagedSeq s[kMaxSeqs];
};

// A warp a row and head, a lane HD / 32 of its dims.
template <int HD>
__global__ void __launch_bounds__(256) paged_simple_kernel(const __grid_constant__ PagedArgs p) {
  constexpr int D = HD / 32;
  pdl_launch_dependents();
  pdl_wait();
  const PagedSeq& s = p.s[blockIdx.z];
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, h = blockIdx.y;
  if (row >= s.n) return;
  const int g = h / (p.n_heads / p.n_kv_heads), kvd = p.n_kv_heads * HD;
  const int limit = max(s.len - s.n + row + 1, s.prefix);
  const size_t at = (size_t(s.q0) + row) * p.n_heads + h;
  float q[D], o[D] = {}, m = -INFINITY, l = 0.0f;
  for (int x = 0; x < D; ++x) q[x] = __bfloat162float(p.q[at * HD + lane * D + x]);
  for (int j = 0; j < limit; ++j) {
    const int page = p.table[size_t(s.seq) * p.max_pages + j / p.page_size];
    if (unsigned(page) >= unsigned(p.n_pages)) {
      if (lane == 0) set_status(p.status, SPD_EINVAL);
      continue;
    }
    const __nv_bfloat16* kr = p.pool + (size_t(page) * p.page_size + j % p.page_size) * (2 * size_t(kvd)) + g * HD + lane * D;
    float d = 0.0f;
    for (int x = 0; x < D; ++x) d = fmaf(q[x], __bfloat162float(kr[x]), d);
    for (int off = 16; off; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
    d *= p.scale;
    const float mn = fmaxf(m, d), f = mn == -INFINITY ? 1.0f : expf(m - mn), w = mn == -INFINITY && !isnan(d) ? 0.0f : expf(d - mn);
    m = mn;
    l = l * f + w;
    for (int x = 0; x < D; ++x) o[x] = o[x] * f + (w == 0.0f ? 0.0f : w * __bfloat162float(kr[kvd + x]));
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  for (int x = 0; x < D; ++x) p.o[at * HD + lane * D + x] = __float2bfloat16(o[x] * inv);
  if (p.lse && lane == 0) p.lse[at] = m + logf(l);
}

}  // namespace

size_t paged_attention_bytes(int, int, int, int) { return 256; }

int paged_attention_run(const void* q, const int32_t* q_cu, const int32_t* len, const int32_t* prefix, int n_seqs,
                        const int32_t* table, int max_pages, const void* pool, int n_pages, int page_size, int n_heads,
                        int n_kv_heads, int head_dim, void* o, float* lse, void*, size_t, int* status, cudaStream_t st) {
  PagedArgs p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.pool = static_cast<const __nv_bfloat16*>(pool);
  p.table = table;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  p.page_size = page_size;
  p.n_heads = n_heads;
  p.n_kv_heads = n_kv_heads;
  p.scale = float(1.0 / sqrt(double(head_dim)));
  p.o = static_cast<__nv_bfloat16*>(o);
  p.lse = lse;
  p.status = status;
  for (int s0 = 0; s0 < n_seqs; s0 += kMaxSeqs) {
    int most = 0;
    p.n_seqs = 0;
    for (int b = s0; b < std::min(n_seqs, s0 + kMaxSeqs); ++b) {
      const int n = q_cu[b + 1] - q_cu[b];
      if (n == 0) continue;
      p.s[p.n_seqs++] = {q_cu[b], n, len[b], prefix ? prefix[b] : 0, b};
      most = std::max(most, n);
    }
    if (p.n_seqs == 0) continue;
    SPD_CUDA_TRY(launch_pdl(head_dim == 128 ? paged_simple_kernel<128> : paged_simple_kernel<64>,
                            dim3((most + 7) / 8, n_heads, p.n_seqs), dim3(256), 0, st, p));
  }
  return SPD_OK;
}

}  // namespace spd

using namespace spd;

extern "C" size_t spd_paged_attention_workspace_size(int n_q, int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  if (n_q < 1 || n_seqs < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads || (head_dim != 64 && head_dim != 128))
    return 0;
  return paged_attention_bytes(n_q, n_heads, n_kv_heads, head_dim);
}

extern "C" int spd_paged_attention(const uint16_t* q, int n_q, const int32_t* q_cu, const int32_t* len, const int32_t* prefix,
                                   int n_seqs, const int32_t* table, int max_pages, const uint16_t* pool, int n_pages,
                                   int page_size, int n_heads, int n_kv_heads, int head_dim, uint16_t* o, float* lse, void* ws,
                                   size_t ws_bytes, void* stream) {
  if (!q || !q_cu || !len || !table || !o || !ws || n_q < 1 || n_seqs < 1 || n_heads < 1 || n_kv_heads < 1 ||
      n_heads % n_kv_heads)
    return fail(SPD_EINVAL, "bad paged attention arguments");
  if (int rc = pool_check(pool, 1, n_pages, page_size, n_kv_heads, head_dim, max_pages)) return rc;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(ws)) & 15)
    return fail(SPD_EINVAL, "q, o and ws must be 16-byte aligned");
  if (int rc = paged_check(q_cu, n_q, len, prefix, n_seqs, max_pages, page_size)) return rc;
  const size_t need = paged_attention_bytes(n_q, n_heads, n_kv_heads, head_dim);
  if (ws_bytes < need) return fail(SPD_ENOSPC, "paged attention workspace too small (%zu < %zu)", ws_bytes, need);
  return paged_attention_run(q, q_cu, len, prefix, n_seqs, table, max_pages, pool, n_pages, page_size, n_heads, n_kv_heads,
                             head_dim, o, lse, ws, ws_bytes, static_cast<int*>(ws), static_cast<cudaStream_t>(stream));
}
