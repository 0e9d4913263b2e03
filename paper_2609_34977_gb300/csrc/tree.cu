// Attention of drafted tokens over a KV cache (the verification of a speculative step; with one node a sequence, a
// decode step whose rotary positions need not be its slots).
//
// Sequence b holds ctx_b committed rows in its cache slot and behind them the rows of its n_b drafts. Node i sees the
// committed rows and the drafts j whose bit is set in its mask (its ancestors and itself for a tree):
//   s_ij = q_i . k_j / sqrt(head_dim),  lse_i = log sum_j e^s_ij,  o_i = sum_j e^(s_ij - lse_i) v_j,
// o = 0 and lse = -inf for a row that sees nothing. Keys a row does not see contribute nothing, whatever they hold.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <vector>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

constexpr int kMaxSeqs = 240;  // sequences whose sizes fit in a launch's parameters
struct TreeSeqs {              // by value in the launch's parameters: no copy, no wait for one
  int cu[kMaxSeqs + 1];
  int ctx[kMaxSeqs];
};
struct TreeArgs {
  const __nv_bfloat16* q;
  const uint32_t* mask;
  int words;
  const __nv_bfloat16* kv;
  int seq0, max_len, n_heads, n_kv_heads;
  float scale;
  __nv_bfloat16* o;
  float* lse;
};

// One CTA a node and head: every warp takes every eighth key, a key's dot product runs over the lanes.
template <int HD>
__global__ void __launch_bounds__(256) tree_kernel(const __grid_constant__ TreeArgs p, const __grid_constant__ TreeSeqs sq) {
  constexpr int D = HD / 32;
  __shared__ float wm[8], wl[8], wo[8][HD];
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.x, g = h / (p.n_heads / p.n_kv_heads), ls = blockIdx.z;
  const int i = blockIdx.y, n = sq.cu[ls + 1] - sq.cu[ls], ctx = sq.ctx[ls];
  if (i >= n) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const size_t row = sq.cu[ls] + i;
  float qf[D], o[D];
#pragma unroll
  for (int e = 0; e < D; ++e) {
    qf[e] = __bfloat162float(p.q[(row * p.n_heads + h) * HD + D * lane + e]);
    o[e] = 0.0f;
  }
  const int kvd = p.n_kv_heads * HD;
  const __nv_bfloat16* base = p.kv + size_t(p.seq0 + ls) * p.max_len * (2 * kvd) + g * HD + D * lane;
  float m = -INFINITY, l = 0.0f;
  for (int k = warp; k < ctx + n; k += 8) {
    const int d = k - ctx;
    if (d >= 0 && (p.mask ? !((p.mask[row * p.words + d / 32] >> (d % 32)) & 1u) : d > i)) continue;
    const __nv_bfloat16* kr = base + size_t(k) * (2 * kvd);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < D; ++e) s = fmaf(qf[e], __bfloat162float(kr[e]), s);
#pragma unroll
    for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    s *= p.scale;
    const float mn = fmaxf(m, s), c = m == -INFINITY ? 0.0f : expf(m - mn), w = expf(s - mn);
    l = l * c + w;
#pragma unroll
    for (int e = 0; e < D; ++e) o[e] = o[e] * c + w * __bfloat162float(kr[kvd + e]);
    m = mn;
  }
  if (lane == 0) {
    wm[warp] = m;
    wl[warp] = l;
  }
#pragma unroll
  for (int e = 0; e < D; ++e) wo[warp][D * lane + e] = o[e];
  __syncthreads();
  float mt = -INFINITY, lt = 0.0f;
  for (int w = 0; w < 8; ++w) mt = fmaxf(mt, wm[w]);
  for (int w = 0; w < 8; ++w) lt += wm[w] == -INFINITY ? 0.0f : wl[w] * expf(wm[w] - mt);
  for (int d = threadIdx.x; d < HD; d += 256) {
    float s = 0.0f;
    for (int w = 0; w < 8; ++w)
      if (wm[w] != -INFINITY) s += wo[w][d] * expf(wm[w] - mt);
    p.o[(row * p.n_heads + h) * HD + d] = __float2bfloat16_rn(mt == -INFINITY ? 0.0f : s / lt);
  }
  if (p.lse && threadIdx.x == 0) p.lse[row * p.n_heads + h] = mt == -INFINITY ? -INFINITY : mt + logf(lt);
}

}  // namespace

size_t tree_attention_bytes(int, int, int, int, int) { return 256; }

int tree_attention_run(const void* q, const int32_t* q_cu, const int32_t* ctx, int n_seqs, const uint32_t* mask, int words,
                       const void* kv, int max_len, int n_heads, int n_kv_heads, int head_dim, void* o, float* lse, void* ws,
                       size_t, cudaStream_t st) {
  (void)ws;
  TreeArgs p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.mask = mask;
  p.words = words;
  p.kv = static_cast<const __nv_bfloat16*>(kv);
  p.max_len = max_len;
  p.n_heads = n_heads;
  p.n_kv_heads = n_kv_heads;
  p.scale = 1.0f / sqrtf(float(head_dim));
  p.o = static_cast<__nv_bfloat16*>(o);
  p.lse = lse;
  for (int s0 = 0; s0 < n_seqs; s0 += kMaxSeqs) {
    TreeSeqs sq;
    const int m = std::min(kMaxSeqs, n_seqs - s0);
    p.seq0 = s0;
    int most = 0;
    double pairs = 0.0, keys = 0.0;
    for (int b = 0; b < m; ++b) {
      const int n = q_cu[s0 + b + 1] - q_cu[s0 + b];
      sq.ctx[b] = ctx[s0 + b];
      most = std::max(most, n);
      keys += ctx[s0 + b] + n;
      pairs += double(n) * (ctx[s0 + b] + n);
    }
    for (int b = 0; b <= m; ++b) sq.cu[b] = q_cu[s0 + b];
    if (most == 0) continue;
    const int slot = trace_begin(st);
    SPD_CUDA_TRY(launch_pdl(head_dim == 128 ? tree_kernel<128> : tree_kernel<64>, dim3(n_heads, most, m), dim3(256), 0, st, p,
                            sq));
    trace_end(slot, st, TR_ATTN, 4.0 * head_dim * n_heads * pairs,
              4.0 * n_kv_heads * head_dim * keys + 4.0 * n_heads * head_dim * (sq.cu[m] - sq.cu[0]));
  }
  return SPD_OK;
}

}  // namespace spd

using namespace spd;

extern "C" int spd_tree_mask(int n_seqs, const int32_t* q_cu, const int32_t* parent, int words, uint32_t* mask,
                             int32_t* depth) {
  if (n_seqs < 1 || !q_cu || !parent || !mask || words < 1 || q_cu[0] != 0) return fail(SPD_EINVAL, "bad tree arguments");
  for (int b = 0; b < n_seqs; ++b) {
    const int n = q_cu[b + 1] - q_cu[b];
    if (n < 0) return fail(SPD_EINVAL, "q_cu decreases at sequence %d", b);
    if (n > 32 * words) return fail(SPD_EINVAL, "sequence %d: %d nodes do not fit in %d mask words", b, n, words);
    for (int i = 0; i < n; ++i) {
      const int up = parent[q_cu[b] + i];
      if (up < -1 || up >= i) return fail(SPD_EINVAL, "sequence %d: the parent of node %d must come before it", b, i);
    }
  }
  for (int b = 0; b < n_seqs; ++b) {
    for (int i = 0; i < q_cu[b + 1] - q_cu[b]; ++i) {
      const int up = parent[q_cu[b] + i];
      uint32_t* row = mask + size_t(q_cu[b] + i) * words;
      for (int w = 0; w < words; ++w) row[w] = up < 0 ? 0u : mask[size_t(q_cu[b] + up) * words + w];
      row[i / 32] |= 1u << (i % 32);
      if (depth) depth[q_cu[b] + i] = up < 0 ? 0 : depth[q_cu[b] + up] + 1;
    }
  }
  return SPD_OK;
}

extern "C" size_t spd_tree_attention_workspace_size(int n_q, int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  if (n_q < 1 || n_seqs < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads || (head_dim != 64 && head_dim != 128))
    return 0;
  return tree_attention_bytes(n_q, n_seqs, n_heads, n_kv_heads, head_dim);
}

extern "C" int spd_tree_attention(const uint16_t* q, int n_q, const int32_t* q_cu, const int32_t* ctx_len, int n_seqs,
                                  const uint32_t* tree_mask, int mask_words, const uint16_t* kv, int max_len, int n_heads,
                                  int n_kv_heads, int head_dim, uint16_t* o, float* lse, void* ws, size_t ws_bytes,
                                  void* stream) {
  if (!q || !q_cu || !ctx_len || !kv || !o || !ws || n_q < 1 || n_seqs < 1 || max_len < 1 || n_heads < 1 || n_kv_heads < 1 ||
      n_heads % n_kv_heads)
    return fail(SPD_EINVAL, "bad tree attention arguments");
  if (head_dim != 64 && head_dim != 128) return fail(SPD_EUNSUPPORTED, "tree attention supports head_dim 64 and 128");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(kv) | reinterpret_cast<uintptr_t>(o)) & 15)
    return fail(SPD_EINVAL, "q, kv and o must be 16-byte aligned");
  if (q_cu[0] != 0 || q_cu[n_seqs] != n_q) return fail(SPD_EINVAL, "q_cu must run from 0 to n_q");
  for (int b = 0; b < n_seqs; ++b) {
    const int n = q_cu[b + 1] - q_cu[b];
    if (n < 0) return fail(SPD_EINVAL, "q_cu decreases at sequence %d", b);
    if (ctx_len[b] < 0 || ctx_len[b] > max_len - n)
      return fail(SPD_EINVAL, "sequence %d: context and drafts exceed max_len", b);
    if (tree_mask && n > 32 * mask_words) return fail(SPD_EINVAL, "sequence %d: %d nodes, %d mask words", b, n, mask_words);
  }
  const size_t need = tree_attention_bytes(n_q, n_seqs, n_heads, n_kv_heads, head_dim);
  if (ws_bytes < need) return fail(SPD_ENOSPC, "tree attention workspace too small (%zu < %zu)", ws_bytes, need);
  return tree_attention_run(q, q_cu, ctx_len, n_seqs, tree_mask, mask_words, kv, max_len, n_heads, n_kv_heads, head_dim, o, lse,
                            ws, ws_bytes, static_cast<cudaStream_t>(stream));
}
