// Rules on a step's logits: penalties for repeated tokens, biases and grammar masks, and the best token left, in
// one pass over the rows.
//
// For row r of sequence b, token t with n_t occurrences among the generated tokens (those of the row's own path
// included):
//   x_t = z_t                                   where t is in neither prompt nor answer, else z_t / rep_b (z_t > 0), z_t rep_b
//   x_t = x_t - freq_b n_t - pres_b             where n_t > 0
//   x_t = x_t + the sequence's biases of t;     x_t = -inf where the row's grammar does not allow t
//   best = the first t of the largest x_t       (-1 when nothing is left)
// every step one fp32 operation in this order.
//
// A row moves 8 V bytes; the occurrence counts live in shared memory (a word a token of the CTA's slice), so they cost no
// traffic and leave no state between calls. Up to 16 CTAs share a row; every one walks the whole history (4 bytes a token from
// L2) and counts what falls into its slice, while its logits are on their way into registers. They meet only at the end,
// for the best token: as a cluster where all rows are on the GPU at once, else by offers to `best`.
//
// What bounds it: latency. A CTA is a chain of dependent loads (sequence, its lists, their entries: 5 us under load) before
// the 2.5 us of its stream, and four CTAs an SM overlap only in part. 192 rows of 152064 words, 2000 tokens of history and 300
// biases a sequence: 57.1 us (234 MB, 4.1 TB/s; a copy of the same bytes 36); 64 rows with up to 4000 tokens
// 26.2 us; one row of 32000 words 5.3 us. Slower: clusters that exchange their counts through distributed shared memory (two
// more barriers, 100 us), persistent clusters with the next row's logits under way in registers or by cp.async (85 to 135
// us: the CTA with the frequent words holds up its cluster).
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

// Four CTAs an SM: fewer and larger ones overlap too little of their starts, more find no room for their counts. 192 and 64 rows
// of 152064 words with 128 x 20 (threads x tokens held), 256 x 20, 320 x 16, 384 x 20 and 512 x 20: 74.3 and 36.2 / 59.5 and
// 26.4 / 57.1 and 26.2 / 82.1 and 35.0 / 74.8 and 30.6 us.
constexpr int kThreads = 320, kWarps = kThreads / 32;
constexpr int kHeld = 16;                   // tokens of its slice that a thread holds in registers
constexpr int kBatch = kThreads * kHeld;     // tokens a CTA holds at once
constexpr int kAhead = 2;                    // loads of four tokens of the history that go ahead of the logits
constexpr int kPlaces = 384;                 // CTAs of rows that clusters still serve as well as CTAs on their own
constexpr int kMaxSlice = 51200;             // tokens a CTA holds counts for (200 KB)
constexpr uint32_t kPrompt = 1u << 31;       // the token is in the prompt
constexpr uint32_t kBiased = 1u << 30;       // the sequence has a bias for it
constexpr uint32_t kCount = kBiased - 1;     // occurrences among the generated tokens

struct LogitRules {
  const float* z;
  float* out;
  int32_t* best;
  int n_rows, vocab, ld_in, ld_out, slice;   // slice: tokens a CTA, a multiple of 32
  const int32_t* seq_of;
  int n_seqs;
  const int32_t *hist, *hist_cu, *gen_start;
  int n_hist;
  bool hist4;  // hist is 16-byte aligned
  const int32_t *path, *path_cu;
  int n_path;
  const float *rep, *freq, *pres;
  const int32_t *bias_cu, *bias_id;
  const float* bias;
  int n_bias;
  const uint32_t* allow;
  int n_rules, words;
  const int32_t* rule;
};

// [cu[i], cu[i + 1]) within [0, n): lists that break their precondition give wrong values, never a read elsewhere.
__device__ __forceinline__ int2 range_of(const int32_t* cu, int i, int n) {
  const int lo = min(max(cu[i], 0), n);
  return make_int2(lo, min(max(cu[i + 1], lo), n));
}

// A value's place in the order of floats (no NaN comes here), the token in the low half so that the first of equals wins.
__device__ __forceinline__ unsigned long long order_key(float x, int token) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (static_cast<unsigned long long>((u >> 31) ? ~u : u | 0x80000000u) << 32) | (0xffffffffu - uint32_t(token));
}

__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t u = uint32_t(key >> 32);
  return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}

// *at = to where it is `from`; what it was. Releases the CTA's writes before it, acquires those before the value it read.
// (192 rows of 152064 words with 256 threads a CTA: 59.5 us, relaxed between fences 63.6, without the acquisition, on the order that a load behind
// its address has anyway, 58.3.)
__device__ __forceinline__ int swap_if(int32_t* at, int from, int to) {
  int was;
  asm volatile("atom.acq_rel.gpu.global.cas.b32 %0, [%1], %2, %3;" : "=r"(was) : "l"(at), "r"(from), "r"(to) : "memory");
  return was;
}

// Whether token i of value v goes before token j of value w.
__device__ __forceinline__ bool goes_before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// CLUSTER: the row's CTAs are a cluster and find its best token together; else each offers its own to best[row], which
// started as -1.
template <int W, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 4) logit_rules_kernel(const __grid_constant__ LogitRules p, int C) {
  extern __shared__ uint4 smem4[];
  __shared__ unsigned long long warp_best[16 * kWarps];  // of every warp of the row, in the cluster's first CTA
  uint32_t* word = reinterpret_cast<uint32_t*>(smem4);   // [slice]
  const int rank = blockIdx.x % C, row = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31;
  const int t0 = rank * p.slice, n = max(0, min(p.slice, p.vocab - t0));  // this CTA's tokens
  if (CLUSTER) cluster_arrive();  // waited for before the first access to another CTA's shared memory
  for (int i = tid; i < p.slice / 4; i += kThreads) smem4[i] = make_uint4(0u, 0u, 0u, 0u);
  pdl_launch_dependents();
  pdl_wait();
  const float* z = p.z + size_t(row) * p.ld_in + t0;
  float* out = p.out + size_t(row) * p.ld_out + t0;
  // W = 4: 16-byte pieces, where the rows are aligned for them; 1: single tokens. The slice's first batch is on its way
  // while the history is counted.
  float x[kHeld];
  auto load = [&](int base) {
#pragma unroll
    for (int k = 0; k < kHeld / W; ++k) {
      const int i = base + W * (k * kThreads + tid);
      if (i >= n) continue;
      if constexpr (W == 4) {
        const float4 v = __ldcs(reinterpret_cast<const float4*>(z + i));
        x[4 * k] = v.x, x[4 * k + 1] = v.y, x[4 * k + 2] = v.z, x[4 * k + 3] = v.w;
      } else {
        x[k] = __ldcs(z + i);
      }
    }
  };
  const int seq = p.seq_of ? p.seq_of[row] : row;
  const bool has_seq = seq >= 0 && seq < p.n_seqs;
  const int2 hl = has_seq && p.hist ? range_of(p.hist_cu, seq, p.n_hist) : make_int2(0, 0);
  const int gen = hl.y > hl.x ? min(max(p.gen_start[seq], hl.x), hl.y) : 0;
  const int2 bl = has_seq && p.bias ? range_of(p.bias_cu, seq, p.n_bias) : make_int2(0, 0);
  const int2 pl = p.path ? range_of(p.path_cu, row, p.n_path) : make_int2(0, 0);
  const int rule = p.allow ? p.rule[row] : -1;
  const uint32_t* allow = rule >= 0 && rule < p.n_rules ? p.allow + size_t(rule) * p.words + t0 / 32 : nullptr;
  const float rep = has_seq && p.rep ? p.rep[seq] : 1.0f;
  const float freq = has_seq && p.freq ? p.freq[seq] : 0.0f, pres = has_seq && p.pres ? p.pres[seq] : 0.0f;
  // four tokens of the history a load, from the 16-byte boundary before its first (those outside it are passed over)
  auto tokens4 = [&](int i) -> int4 {
    if (p.hist4 && i + 3 < p.n_hist) return *reinterpret_cast<const int4*>(p.hist + i);
    int4 t = make_int4(-1, -1, -1, -1);
    if (i < p.n_hist) t.x = p.hist[i];
    if (i + 1 < p.n_hist) t.y = p.hist[i + 1];
    if (i + 2 < p.n_hist) t.z = p.hist[i + 2];
    if (i + 3 < p.n_hist) t.w = p.hist[i + 3];
    return t;
  };
  const int h0 = (hl.x & ~3) + 4 * tid;
  int4 first[kAhead];  // ahead of the logits
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    first[u] = h0 + u * 4 * kThreads < hl.y ? tokens4(h0 + u * 4 * kThreads) : make_int4(-1, -1, -1, -1);
  // the thread's first entry of the bias list, and the logit that it concerns
  const bool has_bias = bl.x + tid < bl.y;
  const int b_id = has_bias ? p.bias_id[bl.x + tid] : -1;
  const uint32_t b_tok = has_bias ? uint32_t(b_id - t0) : ~0u;
  const float b_z = b_tok < uint32_t(n) ? z[b_tok] : 0.0f;
  const float b_add = b_tok < uint32_t(n) ? p.bias[bl.x + tid] : 0.0f;
  load(0);
  __syncthreads();  // the words are zero
  // Placeholders of an image lie outside the vocabulary and so outside every slice. (unsigned: negatives too)
  auto count = [&](int token, int i) {
    const uint32_t t = uint32_t(token) - uint32_t(t0);
    if (token < 0 || t >= uint32_t(n) || i < hl.x || i >= hl.y) return;
    if (i >= gen) atomicAdd(&word[t], 1u);
    else if (!(word[t] & kPrompt)) atomicOr(&word[t], kPrompt);  // a prompt may repeat one token throughout
  };
  auto count4 = [&](const int4& t, int i) {
    count(t.x, i);
    count(t.y, i + 1);
    count(t.z, i + 2);
    count(t.w, i + 3);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) count4(first[u], h0 + u * 4 * kThreads);
  for (int i = h0 + kAhead * 4 * kThreads; i < hl.y; i += 16 * kThreads) {
    int4 t[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      t[u] = i + u * 4 * kThreads < hl.y ? tokens4(i + u * 4 * kThreads) : make_int4(-1, -1, -1, -1);
#pragma unroll
    for (int u = 0; u < 4; ++u) count4(t[u], i + u * 4 * kThreads);
  }
  for (int i = pl.x + tid; i < pl.y; i += kThreads) {
    const uint32_t t = uint32_t(p.path[i] - t0);
    if (t < uint32_t(n)) atomicAdd(&word[t], 1u);
  }
  if (b_tok < uint32_t(n)) atomicOr(&word[b_tok], kBiased);
  for (int i = bl.x + tid + kThreads; i < bl.y; i += kThreads) {
    const uint32_t t = uint32_t(p.bias_id[i] - t0);
    if (t < uint32_t(n)) atomicOr(&word[t], kBiased);
  }
  __syncthreads();

  float best = -INFINITY;
  int best_at = -1;
  auto penalised = [&](float v, uint32_t w) {
    if (w & (kCount | kPrompt)) {
      v = v > 0.0f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
      if (w & kCount) v = __fsub_rn(__fsub_rn(v, __fmul_rn(freq, float(w & kCount))), pres);
    }
    return v;
  };
  auto take = [&](float v, int i) {  // a thread's tokens ascend: the first of equals stays
    if (v > best) {
      best = v;
      best_at = t0 + i;
    }
  };
  // A thread a biased token (the list ascends: at its first entry, which adds up all of the token's). Nobody else
  // touches its logit, so this also holds in place.
  float biased_best = -INFINITY;
  int biased_at = -1;
  auto biased = [&](int i, int id, uint32_t t, float v, float add) {
    if (i > bl.x && p.bias_id[i - 1] == id) return;
    for (int j = i + 1; j < bl.y && p.bias_id[j] == id; ++j) add = __fadd_rn(add, p.bias[j]);
    v = __fadd_rn(penalised(v, word[t]), add);
    if (allow && !((allow[t / 32] >> (t % 32)) & 1u)) v = -INFINITY;
    out[t] = v;
    if (v > biased_best) {
      biased_best = v;
      biased_at = id;
    }
  };
  if (b_tok < uint32_t(n)) biased(bl.x + tid, b_id, b_tok, b_z, b_add);
  for (int i = bl.x + tid + kThreads; i < bl.y; i += kThreads) {
    const int id = p.bias_id[i];
    const uint32_t t = uint32_t(id - t0);
    if (t < uint32_t(n)) biased(i, id, t, z[t], p.bias[i]);
  }
  for (int base = 0; base < n; base += kBatch) {
    if (base > 0) load(base);
#pragma unroll
    for (int k = 0; k < kHeld / W; ++k) {
      const int i = base + W * (k * kThreads + tid);
      if (i >= n) continue;
      uint32_t w[W];
      if constexpr (W == 4) {
        const uint4 q = smem4[i / 4];
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
      } else {
        w[0] = word[i];
      }
      const uint32_t a = allow ? allow[i / 32] >> (i % 32) : 15u;
      float v[W];
      uint32_t any = 0;
#pragma unroll
      for (int c = 0; c < W; ++c) {
        v[c] = x[W * k + c];
        any |= w[c];
      }
      if (any) {
#pragma unroll
        for (int c = 0; c < W; ++c) v[c] = penalised(v[c], w[c]);
      }
#pragma unroll
      for (int c = 0; c < W; ++c)
        if (!((a >> c) & 1u)) v[c] = -INFINITY;
      if (any & kBiased) {  // the biased ones are done
#pragma unroll
        for (int c = 0; c < W; ++c)
          if (!(w[c] & kBiased)) {
            out[i + c] = v[c];
            take(v[c], i + c);
          }
      } else if constexpr (W == 4) {
        *reinterpret_cast<float4*>(out + i) = make_float4(v[0], v[1], v[2], v[3]);
        if (fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) > best) {
#pragma unroll
          for (int c = 0; c < 4; ++c) take(v[c], i + c);
        }
      } else {
        out[i] = v[0];
        take(v[0], i);
      }
    }
  }
  if (p.best) {
    unsigned long long k = best_at >= 0 ? order_key(best, best_at) : 0;  // 0: nothing left
    if (biased_at >= 0) {
      const unsigned long long y = order_key(biased_best, biased_at);
      k = y > k ? y : k;
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      const unsigned long long y = __shfl_xor_sync(0xffffffffu, k, off);
      k = y > k ? y : k;
    }
    if constexpr (!CLUSTER) {
      // offers in any order end with the same token: one is replaced only by a token that goes before it, whose own
      // value is in `out` (written before its offer, which releases it)
      if (lane == 0) warp_best[tid >> 5] = k;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < kWarps; ++w) k = warp_best[w] > k ? warp_best[w] : k;
        if (k) {
          const int id = int32_t(0xffffffffu - uint32_t(k));
          volatile float* row_out = p.out + size_t(row) * p.ld_out;
          const float v = key_value(k);
          for (int cur = -1, was; (was = swap_if(p.best + row, cur, id)) != cur; cur = was)
            if (!goes_before(v, id, row_out[was], was)) break;
        }
      }
      return;
    }
    cluster_wait();  // every CTA of the row has started
    if (lane == 0) {
      const uint32_t to = dsmem_addr(&warp_best[rank * kWarps + (tid >> 5)], 0);
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(k) : "memory");
    }
    __syncwarp();
    cluster_arrive();
    if (rank != 0) return;  // nobody reads this CTA's shared memory
    cluster_wait();
    if (tid < 32) {
      k = 0;
      for (int i = tid; i < C * kWarps; i += 32) k = warp_best[i] > k ? warp_best[i] : k;
#pragma unroll
      for (int off = 16; off; off >>= 1) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, k, off);
        k = y > k ? y : k;
      }
      if (tid == 0) p.best[row] = k ? int32_t(0xffffffffu - uint32_t(k)) : -1;
    }
  }
}

__global__ void no_best_kernel(int32_t* best, int n) {
  pdl_launch_dependents();
  pdl_wait();
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < n) best[i] = -1;
}

}  // namespace

// Cluster and slice for a vocabulary: as few CTAs a row as hold a whole slice in registers, 16 (the most a cluster
// has) where that takes more; slices up to kMaxSlice are read in batches.
static int logits_cluster(int vocab, int* slice) {
  auto per = [&](int k) { return ((vocab + k - 1) / k + 31) / 32 * 32; };
  int c = 1;
  while (c < 16 && per(c) > kBatch) c *= 2;
  *slice = per(c);
  return c;
}

}  // namespace spd

using namespace spd;

extern "C" int spd_logits_process(const float* logits, int n_rows, int vocab, int ld, const spd_logits_rules* r,
                                  float* out, int ld_out, int32_t* best, void* stream) {
  if (!logits || !r || !out || n_rows < 0 || vocab < 1 || ld < vocab || ld_out < vocab)
    return fail(SPD_EINVAL, "bad logits arguments");
  if (r->n_seqs < 0 || r->n_hist < 0 || r->n_path < 0 || r->n_bias < 0 || r->n_rules < 0)
    return fail(SPD_EINVAL, "negative list length");
  if (r->hist && (!r->hist_cu || !r->gen_start)) return fail(SPD_EINVAL, "a history needs hist_cu and gen_start");
  if (r->path && !r->path_cu) return fail(SPD_EINVAL, "paths need path_cu");
  if (r->bias && (!r->bias_cu || !r->bias_id)) return fail(SPD_EINVAL, "biases need bias_cu and bias_id");
  if (r->allow && !r->rule) return fail(SPD_EINVAL, "grammar masks need the rows' rule");
  if (!r->seq_of && (r->hist || r->bias) && r->n_seqs < n_rows)
    return fail(SPD_EINVAL, "without seq_of every row is a sequence");
  if (n_rows == 0) return SPD_OK;
  LogitRules p{};
  const int C = logits_cluster(vocab, &p.slice);
  if (p.slice > kMaxSlice) return fail(SPD_EUNSUPPORTED, "vocabulary of %d tokens (at most %d)", vocab, 16 * kMaxSlice);
  if (n_rows > 0x7fffffff / C) return fail(SPD_EUNSUPPORTED, "%d rows", n_rows);
  p.z = logits;
  p.out = out;
  p.best = best;
  p.n_rows = n_rows;
  p.vocab = vocab;
  p.ld_in = ld;
  p.ld_out = ld_out;
  p.seq_of = r->seq_of;
  p.n_seqs = r->n_seqs;
  p.hist = r->n_hist > 0 ? r->hist : nullptr;
  p.hist_cu = r->hist_cu;
  p.gen_start = r->gen_start;
  p.n_hist = r->n_hist;
  p.hist4 = (reinterpret_cast<uintptr_t>(r->hist) & 15) == 0;
  p.path = r->n_path > 0 ? r->path : nullptr;
  p.path_cu = r->path_cu;
  p.n_path = r->n_path;
  p.rep = r->repetition;
  p.freq = r->frequency;
  p.pres = r->presence;
  p.bias_cu = r->bias_cu;
  p.bias_id = r->bias_id;
  p.bias = r->n_bias > 0 ? r->bias : nullptr;
  p.n_bias = r->n_bias;
  p.allow = reinterpret_cast<const uint32_t*>(r->allow);
  p.n_rules = r->n_rules;
  p.words = (vocab + 31) / 32;
  p.rule = r->rule;
  const bool vec = vocab % 4 == 0 && ld % 4 == 0 && ld_out % 4 == 0 &&
                   ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  // A cluster needs all of its places at once. Where the rows do not fit on the GPU together, CTAs on their own
  // fill it better, at the price of a launch that clears `best`.
  const bool apart = C > 1 && n_rows > kPlaces / C;
  auto kern = vec ? (apart ? logit_rules_kernel<4, false> : logit_rules_kernel<4, true>)
                  : (apart ? logit_rules_kernel<1, false> : logit_rules_kernel<1, true>);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (apart && best)
    SPD_CUDA_TRY(launch_pdl(no_best_kernel, dim3((n_rows + kThreads - 1) / kThreads), dim3(kThreads), 0, st, best, n_rows));
  const size_t smem = size_t(p.slice) * 4;
  static DeviceOnce prepared[4];
  SPD_CUDA_TRY(once_per_device(prepared[2 * vec + apart], [&] {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * 4);
    return e ? e : cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  }));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_rows * C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = apart ? 1 : 2;
  const double by = 8.0 * n_rows * vocab + 4.0 * (double(p.n_hist) + p.n_path + 2.0 * p.n_bias);
  const int slot = trace_begin(cfg.stream);
  SPD_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, p, C));
  trace_end(slot, cfg.stream, TR_ROWS, 0.0, by);
  return SPD_OK;
}
