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
// A row moves 8 V bytes and one occurrence count a token has to be found for it. The counts need no memory of the
// GPU's: a cluster of CTAs shares a row's vocabulary, each holds the counts of its slice in shared memory (one word a
// token), and every CTA adds its share of the history into the slices of all through distributed shared memory.
#include <cooperative_groups.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
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

// A value's place in the order of floats (NaN below all), the token in the low half so that the first of equals wins.
__device__ __forceinline__ unsigned long long order_key(float x, int token) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  const uint32_t k = isnan(x) ? 0u : (u >> 31) ? ~u : u | 0x80000000u;
  return (static_cast<unsigned long long>(k) << 32) | (0xffffffffu - uint32_t(token));
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads) logit_rules_kernel(const LogitRules p) {
  extern __shared__ uint4 smem4[];
  __shared__ unsigned long long warp_best[kThreads / 32];
  __shared__ unsigned long long cta_best;
  uint32_t* word = reinterpret_cast<uint32_t*>(smem4);  // [slice]
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = int(cluster.block_rank()), C = int(cluster.num_blocks());
  const int row = blockIdx.x / C, tid = threadIdx.x;
  const int t0 = rank * p.slice, n = max(0, min(p.slice, p.vocab - t0));  // this CTA's tokens
  for (int i = tid; i < p.slice / 4; i += kThreads) smem4[i] = make_uint4(0u, 0u, 0u, 0u);
  pdl_launch_dependents();
  pdl_wait();
  cluster.sync();
  const int seq = p.seq_of ? p.seq_of[row] : row;
  const bool has_seq = seq >= 0 && seq < p.n_seqs;
  if (has_seq && p.hist) {
    const int2 h = range_of(p.hist_cu, seq, p.n_hist);
    const int gen = p.gen_start[seq];
    for (int i = h.x + rank * kThreads + (tid & ~31); i < h.y; i += C * kThreads) {
      const int at = i + (tid & 31);
      const int t = at < h.y ? p.hist[at] : -1;
      const bool fine = t >= 0 && t < p.vocab;  // placeholders of an image lie outside the vocabulary
      const bool made = at >= gen;
      // texts repeat few tokens: one addition for all of a warp's occurrences
      const unsigned same = __match_any_sync(0xffffffffu, fine ? 2 * t + int(made) : -1);
      if (fine && (tid & 31) == __ffs(same) - 1) {
        uint32_t* w = cluster.map_shared_rank(word, t / p.slice) + t % p.slice;
        if (made) atomicAdd(w, uint32_t(__popc(same)));
        else atomicOr(w, kPrompt);
      }
    }
  }
  if (p.path) {
    const int2 h = range_of(p.path_cu, row, p.n_path);
    for (int i = h.x + tid; i < h.y; i += kThreads) {
      const int t = p.path[i] - t0;
      if (t >= 0 && t < n) atomicAdd(&word[t], 1u);
    }
  }
  int2 bl = make_int2(0, 0);
  if (has_seq && p.bias) {
    bl = range_of(p.bias_cu, seq, p.n_bias);
    for (int i = bl.x + tid; i < bl.y; i += kThreads) {
      const int t = p.bias_id[i] - t0;
      if (t >= 0 && t < n) atomicOr(&word[t], kBiased);
    }
  }
  cluster.sync();  // every CTA's share of the history has arrived

  const float rep = has_seq && p.rep ? p.rep[seq] : 1.0f;
  const float freq = has_seq && p.freq ? p.freq[seq] : 0.0f, pres = has_seq && p.pres ? p.pres[seq] : 0.0f;
  const int rule = p.allow && p.rule ? p.rule[row] : -1;
  const uint32_t* allow = rule >= 0 && rule < p.n_rules ? p.allow + size_t(rule) * p.words + t0 / 32 : nullptr;
  const float* z = p.z + size_t(row) * p.ld_in + t0;
  float* out = p.out + size_t(row) * p.ld_out + t0;
  unsigned long long best = 0;
  auto one = [&](float x, uint32_t w, int i) {
    if (w & (kCount | kPrompt)) {
      x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
      if (w & kCount) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, float(w & kCount))), pres);
    }
    if (w & kBiased) {  // the list ascends: the first entry of the token, then all of its entries in order
      int lo = bl.x, hi = bl.y;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.bias_id[mid] < t0 + i) lo = mid + 1;
        else hi = mid;
      }
      float add = 0.0f;
      for (; lo < bl.y && p.bias_id[lo] == t0 + i; ++lo) add = __fadd_rn(add, p.bias[lo]);
      x = __fadd_rn(x, add);
    }
    return x;
  };
  auto take = [&](float x, int i) {
    const unsigned long long k = order_key(x, t0 + i);
    best = k > best ? k : best;
  };
  if constexpr (VEC) {
    for (int i = 4 * tid; i < n; i += 4 * kThreads) {
      float4 x = *reinterpret_cast<const float4*>(z + i);
      const uint4 w = smem4[i / 4];
      const uint32_t a = allow ? allow[i / 32] >> (i % 32) : 15u;
      if (w.x | w.y | w.z | w.w) {
        x.x = one(x.x, w.x, i);
        x.y = one(x.y, w.y, i + 1);
        x.z = one(x.z, w.z, i + 2);
        x.w = one(x.w, w.w, i + 3);
      }
      if (!(a & 1u)) x.x = -INFINITY;
      if (!(a & 2u)) x.y = -INFINITY;
      if (!(a & 4u)) x.z = -INFINITY;
      if (!(a & 8u)) x.w = -INFINITY;
      *reinterpret_cast<float4*>(out + i) = x;
      take(x.x, i);
      take(x.y, i + 1);
      take(x.z, i + 2);
      take(x.w, i + 3);
    }
  } else {
    for (int i = tid; i < n; i += kThreads) {
      float x = one(z[i], word[i], i);
      if (allow && !((allow[i / 32] >> (i % 32)) & 1u)) x = -INFINITY;
      out[i] = x;
      take(x, i);
    }
  }
  if (p.best) {
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, off);
      best = k > best ? k : best;
    }
    if ((tid & 31) == 0) warp_best[tid >> 5] = best;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kThreads / 32; ++w) best = warp_best[w] > best ? warp_best[w] : best;
      cta_best = best;
    }
    cluster.sync();
    if (rank == 0 && tid == 0) {
      for (int c = 1; c < C; ++c) {
        const unsigned long long k = *cluster.map_shared_rank(&cta_best, c);
        best = k > best ? k : best;
      }
      // nothing left: every value is -inf (order key 0x007fffff) or NaN (0)
      p.best[row] = (best >> 32) <= 0x007fffffull ? -1 : int32_t(0xffffffffu - uint32_t(best));
    }
    cluster.sync();  // the others' shared memory outlives the read
  }
}

}  // namespace

// Cluster and slice for a vocabulary: eight CTAs a row, more where their slices would not fit in shared memory (16 is
// the most a cluster has), fewer below 1024 tokens a CTA.
static int logits_cluster(int vocab, int* slice) {
  int c = 8;
  while (c > 1 && vocab < 1024 * c) c /= 2;
  auto per = [&](int k) { return ((vocab + k - 1) / k + 31) / 32 * 32; };
  if (per(c) > kMaxSlice) c = 16;
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
  auto kern = vec ? logit_rules_kernel<true> : logit_rules_kernel<false>;
  const size_t smem = size_t(p.slice) * 4;
  SPD_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * 4));
  if (C > 8) SPD_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_rows * C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const double by = 8.0 * n_rows * vocab + 4.0 * (double(p.n_hist) + p.n_path + 2.0 * p.n_bias);
  const int slot = trace_begin(cfg.stream);
  SPD_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, p));
  trace_end(slot, cfg.stream, TR_ROWS, 0.0, by);
  return SPD_OK;
}
