// Beam search's selection: of every request's beams and their continuations the best, in one pass over the logits.
//
// total(w, t) = score_w + z_wt - log sum_u exp z_wu; the n_out largest over the live beams w and the tokens t other than `eos`,
// ties to the lower beam, then to the lower token. A beam's end, total(w, eos), counts where fewer than n_out candidates of
// the request, other ends among them, go before it.
//
// A row's tokens are split over CTAs (slices). Of one row the order of the totals is that of the logits, so of a slice only its
// n_out best can be among the request's best. A CTA streams its slice through registers: the maximum and the sum of
// exponentials a thread, and those tokens that beat the n_out-th best so far go to a list in shared memory, which is cut back to
// n_out when it has doubled. The first bound: of n_out or more groups of threads the least of their maxima. Where more tokens beat
// the bound than the list holds (rising or equal logits) the batch's n_out best are taken one by one.
// A CTA a request then takes the n_out lists of the best heads, and of their candidates that are not behind the last of these
// heads the n_out best, by counting how many go before each. Rounded to fp32 totals of one
// beam would tie that differ, and fp64 is slow here, so totals are pairs of fp32 values (a sum and what it was rounded by). The logarithm
// of a beam's sum itself is off by about 2^-20 (exponentials of a few units, sums in fp32), which is what separates beams.
//
// What bounds it: of many rows the stream and the instructions a logit takes (an exponential, two maxima, a comparison): 128 rows
// of 152064 19.4 us with the merge, 78 MB; of one request a chain, 6 us. 256 threads a CTA, or twice as many tokens a thread, took
// longer.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kHeld = 16;                  // tokens a thread holds
constexpr int kBatch = kThreads * kHeld;
constexpr int kMaxBeams = 32;
constexpr int kList = 384;                 // candidates a CTA holds
constexpr int kMergeThreads = 256;
constexpr int kStages = 4;                 // batches on their way into shared memory
constexpr int kCtasSm = 6;                 // CTAs an SM
// Lists a request, of which the merging CTA has one a thread: of 12 and 4 rows of 152064 with up to 48 / 96 / 128 / 192 / 256 lists 18.6 /
// 15.9 / 13.9 / 15.5 / 15.4 and 10.1 / 8.8 / 8.7 / 10.5 / 11.5 us.
constexpr int kMostLists = 128;
static_assert(kMaxBeams <= kMostLists && kMostLists <= kMergeThreads, "a list a thread");

struct BeamArgs {
  const float* z;
  int vocab, ld, n_in, n_out, slices, slice, eos;
  const float* scores;
  unsigned long long* best;  // [row][slice][n_out] order keys, descending, 0 behind the last
  float2* sums;              // [row][slice] maximum, sum of exp(z - maximum)
  int32_t *parent, *token;
  float *out, *ended;
  int* status;
  long long budget;
};

// A value's place in the order of floats, the token in the low half so that the first of equals wins (0: none).
__device__ __forceinline__ unsigned long long order_key(float x, int token) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (static_cast<unsigned long long>((u >> 31) ? ~u : u | 0x80000000u) << 32) | (0xffffffffu - uint32_t(token));
}
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t u = uint32_t(key >> 32);
  return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    const unsigned long long y = __shfl_xor_sync(0xffffffffu, k, off);
    k = y > k ? y : k;
  }
  return k;
}

// exp(x - m): the difference first, so that large logits lose nothing.
__device__ __forceinline__ float exp_less(float x, float m) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"((x - m) * 1.4426950408889634f));
  return y;
}
// The least value above a key's.
__device__ __forceinline__ float above(unsigned long long key) { return key_value(key + (1ull << 32)); }
// The sum of states (maximum, sum): NaN stays, -inf adds nothing.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);
  return make_float2(m, a.y * exp_less(a.x, m) + b.y * exp_less(b.x, m));
}

// Waits for the batches from `first` on that were fetched: they land before the CTA exits.
__device__ __noinline__ void land(uint64_t* full, int first, int n, long long budget) {
  volatile int no_abort = 0;
  for (int i = first; i < first + kStages && i * kBatch < n; ++i) mbar_wait(&full[i % kStages], (i / kStages) & 1, &no_abort, budget);
}

// W = 4: rows whose 16-byte pieces are aligned, batches by bulk copies into shared memory; 1: any rows, through registers.
template <int W>
__global__ void __launch_bounds__(kThreads, kCtasSm) beam_slice_kernel(const __grid_constant__ BeamArgs p) {
  extern __shared__ __align__(128) float ring[];  // [kStages][kBatch]
  __shared__ uint64_t full[kStages];
  __shared__ int aborted;  // 1 + the first batch that a thread gave up waiting for; none is fetched from then on
  __shared__ unsigned long long list[kList], top[kMaxBeams], wbest[2][kWarps];
  __shared__ float group[kMaxBeams];
  __shared__ float2 wsum[kWarps];
  __shared__ int pushed[3];
  const int row = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = p.n_out;
  const int t0 = blockIdx.x * p.slice, n = max(0, min(p.slice, p.vocab - t0));
  if (tid < 3) pushed[tid] = 0;
  if (tid < kMaxBeams) top[tid] = 0;
  pdl_launch_dependents();
  pdl_wait();
  const float* z = p.z + size_t(row) * p.ld + t0;
  auto place = [&](int base, int k) { return base + (W == 4 ? (k >> 2) * (4 * kThreads) + 4 * tid + (k & 3) : k * kThreads + tid); };
  float next[W == 4 ? 1 : kHeld];
  auto fetch = [&](int base, int b) {
    if constexpr (W == 4) {
      if (tid == 0 && base < n && !aborted) {
        const uint32_t bytes = 4u * uint32_t(min(kBatch, n - base));  // (slices are multiples of four)
        mbar_arrive_expect_tx(&full[b % kStages], bytes);
        bulk_load(ring + (b % kStages) * kBatch, z + base, bytes, &full[b % kStages]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const int i = place(base, k);
        next[k] = i < n ? __ldcs(z + i) : -INFINITY;
      }
    }
  };
  if constexpr (W == 4) {
    if (tid == 0) {
      aborted = 0;
      for (int b = 0; b < kStages; ++b) mbar_init(&full[b], 1);
      fence_mbar_init();
      for (int b = 0; b < kStages; ++b) fetch(b * kBatch, b);
    }
  } else {
    fetch(0, 0);
  }
  float m = -INFINITY, s = 0.0f;   // of the thread's tokens
  float low = 0.0f;                // a later token below it is not among the best
  int have = 0;                    // entries of the list
  bool sorted = true;
  __syncthreads();
  // cuts the list's `all` entries back to the K best, in order, in top and list
  auto cut = [&](int all) {
    for (int i = tid; i < all; i += kThreads) {
      const unsigned long long mine = list[i];
      int ahead = 0;
      for (int j = 0; j < all; ++j) ahead += list[j] > mine;
      if (ahead < K) top[ahead] = mine;
    }
    __syncthreads();
    if (tid < min(all, K)) list[tid] = top[tid];
    have = min(all, K);
    sorted = true;
    if (have == K) low = above(top[K - 1]);
  };
  for (int base = 0, b = 0; base < n; base += kBatch, ++b) {
    float x[kHeld];
    if constexpr (W == 4) {
      if (!mbar_wait(&full[b % kStages], (b / kStages) & 1, &aborted, p.budget)) {
        if (!aborted) aborted = b + 1;
        set_status(p.status, SPD_ETIMEOUT);
      }
#pragma unroll
      for (int k = 0; k < kHeld; k += 4) {
        const int i = place(base, k);
        float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (i < n) v = *reinterpret_cast<const float4*>(ring + (b % kStages) * kBatch + i - base);
        x[k] = v.x, x[k + 1] = v.y, x[k + 2] = v.z, x[k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < kHeld; ++k) x[k] = next[k];
      if (base + kBatch < n) fetch(base + kBatch, b + 1);
    }
    float t4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int k = 4; k < kHeld; ++k) t4[k & 3] = fmaxf(t4[k & 3], x[k]);
    float most = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
    const float mn = fmaxf(m, most), ref = mn == -INFINITY ? 0.0f : mn;
    float s4[4] = {s * exp_less(m, ref), 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kHeld; ++k) s4[k & 3] += exp_less(x[k], ref);
    m = mn;
    s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
    if (unsigned(p.eos - t0 - base) < unsigned(kBatch)) {  // the end is no continuation
      most = -INFINITY;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (t0 + place(base, k) == p.eos) x[k] = -INFINITY;
        most = fmaxf(most, x[k]);
      }
    }
    const bool first = base == 0;
    if (first) {  // the least of the maxima of 4, 8, 16 or 32 groups of threads
      const int width = K <= 4 ? 32 : K <= 8 ? 16 : K <= 16 ? 8 : 4;
      float g = most;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const float y = __shfl_xor_sync(0xffffffffu, g, off);
        if (off < width) g = fmaxf(g, y);
      }
      if ((lane & 3) == 0) group[tid >> 2] = g;
      __syncthreads();
      g = group[lane];
#pragma unroll
      for (int off = 16; off; off >>= 1) g = fminf(g, __shfl_xor_sync(0xffffffffu, g, off));
      low = fmaxf(g, -3.402823466e38f);  // (-inf is no candidate)
    }
    if (most >= low) {
      uint32_t some = 0;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) some |= x[k] >= low ? 1u << k : 0u;
      int at = have + atomicAdd(&pushed[b % 3], __popc(some));
      if constexpr (W == 4) {
        for (; some && at < kList; some &= some - 1, ++at) {
          const int i = place(base, __ffs(some) - 1);
          list[at] = order_key(ring[(b % kStages) * kBatch + i - base], t0 + i);
        }
      } else {
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
          if (((some >> k) & 1u) && at < kList) list[at++] = order_key(x[k], t0 + place(base, k));
      }
    }
    if (tid == 0) pushed[(b + 1) % 3] = 0;  // (read last before the barrier of the batch before)
    __syncthreads();
    if constexpr (W == 4) fetch(base + kStages * kBatch, b + kStages);  // (the batch is in registers)
    const int all = have + pushed[b % 3];
    if (all > kList) {
      // the list as it was, and this batch's tokens one by one: the k-th largest of both in round k
      cut(have);
      __syncthreads();
      unsigned long long mine[kHeld], big = 0, old = tid < have ? list[tid] : 0;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        mine[k] = x[k] > -INFINITY ? order_key(x[k], t0 + place(base, k)) : 0;
        big = mine[k] > big ? mine[k] : big;
      }
      have = 0;
      for (int k = 0; k < K; ++k) {
        const unsigned long long c = warp_max(big > old ? big : old);
        if (lane == 0) wbest[k & 1][warp] = c;
        __syncthreads();
        unsigned long long a = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) a = wbest[k & 1][w] > a ? wbest[k & 1][w] : a;
        if (a == 0) continue;
        ++have;
        if (tid == 0) top[k] = list[k] = a;
        if (old == a) old = 0;
        if (big == a) {
          big = 0;
#pragma unroll
          for (int e = 0; e < kHeld; ++e) {
            if (mine[e] == a) mine[e] = 0;
            big = mine[e] > big ? mine[e] : big;
          }
        }
      }
      __syncthreads();
      sorted = true;
      if (have == K) low = above(top[K - 1]);
    } else if (all > have) {
      if (first || all > 2 * K) {
        cut(all);
      } else {
        have = all;
        sorted = false;
      }
    }
  }
  if (!sorted) {
    __syncthreads();
    cut(have);
  }
  float2 sum = make_float2(m, s);
#pragma unroll
  for (int off = 16; off; off >>= 1)
    sum = join(sum, make_float2(__shfl_down_sync(0xffffffffu, sum.x, off), __shfl_down_sync(0xffffffffu, sum.y, off)));
  if (lane == 0) wsum[warp] = sum;
  __syncthreads();
  const size_t at = size_t(row) * p.slices + blockIdx.x;
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w) sum = join(sum, wsum[w]);
    p.sums[at] = sum;
  }
  if (tid < K) p.best[at * K + tid] = tid < have ? top[tid] : 0;
  if (W == 4 && tid == 0 && aborted) land(full, aborted - 1, n, p.budget);
}

// hi + lo = a + b exactly, hi the rounded sum.
__device__ __forceinline__ float2 two_sum(float a, float b) {
  const float hi = __fadd_rn(a, b), x = __fsub_rn(hi, a);
  return make_float2(hi, __fadd_rn(__fsub_rn(a, __fsub_rn(hi, x)), __fsub_rn(b, x)));
}
// (a.x + a.y) + b as such a pair.
__device__ __forceinline__ float2 add_pair(float2 a, float b) {
  const float2 s = two_sum(a.x, b);
  return two_sum(s.x, __fadd_rn(s.y, a.y));
}
// The natural logarithm of l > 0 as a pair: l = 2^k f with f in [3/4, 3/2), k ln 2 in two parts.
__device__ __forceinline__ float2 log_pair(float l) {
  int k;
  float f = frexpf(l, &k);  // [1/2, 1)
  if (f < 0.75f) {
    f *= 2.0f;
    --k;
  }
  const float kh = float(k) * 0.693145751953125f;  // 16 bits of ln 2: exact
  return add_pair(two_sum(kh, float(k) * 1.42860682030941723e-6f), log1pf(f - 1.0f));
}

__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t u) { return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u); }
// A candidate's total as an integer of the same order (the pair's values), where the beam's logits are added to `norm`; 0: none.
using Total = unsigned long long;
__device__ __forceinline__ Total total_of(float2 norm, float z) {
  const float2 s = add_pair(norm, z);
  return isfinite(s.x) ? (Total(order_of(s.x)) << 32) | order_of(s.y) : 0;
}
// Whether candidate i of total a goes before candidate j of total b: lists ascend in beam and slice, and in a list equal totals in
// their tokens, so places tell the order of equals. (No branches: 64 of them in a row are 4500 cycles.)
__device__ __forceinline__ int before(Total a, int i, Total b, int j) { return int(a > b) | (int(a == b) & int(i < j)); }

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const __grid_constant__ BeamArgs p) {
  constexpr int kFronts = kMaxBeams * (kMaxBeams + 1) / 2;
  __shared__ float2 norm[kMaxBeams];  // what a beam's logits are added to: score - log sum; NaN where it offers nothing
  __shared__ Total ends[kMaxBeams], head[kMostLists], front[kFronts], last_total;
  __shared__ int chosen[kMaxBeams], front_at[kFronts], front_token[kFronts], fronts, last_at;
  const int req = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lists = p.n_in * p.slices, K = p.n_out;
  int stages = 1;  // of a sum over the slices
  while (stages < p.slices && stages < 32) stages *= 2;
  if (tid == 0) {
    fronts = 0;
    last_total = 0;  // fewer lists than places: nothing is behind it
    last_at = 0x7fffffff;
  }
  pdl_launch_dependents();
  pdl_wait();
  const unsigned long long* best = p.best + size_t(req) * lists * K;
  const unsigned long long head_key = tid < lists ? best[size_t(tid) * K] : 0;  // on its way while the sums are added up
  for (int w = warp; w < p.n_in; w += kMergeThreads / 32) {
    const size_t row = size_t(req) * p.n_in + w;
    const float score = p.scores[row];
    const float end = p.eos >= 0 ? p.z[row * p.ld + p.eos] : -INFINITY;
    const float2* sums = p.sums + row * p.slices;
    const float2 mine = lane < p.slices ? sums[lane] : make_float2(-INFINITY, 0.0f);
    float m = mine.x;
    for (int i = lane + 32; i < p.slices; i += 32) m = fmaxf(m, sums[i].x);
    for (int off = stages / 2; off; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    auto part = [&](float2 s) { return s.x == -INFINITY ? s.y : s.y * expf(s.x - m); };
    float2 l = make_float2(part(mine), 0.0f);  // a sum, and what it was rounded by
    auto add = [&](float x, float y) {
      const float2 t = two_sum(l.x, x);
      l = make_float2(t.x, t.y + (l.y + y));
    };
    for (int i = lane + 32; i < p.slices; i += 32) add(part(sums[i]), 0.0f);
    for (int off = stages / 2; off; off >>= 1) add(__shfl_xor_sync(0xffffffffu, l.x, off), __shfl_xor_sync(0xffffffffu, l.y, off));
    if (lane == 0) {
      const float2 g = log_pair(l.x);
      float2 c = add_pair(two_sum(score, -m), -g.x);
      c = add_pair(c, -g.y - l.y / l.x);
      norm[w] = isfinite(c.x) && isfinite(c.y) ? c : make_float2(NAN, NAN);
      ends[w] = total_of(norm[w], end);
    }
  }
  __syncthreads();
  auto total_at = [&](int list, unsigned long long key) { return key ? total_of(norm[list / p.slices], key_value(key)) : 0; };
  // the n_out best heads
  if (tid < lists) head[tid] = total_at(tid, head_key);
  __syncthreads();
  if (tid < lists) {
    const Total mine = head[tid];
    int first = 0;
#pragma unroll 8
    for (int j = 0; j < lists; ++j) first += before(head[j], j, mine, tid);
    if (first < K) chosen[first] = tid;
    if (first == K - 1) {
      last_total = mine;
      last_at = tid * K;
    }
  }
  __syncthreads();
  // Their candidates, but for what goes behind the last of these heads. What is k-th of the list whose head is r-th has r + k before it.
  const Total last = last_total;
  const int behind = last_at;
  for (int x = tid; x < min(K, lists) * K; x += kMergeThreads) {
    const int r = x / K, k = x - r * K, list = chosen[r], i = list * K + k;
    if (r + k >= K) continue;
    const unsigned long long key = best[i];
    const Total c = total_at(list, key);
    if (c == 0 || before(last, behind, c, i)) continue;
    const int y = atomicAdd(&fronts, 1);
    front[y] = c;
    front_at[y] = i;
    front_token[y] = int(0xffffffffu - uint32_t(key));
  }
  __syncthreads();
  const int n = fronts;
  for (int i = tid; i < n; i += kMergeThreads) {
    const Total c = front[i];
    const int from = front_at[i];
    int first = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) first += before(front[j], front_at[j], c, from);
    if (first >= K) continue;
    const size_t at = size_t(req) * K + first;
    p.parent[at] = req * p.n_in + from / (p.slices * K);
    p.token[at] = front_token[i];
    p.out[at] = order_value(uint32_t(c >> 32));
  }
  for (int i = n + tid; i < K; i += kMergeThreads) {
    const size_t at = size_t(req) * K + i;
    p.parent[at] = p.token[at] = -1;
    p.out[at] = -INFINITY;
  }
  if (p.ended && tid >= kMergeThreads - p.n_in) {  // (other warps than those of the few fronts)
    const int w = tid - (kMergeThreads - p.n_in), own = p.slices * K;
    const Total e = ends[w];
    int first = 0;  // candidates that go before it: were they n_out in all, those of the fronts are as many
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const Total c = front[j];
      const int at = front_at[j];
      // of equal totals those of a lower beam, and of the beam's own the lower tokens
      first += int(c > e) | (int(c == e) & (int(at < w * own) | (int(at < (w + 1) * own) & int(front_token[j] < p.eos))));
    }
    for (int v = 0; v < p.n_in; ++v) first += before(ends[v], v, e, w);
    p.ended[size_t(req) * p.n_in + w] = e && first < K ? order_value(uint32_t(e >> 32)) : -INFINITY;
  }
}

// Slices a row: as many as fill the GPU (kCtasSm CTAs on each of 152 SMs), of a batch at least, kMostLists lists a request at most.
int slices_of(int n_seqs, int n_in, int vocab) {
  const int most = std::min((vocab + kBatch - 1) / kBatch, kMostLists / n_in);
  return std::max(1, std::min(most, kCtasSm * 152 / std::max(1, n_seqs * n_in)));
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" size_t spd_beam_select_workspace_size(int n_seqs, int n_in, int n_out, int vocab) {
  if (n_seqs < 1 || n_in < 1 || n_out < 1 || vocab < 1 || n_in > kMaxBeams || n_out > kMaxBeams) return 0;
  const size_t lists = size_t(n_seqs) * n_in * slices_of(n_seqs, n_in, vocab);
  Carve cv(nullptr, ~size_t(0));
  cv.take<unsigned long long>(lists * n_out);
  cv.take<float2>(lists);
  return cv.used;
}

extern "C" int spd_beam_select(const float* logits, int n_seqs, int n_in, int vocab, int ld, const float* scores, int n_out, int eos,
                               int32_t* parent, int32_t* token, float* scores_out, float* ended, void* ws, size_t ws_bytes,
                               void* stream) {
  if (!logits || !scores || !parent || !token || !scores_out || !ws || n_seqs < 1 || n_in < 1 || n_out < 1 || vocab < 1 || ld < vocab)
    return fail(SPD_EINVAL, "bad beam arguments");
  if (n_in > kMaxBeams || n_out > kMaxBeams) return fail(SPD_EUNSUPPORTED, "more than %d beams", kMaxBeams);
  if (vocab > 1 << 30) return fail(SPD_EUNSUPPORTED, "vocabulary of %d tokens", vocab);
  if ((long long)n_seqs * n_in > 65535) return fail(SPD_EUNSUPPORTED, "more than 65535 beams in all");
  if (eos < -1 || eos >= vocab) return fail(SPD_EINVAL, "eos outside the vocabulary (-1: none)");
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(SPD_EINVAL, "ws must be 16-byte aligned");
  BeamArgs p{};
  p.z = logits;
  p.vocab = vocab;
  p.ld = ld;
  p.n_in = n_in;
  p.n_out = n_out;
  p.slices = slices_of(n_seqs, n_in, vocab);
  p.slice = ((vocab + p.slices - 1) / p.slices + 3) & ~3;
  p.eos = eos;
  p.scores = scores;
  const size_t lists = size_t(n_seqs) * n_in * p.slices;
  Carve cv(ws, ws_bytes);
  p.best = cv.take<unsigned long long>(lists * n_out);
  p.sums = cv.take<float2>(lists);
  if (!cv.fits()) return fail(SPD_ENOSPC, "beam workspace too small (%zu < %zu)", ws_bytes, cv.used);
  if (scores_out == scores && n_in != n_out) return fail(SPD_EINVAL, "scores_out may be scores only where n_in is n_out");
  p.parent = parent;
  p.token = token;
  p.out = scores_out;
  p.ended = ended;
  p.status = cv.status();
  p.budget = kWaitBudget;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int slot = trace_begin(st);
  const bool vec = vocab % 4 == 0 && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(logits) & 15) == 0;
  constexpr int kRing = kStages * kBatch * 4;
  static DeviceOnce once;
  SPD_CUDA_TRY(once_per_device(once, [] {
    return cudaFuncSetAttribute(beam_slice_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
  }));
  SPD_CUDA_TRY(launch_pdl(vec ? beam_slice_kernel<4> : beam_slice_kernel<1>, dim3(p.slices, n_seqs * n_in), dim3(kThreads),
                          vec ? kRing : 0, st, p));
  SPD_CUDA_TRY(launch_pdl(beam_merge_kernel, dim3(n_seqs), dim3(kMergeThreads), 0, st, p));
  trace_end(slot, st, TR_ROWS, 0.0, 4.0 * n_seqs * n_in * double(vocab));
  return SPD_OK;
}
