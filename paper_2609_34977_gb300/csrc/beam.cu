// Beam search's selection: of every request's beams and their continuations the best, in one pass over the logits.
//
// total(w, t) = score_w + z_wt - log sum_u exp z_wu; the n_out largest over the live beams w and the tokens t other than `eos`,
// ties to the lower beam, then to the lower token. A beam's end, total(w, eos), counts where fewer than n_out candidates of
// the request, other ends among them, go before it.
//
// A row's tokens are split over CTAs (slices). Of one row the order of the totals is that of the logits, so of a slice only its
// n_out best can be among the request's best. A CTA streams its slice through registers: the maximum and the sum of
// exponentials a thread, and those tokens that beat the n_out-th best so far go to a list in shared memory, which is cut back to
// n_out when it has grown. The first bound: of n_out or more groups of threads the least of their maxima. Where more tokens beat
// the bound than the list holds (rising or equal logits) the batch's n_out best are taken one by one.
// A warp a request then takes the best of the lists' heads n_out times. Totals are fp64, the sums of the slices too: candidates
// of different beams may lie closer together than fp32 tells.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kHeld = 16;                  // tokens a thread holds
constexpr int kBatch = kThreads * kHeld;
constexpr int kMaxBeams = 32;
constexpr int kList = 512;                 // candidates a CTA holds
constexpr int kFull = 256;                 // cut back to n_out from here on
constexpr int kMergeThreads = 256;

struct BeamArgs {
  const float* z;
  int vocab, ld, n_in, n_out, slices, slice, eos;
  const float* scores;
  unsigned long long* best;  // [row][slice][n_out] order keys, descending, 0 behind the last
  float2* sums;              // [row][slice] maximum, sum of exp(z - maximum)
  int32_t *parent, *token;
  float *out, *ended;
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
// The sum of states (maximum, sum): NaN stays, -inf adds nothing.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);
  return make_float2(m, a.y * exp_less(a.x, m) + b.y * exp_less(b.x, m));
}

// W = 4: rows whose 16-byte pieces are aligned; 1: any.
template <int W>
__global__ void __launch_bounds__(kThreads, 4) beam_slice_kernel(const __grid_constant__ BeamArgs p) {
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
  float next[kHeld];
  auto load = [&](int base) {
#pragma unroll
    for (int k = 0; k < kHeld; k += W) {
      const int i = place(base, k);
      if constexpr (W == 4) {  // (slices are multiples of four)
        float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (i < n) v = __ldcs(reinterpret_cast<const float4*>(z + i));
        next[k] = v.x, next[k + 1] = v.y, next[k + 2] = v.z, next[k + 3] = v.w;
      } else {
        next[k] = i < n ? __ldcs(z + i) : -INFINITY;
      }
    }
  };
  load(0);
  float m = -INFINITY, s = 0.0f;   // of the thread's tokens
  float bound = -INFINITY;         // a token that is not above it is not among the best
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
    if (have == K) bound = key_value(top[K - 1]);
  };
  for (int base = 0, b = 0; base < n; base += kBatch, ++b) {
    float x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) x[k] = next[k];
    if (base + kBatch < n) load(base + kBatch);
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
    if (first) {  // the least of the maxima of 8 warps, or of 32 groups of eight threads
      float g = most;
#pragma unroll
      for (int off = 1; off < 8; off <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, off));
      if (K <= kWarps) {
#pragma unroll
        for (int off = 8; off < 32; off <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, off));
      }
      if ((lane & 7) == 0) group[tid >> 3] = g;
      __syncthreads();
      g = group[lane];
#pragma unroll
      for (int off = 16; off; off >>= 1) g = fminf(g, __shfl_xor_sync(0xffffffffu, g, off));
      bound = g;
    }
    if (most > bound || (first && most == bound && most > -INFINITY)) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (x[k] > bound || (first && x[k] == bound && x[k] > -INFINITY)) {
          const int at = have + atomicAdd(&pushed[b % 3], 1);
          if (at < kList) list[at] = order_key(x[k], t0 + place(base, k));
        }
      }
    }
    if (tid == 0) pushed[(b + 1) % 3] = 0;  // (read last before the barrier of the batch before)
    __syncthreads();
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
      if (have == K) bound = key_value(top[K - 1]);
    } else if (all > have) {
      if (first || all > kFull) {
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
}

// A candidate's order: its total, then the beam, then the token.
struct Candidate {
  uint32_t hi, lo;  // the total as an integer of the same order, 0: none
  uint32_t beam, token;
};
__device__ __forceinline__ void set_total(Candidate& c, double t) {
  const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(t + 0.0));
  const unsigned long long k = (u >> 63) ? ~u : u | (1ull << 63);
  c.hi = uint32_t(k >> 32);
  c.lo = uint32_t(k);
}
__device__ __forceinline__ double total_of(const Candidate& c) {
  const unsigned long long k = (static_cast<unsigned long long>(c.hi) << 32) | c.lo;
  return __longlong_as_double(static_cast<long long>((k >> 63) ? k & ~(1ull << 63) : ~k));
}
__device__ __forceinline__ bool none(const Candidate& c) { return (c.hi | c.lo) == 0; }
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) {
  if (a.hi != b.hi) return a.hi > b.hi;
  if (a.lo != b.lo) return a.lo > b.lo;
  return !none(a) && (a.beam != b.beam ? a.beam < b.beam : a.token < b.token);
}

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const __grid_constant__ BeamArgs p) {
  __shared__ double norm[kMaxBeams];  // what a beam's logits are added to: score - log sum; NaN where it offers nothing
  __shared__ Candidate got[kMaxBeams], ends[kMaxBeams];
  extern __shared__ unsigned long long keys[];  // [n_in * slices][n_out], then the heads of the lists
  const int req = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lists = p.n_in * p.slices, K = p.n_out;
  uint8_t* head = reinterpret_cast<uint8_t*>(keys + size_t(lists) * K);
  for (int i = tid; i < lists; i += kMergeThreads) head[i] = 0;
  pdl_launch_dependents();
  pdl_wait();
  const unsigned long long* best = p.best + size_t(req) * lists * K;
  for (int i = tid; i < lists * K; i += kMergeThreads) keys[i] = best[i];
  for (int w = warp; w < p.n_in; w += kMergeThreads / 32) {
    const size_t row = size_t(req) * p.n_in + w;
    const float score = p.scores[row];
    const float end = p.eos >= 0 ? p.z[row * p.ld + p.eos] : -INFINITY;
    const float2* sums = p.sums + row * p.slices;
    const float2 mine = lane < p.slices ? sums[lane] : make_float2(-INFINITY, 0.0f);
    float m = mine.x;
    for (int i = lane + 32; i < p.slices; i += 32) m = fmaxf(m, sums[i].x);
#pragma unroll
    for (int off = 16; off; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    auto part = [&](float2 s) { return s.x == -INFINITY ? double(s.y) : double(s.y) * double(expf(s.x - m)); };
    double l = part(mine);
    for (int i = lane + 32; i < p.slices; i += 32) l += part(sums[i]);
#pragma unroll
    for (int off = 16; off; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    const double c = double(score) - (double(m) + log(l));
    if (lane == 0) {
      norm[w] = isfinite(c) ? c : nan("");
      Candidate e{0u, 0u, uint32_t(w), uint32_t(p.eos)};
      if (isfinite(c) && end > -INFINITY) set_total(e, c + double(end));
      ends[w] = e;
    }
  }
  __syncthreads();
  if (warp > 0) return;
  Candidate mine;
  int from = 0;
  auto refresh = [&]() {  // the best head of the lane's lists
    mine = Candidate{0u, 0u, 0u, 0u};
    for (int i = lane; i < lists; i += 32) {
      const int w = i / p.slices, k = head[i];
      const unsigned long long key = k < K ? keys[i * K + k] : 0;
      if (key == 0 || isnan(norm[w])) continue;
      Candidate c{0u, 0u, uint32_t(w), 0xffffffffu - uint32_t(key)};
      set_total(c, norm[w] + double(key_value(key)));
      if (before(c, mine)) {
        mine = c;
        from = i;
      }
    }
  };
  refresh();
  for (int k = 0; k < K; ++k) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, mine.hi);
    bool in = mine.hi == hi;
    const uint32_t lo = __reduce_max_sync(0xffffffffu, in ? mine.lo : 0u);
    in &= mine.lo == lo;
    const uint32_t beam = __reduce_min_sync(0xffffffffu, in ? mine.beam : 0xffffffffu);
    in &= mine.beam == beam;
    const uint32_t token = __reduce_min_sync(0xffffffffu, in ? mine.token : 0xffffffffu);
    in &= mine.token == token;
    const bool any = (hi | lo) != 0;
    if (lane == 0) got[k] = Candidate{hi, lo, beam, token};
    if (any && in) {
      ++head[from];
      refresh();
    }
    __syncwarp();
  }
  for (int i = lane; i < K; i += 32) {
    const Candidate c = got[i];
    const size_t at = size_t(req) * K + i;
    p.parent[at] = none(c) ? -1 : req * p.n_in + int(c.beam);
    p.token[at] = none(c) ? -1 : int(c.token);
    p.out[at] = none(c) ? -INFINITY : float(total_of(c));
  }
  if (p.ended && lane < p.n_in) {
    const Candidate e = ends[lane];
    int ahead = 0;
    for (int k = 0; k < K; ++k) ahead += before(got[k], e);
    for (int w = 0; w < p.n_in; ++w) ahead += before(ends[w], e);
    p.ended[size_t(req) * p.n_in + lane] = !none(e) && ahead < K ? float(total_of(e)) : -INFINITY;
  }
}

// Slices a row: as many as fill the GPU (four CTAs on each of 152 SMs), of a batch at least.
int slices_of(int rows, int vocab) {
  const int most = (vocab + kBatch - 1) / kBatch;
  return std::max(1, std::min(most, 4 * 152 / std::max(1, rows)));
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" size_t spd_beam_select_workspace_size(int n_seqs, int n_in, int n_out, int vocab) {
  if (n_seqs < 1 || n_in < 1 || n_out < 1 || vocab < 1 || n_in > kMaxBeams || n_out > kMaxBeams) return 0;
  const size_t lists = size_t(n_seqs) * n_in * slices_of(n_seqs * n_in, vocab);
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
  if ((long long)n_seqs * n_in > 65535) return fail(SPD_EUNSUPPORTED, "more than 65535 beams in all");
  if (eos < -1 || eos >= vocab) return fail(SPD_EINVAL, "eos outside the vocabulary (-1: none)");
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(SPD_EINVAL, "ws must be 16-byte aligned");
  BeamArgs p{};
  p.z = logits;
  p.vocab = vocab;
  p.ld = ld;
  p.n_in = n_in;
  p.n_out = n_out;
  p.slices = slices_of(n_seqs * n_in, vocab);
  p.slice = ((vocab + p.slices - 1) / p.slices + 3) & ~3;
  p.eos = eos;
  p.scores = scores;
  const size_t lists = size_t(n_seqs) * n_in * p.slices;
  Carve cv(ws, ws_bytes);
  p.best = cv.take<unsigned long long>(lists * n_out);
  p.sums = cv.take<float2>(lists);
  if (!cv.fits()) return fail(SPD_ENOSPC, "beam workspace too small (%zu < %zu)", ws_bytes, cv.used);
  p.parent = parent;
  p.token = token;
  p.out = scores_out;
  p.ended = ended;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int slot = trace_begin(st);
  const bool vec = vocab % 4 == 0 && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(logits) & 15) == 0;
  const size_t smem = size_t(n_in) * p.slices * (8 * size_t(n_out) + 1);
  static DeviceOnce once;
  SPD_CUDA_TRY(once_per_device(once, [] {
    return cudaFuncSetAttribute(beam_merge_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  }));
  SPD_CUDA_TRY(launch_pdl(vec ? beam_slice_kernel<4> : beam_slice_kernel<1>, dim3(p.slices, n_seqs * n_in), dim3(kThreads), 0, st, p));
  SPD_CUDA_TRY(launch_pdl(beam_merge_kernel, dim3(n_seqs), dim3(kMergeThreads), smem, st, p));
  trace_end(slot, st, TR_ROWS, 0.0, 4.0 * n_seqs * n_in * double(vocab));
  return SPD_OK;
}
