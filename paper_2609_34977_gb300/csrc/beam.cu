// Beam search's selection: of every request's beams and their continuations the best, in one pass over the logits.
//
// total(w, t) = score_w + z_wt - log sum_u exp z_wu; the n_out largest over the live beams w and the tokens t other than `eos`,
// ties to the lower beam, then to the lower token. A beam's end, total(w, eos), counts where fewer than n_out candidates of
// the request, other ends among them, go before it.
//
// A row's tokens are split over CTAs. Each finds its slice's maximum, sum of exponentials and n_out best tokens (of one row
// the order of the totals is that of the logits, so nothing else can be among the request's best), in registers by n_out
// rounds of a maximum over the block. A CTA a request then adds the sums up in fp64, in the order of the slices, and takes
// the best of the lists' heads n_out times. Totals are fp64: candidates of different beams may lie closer together than fp32 tells.
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
constexpr int kMergeThreads = 512;

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

__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    const unsigned long long y = __shfl_xor_sync(0xffffffffu, k, off);
    k = y > k ? y : k;
  }
  return k;
}

// The sum of states (maximum, sum): NaN stays, -inf adds nothing.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);
  return make_float2(m, a.y * expf(a.x - m) + b.y * expf(b.x - m));
}

__global__ void __launch_bounds__(kThreads) beam_slice_kernel(const __grid_constant__ BeamArgs p) {
  __shared__ unsigned long long wbest[2][kWarps], top[kMaxBeams];
  __shared__ float2 wsum[kWarps];
  const int row = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t0 = blockIdx.x * p.slice, n = max(0, min(p.slice, p.vocab - t0));
  pdl_launch_dependents();
  pdl_wait();
  const float* z = p.z + size_t(row) * p.ld + t0;
  if (tid < kMaxBeams) top[tid] = 0;
  float2 sum = make_float2(-INFINITY, 0.0f);
  for (int base = 0; base < n; base += kBatch) {
    float x[kHeld];
    unsigned long long mine[kHeld], most = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const int i = base + k * kThreads + tid;
      x[k] = i < n ? z[i] : -INFINITY;
      mine[k] = i < n && x[k] > -INFINITY && t0 + i != p.eos ? order_key(x[k], t0 + i) : 0;
      most = mine[k] > most ? mine[k] : most;
    }
    float m = sum.x;
    bool odd = false;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      m = fmaxf(m, x[k]);
      odd |= isnan(x[k]);
    }
    if (m > -INFINITY) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) s += expf(x[k] - m);
      sum = make_float2(m, sum.y * expf(sum.x - m) + s);
    }
    if (odd) sum.y = NAN;
    __syncthreads();
    // the best of the list so far and of this batch: the k-th largest of both in round k
    unsigned long long old = tid < p.n_out ? top[tid] : 0;
    for (int k = 0; k < p.n_out; ++k) {
      const unsigned long long c = warp_max(most > old ? most : old);
      if (lane == 0) wbest[k & 1][warp] = c;
      __syncthreads();
      unsigned long long b = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) b = wbest[k & 1][w] > b ? wbest[k & 1][w] : b;
      if (tid == 0) top[k] = b;
      if (b == 0) continue;
      if (old == b) old = 0;
      if (most == b) {
        most = 0;
#pragma unroll
        for (int e = 0; e < kHeld; ++e) {
          if (mine[e] == b) mine[e] = 0;
          most = mine[e] > most ? mine[e] : most;
        }
      }
    }
    __syncthreads();
  }
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
  if (tid < p.n_out) p.best[at * p.n_out + tid] = top[tid];
}

struct Candidate {
  double total;
  unsigned long long at;  // beam and token, ~0: none
};
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) {
  return a.at != ~0ull && (b.at == ~0ull || a.total > b.total || (a.total == b.total && a.at < b.at));
}

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const __grid_constant__ BeamArgs p) {
  __shared__ double norm[kMaxBeams];    // what a beam's logits are added to: score - log sum; NaN where it offers nothing
  __shared__ Candidate wbest[2][kMergeThreads / 32], got[kMaxBeams], ends[kMaxBeams];
  extern __shared__ uint16_t next[];  // [n_in * slices] heads of the lists
  const int req = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lists = p.n_in * p.slices;
  pdl_launch_dependents();
  pdl_wait();
  for (int w = warp; w < p.n_in; w += kMergeThreads / 32) {
    const float2* s = p.sums + (size_t(req) * p.n_in + w) * p.slices;
    float m = -INFINITY;
    for (int i = lane; i < p.slices; i += 32) m = fmaxf(m, s[i].x);
#pragma unroll
    for (int off = 16; off; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    double l = 0.0;
    for (int i = lane; i < p.slices; i += 32) l += s[i].x == -INFINITY ? double(s[i].y) : double(s[i].y) * exp(double(s[i].x) - double(m));
#pragma unroll
    for (int off = 16; off; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    const float score = p.scores[size_t(req) * p.n_in + w];
    const double c = double(score) - (double(m) + log(l));
    if (lane == 0) {
      norm[w] = isfinite(c) ? c : nan("");
      Candidate e{0.0, ~0ull};
      if (unsigned(p.eos) < unsigned(p.vocab)) {
        const float z = p.z[(size_t(req) * p.n_in + w) * p.ld + p.eos];
        if (isfinite(c) && z > -INFINITY) e = {c + double(z), size_t(w) * p.vocab + p.eos};
      }
      ends[w] = e;
    }
  }
  for (int i = tid; i < lists; i += kMergeThreads) next[i] = 0;
  __syncthreads();
  const unsigned long long* best = p.best + size_t(req) * lists * p.n_out;
  auto head = [&](int i) {
    const int w = i / p.slices, k = next[i];
    const unsigned long long key = k < p.n_out ? best[size_t(i) * p.n_out + k] : 0;
    if (key == 0 || isnan(norm[w])) return Candidate{0.0, ~0ull};
    const uint32_t u = uint32_t(key >> 32);
    const float z = __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
    return Candidate{norm[w] + double(z), size_t(w) * p.vocab + (0xffffffffu - uint32_t(key))};
  };
  Candidate mine{0.0, ~0ull};
  int from = -1;
  auto refresh = [&]() {
    mine.at = ~0ull;
    for (int i = tid; i < lists; i += kMergeThreads) {
      const Candidate c = head(i);
      if (before(c, mine)) {
        mine = c;
        from = i;
      }
    }
  };
  refresh();
  for (int k = 0; k < p.n_out; ++k) {
    Candidate c = mine;
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      const Candidate d{__shfl_xor_sync(0xffffffffu, c.total, off), __shfl_xor_sync(0xffffffffu, c.at, off)};
      if (before(d, c)) c = d;
    }
    if (lane == 0) wbest[k & 1][warp] = c;
    __syncthreads();
    c = wbest[k & 1][0];
    for (int w = 1; w < kMergeThreads / 32; ++w)
      if (before(wbest[k & 1][w], c)) c = wbest[k & 1][w];
    if (tid == 0) got[k] = c;
    if (c.at != ~0ull && c.at == mine.at) {
      ++next[from];
      refresh();
    }
  }
  __syncthreads();
  if (tid < p.n_out) {
    const Candidate c = got[tid];
    const size_t at = size_t(req) * p.n_out + tid;
    p.parent[at] = c.at == ~0ull ? -1 : req * p.n_in + int(c.at / p.vocab);
    p.token[at] = c.at == ~0ull ? -1 : int(c.at % p.vocab);
    p.out[at] = c.at == ~0ull ? -INFINITY : float(c.total);
  }
  if (p.ended && tid < p.n_in) {
    const Candidate e = ends[tid];
    int ahead = 0;
    for (int k = 0; k < p.n_out; ++k) ahead += before(got[k], e);
    for (int w = 0; w < p.n_in; ++w) ahead += before(ends[w], e);
    p.ended[size_t(req) * p.n_in + tid] = e.at != ~0ull && ahead < p.n_out ? float(e.total) : -INFINITY;
  }
}

// Slices a row: as many as fill the GPU, of a batch at least.
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
  SPD_CUDA_TRY(launch_pdl(beam_slice_kernel, dim3(p.slices, n_seqs * n_in), dim3(kThreads), 0, st, p));
  SPD_CUDA_TRY(launch_pdl(beam_merge_kernel, dim3(n_seqs), dim3(kMergeThreads), size_t(n_in) * p.slices * 2, st, p));
  trace_end(slot, st, TR_ROWS, 0.0, 4.0 * n_seqs * n_in * double(vocab));
  return SPD_OK;
}
