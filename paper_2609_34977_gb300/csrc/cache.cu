// Keeping a KV cache within a budget: the eviction of the rows that receive least attention, and the move of an accepted
// path of drafts to the end of the context.
//
// Cache rows are [K of every K/V head | V of every K/V head], bf16, at row (layer * n_seqs + seq) * max_len + slot. A
// "unit" is one layer, sequence and K/V head: rows of a unit are evicted by the unit's own weights, so a slot holds
// different tokens in different units, and `pos` (int32 a unit and slot) says which.
#include <cooperative_groups.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <exception>
#include <vector>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

namespace cg = cooperative_groups;

// ---- eviction ------------------------------------------------------------------------------------
// Of a unit's n rows the `keep` best stay: those that `pos` protects (the first n_sink positions and the n_recent
// before next_pos), then by accumulated weight, the lower slot first among equals. Kept rows below slot `keep` stay
// where they are; the j-th kept row past it moves into the j-th hole. Sources and targets of the moves are disjoint,
// so they run in place, all at once, and a step that evicts a few rows of a long cache moves a few rows. (Closing the
// gaps in order would move every row behind the first hole.)
//
// Selection: the weights as order-preserving 32-bit keys in shared memory (a cluster of CTAs where a unit has more than
// one holds), the keep-th largest by a radix search of 11, 11 and 10 bits: the first digit, sign, exponent and two bits of
// the mantissa, spreads weights of any scale over enough counters that the additions do not queue, and the search ends as
// soon as a digit's keys are all kept, after two digits as a rule. (Counting the keys that reach three candidates a round, two
// bits at a time and without atomics, took 16 rounds of 1000 cycles, more than all the rest.)
// A CTA is one chain of loads, passes and prefix sums: units of up to kSelSmall slots get 512 threads where all of them are
// on the GPU at once (three an SM), 256 (six an SM) beyond. Whole calls, 256 / 512 / 1024 threads: 896 units of 1029 slots
// 14.3 / 17.9 / 26.8 us, 256 units of 3008 (of which the moves take 25) 50.5 / 44.2 / 44.0.
constexpr int kSelSmall = 4096;
constexpr int kSelWide = 1024;      // threads for longer ones
constexpr int kBins = 2048;
constexpr int kSelMost = 49152;     // keys a CTA holds (192 KB)
constexpr int kSelMaxCluster = 8;
// Units that lose few rows move them in the selecting kernel. 896 units that evict 7 / 32 / 64 / 256 rows of 1024, one
// launch and two: 14.5 and 17.4 / 19.3 and 23.0 / 25.8 and 28.2 / 49.7 and 48.9 us.
constexpr int kFusedMoves = 64;
constexpr int kMaxSeqs = 240;       // sequences whose sizes fit in a launch's parameters
constexpr uint32_t kHeld = 0xffffffffu;

struct EvictSeqs {  // by value in the launch's parameters: no copy, no wait for one
  int len[kMaxSeqs];
  int next_pos[kMaxSeqs];
};

struct EvictArgs {
  int n_seqs, seq0, launch_seqs, n_kv_heads, max_len, budget, n_sink, n_recent;
  const float* acc_in;
  const int32_t* pos_in;
  float* acc_out;
  int32_t* pos_out;
  int32_t* src;
  int32_t *fill, *hole, *moves;  // [unit][budget] x 2, [unit]
};

__device__ __forceinline__ uint32_t weight_key(float a) {
  if (isnan(a)) a = -INFINITY;
  const uint32_t u = __float_as_uint(a + 0.0f);  // -0 as 0
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// Exclusive prefix sum over the T threads of the block; *total the block's sum. tmp: T / 32 ints.
template <int T>
__device__ int block_before(int v, int* tmp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
  if (lane == 31) tmp[warp] = x;
  __syncthreads();
  int w = lane < T / 32 ? tmp[lane] : 0;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, off);
    if (lane >= off) w += y;
  }
  const int before = (warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0) + x - v;
  *total = __shfl_sync(0xffffffffu, w, 31);
  __syncthreads();
  return before;
}

// HD > 0: the kernel also moves the rows (a step's few), else evict_move_kernel does.
template <int T, int HD>
__global__ void __launch_bounds__(T, T == 256 ? 6 : T == 512 ? 3 : 1)
    evict_select_kernel(uint16_t* kv, const __grid_constant__ EvictArgs p, const __grid_constant__ EvictSeqs seqs, int per) {
  constexpr int kWarps = T / 32, kEach = kBins / T;  // counters a thread
  extern __shared__ uint32_t smem[];
  uint32_t* bins = smem;               // [2][kBins]
  uint32_t* key = smem + 2 * kBins;    // [per]: this CTA's slots
  __shared__ int tmp[kWarps];
  __shared__ int found[3];             // the digit, keys above it, keys with it
  __shared__ int ties_here, moves_here[2];
  __shared__ int list[2][kFusedMoves];
  cg::cluster_group cluster = cg::this_cluster();
  const int C = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per_layer = p.launch_seqs * p.n_kv_heads;
  const int local = int(blockIdx.x) / C, layer = local / per_layer, at = local - layer * per_layer;
  const int ls = at / p.n_kv_heads, g = at - ls * p.n_kv_heads;
  const size_t unit = (size_t(layer) * p.n_seqs + p.seq0 + ls) * p.n_kv_heads + g;
  const int n = seqs.len[ls], keep = min(n, p.budget), next = seqs.next_pos[ls];
  auto meet = [&]() {
    if (C > 1) cluster.sync();
    else __syncthreads();
  };
  pdl_launch_dependents();
  pdl_wait();
  const float* acc = p.acc_in + unit * p.max_len;
  const int32_t* pos = p.pos_in ? p.pos_in + unit * p.max_len : nullptr;
  float* acc_out = p.acc_out + unit * p.max_len;
  int32_t* pos_out = p.pos_out ? p.pos_out + unit * p.max_len : nullptr;
  int32_t* src = p.src ? p.src + unit * p.budget : nullptr;
  const int lo = min(n, rank * per), cnt = min(n, lo + per) - lo;  // this CTA's slots
  if (n <= p.budget) {  // nothing leaves (every CTA of the cluster agrees)
    for (int i = tid; i < cnt; i += T) {
      acc_out[lo + i] = acc[lo + i];
      if (pos_out) pos_out[lo + i] = pos ? pos[lo + i] : lo + i;
      if (src) src[lo + i] = lo + i;
    }
    if (HD == 0 && rank == 0 && tid == 0) p.moves[unit] = 0;
    return;
  }
  for (int i = tid; i < 2 * kBins; i += T) bins[i] = 0;
#pragma unroll 4
  for (int i = tid; i < cnt; i += T) {
    const int q = pos ? pos[lo + i] : lo + i;
    const float a = acc[lo + i];
    key[i] = q < p.n_sink || q >= next - p.n_recent ? kHeld : weight_key(a);
  }
  __syncthreads();
  // the keep-th largest key: thr, and how many of its equals stay (the lowest slots)
  uint32_t thr = 0;
  int need = keep, equal = n;
  for (int pass = 0, shift = 21; pass < 3 && equal != need; ++pass) {
    const int width = pass < 2 ? 11 : 10;
    uint32_t* bin = bins + (pass & 1) * kBins;
    for (int i = tid; i < cnt; i += T)
      if (pass == 0 || (key[i] >> (shift + width)) == (thr >> (shift + width)))
        atomicAdd(&bin[(key[i] >> shift) & ((1u << width) - 1)], 1u);
    meet();
    // counters from the largest digit down: thread t has kEach of them
    const int top = kBins - kEach * (tid + 1);
    uint32_t here[kEach] = {};
    for (int c = 0; c < C; ++c) {
      const uint32_t* b = C > 1 ? cluster.map_shared_rank(bin, c) : bin;
#pragma unroll
      for (int u = 0; u < kEach; ++u) here[u] += b[top + u];
    }
    if (pass > 0)  // the counters of the pass before, which nobody reads any more
      for (int i = tid; i < kBins; i += T) bins[((pass & 1) ^ 1) * kBins + i] = 0;
    int sum = 0, all;
#pragma unroll
    for (int u = 0; u < kEach; ++u) sum += int(here[u]);
    int above = block_before<T>(sum, tmp, &all);
    if (above < need && need <= above + sum) {
#pragma unroll
      for (int u = kEach - 1; u >= 0; --u) {
        if (above < need && need <= above + int(here[u])) {
          found[0] = top + u;
          found[1] = above;
          found[2] = int(here[u]);
        }
        above += int(here[u]);
      }
    }
    __syncthreads();
    thr |= uint32_t(found[0]) << shift;
    need -= found[1];
    equal = found[2];
    shift -= pass == 0 ? 11 : 10;
    __syncthreads();  // found has been read
  }
  // kept: key > thr's digits, and of those with thr's digits the first `need` by slot (all of them where equal == need). A
  // thread's slots are consecutive, so that prefix sums run in slot order.
  const int each = (per + T - 1) / T;
  const int i0 = min(cnt, tid * each), i1 = min(cnt, i0 + each);
  const bool split = equal != need;  // only after the last pass: thr is a whole key
  int ties = 0;
  if (split) {
    for (int i = i0; i < i1; ++i) ties += key[i] == thr;
    int all;
    ties = block_before<T>(ties, tmp, &all);
    if (tid == 0) ties_here = all;
    meet();
    for (int c = 0; c < rank; ++c) ties += *cluster.map_shared_rank(&ties_here, c);
  }
  int both = 0;  // holes in the low half, fills in the high half
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key[i];
    const bool kept = split ? k > thr || (k == thr && ties++ < need) : k >= thr;
    both += lo + i < keep ? !kept : int(kept) << 16;
    key[i] = kept;  // from here on
  }
  int total;
  both = block_before<T>(both, tmp, &total);
  int hole_at = both & 0xffff, fill_at = int(uint32_t(both) >> 16), moves = total & 0xffff;
  if (C > 1) {
    if (tid == 0) {
      moves_here[0] = total & 0xffff;
      moves_here[1] = int(uint32_t(total) >> 16);
    }
    cluster.sync();
    moves = 0;
    for (int c = 0; c < C; ++c) {
      const int* q = cluster.map_shared_rank(moves_here, c);
      moves += q[0];
      if (c < rank) {
        hole_at += q[0];
        fill_at += q[1];
      }
    }
  }
  // the lists; a CTA on its own with few moves keeps them to itself
  const bool in_smem = HD > 0 && C == 1;
  int32_t *fill = in_smem ? list[0] : p.fill + unit * p.budget, *hole = in_smem ? list[1] : p.hole + unit * p.budget;
  if (moves > 0)
    for (int i = i0; i < i1; ++i) {
      const int s = lo + i;
      if (s < keep && !key[i]) hole[hole_at++] = s;
      if (s >= keep && key[i]) fill[fill_at++] = s;
    }
  if (!in_smem) __threadfence();  // for the other CTAs of the cluster
  meet();
  if constexpr (HD > 0) {
    // a warp a move, 16 bytes a lane: K's row, V's row (HD = 64: in half of the lanes)
    constexpr int VEC = HD / 8;
    const int kvd = p.n_kv_heads * HD, col = (lane / VEC) * kvd + g * HD + (lane % VEC) * 8;
    uint16_t* base = kv + (unit / p.n_kv_heads) * p.max_len * (2 * size_t(kvd)) + col;
    for (int j = rank * kWarps + warp; j < moves; j += C * kWarps) {
      const int s = *(volatile int32_t*)(hole + j), f = *(volatile int32_t*)(fill + j);
      if (lane < 2 * VEC)
        *reinterpret_cast<uint4*>(base + size_t(s) * (2 * kvd)) = *reinterpret_cast<const uint4*>(base + size_t(f) * (2 * kvd));
    }
  } else {
    if (rank == 0 && tid == 0) p.moves[unit] = moves;
  }
  // rows that stay in their slots (four of a thread's in flight)
  const int stay = min(cnt, keep - lo);
  for (int i = tid; i < stay; i += 4 * T) {
    float a[4];
    int q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = i + u * T;
      if (x < stay && key[x]) {
        a[u] = acc[lo + x];
        q[u] = pos ? pos[lo + x] : lo + x;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = i + u * T;
      if (x < stay && key[x]) {
        acc_out[lo + x] = a[u];
        if (pos_out) pos_out[lo + x] = q[u];
        if (src) src[lo + x] = lo + x;
      }
    }
  }
  for (int j = rank * T + tid; j < moves; j += C * T) {
    const int s = *(volatile int32_t*)(hole + j), f = *(volatile int32_t*)(fill + j);
    acc_out[s] = acc[f];
    if (pos_out) pos_out[s] = pos ? pos[f] : f;
    if (src) src[s] = f;
  }
  meet();  // before the slots past the budget are cleared, which may be the ones read above
  for (int s = keep + rank * T + tid; s < n; s += C * T) {
    acc_out[s] = 0.0f;
    if (pos_out) pos_out[s] = -1;
  }
}

using SelectKernel = void (*)(uint16_t*, EvictArgs, EvictSeqs, int);
template <int T>
SelectKernel pick_select(int move) {
  return move == 128 ? evict_select_kernel<T, 128> : move == 64 ? evict_select_kernel<T, 64> : evict_select_kernel<T, 0>;
}

// The rows themselves: a warp a move, 16 bytes a lane (half a warp K, half V; HD = 64: a quarter each), four moves in
// flight a warp; `ctas` CTAs a unit, side by side. HBM: 175 K moves of 1 KB (read and written) in 25 us, 7.1 TB/s. Moving
// inside the selecting kernel saves a launch and loses the occupancy: 46.8 against 44.1 us for the whole call.
constexpr int kMoveWarps = 8, kMoveDepth = 4;
template <int HD>
__global__ void __launch_bounds__(kMoveWarps * 32) evict_move_kernel(uint16_t* kv, const __grid_constant__ EvictArgs p, int ctas) {
  constexpr int VEC = HD / 8;  // 16-byte pieces of a head's K or V row
  constexpr int ROWS = 32 / (2 * VEC);  // moves a warp takes at once
  pdl_launch_dependents();
  pdl_wait();
  const int local = int(blockIdx.x / uint32_t(ctas)), per_layer = p.launch_seqs * p.n_kv_heads, layer = local / per_layer;
  const int at = local - layer * per_layer, ls = at / p.n_kv_heads, g = at - ls * p.n_kv_heads;
  const size_t seq = size_t(layer) * p.n_seqs + p.seq0 + ls, unit = seq * p.n_kv_heads + g;
  const int moves = p.moves[unit];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = lane / (2 * VEC), e = lane % (2 * VEC), kvd = p.n_kv_heads * HD;
  const int col = (e / VEC) * kvd + g * HD + (e % VEC) * 8;
  uint16_t* base = kv + seq * p.max_len * (2 * size_t(kvd)) + col;
  const int32_t *fill = p.fill + unit * p.budget, *hole = p.hole + unit * p.budget;
  const int j0 = (int(blockIdx.x - uint32_t(local) * ctas) * kMoveWarps + warp) * (kMoveDepth * ROWS) + sub;
  uint4 v[kMoveDepth];
#pragma unroll
  for (int u = 0; u < kMoveDepth; ++u)
    if (j0 + u * ROWS < moves)
      v[u] = *reinterpret_cast<const uint4*>(base + size_t(fill[j0 + u * ROWS]) * (2 * kvd));
#pragma unroll
  for (int u = 0; u < kMoveDepth; ++u)
    if (j0 + u * ROWS < moves) *reinterpret_cast<uint4*>(base + size_t(hole[j0 + u * ROWS]) * (2 * kvd)) = v[u];
}

// ---- commit ----------------------------------------------------------------------------------------
// Sequence b's accepted drafts path[cu[b] .. cu[b + 1]) (ascending node numbers) move from slots ctx + node to slots
// ctx, ctx + 1, ... of every layer. A target is at or before its source and before every later source, so one thread
// that walks a column of the row through the path in order needs no second buffer.
struct CommitArgs {
  int n_seqs, max_len, row16;  // row16: 16-byte pieces of a cache row
  int n_kv_heads;
  const int32_t *path, *cu, *ctx, *pos0;
  int32_t* pos;                // [unit][max_len] or null
  float* acc;                  // [unit][max_len] or null
};
__global__ void __launch_bounds__(256) commit_kernel(uint4* kv, const __grid_constant__ CommitArgs p) {
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.y, layer = blockIdx.z;
  const int c0 = p.cu[b], n = p.cu[b + 1] - c0, ctx = p.ctx[b];
  const size_t seq = size_t(layer) * p.n_seqs + b;
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col < p.row16) {
    uint4* base = kv + (seq * p.max_len + ctx) * p.row16 + col;
    for (int i0 = 0; i0 < n; i0 += 8) {  // eight rows in flight: later targets lie before their sources
      uint4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u < n) v[u] = base[size_t(p.path[c0 + i0 + u]) * p.row16];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u < n && p.path[c0 + i0 + u] != i0 + u) base[size_t(i0 + u) * p.row16] = v[u];
    }
  }
  if (blockIdx.x == 0) {
    for (int e = threadIdx.x; e < n * p.n_kv_heads; e += 256) {
      const size_t at = (seq * p.n_kv_heads + e / n) * p.max_len + ctx + e % n;
      if (p.pos) p.pos[at] = p.pos0[b] + e % n;
      if (p.acc) p.acc[at] = 0.0f;
    }
  }
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" size_t spd_cache_evict_workspace_size(int n_layers, int n_seqs, int n_kv_heads, int budget) {
  if (n_layers < 1 || n_seqs < 1 || n_kv_heads < 1 || budget < 1) return 0;
  const size_t units = size_t(n_layers) * n_seqs * n_kv_heads;
  Carve cv(nullptr, ~size_t(0));
  cv.take<int32_t>(units * budget);
  cv.take<int32_t>(units * budget);
  cv.take<int32_t>(units);
  return cv.used;
}

extern "C" int spd_cache_evict(uint16_t* kv_cache, int n_layers, int n_seqs, const int32_t* lens, int max_len,
                               int n_kv_heads, int head_dim, int budget, int n_sink, int n_recent,
                               const int32_t* next_pos, const float* acc_in, const int32_t* pos_in, float* acc_out,
                               int32_t* pos_out, int32_t* src, void* ws, size_t ws_bytes, void* stream) {
  if (!kv_cache || !lens || !acc_in || !acc_out || !ws || n_layers < 1 || n_seqs < 1 || n_kv_heads < 1 || max_len < 1 ||
      budget < 1 || n_sink < 0 || n_recent < 0)
    return fail(SPD_EINVAL, "bad eviction arguments");
  if (head_dim != 64 && head_dim != 128) return fail(SPD_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (pos_in && !next_pos) return fail(SPD_EINVAL, "positions need next_pos");
  if (pos_in && !pos_out) return fail(SPD_EINVAL, "positions need pos_out");
  if ((reinterpret_cast<uintptr_t>(kv_cache) | reinterpret_cast<uintptr_t>(ws)) & 15)
    return fail(SPD_EINVAL, "the cache and ws must be 16-byte aligned");
  int longest = 0, most_moves = 0;
  for (int b = 0; b < n_seqs; ++b) {
    if (lens[b] < 0 || lens[b] > max_len) return fail(SPD_EINVAL, "length of sequence %d outside [0, max_len]", b);
    if (lens[b] > budget) {
      longest = std::max(longest, lens[b]);
      most_moves = std::max(most_moves, std::min(budget, lens[b] - budget));
    }
  }
  if (longest > kSelMost * kSelMaxCluster)
    return fail(SPD_EUNSUPPORTED, "eviction from more than %d rows", kSelMost * kSelMaxCluster);
  const size_t units = size_t(n_layers) * n_seqs * n_kv_heads;
  Carve cv(ws, ws_bytes);
  EvictArgs p{};
  p.fill = cv.take<int32_t>(units * budget);
  p.hole = cv.take<int32_t>(units * budget);
  p.moves = cv.take<int32_t>(units);
  if (!cv.fits()) return fail(SPD_ENOSPC, "eviction workspace too small (%zu < %zu)", ws_bytes, cv.used);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  p.n_seqs = n_seqs;
  p.n_kv_heads = n_kv_heads;
  p.max_len = max_len;
  p.budget = budget;
  p.n_sink = n_sink;
  p.n_recent = n_recent;
  p.acc_in = acc_in;
  p.pos_in = pos_in;
  p.acc_out = acc_out;
  p.pos_out = pos_out;
  p.src = src;
  int C = 1;
  // more CTAs a unit where one would hold over 16384 keys, and over 8192 while a quarter of the SMs stay idle (clusters do
  // not find room on all). 112 units of 16384 slots with 1 / 2 / 4: 30.1 / 35.1 / 49.6 us; 16 units of 32768: 74 / 32.3 / 21.5; 16 of 12000: 14.6 /
  // 13.9 / 20.7; 16 of 65521 with 4 / 8: 50 / 68
  while (C < kSelMaxCluster && (longest > 16384 * C || (longest > 8192 * C && 4 * units * 2 * C <= 3 * size_t(num_sms())))) C *= 2;
  int per = (std::max(longest, 1) + C - 1) / C;
  for (int b = 0; b < n_seqs; ++b) per = std::max(per, (std::min(lens[b], budget) + C - 1) / C);
  per = (per + 3) & ~3;
  // moves that the selecting CTA makes itself: where a unit has few of them, the second launch costs more
  const bool fused = most_moves <= kFusedMoves, small = per <= kSelSmall;
  const int rows_cta = kMoveWarps * kMoveDepth * (128 / head_dim), ctas = (most_moves + rows_cta - 1) / rows_cta;
  if (units * std::max(C, ctas) > 0x7fffffff)
    return fail(SPD_EUNSUPPORTED, "eviction from %zu layers x sequences x K/V heads of up to %d rows", units, longest);
  const int threads = !small ? kSelWide : units * C > 3 * size_t(num_sms()) ? 256 : 512;
  const int move = fused ? head_dim : 0;
  const auto select = threads == 256   ? pick_select<256>(move)
                      : threads == 512 ? pick_select<512>(move)
                                       : pick_select<kSelWide>(move);
  if (!small) SPD_CUDA_TRY(cudaFuncSetAttribute(select, cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * kBins + 4 * kSelMost));
  const size_t smem = longest ? 8 * size_t(kBins) + 4 * size_t(per) : 16;
  for (int s0 = 0; s0 < n_seqs; s0 += kMaxSeqs) {
    EvictSeqs sq;
    p.seq0 = s0;
    p.launch_seqs = std::min(kMaxSeqs, n_seqs - s0);
    double rows = 0.0, moved = 0.0;
    for (int b = 0; b < p.launch_seqs; ++b) {
      sq.len[b] = lens[s0 + b];
      sq.next_pos[b] = next_pos ? next_pos[s0 + b] : lens[s0 + b];
      rows += lens[s0 + b];
      if (lens[s0 + b] > budget) moved += std::min(budget, lens[s0 + b] - budget);
    }
    const int n = n_layers * p.launch_seqs * n_kv_heads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n * C);
    cfg.blockDim = dim3(threads);
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
    cfg.numAttrs = 2;
    int slot = trace_begin(st);
    SPD_CUDA_TRY(cudaLaunchKernelEx(&cfg, select, kv_cache, p, sq, per));
    trace_end(slot, st, TR_ROWS, 0.0, 16.0 * rows * n_layers * n_kv_heads);
    if (!fused) {
      slot = trace_begin(st);
      SPD_CUDA_TRY(launch_pdl(head_dim == 128 ? evict_move_kernel<128> : evict_move_kernel<64>, dim3(unsigned(n) * ctas),
                              dim3(kMoveWarps * 32), 0, st, kv_cache, p, ctas));
      trace_end(slot, st, TR_ROWS, 0.0, 8.0 * head_dim * moved * n_layers * n_kv_heads);
    }
  }
  return SPD_OK;
}

extern "C" size_t spd_tree_commit_workspace_size(int n_seqs, int n_path) {
  if (n_seqs < 1 || n_path < 0) return 0;
  Carve cv(nullptr, ~size_t(0));
  cv.take<int32_t>(size_t(n_path) + 3 * size_t(n_seqs) + 1);
  return cv.used;
}

extern "C" int spd_tree_commit(uint16_t* kv_cache, int n_layers, int n_seqs, const int32_t* path, const int32_t* path_cu,
                               const int32_t* ctx_len, int max_len, int n_kv_heads, int head_dim, const int32_t* next_pos,
                               int32_t* pos, float* acc, void* ws, size_t ws_bytes, void* stream) try {
  if (!kv_cache || !path_cu || !ctx_len || !ws || n_layers < 1 || n_seqs < 1 || max_len < 1 || n_kv_heads < 1)
    return fail(SPD_EINVAL, "bad commit arguments");
  if (head_dim != 64 && head_dim != 128) return fail(SPD_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (pos && !next_pos) return fail(SPD_EINVAL, "positions need next_pos");
  if ((reinterpret_cast<uintptr_t>(kv_cache) | reinterpret_cast<uintptr_t>(ws)) & 15)
    return fail(SPD_EINVAL, "the cache and ws must be 16-byte aligned");
  if (n_seqs > 65535 || n_layers > 65535) return fail(SPD_EUNSUPPORTED, "more than 65535 sequences or layers");
  if (path_cu[0] != 0) return fail(SPD_EINVAL, "path_cu must start at 0");
  for (int b = 0; b < n_seqs; ++b)
    if (path_cu[b + 1] < path_cu[b]) return fail(SPD_EINVAL, "path_cu decreases at sequence %d", b);
  for (int b = 0; b < n_seqs; ++b) {  // (path holds path_cu[n_seqs] entries, which no range passes now)
    if (ctx_len[b] < 0 || ctx_len[b] > max_len) return fail(SPD_EINVAL, "context of sequence %d outside [0, max_len]", b);
    for (int i = path_cu[b]; i < path_cu[b + 1]; ++i) {
      if (!path) return fail(SPD_EINVAL, "null path");
      if (path[i] < (i > path_cu[b] ? path[i - 1] + 1 : 0) || path[i] >= max_len - ctx_len[b])
        return fail(SPD_EINVAL, "sequence %d: path nodes must ascend within the cache slot", b);
    }
  }
  const int n_path = path_cu[n_seqs];
  if (n_path == 0) return SPD_OK;
  Carve cv(ws, ws_bytes);
  const size_t ints = size_t(n_path) + 3 * size_t(n_seqs) + 1;
  int32_t* d = cv.take<int32_t>(ints);
  if (!cv.fits()) return fail(SPD_ENOSPC, "commit workspace too small (%zu < %zu)", ws_bytes, cv.used);
  static thread_local std::vector<int32_t> host;
  host.resize(ints);
  memcpy(host.data(), path, n_path * 4);
  memcpy(host.data() + n_path, path_cu, (n_seqs + 1) * 4);
  memcpy(host.data() + n_path + n_seqs + 1, ctx_len, n_seqs * 4);
  for (int b = 0; b < n_seqs; ++b) host[n_path + 2 * n_seqs + 1 + b] = next_pos ? next_pos[b] : 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  SPD_CUDA_TRY(cudaMemcpyAsync(d, host.data(), ints * 4, cudaMemcpyHostToDevice, st));
  CommitArgs p{};
  p.n_seqs = n_seqs;
  p.max_len = max_len;
  p.row16 = n_kv_heads * head_dim / 4;
  p.n_kv_heads = n_kv_heads;
  p.path = d;
  p.cu = d + n_path;
  p.ctx = d + n_path + n_seqs + 1;
  p.pos0 = d + n_path + 2 * n_seqs + 1;
  p.pos = pos;
  p.acc = acc;
  const int slot = trace_begin(st);
  SPD_CUDA_TRY(launch_pdl(commit_kernel, dim3((p.row16 + 255) / 256, n_seqs, n_layers), dim3(256), 0, st,
                          reinterpret_cast<uint4*>(kv_cache), p));
  trace_end(slot, st, TR_ROWS, 0.0, 32.0 * p.row16 * n_path * n_layers);
  return SPD_OK;
} catch (const std::exception&) {  // the host list
  return fail(SPD_EUNSUPPORTED, "commit: out of host memory");
}
