// The attention weight that cached rows receive, on the tcgen05 tensor cores.
//
// For slot k of a unit (layer, sequence, K/V head g) and the sequence's n rows i with the heads h of g's group:
//   acc_out[k] = decay acc_in[k] + sum_ih exp(q_ih . k / sqrt(head_dim) - lse_ih)      (k visible to row i)
// The normalisers are known, so nothing has to be carried from key to key and V is not read: the call is one pass over K
// (2 head_dim bytes a slot and K/V head) and one exponential a (slot, row, head).
//
// The product is taken the other way round than in attention: S^T = K Q^T with 128 keys as the MMA's M and up to 64 (row,
// head) pairs as its N. A thread then owns a key (TMEM lane), its sum over the rows stays in its registers, and a
// decode step's few rows cost few columns instead of 128 mostly empty rows. More than 128 pairs take further passes over the
// item's keys (from L2), added in order by the same thread. Sums have a fixed order: the same bits in every run.
//
// A weight is as exact as its exponent, which can be large where lse is another step's: the two halves of a head have
// accumulators of their own (a chain over the whole head loses low bits in the tensor pipe), and they and the constants' low
// parts are added to -lse, not to each other. Against 64 bits 1.0e-7 to 1.7e-6 of the result, 0.4 to 1.6 (once 2.2) times an
// fp32 computation's error; one chain and one constant 1.0 to 3.1 times, for 3 to 4 % less time.
//   warp 4  TMA producer: blocks of 128 keys into a ring;  warp 5  MMA issuer, TMEM double-buffered
//   warps 0-3  Q tile and normalisers of the pass to shared memory, then a key a thread
//
// What bounds it: the K stream. 28 layers of four sequences of 1024 to 3977 slots, 28 heads on 4 of 128, a row each (270
// MB): 45.4 us, 5.9 TB/s, 0.87 of the copy rate; 8 layers of 3008 slots, 32 heads, 32 rows (205 MB): 36.2 us, 5.7 TB/s.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

constexpr int kMaxSeqs = 112;            // sequences whose sizes fit in a launch's parameters (4 KB)
constexpr int kTile = 128;               // keys a block, and (row, head) pairs a pass
constexpr int kSub = 64;                 // pairs a product (each half of the head has an accumulator of its own)
constexpr float kLog2eHi = 1.44269502f, kLog2eLo = 1.92596303e-8f;
constexpr uint32_t kBox = kTile * 128;   // 64 columns of 128 rows
constexpr int kThreads = 192;
constexpr int kStages = 2;
constexpr uint32_t kTmemCols = 256;      // two buffers of 2 x 64 columns
constexpr int kPlaces = 304;             // CTAs the GPU holds at once (two on each of 152 SMs)

struct WeightSeq {  // item0: the sequence's first item (K/V head, part of the keys)
  int item0, len, rows, row0, blocks, parts, pad[2];
};
struct WeightSeqs {  // by value in the launch's parameters
  int n, pad[7];
  WeightSeq s[kMaxSeqs];
};
struct WeightArgs {
  const __nv_bfloat16* q;
  const float* lse;
  const int32_t* rows;
  int n_q, n_seqs, seq0, max_len, n_heads, n_kv_heads;
  float scale_hi, scale_lo, decay;  // log2(e) / sqrt(head_dim) to twice the bits
  const float* acc_in;
  float* acc_out;
  int* status;
  long long budget;
  unsigned long long* stamp;
};

template <int HD>
struct WeightSmem {
  static constexpr int kChunks = HD / 64;
  static constexpr uint32_t q = 0;
  static constexpr uint32_t k = kChunks * kBox;
  static constexpr uint32_t lse = k + kStages * kChunks * kBox;  // [128] log2 units, high and low part
  static constexpr uint32_t lim = lse + kTile * 8;               // [128] slots the pair's row sees
  static constexpr uint32_t bars = lim + kTile * 4;
  static constexpr uint32_t bytes = bars + 128 + 1024;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <int HD>
__global__ void __launch_bounds__(kThreads, 2)
    weights_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ WeightArgs p,
                   const __grid_constant__ WeightSeqs sq) {
  using L = WeightSmem<HD>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float2* s_lse = reinterpret_cast<float2*>(smem + L::lse);
  int* s_lim = reinterpret_cast<int*>(smem + L::lim);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + L::bars);  // [kStages]
  uint64_t* k_empty = k_full + kStages;                            // [kStages]
  uint64_t* q_full = k_empty + kStages;  // the pass's Q tile is in shared memory
  uint64_t* d_full = q_full + 1;         // [2] scores of a block are in TMEM
  uint64_t* d_empty = d_full + 2;        // [2] they have been read
  uint64_t* meet = d_empty + 2;          // warps 0-3 among themselves (bounded, unlike bar.sync)
  uint64_t* drain = meet + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int e = 0;
  for (int hi = sq.n; hi - e > 1;) {
    const int mid = (e + hi) >> 1;
    if (sq.s[mid].item0 <= int(blockIdx.x)) e = mid;
    else hi = mid;
  }
  const WeightSeq& sh = sq.s[e];
  const int len = sh.len, n = sh.rows, G = p.n_heads / p.n_kv_heads, pairs = n * G, blocks = sh.blocks, parts = sh.parts;
  const uint32_t local = blockIdx.x - uint32_t(sh.item0);
  const int part = int(local % uint32_t(parts)), hk = int(local / uint32_t(parts)), layer = blockIdx.y;
  const int even = int(uint32_t(blocks) / uint32_t(parts)), more = blocks - even * parts;  // the first `more` parts have one more
  const int b0 = part * even + min(part, more), nb = even + (part < more);
  const int passes = (pairs + kTile - 1) / kTile;
  const int seq = layer * p.n_seqs + p.seq0 + e, row_k = seq * p.max_len;  // first row of the cache slot
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
    }
    mbar_init(q_full, 4);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&d_full[s], 1);
      mbar_init(&d_empty[s], 4);
    }
    mbar_init(meet, 4);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&map_k);
  }
  if (warp == 4) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x == 0) stamp_start(p.stamp);

  const int steps = passes * nb;  // blocks of all passes
  int issued = 0;
  if (warp == 4) {
    if (lane == 0) {
      // ---- TMA producer ----
      const uint64_t pol = passes > 1 ? policy_evict_last() : policy_evict_first();
      for (int it = 0; it < steps; ++it) {
        const int s = it % kStages;
        if (it >= kStages && !mbar_wait(&k_empty[s], (it / kStages - 1) & 1, abort_flag, p.budget)) {
          *abort_flag = 1;
          set_status(p.status, SPD_ETIMEOUT);
          break;
        }
        mbar_arrive_expect_tx(&k_full[s], L::kChunks * kBox);
        for (int c = 0; c < L::kChunks; ++c)
          tma_load_2d(smem + L::k + (s * L::kChunks + c) * kBox, &map_k, &k_full[s], hk * HD + c * 64,
                      row_k + (b0 + it % nb) * kTile, pol);
        issued = it + 1;
      }
    }
  } else if (warp == 5) {
    if (lane == 0) {
      // ---- MMA issuer ----
      const uint32_t sb = smem_u32(smem + L::q);
      bool ok = true;
      int st = 0;  // products so far
      for (int it = 0; it < steps && ok; ++it) {
        const int s = it % kStages, pass = it / nb, cols = min(kTile, pairs - pass * kTile);
        if (it % nb == 0 && !(ok = mbar_wait(q_full, pass & 1, abort_flag, p.budget))) break;
        if (!(ok = mbar_wait(&k_full[s], (it / kStages) & 1, abort_flag, p.budget))) break;
        const uint32_t sk = smem_u32(smem + L::k + s * L::kChunks * kBox);
        for (int c0 = 0; c0 < cols; c0 += kSub, ++st) {
          if (st > 1 && !(ok = mbar_wait(&d_empty[st & 1], ((st >> 1) - 1) & 1, abort_flag, p.budget))) break;
          tc_fence_after();
          const uint32_t id = idesc_bf16_f32(kTile, (min(kSub, cols - c0) + 15) & ~15);
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk)  // each half of the head from zero, in columns of its own
            mma_bf16(tmem + kTile * (st & 1) + (kk / (HD / 32)) * kSub, sdesc_k128(sk + (kk >> 2) * kBox + (kk & 3) * 32),
                     sdesc_k128(sb + c0 * 128 + (kk >> 2) * kBox + (kk & 3) * 32), id, kk % (HD / 32) > 0 ? 1u : 0u);
          mma_commit(&d_full[st & 1]);
        }
        if (!ok) break;
        mma_commit(&k_empty[s]);
      }
      if (!ok) {
        *abort_flag = 1;
        set_status(p.status, SPD_ETIMEOUT);
      }
      if (st > 0) mma_commit(drain);
      else mbar_arrive(drain);
      volatile int no_abort = 0;
      if (!mbar_wait(drain, 0, &no_abort, p.budget)) set_status(p.status, SPD_ETIMEOUT);
    }
  } else {
    // ---- warps 0-3: thread t owns key t of a block (TMEM lane t) ----
    const int t = threadIdx.x;
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    const float* acc = p.acc_in + (size_t(seq) * p.n_kv_heads + hk) * p.max_len;
    float* out = p.acc_out + (size_t(seq) * p.n_kv_heads + hk) * p.max_len;
    if (passes == 0)
      for (int k = b0 * kTile + t; k < min(len, (b0 + nb) * kTile); k += kTile) out[k] = p.decay * acc[k];
    bool ok = true;
    int met = 0, st = 0;
    auto all_meet = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(meet);
      return __all_sync(0xffffffffu, mbar_wait(meet, met++ & 1, abort_flag, p.budget));
    };
    for (int it = 0; it < steps; ++it) {
      const int pass = it / nb, kb = (b0 + it % nb) * kTile, key = kb + t;
      const int cols = min(kTile, pairs - pass * kTile);
      if (it % nb == 0) {
        // the pass's pairs, in the 128-byte swizzle (16-byte piece j of row t at j ^ (t % 8)); pairs past the
        // last, and rows outside the queries, as zeros with a normaliser that leaves no weight
        const int x = pass * kTile + t, i = x / G, at = x < pairs ? (p.rows ? p.rows[sh.row0 + i] : sh.row0 + i) : -1;
        const bool have = at >= 0 && at < p.n_q;
        const size_t row = (size_t(layer) * p.n_q + (have ? at : 0)) * p.n_heads + hk * G + (x < pairs ? x % G : 0);
        if (it > 0 && !(ok = all_meet())) break;  // every warp is done with the last pass's normalisers, the MMAs with its Q
        if (t < ((cols + 15) & ~15)) {
          uint4 v[HD / 8];
#pragma unroll
          for (int j = 0; j < HD / 8; ++j)
            v[j] = have ? reinterpret_cast<const uint4*>(p.q + row * HD)[j] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int j = 0; j < HD / 8; ++j)
            *reinterpret_cast<uint4*>(smem + L::q + (j >> 3) * kBox + t * 128 + (((j & 7) ^ (t & 7)) << 4)) = v[j];
        }
        // lse log2(e) to twice the bits (an infinite one leaves no weight, of either sign)
        const float l = have ? p.lse[row] : -INFINITY, hi = l * kLog2eHi;
        s_lse[t] = isinf(l) ? make_float2(INFINITY, 0.0f) : make_float2(hi, fmaf(l, kLog2eHi, -hi) + l * kLog2eLo);
        s_lim[t] = len - n + i + 1;
        fence_proxy_async_smem();
        if (!(ok = all_meet())) break;
        if (lane == 0) mbar_arrive(q_full);
      }
      float sum = 0.0f;
      const float before = key < len ? (pass == 0 ? p.decay * acc[key] : out[key]) : 0.0f;
      const bool masked = kb + kTile > len - n + 1;  // some row does not see the whole block
      // the exponent s scale - lse in log2 units: the halves' products and the constants' low parts are added where the sum
      // is small already, so its only rounding of note is that of its own size
      auto add = [&](float s0, float s1, int c) {
        const float2 z = s_lse[c];
        const float low = fmaf(s0 + s1, p.scale_lo, -z.y);
        const float w = ex2(fmaf(s0, p.scale_hi, fmaf(s1, p.scale_hi, -z.x)) + low);
        sum += !masked || key < s_lim[c] ? w : 0.0f;
      };
      for (int c0 = 0; c0 < cols; c0 += kSub, ++st) {
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(&d_full[st & 1], (st >> 1) & 1, abort_flag, p.budget)))) break;
        tc_fence_after();
        const uint32_t td = tmem + kTile * (st & 1) + lanes;
        const int m = min(kSub, cols - c0);
        const float was = sum;
        if (m <= 8) {
          float v[8], u[8];
          tmem_ld8x2(td, v, td + kSub, u);
#pragma unroll
          for (int c = 0; c < 8; ++c) add(v[c], u[c], c0 + c);
        } else {
          for (int d = 0; d < m; d += 32) {
            float v[32], u[32];
            tmem_ld32(td + d, v);
            tmem_ld32(td + kSub + d, u);
            if (m - d > 16) {
#pragma unroll
              for (int c = 0; c < 32; ++c) add(v[c], u[c], c0 + d + c);
            } else {
#pragma unroll
              for (int c = 0; c < 16; ++c) add(v[c], u[c], c0 + d + c);
            }
          }
        }
        if (__any_sync(0xffffffffu, isnan(sum))) {
          // a key that is not finite: again without the pairs that add nothing, whose zeros became NaN
          sum = was;
#pragma unroll 1
          for (int d = 0; d < m; d += 8) {
            float v[8], u[8];
            tmem_ld8x2(td + d, v, td + kSub + d, u);
#pragma unroll
            for (int c = 0; c < 8; ++c)
              if (!isinf(s_lse[c0 + d + c].x)) add(v[c], u[c], c0 + d + c);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&d_empty[st & 1]);
      }
      if (!ok) break;
      if (key < len) out[key] = before + sum;
    }
    if (!ok) {
      *abort_flag = 1;
      set_status(p.status, SPD_ETIMEOUT);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 128 && *abort_flag) {  // loads issued but never consumed land before the CTA exits
    volatile int no_abort = 0;
    for (int it = max(0, issued - kStages); it < issued; ++it)
      mbar_wait(&k_full[it % kStages], (it / kStages) & 1, &no_abort, p.budget);
  }
  __syncwarp();
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, kTmemCols);
  if (threadIdx.x == 0) stamp_end(p.stamp);
}

}  // namespace
}  // namespace spd

using namespace spd;

extern "C" int spd_cache_weights(const uint16_t* q, const float* lse, int n_q, const int32_t* rows, const int32_t* rows_cu,
                                 const uint16_t* kv_cache, int n_layers, int n_seqs, const int32_t* lens, int max_len,
                                 int n_heads, int n_kv_heads, int head_dim, float decay, const float* acc_in, float* acc_out,
                                 void* ws, size_t ws_bytes, void* stream) {
  if (!q || !lse || !rows_cu || !kv_cache || !lens || !acc_in || !acc_out || n_q < 0 || n_layers < 1 || n_seqs < 1 ||
      max_len < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads)
    return fail(SPD_EINVAL, "bad cache weight arguments");
  if (head_dim != 64 && head_dim != 128) return fail(SPD_EUNSUPPORTED, "head_dim must be 64 or 128");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(kv_cache)) & 15)
    return fail(SPD_EINVAL, "q and kv_cache must be 16-byte aligned");
  if (ws && ws_bytes < sizeof(int)) return fail(SPD_ENOSPC, "cache weight workspace too small (%zu < 4)", ws_bytes);
  if (rows_cu[0] != 0) return fail(SPD_EINVAL, "rows_cu must start at 0");
  if ((long long)n_layers * n_seqs * max_len > 0x7fffffffLL) return fail(SPD_EUNSUPPORTED, "more than 2^31 - 1 cache rows");
  if (n_layers > 65535) return fail(SPD_EUNSUPPORTED, "more than 65535 layers");
  for (int b = 0; b < n_seqs; ++b) {
    if (lens[b] < 0 || lens[b] > max_len) return fail(SPD_EINVAL, "length of sequence %d outside [0, max_len]", b);
    if (rows_cu[b + 1] < rows_cu[b] || rows_cu[b + 1] - rows_cu[b] > lens[b])
      return fail(SPD_EINVAL, "sequence %d: rows_cu decreases, or more rows than cached tokens", b);
    const long long pairs = (long long)(rows_cu[b + 1] - rows_cu[b]) * (n_heads / n_kv_heads);
    if ((pairs + kTile - 1) / kTile * ((lens[b] + kTile - 1) / kTile) > 0x7fffffffLL / kTile)
      return fail(SPD_EUNSUPPORTED, "sequence %d: too many (row, head, slot) triples", b);
  }
  if (!rows && rows_cu[n_seqs] > n_q) return fail(SPD_EINVAL, "rows_cu runs past the queries");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  CUtensorMap map;
  if (int rc = make_operand_map(&map, kv_cache, 2 * n_kv_heads * head_dim, n_layers * n_seqs * max_len, kTile)) return rc;
  WeightArgs p{};
  p.q = reinterpret_cast<const __nv_bfloat16*>(q);
  p.lse = lse;
  p.rows = rows;
  p.n_q = n_q;
  p.n_seqs = n_seqs;
  p.max_len = max_len;
  p.n_heads = n_heads;
  p.n_kv_heads = n_kv_heads;
  const double scale = 1.4426950408889634 / sqrt(double(head_dim));
  // rounded down, so that the low part is positive and an infinite score stays what it is
  p.scale_hi = float(scale) > scale ? nextafterf(float(scale), 0.0f) : float(scale);
  p.scale_lo = float(scale - double(p.scale_hi));
  p.decay = decay;
  p.acc_in = acc_in;
  p.acc_out = acc_out;
  p.status = static_cast<int*>(ws);
  p.budget = kWaitBudget;
  const auto kernel = head_dim == 128 ? weights_kernel<128> : weights_kernel<64>;
  const size_t smem = head_dim == 128 ? WeightSmem<128>::bytes : WeightSmem<64>::bytes;
  static DeviceOnce attr[2];
  SPD_CUDA_TRY(once_per_device(attr[head_dim == 128], [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  }));
  for (int s0 = 0; s0 < n_seqs; s0 += kMaxSeqs) {
    WeightSeqs sq{};
    sq.n = std::min(kMaxSeqs, n_seqs - s0);
    p.seq0 = s0;
    double keys = 0.0, pairs = 0.0;
    long long work = 0;
    for (int b = s0; b < s0 + sq.n; ++b) work += (long long)((lens[b] + kTile - 1) / kTile) * n_kv_heads * n_layers;
    // blocks an item: few and long ones, since a CTA's start (Q tile, normalisers, first block) costs several blocks'
    // time: one wave of CTAs where the units allow it, else about two. 8 layers of 32 heads, 24 blocks each, with 6 / 8 / 12 /
    // 24 blocks an item: 45.1 / 42.3 / 39.4 / 35.5 us; 448 units of 8 to 32 blocks with 4 / 7 / 12 / 16 / 24: 50.7 / 46.9 / 44.9 /
    // 49.3 / 46.1.
    auto wave = [&](long long share) {
      long long k = 0;
      for (int b = s0; b < s0 + sq.n; ++b) k += ((lens[b] + kTile - 1) / kTile + share - 1) / share;
      return k * n_kv_heads * n_layers;
    };
    const bool fits = wave(1 << 24) <= kPlaces;  // the units do, whole
    const int waves = fits ? 1 : 2;
    long long share = std::max<long long>(2, (work + waves * kPlaces - 1) / (waves * kPlaces));
    while (fits && wave(share) > kPlaces) share += (share + 15) / 16;
    long long items = 0;
    for (int i = 0; i < sq.n; ++i) {
      const int b = s0 + i, blocks = (lens[b] + kTile - 1) / kTile;
      const int parts = int((blocks + share - 1) / share), rows_b = rows_cu[b + 1] - rows_cu[b];
      sq.s[i] = {int(items), lens[b], rows_b, rows_cu[b], blocks, parts, {}};
      items += (long long)n_kv_heads * parts;
      keys += lens[b];
      pairs += double(lens[b]) * rows_b;
    }
    if (items > 0x7fffffff) return fail(SPD_EUNSUPPORTED, "cache weights of more than 2^31 blocks");
    if (items == 0) continue;
    const double fl = 2.0 * head_dim * n_heads * pairs * n_layers, by = keys * n_layers * n_kv_heads * (2.0 * head_dim + 8.0);
    p.stamp = stamp_slot(TR_ATTN, fl, by);
    const int slot = trace_begin(st);
    SPD_CUDA_TRY(launch_pdl(kernel, dim3(unsigned(items), n_layers), dim3(kThreads), smem, st, map, p, sq));
    trace_end(slot, st, TR_ATTN, fl, by);
  }
  return SPD_OK;
}
