// Attention of drafted tokens over a KV cache (the verification of a speculative step; with one node a sequence, a
// decode step whose rotary positions need not be its slots).
//
// Sequence b holds ctx_b committed rows in its cache slot and behind them the rows of its n_b drafts. Node i sees the
// committed rows and the drafts j whose bit is set in its mask (its ancestors and itself for a tree):
//   s_ij = q_i . k_j / sqrt(head_dim),  lse_i = log sum_j e^s_ij,  o_i = sum_j e^(s_ij - lse_i) v_j,
// o = 0 and lse = -inf for a row that sees nothing. Keys a row does not see contribute nothing, whatever they hold.
//
// The K/V stream is what a call cannot do without (4 head_dim bytes a key and K/V head), so every key is read once for
// all the rows that see it: the up to 128 rows of an MMA tile are the nodes of a sequence times the query heads of a
// K/V head's group. An item is one such tile over a range of keys; the ranges are cut so that the items fill the GPU
// (two CTAs an SM) and every item of a batch of different lengths has about the same number of keys. Parts of a row's
// keys leave states (m, l, O) in fp32, merged in the order of the keys (the same bits in every run): those of a cluster of up to 8
// items through distributed shared memory, and where a row's keys take more than one cluster, the clusters' by
// tree_merge_kernel.
//   warp 4     TMA producer: blocks of 64 keys of K and of V into rings
//   warp 5     MMA issuer: S = Q K^T into TMEM, then O += P V with P read from TMEM, V in place as an MN-major operand
//   warps 0-3  a thread a row: the block's 64 scores in registers, online softmax in fp32; a weight is held as the sum of
//              three bf16 terms, all 24 bits of it (three products: the tensor pipe has the time while K and V stream): two
//              over the scores in TMEM, where O leaves no room for more, the third in shared memory
// Only blocks that reach past the committed rows are masked; there the softmax warps also clear the rows of V behind the last
// draft (recycled memory) and those that are not finite, which a weight of zero would turn into NaN for rows that
// do not see them; rows that do see one add it at the end.
//
// What bounds it: the tensor pipe and the K/V stream about alike. With two CTAs an SM a block of 64 keys takes 0.77 us of the
// SM (0.70 with heads of 64) where K and V come from L2, 1150 of its 1500 cycles in products (S 384, P V 768); its share
// of HBM is 0.73. Two terms a weight took 256 cycles less, and 35.5 instead of 40.5 us a call for the first of the
// cases below. A single CTA takes 1.2 us a block, S and P V waiting for each other. A CTA costs about 6 us besides: launch and
// set-up 1, the first loads 2 to 3 (everybody asks at once), the last products, state and merge 2 to 3. 16 nodes on 65521 keys,
// 28 heads on 4 of 128: 39.7 us, 3.4 TB/s (the merge through memory 4); eight trees of 48 on 640 to 1417 keys, 32 K/V heads:
// 41.8 us, 3.5 TB/s (the SMs with the two longest sequences); 32 trees on 300 to 1943 keys: 31.3 us; one token, 321 keys, 32
// heads: 9.2 us.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

constexpr int kMaxSeqs = 112;          // sequences whose sizes fit in a launch's parameters (4 KB)
constexpr int kTK = 64;                // keys a block
constexpr uint32_t kQBox = 128 * 128;  // 64 columns of the Q tile
constexpr uint32_t kKBox = kTK * 128;  // 64 columns of a block of K or V
constexpr int kThreads = 192;
constexpr uint32_t kTmemCols = 256;    // S: two buffers [0, 64) and [64, 128); O: [128, 128 + HD)
constexpr int kItems = 304;            // items that fill the GPU: two CTAs on each of 152 SMs
// The reference that a row's exponentials are taken against is renewed once its maximum has grown by this much (log2
// units): weights stay below 2^8, their two terms and the fp32 sums are relative to them, and almost no block pays for the
// round trip of O through the registers.
constexpr float kGrown = 8.0f;
constexpr int kMaxCluster = 8;

// Sequences of a launch, the longest first, in the launch's parameters (no copy, no wait for one). Clusters from item0 on are
// the sequence's: (K/V head, group of parts of the keys, tile), the tile fastest, so that the tiles that read the same keys
// run side by side; the CTAs of a cluster are the parts of its group. A CTA reads one entry, half a line of parameter
// memory: with an array a field the look-up took 1400 to 2100 cycles.
struct TreeSeq {
  int item0, q0, nodes, ctx, seq, tiles, groups;
  int part0;  // first slot of the sequence's states in the workspace (groups > 1)
};
struct TreeSeqs {
  int n, pad[7];
  TreeSeq s[kMaxSeqs];
};
struct TreeArgs {
  const __nv_bfloat16* q;
  const uint32_t* mask;
  int words;
  const __nv_bfloat16* kv;
  int max_len, n_heads, n_kv_heads;
  int group, chunk, chunks, nodes_tile;  // heads a group; of them in a tile; tiles across; nodes a tile
  float scale_log2;
  __nv_bfloat16* o;
  float* lse;
  int cluster;     // CTAs a cluster
  float* part_o;   // [cluster][rows_part][HD] states of sequences of several groups
  float2* part_ml; // [cluster][rows_part]: maximum (log2 units), sum
  int rows_part;
  int* status;
  long long budget;
  unsigned long long* stamp;
};

template <int HD>
struct TreeSmem {
  static constexpr int kChunks = HD / 64;
  static constexpr int kStages = 256 / HD;  // 64 KB of K and V in flight a CTA
  static constexpr uint32_t q = 0;
  static constexpr uint32_t k = q + kChunks * kQBox;
  static constexpr uint32_t v = k + kStages * kChunks * kKBox;
  static constexpr uint32_t p3 = v + kStages * kChunks * kKBox;  // [128][64] third terms of a block's weights
  static constexpr uint32_t bars = p3 + 128 * 128;
  static constexpr uint32_t bytes = bars + 256;  // (two CTAs an SM: at most 113 KB)
  // after the last product, of a cluster's merge
  static constexpr uint32_t ml = q;     // [128] a row's maximum and sum, over the Q tile
  static constexpr uint32_t state = k;  // [128][HD] fp32 O, over the rings
  static_assert(128 * HD * 4 <= p3 - k, "the rings hold the tile's O");
  static_assert(bytes <= 113 * 1024, "two CTAs an SM");
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ bool not_finite(uint32_t two) {  // either of two bf16
  return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u;
}

// Bits d0 .. d0 + 63 of what node i (mask row `row`) of n sees; d < 0: a committed row, which every node sees.
__device__ __forceinline__ uint64_t seen64(const TreeArgs& p, size_t row, int i, int n, int d0) {
  const int at = max(d0, 0);
  uint64_t bits;
  if (!p.mask) {
    bits = i >= at ? (i - at >= 63 ? ~0ull : (2ull << (i - at)) - 1) : 0ull;
  } else {
    const uint32_t* m = p.mask + row * p.words;
    const int w = at >> 5;
    const uint32_t a = w < p.words ? m[w] : 0u, b = w + 1 < p.words ? m[w + 1] : 0u, c = w + 2 < p.words ? m[w + 2] : 0u;
    bits = (uint64_t(__funnelshift_r(b, c, at & 31)) << 32) | __funnelshift_r(a, b, at & 31);
  }
  const int left = n - at;  // drafts there are
  if (left < 64) bits &= left > 0 ? (1ull << left) - 1 : 0ull;
  if (d0 <= -64) return ~0ull;
  return d0 < 0 ? (bits << -d0) | ((1ull << -d0) - 1) : bits;
}

template <int HD>
__global__ void __launch_bounds__(kThreads, 2)
    tree_attn_kernel(const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ TreeArgs p,
                     const __grid_constant__ TreeSeqs sq) {
  using L = TreeSmem<HD>;
  constexpr int NS = L::kStages;
  extern __shared__ __align__(1024) uint8_t smem[];  // (the swizzle's atoms; no room to round the address up)
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + L::bars);  // [NS] K block landed
  uint64_t* k_empty = k_full + NS;                                 // [NS] its S product has completed
  uint64_t* v_full = k_empty + NS;                                 // [NS] V block landed
  uint64_t* v_empty = v_full + NS;                                 // [NS] its PV products have completed
  uint64_t* q_full = v_empty + NS;   // the Q tile is in shared memory
  uint64_t* s_full = q_full + 1;     // [2] S of block j is in TMEM buffer j % 2
  uint64_t* p_full = s_full + 2;     // [2] P of block j written and O rescaled
  uint64_t* o_done = p_full + 2;     // PV products of the current block completed
  uint64_t* drain = o_done + 1;      // every MMA completed: O is final
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* odd_v = reinterpret_cast<int*>(tmem_slot + 2);  // some visible V is not finite

  if (smem_u32(smem) & 1023) {  // every CTA alike
    pdl_wait();
    if (threadIdx.x == 0) set_status(p.status, SPD_ECUDA);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the cluster's sequence: the last entry that starts at or before it
  const int C = p.cluster, rank = int(blockIdx.x) & (C - 1);
  uint32_t u = blockIdx.x / uint32_t(C);
  int e = 0;
  for (int hi = sq.n; hi - e > 1;) {
    const int mid = (e + hi) >> 1;
    if (uint32_t(sq.s[mid].item0) <= u) e = mid;
    else hi = mid;
  }
  const TreeSeq& sh = sq.s[e];
  const int n = sh.nodes, ctx = sh.ctx, groups = sh.groups, parts = groups * C, tiles = sh.tiles;
  u -= uint32_t(sh.item0);
  const int slot = sh.part0 + int(u);
  const int tile = int(u % uint32_t(tiles));
  u /= uint32_t(tiles);
  const int part = int(u % uint32_t(groups)) * C + rank, hk = int(u / uint32_t(groups));
  const int n0 = tile / p.chunks * p.nodes_tile, h0 = tile % p.chunks * p.chunk;  // first node, first head of the group
  const int nodes = min(p.nodes_tile, n - n0), rows = nodes * p.chunk;
  const int heads = min(p.chunk, p.group - h0);  // of the chunk's heads, those there are
  const int total = ctx + n, blocks = (total + kTK - 1) / kTK;
  const int even = int(uint32_t(blocks) / uint32_t(parts)), more = blocks - even * parts;  // the first `more` parts have one more
  const int b0 = part * even + min(part, more), nkb = even + (part < more);
  const int row0 = sh.seq * p.max_len;  // the cache slot's first row
  const int nw = (rows + 31) / 32;         // softmax warps with rows
  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_full[s], 1);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(q_full, nw);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&p_full[s], nw);  // one arrival per softmax warp
    }
    mbar_init(o_done, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    *odd_v = 0;
    fence_mbar_init();
    prefetch_tmap(&map_kv);
  }
  if (warp == 4) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t t_o = tmem + 2 * kTK;

  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x == 0) stamp_start(p.stamp);

  int issued_k = 0, issued_v = 0;
  if (warp == 4) {
    if (lane == 0) {
      // ---- TMA producer ----
      const uint64_t pol = tiles > 1 ? policy_evict_last() : policy_evict_first();
      auto load = [&](int j, uint64_t* full, uint64_t* empty, uint32_t at, int x0) -> bool {
        const int s = j % NS;
        if (j >= NS && !mbar_wait(&empty[s], (j / NS - 1) & 1, abort_flag, p.budget)) {
          *abort_flag = 1;
          set_status(p.status, SPD_ETIMEOUT);
          return false;
        }
        mbar_arrive_expect_tx(&full[s], L::kChunks * kKBox);
        for (int c = 0; c < L::kChunks; ++c)
          tma_load_2d(smem + at + (s * L::kChunks + c) * kKBox, &map_kv, &full[s], x0 + hk * HD + c * 64,
                      row0 + (b0 + j) * kTK, pol);
        return true;
      };
      for (int j = 0; j < nkb; ++j) {
        if (!load(j, k_full, k_empty, L::k, 0)) break;
        issued_k = j + 1;
        if (!load(j, v_full, v_empty, L::v, p.n_kv_heads * HD)) break;
        issued_v = j + 1;
      }
    }
  } else if (warp == 5) {
    if (lane == 0) {
      // ---- MMA issuer ----
      const uint32_t id_s = idesc_bf16_f32(128, kTK);
      const uint32_t id_o = idesc_bf16_f32(128, HD) | (1u << 16);  // V is MN-major
      const uint32_t sa = smem_u32(smem + L::q), sp = smem_u32(smem + L::p3);
      bool ok = mbar_wait(q_full, 0, abort_flag, p.budget);
      auto issue_s = [&](int j) -> bool {
        const int s = j % NS;
        if (!mbar_wait(&k_full[s], (j / NS) & 1, abort_flag, p.budget)) return false;
        // S buffer j % 2 holds P of block j - 2 until its PV products have completed
        if (j > 1 && !mbar_wait(o_done, j & 1, abort_flag, p.budget)) return false;
        tc_fence_after();
        const uint32_t sk = smem_u32(smem + L::k + s * L::kChunks * kKBox);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk)
          mma_bf16(tmem + kTK * (j & 1), sdesc_k128(sa + (kk >> 2) * kQBox + (kk & 3) * 32),
                   sdesc_k128(sk + (kk >> 2) * kKBox + (kk & 3) * 32), id_s, kk > 0 ? 1u : 0u);
        mma_commit(&s_full[j & 1]);
        mma_commit(&k_empty[s]);
        return true;
      };
      if (ok && nkb > 0) ok = issue_s(0);  // (a short sequence's parts may be empty)
      for (int j = 0; j < nkb && ok; ++j) {
        const int s = j % NS;
        if (j + 1 < nkb && !(ok = issue_s(j + 1))) break;
        if (!(ok = mbar_wait(&v_full[s], (j / NS) & 1, abort_flag, p.budget))) break;
        if (!(ok = mbar_wait(&p_full[j & 1], (j >> 1) & 1, abort_flag, p.budget))) break;
        tc_fence_after();
        const uint32_t sv = smem_u32(smem + L::v + s * L::kChunks * kKBox);
#pragma unroll
        for (int kk = 0; kk < 2 * (kTK / 16); ++kk) {  // the weights' first terms, then their second, then their third
          const int x = kk % (kTK / 16), term = kk / (kTK / 16);
          mma_bf16_ts(t_o, tmem + kTK * (j & 1) + 16 * x + 8 * term, sdesc_mn128(sv + x * 2048, kKBox),
                      id_o, (j > 0 || kk > 0) ? 1u : 0u);
        }
#pragma unroll
        for (int x = 0; x < kTK / 16; ++x)
          mma_bf16(t_o, sdesc_k128(sp + x * 32), sdesc_mn128(sv + x * 2048, kKBox), id_o, 1u);
        mma_commit(o_done);
        mma_commit(&v_empty[s]);
      }
      if (!ok) {
        *abort_flag = 1;
        set_status(p.status, SPD_ETIMEOUT);
      }
      if (nkb > 0) mma_commit(drain);  // arrives once every MMA issued above has completed
      else mbar_arrive(drain);
      volatile int no_abort = 0;
      if (!mbar_wait(drain, 0, &no_abort, p.budget)) set_status(p.status, SPD_ETIMEOUT);
    }
  } else if (warp < nw) {
    // ---- softmax: warp w reads TMEM lanes [32 w, 32 w + 32) ----
    const int r = warp * 32 + lane, T = nw * 32;
    const int node = n0 + min(r / p.chunk, nodes - 1), hc = r % p.chunk;
    const bool valid = r < rows && hc < heads;
    const int head = hk * p.group + h0 + min(hc, heads - 1);
    const size_t qrow = sh.q0 + node;  // rows without a node repeat the last one's, and are not stored
    const __nv_bfloat16* qsrc = p.q + (qrow * p.n_heads + head) * HD;
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    {  // the Q tile in the 128-byte swizzle: 16-byte piece j of row r at j ^ (r % 8)
      uint4 v[HD / 8];
#pragma unroll
      for (int j = 0; j < HD / 8; ++j) v[j] = reinterpret_cast<const uint4*>(qsrc)[j];
#pragma unroll
      for (int j = 0; j < HD / 8; ++j)
        *reinterpret_cast<uint4*>(smem + L::q + (j >> 3) * kQBox + r * 128 + (((j & 7) ^ (r & 7)) << 4)) = v[j];
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    }
    float m_run = -INFINITY, l_run = 0.0f;  // the row's maximum so far (raw scores) and sum of weights
    bool ok = true;
    for (int j = 0; j < nkb; ++j) {
      const uint32_t t_s = tmem + kTK * (j & 1) + lanes;
      const int kb = (b0 + j) * kTK;
      const bool drafts = kb + kTK > ctx;  // the block holds keys that not every row sees, or none at all
      if (drafts) {
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(&v_full[j % NS], (j / NS) & 1, abort_flag, p.budget)))) break;
        bool odd = false;
        for (int x = threadIdx.x; x < kTK * L::kChunks; x += T) {
          uint4* vr = reinterpret_cast<uint4*>(smem + L::v + (j % NS) * L::kChunks * kKBox + x * 128);
          bool clear = kb + x % kTK >= total;
          if (!clear && kb + x % kTK >= ctx) {
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              const uint4 w = vr[y];
              clear |= not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w);
            }
            odd |= clear;
          }
          if (clear) {
#pragma unroll
            for (int y = 0; y < 8; ++y) vr[y] = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        if (odd) atomicOr(odd_v, 1);
        fence_proxy_async_smem();
        // (every softmax warp arrives on p_full after its share, so the products see all of them)
      }
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(&s_full[j & 1], (j >> 1) & 1, abort_flag, p.budget)))) break;
      tc_fence_after();
      float v[kTK];
      tmem_ld64(t_s, v);
      if (drafts) {
        const uint64_t see = seen64(p, qrow, node, n, kb - ctx);
        const uint32_t lo = uint32_t(see), hi = uint32_t(see >> 32);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if (!((lo >> i) & 1u)) v[i] = -INFINITY;
          if (!((hi >> i) & 1u)) v[32 + i] = -INFINITY;
        }
      }
      float m4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
      for (int i = 4; i < kTK; ++i) m4[i & 3] = fmaxf(m4[i & 3], v[i]);
      const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
      if (j == 0) {
        m_run = mx;
      } else if (__any_sync(0xffffffffu, (mx - m_run) * p.scale_log2 > kGrown)) {
        // a row's weights have outgrown its reference. The previous products have completed (those before had when
        // these scores came): O can be rescaled
        if (!(ok = __all_sync(0xffffffffu, mbar_wait(o_done, (j - 1) & 1, abort_flag, p.budget)))) break;
        tc_fence_after();
        const float m_new = fmaxf(m_run, mx);
        const float corr = m_new == m_run ? 1.0f : ex2((m_run - m_new) * p.scale_log2);
        m_run = m_new;
        l_run *= corr;
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          float ov[32];
          tmem_ld32(t_o + lanes + c * 32, ov);
#pragma unroll
          for (int i = 0; i < 32; ++i) ov[i] *= corr;
          tmem_st32(t_o + lanes + c * 32, ov);
        }
      }
      const float off = m_run == -INFINITY ? 0.0f : m_run * p.scale_log2;  // nothing seen yet: all weights are 0
      float r4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      uint32_t third[kTK / 2];  // keys 2 i and 2 i + 1 in word i
#pragma unroll
      for (int x = 0; x < kTK / 16; ++x) {
        float first[8], second[8];  // the terms of keys 16 x + 2 i and 16 x + 2 i + 1 in word i
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = 16 * x + 2 * i;
          const float p0 = ex2(fmaf(v[k], p.scale_log2, -off)), p1 = ex2(fmaf(v[k + 1], p.scale_log2, -off));
          r4[k & 2] += p0;
          r4[(k & 2) + 1] += p1;
          const uint32_t hi = pack_bf16(p0, p1);
          const float a = p0 - __uint_as_float(hi << 16), b = p1 - __uint_as_float(hi & 0xffff0000u);
          const uint32_t mid = pack_bf16(a, b);
          first[i] = __uint_as_float(hi);
          second[i] = __uint_as_float(mid);
          third[k >> 1] = pack_bf16(a - __uint_as_float(mid << 16), b - __uint_as_float(mid & 0xffff0000u));
        }
        tmem_st8(t_s + 16 * x, first);  // over the scores
        tmem_st8(t_s + 16 * x + 8, second);
      }
      l_run += (r4[0] + r4[1]) + (r4[2] + r4[3]);
      // the third terms' place is free when the block before has been multiplied
      if (j > 0 && !(ok = __all_sync(0xffffffffu, mbar_wait(o_done, (j - 1) & 1, abort_flag, p.budget)))) break;
#pragma unroll
      for (int y = 0; y < 8; ++y)
        *reinterpret_cast<uint4*>(smem + L::p3 + r * 128 + ((y ^ (r & 7)) << 4)) =
            make_uint4(third[4 * y], third[4 * y + 1], third[4 * y + 2], third[4 * y + 3]);
      fence_proxy_async_smem();
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[j & 1]);
    }
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait(drain, 0, abort_flag, p.budget));
    if (!ok) {
      *abort_flag = 1;
      set_status(p.status, SPD_ETIMEOUT);
      if (C > 1) *reinterpret_cast<float2*>(smem + L::ml + r * 8) = make_float2(-INFINITY, 0.0f);
    } else {
      tc_fence_after();
      // A committed V that is infinite: the products of a weight's terms, which can be 0 or negative, are NaN together. Which
      // infinity a column has is the same for every row (all see every committed key, with a weight above 0).
      float sick = 0.0f;  // NaN where a column is not finite
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {
        float ov[32];
        tmem_ld32(t_o + lanes + c * 32, ov);
#pragma unroll
        for (int i = 0; i < 32; ++i) sick = fmaf(ov[i], 0.0f, sick);
      }
      const bool mend = valid && isnan(sick) && !isnan(l_run);  // (scores that are NaN leave the row NaN)
      if (__any_sync(0xffffffffu, mend)) {
        constexpr int E = HD / 32;  // columns a lane looks through
        const size_t ld = 2 * size_t(p.n_kv_heads) * HD;
        const __nv_bfloat16* vc = p.kv + size_t(row0) * ld + (size_t(p.n_kv_heads) + hk) * HD + E * lane;
        uint32_t has = 0;  // of column e in bits 4 e: +inf, -inf, NaN
        for (int k = b0 * kTK; k < min(ctx, (b0 + nkb) * kTK); ++k)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float x = __bfloat162float(vc[k * ld + e]);
            has |= (isnan(x) ? 4u : x == INFINITY ? 1u : x == -INFINITY ? 2u : 0u) << (4 * e);
          }
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          float ov[32];
          tmem_ld32(t_o + lanes + c * 32, ov);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const uint32_t h = (__shfl_sync(0xffffffffu, has, (c * 32 + i) / E) >> (4 * (i % E))) & 15u;
            if (mend && isnan(ov[i]) && (h == 1u || h == 2u)) ov[i] = h == 1u ? INFINITY : -INFINITY;
          }
          tmem_st32(t_o + lanes + c * 32, ov);
        }
      }
      if (*reinterpret_cast<volatile int*>(odd_v)) {
        // drafts whose V was cleared: rows that see one add p v in fp32 (the score again from q and k)
        const float off = m_run == -INFINITY ? 0.0f : m_run * p.scale_log2;
        for (int d = max(0, b0 * kTK - ctx); d < min(n, (b0 + nkb) * kTK - ctx); ++d) {
          const bool sees = valid && (seen64(p, qrow, node, n, d) & 1ull);
          const __nv_bfloat16* kr = p.kv + size_t(row0 + ctx + d) * (2 * size_t(p.n_kv_heads) * HD) + hk * HD;
          const __nv_bfloat16* vr = kr + size_t(p.n_kv_heads) * HD;
          for (int c = 0; c < L::kChunks; ++c) {
            const uint32_t two = *reinterpret_cast<const uint32_t*>(vr + c * 64 + 2 * lane);
            if (!__any_sync(0xffffffffu, not_finite(two))) continue;
            float s = 0.0f;
            if (sees)
              for (int x = 0; x < HD; ++x) s = fmaf(__bfloat162float(qsrc[x]), __bfloat162float(kr[x]), s);
            const float w = ex2(fmaf(s, p.scale_log2, -off));
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
              float ov[32];
              tmem_ld32(t_o + lanes + c * 64 + b * 32, ov);
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (sees) ov[i] = fmaf(w, __bfloat162float(vr[c * 64 + b * 32 + i]), ov[i]);
              tmem_st32(t_o + lanes + c * 64 + b * 32, ov);
            }
          }
        }
      }
      const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
      const float m2 = m_run * p.scale_log2;
      if (C > 1) {  // to this CTA's shared memory: 16-byte piece j of row r at j ^ r, so that neither side meets in a bank
        *reinterpret_cast<float2*>(smem + L::ml + r * 8) = make_float2(m2, l_run);
        if (nkb > 0) {
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            float v[32];
            tmem_ld32(t_o + lanes + c * 32, v);
#pragma unroll
            for (int y = 0; y < 8; ++y)
              *reinterpret_cast<float4*>(smem + L::state + r * (HD * 4) + (((c * 8 + y) ^ (r & (HD / 4 - 1))) << 4)) =
                  make_float4(v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
          }
        }
      } else if (parts > 1) {
        float* po = p.part_o + (size_t(slot) * p.rows_part + r) * HD;
        if (valid) p.part_ml[size_t(slot) * p.rows_part + r] = make_float2(m2, l_run);
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          float v[32];
          tmem_ld32(t_o + lanes + c * 32, v);
          if (valid) {
#pragma unroll
            for (int y = 0; y < 8; ++y)
              reinterpret_cast<float4*>(po + c * 32)[y] = make_float4(v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
          }
        }
      } else {
        __nv_bfloat16* orow = p.o + (qrow * p.n_heads + head) * HD;
        if (valid && p.lse) p.lse[qrow * p.n_heads + head] = fmaf(m2, 0.6931471805599453f, logf(l_run));
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          float v[32];
          tmem_ld32(t_o + lanes + c * 32, v);
          if (valid) {
#pragma unroll
            for (int y = 0; y < 4; ++y)
              reinterpret_cast<uint4*>(orow + c * 32)[y] =
                  make_uint4(pack_bf16(v[8 * y] * inv, v[8 * y + 1] * inv), pack_bf16(v[8 * y + 2] * inv, v[8 * y + 3] * inv),
                             pack_bf16(v[8 * y + 4] * inv, v[8 * y + 5] * inv), pack_bf16(v[8 * y + 6] * inv, v[8 * y + 7] * inv));
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 128 && *abort_flag) {
    // loads issued but never consumed land before the CTA exits
    volatile int no_abort = 0;
    for (int j = max(0, issued_k - NS); j < issued_k; ++j) mbar_wait(&k_full[j % NS], (j / NS) & 1, &no_abort, p.budget);
    for (int j = max(0, issued_v - NS); j < issued_v; ++j) mbar_wait(&v_full[j % NS], (j / NS) & 1, &no_abort, p.budget);
  }
  __syncwarp();
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, kTmemCols);
  if (C > 1) {
    // every CTA merges its share of the tile's rows, in rank order
    cluster_arrive();
    cluster_wait();
    constexpr int P = HD / 4;  // 16-byte pieces a row
    const int r1 = rows * (rank + 1) / C;
    for (int x = rows * rank / C * P + int(threadIdx.x); x < r1 * P; x += kThreads) {
      const int r = x / P, j = x % P, hc = r % p.chunk;
      const uint32_t at_ml = smem_u32(smem + L::ml + r * 8);
      const uint32_t at_o = smem_u32(smem + L::state + r * (HD * 4) + ((j ^ (r & (P - 1))) << 4));
      float2 ml[kMaxCluster];
      float4 v[kMaxCluster];
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) {
        ml[k] = make_float2(-INFINITY, 0.0f);
        if (k < C) {
          uint32_t a, b;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at_ml), "r"(k));
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(at_o), "r"(k));
          ml[k] = ld_dsmem_v2(a);
          v[k] = ld_dsmem_v4(b);
        }
      }
      float m = -INFINITY, l = 0.0f;
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) m = fmaxf(m, ml[k].x);
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < kMaxCluster; ++k) {
        if (ml[k].y == 0.0f) continue;  // a part in which the row sees nothing
        const float f = exp2f(ml[k].x - m);
        l = fmaf(ml[k].y, f, l);
        o.x = fmaf(v[k].x, f, o.x);
        o.y = fmaf(v[k].y, f, o.y);
        o.z = fmaf(v[k].z, f, o.z);
        o.w = fmaf(v[k].w, f, o.w);
      }
      if (groups > 1) {
        const size_t at = size_t(slot) * p.rows_part + r;
        if (j == 0) p.part_ml[at] = make_float2(m, l);
        reinterpret_cast<float4*>(p.part_o + at * HD)[j] = o;
      } else if (hc < heads) {
        const size_t at = size_t(sh.q0 + n0 + r / p.chunk) * p.n_heads + hk * p.group + h0 + hc;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        reinterpret_cast<uint2*>(p.o + at * HD)[j] = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        if (j == 0 && p.lse) p.lse[at] = fmaf(m, 0.6931471805599453f, logf(l));
      }
    }
    cluster_arrive();  // the others' shared memory outlives the reads
    cluster_wait();
  }
  if (threadIdx.x == 0) stamp_end(p.stamp);
}

// Rows whose keys took several clusters: states (m_i, l_i, O_i) merged in key order, m = max m_i, l = sum l_i 2^(m_i - m),
// O = sum O_i 2^(m_i - m). A part in which the row sees nothing has l_i = 0. (Its maximum does not tell: fmaxf passes over
// those of parts whose scores are all NaN, whose sums are NaN and stay so.) W warps a row (node and head), each a range of the
// parts, four of them in flight; the kernel is a handful of dependent loads, so long rows of parts want more warps, not longer
// loops. Whole calls with 4 / 8 parts in flight, before weights had a third term: 32 trees in 2 to 4 parts 27.8 / 28.6 us, one
// in 18 parts 35.1 / 35.0; four warps a CTA instead of eight 27.6 and 36.7. Where a row's states are is worked out before the
// wait for them (27.5 and 34.8).
constexpr int kMergeWarps = 8, kMergeAhead = 4;
template <int HD>
__global__ void __launch_bounds__(kMergeWarps * 32)
    tree_merge_kernel(const __grid_constant__ TreeArgs p, const __grid_constant__ TreeSeqs sq, int W) {
  constexpr int D = HD / 32;  // dims a lane
  __shared__ float2 wml[kMergeWarps];
  __shared__ float wo[kMergeWarps][HD];
  pdl_launch_dependents();
  const TreeSeq& sh = sq.s[blockIdx.y];
  const uint32_t parts = sh.groups, tiles = sh.tiles;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp & (W - 1);
  const uint32_t row = (blockIdx.x * kMergeWarps + warp) / uint32_t(W);
  const bool have = row < uint32_t(sh.nodes * p.n_heads);
  float m = -INFINITY, l = 0.0f, o[D];
#pragma unroll
  for (int x = 0; x < D; ++x) o[x] = 0.0f;
  const uint32_t node = row / uint32_t(p.n_heads), head = row - node * p.n_heads;
  const uint32_t hk = head / uint32_t(p.group), hg = head - hk * p.group, chunk = hg / uint32_t(p.chunk);
  const uint32_t across = node / uint32_t(p.nodes_tile), tile = across * p.chunks + chunk;
  const uint32_t r = (node - across * p.nodes_tile) * p.chunk + hg - chunk * p.chunk;
  const size_t first = (size_t(sh.part0) + size_t(hk) * parts * tiles + tile) * p.rows_part + r;
  const size_t step = size_t(tiles) * p.rows_part;
  const int s1 = int((w + 1) * parts / uint32_t(W));
  pdl_wait();
  if (have) {
    for (int s0 = int(w * parts / uint32_t(W)); s0 < s1; s0 += kMergeAhead) {
      float2 ml[kMergeAhead];
      float v[kMergeAhead][D];
#pragma unroll
      for (int u = 0; u < kMergeAhead; ++u) {
        ml[u] = make_float2(-INFINITY, 0.0f);
        if (s0 + u >= s1) continue;
        const size_t at = first + (s0 + u) * step;
        ml[u] = p.part_ml[at];
        const float* po = p.part_o + at * HD + D * lane;
        if constexpr (D == 4) {
          const float4 f = *reinterpret_cast<const float4*>(po);
          v[u][0] = f.x, v[u][1] = f.y, v[u][2] = f.z, v[u][3] = f.w;
        } else {
          const float2 f = *reinterpret_cast<const float2*>(po);
          v[u][0] = f.x, v[u][1] = f.y;
        }
      }
      float top = m;
      bool some = false;
#pragma unroll
      for (int u = 0; u < kMergeAhead; ++u) {
        top = fmaxf(top, ml[u].x);
        some |= ml[u].y != 0.0f;
      }
      if (!some) continue;
      const float keep = exp2f(m - top);
      m = top;
      l *= keep;
#pragma unroll
      for (int x = 0; x < D; ++x) o[x] *= keep;
#pragma unroll
      for (int u = 0; u < kMergeAhead; ++u) {
        if (ml[u].y == 0.0f) continue;  // a part in which the row sees nothing
        const float f = exp2f(ml[u].x - m);
        l = fmaf(ml[u].y, f, l);
#pragma unroll
        for (int x = 0; x < D; ++x) o[x] = fmaf(v[u][x], f, o[x]);
      }
    }
  }
  if (W > 1) {
    if (lane == 0) wml[warp] = make_float2(m, l);
#pragma unroll
    for (int x = 0; x < D; ++x) wo[warp][D * lane + x] = o[x];
    __syncthreads();
    if (w > 0) return;
    for (int k = 1; k < W; ++k) m = fmaxf(m, wml[warp + k].x);
    l = 0.0f;
#pragma unroll
    for (int x = 0; x < D; ++x) o[x] = 0.0f;
    for (int k = 0; k < W; ++k) {
      const float2 ml = wml[warp + k];
      if (ml.y == 0.0f) continue;
      const float f = exp2f(ml.x - m);
      l = fmaf(ml.y, f, l);
#pragma unroll
      for (int x = 0; x < D; ++x) o[x] = fmaf(wo[warp + k][D * lane + x], f, o[x]);
    }
  }
  if (!have) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const size_t at = size_t(sh.q0 + node) * p.n_heads + head;
  uint32_t* to = reinterpret_cast<uint32_t*>(p.o + at * HD + D * lane);
#pragma unroll
  for (int x = 0; x < D / 2; ++x) to[x] = pack_bf16(o[2 * x] * inv, o[2 * x + 1] * inv);
  if (p.lse && lane == 0) p.lse[at] = fmaf(m, 0.6931471805599453f, logf(l));
}

struct TreeTile {
  int group, chunk, chunks, nodes;
};
TreeTile tree_tile(int n_heads, int n_kv_heads) {
  TreeTile t;
  t.group = n_heads / n_kv_heads;
  t.chunk = std::min(t.group, 128);
  t.chunks = (t.group + 127) / 128;
  t.nodes = 128 / t.chunk;
  return t;
}
// Rows of a state in the workspace.
int rows_of_part(const TreeTile& t, int n_q) { return std::min(t.nodes, n_q) * t.chunk; }

// How the keys of a launch are split: clusters of `cluster` CTAs, and as many of them a tile as leave a CTA `share` blocks
// of keys. The choice minimises an estimate of the launch's time from what CTAs were measured to take (us, GB300): a CTA
// kCtaTime besides its blocks (its launch, the first loads, the last products), a block `alone` with the SM to itself and
// `pair` beside a second CTA (half an SM's share of HBM), a merge in the cluster, one through memory by the rows of its states.
// Where the CTAs do not fit on the GPU at once, later ones start as earlier ones end, at 1.3 times the even share of the
// work. Estimated / measured: one token, 321 keys, 32 heads, cluster 1 / 2 / 4 / 8: 13.2 / 10.6 / 8.8 / 8.2 and 12.6 / 11.4 / 8.6 /
// 9.2; 32 trees on 300 to 1958 keys, 4 K/V heads, no split / cluster 2 / 10 blocks a CTA, merged through memory: 43.2 / 30.9 /
// 29.8 and 53.7 / 37.9 / 31.3; eight of 48 nodes, 32 K/V heads, cluster 1 / 2 / 4: 41.4 / 49.2 / 65.4 and 41.8 / 48.0 / 63.2. A
// batch with more units than the GPU holds CTAs is not split by length: its time is that of its longest sequence.
constexpr double kCtaTime = 6.0, kClusterTime = 1.0, kMergeTime = 4.0, kMergeRow = 0.25e-3, kWaveFactor = 1.3;
constexpr int kMaxStates = kItems;  // states in memory of a launch: those of plans that fit on the GPU at once
struct TreeWork {  // a sequence of the launch: key blocks, (tile, K/V head) pairs, (node, head) rows
  int seq, blocks;
  long long units, rows;
};
struct TreePlan {
  int cluster = 1, share = 1 << 24;
  int groups(int blocks) const { return std::max(1, (blocks + share * cluster - 1) / (share * cluster)); }
};
struct TreeWorkList {
  TreeWork w[kMaxSeqs];
  int n = 0;
  const TreeWork* begin() const { return w; }
  const TreeWork* end() const { return w + n; }
};
// work: the longest first; places: CTAs the GPU holds at once.
TreePlan tree_plan(const TreeWorkList& work, int places, int head_dim) {
  const double alone = head_dim == 128 ? 1.2 : 1.1, pair = head_dim == 128 ? 1.54 : 1.39;
  TreePlan best;
  double least = 1e30;
  long long units = 0;
  double blocks_all = 0.0;
  for (const TreeWork& w : work) {
    units += w.units;
    blocks_all += double(w.units) * w.blocks;
  }
  for (int c = 1; c <= kMaxCluster; c *= 2) {
    // CTAs that fit in clusters: 304, 304, 288 and 256 of the 304 places of 152 SMs (the largest launches that ran as one wave)
    const int room = std::max(c, places - (c == 4 ? places / 19 : c == 8 ? 3 * places / 19 : 0));
    // the estimate of a plan, its CTAs in *ctas
    auto weigh = [&](const TreePlan& t, long long* ctas) {
      double longest = 0.0, merge = 0.0;
      long long all = 0, states = 0;
      for (const TreeWork& w : work) {
        const int g = t.groups(w.blocks);
        all += w.units * g * c;
        longest = std::max(longest, double(w.blocks) / (g * c));
        if (g > 1) {
          states += w.units * g;
          merge += kMergeRow * double(w.rows) * g;
        }
      }
      *ctas = all;
      double cost = kCtaTime + longest * (2 * all > room ? pair : alone);
      if (all > room) cost = std::max(cost, kCtaTime + kWaveFactor * (all * kCtaTime + blocks_all * pair) / room);
      cost += (c > 1 ? kClusterTime : 0.0) + (states ? kMergeTime + merge : 0.0);
      if (cost < least && states <= kMaxStates) {
        least = cost;
        best = t;
      }
    };
    long long ctas;
    TreePlan t;  // one group a sequence
    t.cluster = c;
    weigh(t, &ctas);
    if (ctas >= room || work.w[0].blocks <= c) continue;
    // more groups while all CTAs fit: the share can be no smaller than an even one
    int share = std::max(1, int(blocks_all / room));
    for (const int whole = (work.w[0].blocks + c - 1) / c; share < whole; share += share / 16 + 1) {
      t.share = share;
      const double before = least;
      const TreePlan was = best;
      weigh(t, &ctas);
      if (ctas <= room) break;
      least = before;
      best = was;
    }
  }
  return best;
}

}  // namespace

size_t tree_attention_bytes(int n_q, int n_heads, int n_kv_heads, int head_dim) {
  const size_t rows = size_t(kMaxStates) * rows_of_part(tree_tile(n_heads, n_kv_heads), n_q);
  Carve cv(nullptr, ~size_t(0));
  cv.take<float>(rows * head_dim);
  cv.take<float2>(rows);
  return cv.used;
}

int tree_attention_check(const int32_t* q_cu, int n_q, const int32_t* ctx, int n_seqs, const uint32_t* mask, int words,
                         int max_len) {
  if (q_cu[0] != 0 || q_cu[n_seqs] != n_q) return fail(SPD_EINVAL, "q_cu must run from 0 to n_q");
  for (int b = 0; b < n_seqs; ++b) {
    const int n = q_cu[b + 1] - q_cu[b];
    if (n < 0) return fail(SPD_EINVAL, "q_cu decreases at sequence %d", b);
    if (ctx[b] < 0 || ctx[b] > max_len - n)
      return fail(SPD_EINVAL, "sequence %d: context and drafts exceed max_len", b);
    if (mask && n > 32 * words) return fail(SPD_EINVAL, "sequence %d: %d nodes, %d mask words", b, n, words);
  }
  if ((long long)n_seqs * max_len > 0x7fffffffLL) return fail(SPD_EUNSUPPORTED, "more than 2^31 - 1 cache rows in a layer");
  return SPD_OK;
}

int tree_attention_run(const void* q, const int32_t* q_cu, const int32_t* ctx, int n_seqs, const uint32_t* mask, int words,
                       const void* kv, int max_len, int n_heads, int n_kv_heads, int head_dim, void* o, float* lse, void* ws,
                       size_t ws_bytes, int* status, cudaStream_t st) {
  const TreeTile t = tree_tile(n_heads, n_kv_heads);
  const int kvd = n_kv_heads * head_dim;
  CUtensorMap map;
  if (int rc = make_operand_map(&map, kv, 2 * kvd, n_seqs * max_len, kTK)) return rc;
  TreeArgs p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.mask = mask;
  p.words = words;
  p.kv = static_cast<const __nv_bfloat16*>(kv);
  p.max_len = max_len;
  p.n_heads = n_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = t.group;
  p.chunk = t.chunk;
  p.chunks = t.chunks;
  p.nodes_tile = t.nodes;
  p.scale_log2 = float(1.4426950408889634 / sqrt(double(head_dim)));
  p.o = static_cast<__nv_bfloat16*>(o);
  p.lse = lse;
  Carve cv(ws, ws_bytes);
  p.rows_part = rows_of_part(t, q_cu[n_seqs]);
  const size_t rows = size_t(kMaxStates) * p.rows_part;
  p.part_o = cv.take<float>(rows * head_dim);
  p.part_ml = cv.take<float2>(rows);
  p.status = status;
  p.budget = kWaitBudget;
  const auto kernel = head_dim == 128 ? tree_attn_kernel<128> : tree_attn_kernel<64>;
  const size_t smem = head_dim == 128 ? TreeSmem<128>::bytes : TreeSmem<64>::bytes;
  static DeviceOnce attr[2];
  SPD_CUDA_TRY(once_per_device(attr[head_dim == 128], [&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  }));
  const int places = std::min(kItems, 2 * num_sms());
  TreeWorkList work;
  for (int s0 = 0; s0 < n_seqs; s0 += kMaxSeqs) {
    const int m = std::min(kMaxSeqs, n_seqs - s0);
    work.n = 0;
    double pairs = 0.0, keys = 0.0;
    for (int b = s0; b < s0 + m; ++b) {
      const int n = q_cu[b + 1] - q_cu[b];
      if (n == 0) continue;
      work.w[work.n++] = {b, (ctx[b] + n + kTK - 1) / kTK,
                          (long long)((n + t.nodes - 1) / t.nodes) * t.chunks * n_kv_heads,
                          (long long)n * n_heads};
      keys += ctx[b] + n;
      pairs += double(n) * (ctx[b] + n);
    }
    if (work.n == 0) continue;
    std::stable_sort(work.w, work.w + work.n, [](const TreeWork& x, const TreeWork& y) { return x.blocks > y.blocks; });
    const TreePlan plan = tree_plan(work, places, head_dim);
    const int C = plan.cluster;
    TreeSeqs sq{};
    long long items = 0;
    int states = 0, most = 0, most_groups = 0, split = 0;  // split: sequences of several groups, the first ones
    for (const TreeWork& w : work) {
      const int n = q_cu[w.seq + 1] - q_cu[w.seq], k = plan.groups(w.blocks);
      sq.s[sq.n++] = {int(items), q_cu[w.seq], n, ctx[w.seq], w.seq, (n + t.nodes - 1) / t.nodes * t.chunks, k, states};
      if (k > 1) {
        ++split;
        states += int(w.units) * k;
        most = std::max(most, n);
        most_groups = std::max(most_groups, k);
      }
      items += w.units * k;
    }
    if (items * C > 0x7fffffff) return fail(SPD_EUNSUPPORTED, "tree attention of more than 2^31 tiles");
    if (states > kMaxStates) return fail(SPD_EUNSUPPORTED, "tree attention plan of %d states", states);
    p.cluster = C;
    const double fl = 4.0 * head_dim * n_heads * pairs;
    const double by = 4.0 * kvd * keys + 4.0 * n_heads * head_dim * (q_cu[s0 + m] - q_cu[s0]);
    p.stamp = stamp_slot(TR_ATTN, fl, by);
    const int slot = trace_begin(st);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(items) * C);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute la[2];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    la[1].id = cudaLaunchAttributeClusterDimension;
    la[1].val.clusterDim.x = C;
    la[1].val.clusterDim.y = 1;
    la[1].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = 2;
    SPD_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, map, p, sq));
    if (most > 0) {
      int W = 1;
      while (W < kMergeWarps && most_groups > kMergeAhead * W) W *= 2;
      SPD_CUDA_TRY(launch_pdl(head_dim == 128 ? tree_merge_kernel<128> : tree_merge_kernel<64>,
                              dim3((most * n_heads * W + kMergeWarps - 1) / kMergeWarps, split), dim3(kMergeWarps * 32), 0, st, p,
                              sq, W));
    }
    trace_end(slot, st, TR_ATTN, fl, by);
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
  }
  for (int b = 0; b < n_seqs; ++b) {  // (parent holds q_cu[n_seqs] entries, which no range passes now)
    for (int i = 0; i < q_cu[b + 1] - q_cu[b]; ++i) {
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
  return tree_attention_bytes(n_q, n_heads, n_kv_heads, head_dim);
}

extern "C" int spd_tree_attention(const uint16_t* q, int n_q, const int32_t* q_cu, const int32_t* ctx_len, int n_seqs,
                                  const uint32_t* tree_mask, int mask_words, const uint16_t* kv, int max_len, int n_heads,
                                  int n_kv_heads, int head_dim, uint16_t* o, float* lse, void* ws, size_t ws_bytes,
                                  void* stream) {
  if (!q || !q_cu || !ctx_len || !kv || !o || !ws || n_q < 1 || n_seqs < 1 || max_len < 1 || n_heads < 1 || n_kv_heads < 1 ||
      n_heads % n_kv_heads)
    return fail(SPD_EINVAL, "bad tree attention arguments");
  if (head_dim != 64 && head_dim != 128) return fail(SPD_EUNSUPPORTED, "tree attention supports head_dim 64 and 128");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(kv) | reinterpret_cast<uintptr_t>(o) |
       reinterpret_cast<uintptr_t>(ws)) & 15)
    return fail(SPD_EINVAL, "q, kv, o and ws must be 16-byte aligned");
  if (int rc = tree_attention_check(q_cu, n_q, ctx_len, n_seqs, tree_mask, mask_words, max_len)) return rc;
  const size_t need = tree_attention_bytes(n_q, n_heads, n_kv_heads, head_dim);
  if (ws_bytes < need) return fail(SPD_ENOSPC, "tree attention workspace too small (%zu < %zu)", ws_bytes, need);
  return tree_attention_run(q, q_cu, ctx_len, n_seqs, tree_mask, mask_words, kv, max_len, n_heads, n_kv_heads, head_dim, o, lse,
                            ws, ws_bytes, static_cast<int*>(ws), static_cast<cudaStream_t>(stream));
}
