// Attention of new tokens over a paged KV cache: chunks of prompts (paged_attn_kernel), single tokens (paged_token_kernel).
//
// New token i of sequence b, one of its n, sees rows 0 .. lim_i - 1 with lim_i = max(len - n + i + 1, prefix):
//   s_ij = q_i . k_j / sqrt(head_dim),  lse_i = log sum_j e^s_ij,  o_i = sum_j e^(s_ij - lse_i) v_j.
// What a row does not see contributes nothing, whatever it holds.
//
// A unit is a tile of up to 128 rows (tokens times the query heads of a K/V head's group) over the keys that its last token
// sees, in blocks of 64. A CTA has one unit, the longest units first, where that is about as even as it gets. Else all blocks of a
// launch form one list, unit after unit, and every CTA takes an equal stretch of it, whole units and parts of two: no CTA waits
// for a longest sequence, and 1.5 tiles a CTA cost 1.5 tiles. Parts of a unit leave states (m, l, O) in fp32, which
// paged_merge_kernel joins in the order of the keys (the same bits in every run).
//   warps 0-3  a thread a row: online softmax in fp32; a weight is held as the sum of two bf16 terms, 16 bits of it, both over
//              the scores in TMEM
//   warp 4     TMA producer: Q, and K and V blocks into rings, a lane a box of rows that lie in one page
//   warps 5, 6 MMA issuers: S = Q K^T into TMEM; O += P V with P read from TMEM, V in place as an MN-major operand
// Only blocks that reach past the first token's limit are masked; there the softmax warps also clear the values of V that are
// not finite (recycled memory behind the sequence among them), which a weight of zero would turn into NaN for rows that do not
// see them; rows that do see one add it at the end.
//
// What bounds chunks: the tensor pipe, with two products of P V a block 1792 cycles for a block of each of an SM's two CTAs at
// heads of 128 (a product of 128 x 64 x 16 with both operands in shared memory takes 48 cycles, not 32: it reads 6 KB), 900 at
// heads of 64, and what an SM's pairs of blocks take is 2050 and 1770. 2048 tokens behind 14333 rows, 28 heads on 4: 434 us, 1.04
// PFLOP/s of S and P V, 1.56 of what is issued; 2048 behind 14000, 16 heads of 64 on 8: 185 us. Heads of 64 are bound by the chain
// of a block: 350 cycles for scores and maximum, 600 for exponentials and terms, 300 between, 400 waiting for S.
// One warp that issued both products took 437 and 205 us (its instructions for a block were 1000 cycles and on the chain); two
// threads a row, with a barrier a block for what they have to agree on, 449 and 218.
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
constexpr int kThreads = 224;
constexpr uint32_t kTmemCols = 256;    // two buffers of S (64 columns) and 128 of O, or three and 64: half of an SM's 512
constexpr int kCtas = 304;             // CTAs that fill the GPU: two on each of 152 SMs
// The reference that a row's exponentials are taken against is renewed once its maximum has grown by this much (log2
// units): weights stay below 2^8, their terms and the fp32 sums are relative to them, and almost no block pays for the
// round trip of O through the registers.
constexpr float kGrown = 8.0f;

// A sequence with new tokens. Its units are (K/V head, tile), the tile fastest; the tiles of a head have head_blocks blocks.
struct PagedSeq {
  int block0;  // its first block in the launch's list
  int q0, n, len, prefix, seq, head_blocks, tiles;
};
struct PagedSeqs {
  int n, pad[7];
  PagedSeq s[kMaxSeqs];
};
struct PagedArgs {
  const __nv_bfloat16 *q, *pool;
  const int32_t* table;
  int max_pages, n_pages, page_size, box;  // box: rows that one TMA load brings (they divide the page and the block)
  int n_heads, n_kv_heads;
  int group, chunk, chunks, tokens;  // heads a group; of them in a tile; tiles across; tokens a tile
  int keys;                          // a block's
  float scale_log2;
  __nv_bfloat16* o;
  float* lse;
  bool whole;                        // a CTA has one unit (block0: a sequence's first), not an equal stretch of all blocks
  int box_rows;                      // tokens that a load of Q brings
  int total, ctas, share, more;      // stretches of share blocks, the first `more` of one more
  int warps;                         // of 32 rows of the tile
  float* part_o;                     // [2 ctas][rows_part HD] states of parts: slot 2 c of the part that goes on with a unit (CTA
  float2* part_ml;                   // c), 2 c + 1 of the one that begins one; [2 ctas][rows_part] maximum (log2 units) and sum
  int rows_part;
  bool by_row;                       // states [rows_part][HD], else [HD / 4][rows_part][4]
  int* status;
  long long budget;
  unsigned long long* stamp;
};

// Two terms a weight leave 2^-16 of it out, 1/256 of the step that the bf16 outputs are rounded by, and the sum of weights that
// divides them and gives lse is of the whole weights in fp32. A third term, as single tokens have it, is a third more products and
// needs shared memory that K or V then lack: 2048 tokens behind 14000, 28 heads of 128: 547 us, with two 449; 16 of 64: 260, 218.
// One term would be as coarse as the outputs.
template <int HD>
struct PagedSmem {
  static constexpr int kChunks = HD / 64;
  static constexpr int kBufs = HD == 128 ? 2 : 3;      // of S in TMEM, behind them O
  static constexpr int kStages = 3;                    // of K
  static constexpr int kStagesV = HD == 128 ? 2 : 3;
  static constexpr uint32_t q = 0;
  static constexpr uint32_t k = q + kChunks * kQBox;
  static constexpr uint32_t v = k + kStages * kChunks * kKBox;
  static constexpr uint32_t bars = v + kStagesV * kChunks * kKBox;
  static constexpr uint32_t bytes = bars + 256;  // (two CTAs an SM: at most 113 KB)
  static_assert(bytes <= 113 * 1024, "two CTAs an SM");
  static_assert(8 * (2 * kStages + 2 * kStagesV + 2 + 3 * kBufs + 1) + 12 <= bytes - bars, "room for the barriers");
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
// Two fp32 operations in one instruction.
struct Two {
  float lo, hi;
};
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.lo), "=f"(d.hi)
      : "f"(a.lo), "f"(a.hi), "f"(b.lo), "f"(b.hi), "f"(c.lo), "f"(c.hi));
  return d;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  Two d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.lo), "=f"(d.hi)
      : "f"(a.lo), "f"(a.hi), "f"(b.lo), "f"(b.hi));
  return d;
}
// The values of two bf16.
__device__ __forceinline__ Two two_of(uint32_t w) { return Two{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)}; }
__device__ __forceinline__ bool not_finite(uint32_t two) {  // either of two bf16
  return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite_of(uint32_t two) {  // those of two bf16 that are finite, 0 for the others
  if ((two & 0x7f80u) == 0x7f80u) two &= 0xffff0000u;
  return (two & 0x7f800000u) == 0x7f800000u ? two & 0xffffu : two;
}

// Rows that token i of a sequence sees.
__host__ __device__ __forceinline__ int limit_of(const PagedSeq& s, int i) {
  const int own = s.len - s.n + i + 1;
  return own > s.prefix ? own : s.prefix;
}
// Blocks of the tiles that begin with token i.
__host__ __device__ __forceinline__ int blocks_at(const PagedSeq& s, int i, int tokens, int keys) {
  const int last = i + tokens < s.n ? i + tokens : s.n;
  return int(uint32_t(limit_of(s, last - 1) + keys - 1) / uint32_t(keys));
}
// First block of CTA c's stretch.
__device__ __forceinline__ int first_block(const PagedArgs& p, int c) { return c * p.share + min(c, p.more); }
// CTAs whose stretches begin before block `at`.
__device__ __forceinline__ int ctas_before(const PagedArgs& p, int at) {
  const int wide = p.more * (p.share + 1);  // blocks of the stretches of one more
  return at <= wide ? int((uint32_t(at) + uint32_t(p.share)) / uint32_t(p.share + 1))
                    : p.more + int((uint32_t(at - wide) + uint32_t(p.share) - 1u) / uint32_t(p.share));
}

// A CTA's place in the list of blocks: the unit (sequence e, K/V head hk, tile), its blocks, and the stretch's blocks lo .. hi - 1
// of them.
struct Place {
  int e, hk, tile, blocks, lo, hi, left;  // left: blocks of the stretch from lo on
  __device__ __forceinline__ void size(const PagedArgs& p, const PagedSeqs& sq) {
    blocks = blocks_at(sq.s[e], tile / p.chunks * p.tokens, p.tokens, p.keys);
    hi = min(blocks, lo + left);
  }
  // CTA c's stretch (a whole warp, all lanes with the same arguments); its number of blocks.
  __device__ __forceinline__ int begin(const PagedArgs& p, const PagedSeqs& sq, int c) {
    if (!p.whole) {
      const int at = first_block(p, c);
      seek(p, sq, at, first_block(p, c + 1) - at);
      return left;
    }
    find(sq, c);  // a sequence's last tiles, the longest, first
    const int x = c - sq.s[e].block0, back = int(uint32_t(x) / uint32_t(p.n_kv_heads));
    hk = x - back * p.n_kv_heads;
    tile = sq.s[e].tiles - 1 - back;
    lo = 0;
    left = 1 << 30;
    size(p, sq);
    return left = blocks;
  }
  // The last sequence that begins at or before `at`.
  __device__ __forceinline__ void find(const PagedSeqs& sq, int at) {
    e = 0;
    for (int top = sq.n; top - e > 1;) {
      const int mid = (e + top) >> 1;
      if (sq.s[mid].block0 <= at) e = mid;
      else top = mid;
    }
  }
  // The unit of block `at` of the list, `n` blocks from there on.
  __device__ __forceinline__ void seek(const PagedArgs& p, const PagedSeqs& sq, int at, int n) {
    find(sq, at);
    const PagedSeq& s = sq.s[e];
    lo = at - s.block0;
    hk = int(uint32_t(lo) / uint32_t(s.head_blocks));
    lo -= hk * s.head_blocks;
    const int lane = threadIdx.x & 31;
    for (int t0 = 0;; t0 += 32) {
      const int t = t0 + lane, mine = t < s.tiles ? blocks_at(s, t / p.chunks * p.tokens, p.tokens, p.keys) : 0;
      int sum = mine;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, off);
        if (lane >= off) sum += y;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, sum > lo);
      if (past || t0 + 32 >= s.tiles) {
        const int at_lane = past ? __ffs(past) - 1 : 0;
        lo -= __shfl_sync(0xffffffffu, sum - mine, at_lane);
        tile = t0 + at_lane;
        break;
      }
      lo -= __shfl_sync(0xffffffffu, sum, 31);
    }
    left = n;
    size(p, sq);
  }
  __device__ __forceinline__ bool next(const PagedArgs& p, const PagedSeqs& sq) {
    left -= hi - lo;
    if (left <= 0) return false;
    lo = 0;
    if (++tile == sq.s[e].tiles) {
      tile = 0;
      if (++hk == p.n_kv_heads) {
        hk = 0;
        ++e;
      }
    }
    size(p, sq);
    return true;
  }
};

// Products and commits by a whole warp in step, of which one lane issues: descriptors then stay in uniform registers. (A lane on
// its own moves every operand there for each product: 1000 cycles a block of keys, and more than the products take.)
__device__ __forceinline__ void issue_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
      : "memory");
}
__device__ __forceinline__ void issue_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
      : "memory");
}
__device__ __forceinline__ void issue_commit(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
      : "memory");
}
// A value that all lanes hold, in a uniform register.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_max_sync(0xffffffffu, x); }

// Row of the pool that holds row `key` of a sequence; behind the pool (loads there read zeros) where its page is none.
__device__ __forceinline__ int pool_row(const PagedArgs& p, int seq, int key) {
  const int k = int(uint32_t(key) / uint32_t(p.page_size)), page = p.table[size_t(seq) * p.max_pages + k];
  if (unsigned(page) >= unsigned(p.n_pages)) {
    set_status(p.status, SPD_EINVAL);
    return p.n_pages * p.page_size;
  }
  return page * p.page_size + (key - k * p.page_size);
}

template <int HD>
__global__ void __launch_bounds__(kThreads, 2)
    paged_attn_kernel(const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_q,
                      const __grid_constant__ PagedArgs p,
                      const __grid_constant__ PagedSeqs sq) {
  using L = PagedSmem<HD>;
  constexpr int NS = L::kStages, NV = L::kStagesV, NB = L::kBufs;
  extern __shared__ __align__(1024) uint8_t smem[];  // (the swizzle's atoms; no room to round the address up)
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + L::bars);  // [NS] K block landed
  uint64_t* k_empty = k_full + NS;                                 // [NS] its S product has completed
  uint64_t* v_full = k_empty + NS;                                 // [NV] V block landed
  uint64_t* v_empty = v_full + NV;                                 // [NV] its PV products have completed
  uint64_t* q_full = v_empty + NV;   // a unit's Q tile is in shared memory
  uint64_t* q_empty = q_full + 1;    // its S products have completed
  uint64_t* s_full = q_empty + 1;    // [NB] S of block j is in TMEM buffer j % NB
  uint64_t* p_full = s_full + NB;    // [NB] P of block j written and O rescaled
  uint64_t* o_done = p_full + NB;    // [NB] PV products of block j completed
  uint64_t* drain = o_done + NB;     // every MMA completed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* odd_v = reinterpret_cast<int*>(tmem_slot + 2);  // the last unit (counted from 1) with a V that is not finite

  if (smem_u32(smem) & 1023) {  // every CTA alike
    pdl_wait();
    if (threadIdx.x == 0) set_status(p.status, SPD_ECUDA);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nw = p.warps;
  Place at;
  const int count = at.begin(p, sq, int(blockIdx.x));
  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
    }
    for (int s = 0; s < NV; ++s) {
      mbar_init(&v_full[s], 1);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int s = 0; s < NB; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&p_full[s], nw);  // one arrival per softmax warp
      mbar_init(&o_done[s], 1);
    }
    mbar_init(drain, 2);
    *abort_flag = 0;
    *odd_v = 0;
    fence_mbar_init();
    prefetch_tmap(&map_kv);
    prefetch_tmap(&map_q);
  }
  if (warp == 4) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t t_o = tmem + NB * kTK;

  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x == 0) stamp_start(p.stamp);

  int issued_q = 0, issued_k = 0, issued_v = 0;
  if (warp == 4) {
    // ---- TMA producer ----
    const uint64_t pol = policy_evict_last();
    const int boxes = kTK / p.box;
    int j = 0;  // block of the CTA
    bool ok = true;
    do {
      const PagedSeq& s = sq.s[at.e];
      {  // the tile's rows: `chunk` heads of a token side by side
        if (issued_q > 0 && !(ok = __all_sync(0xffffffffu, mbar_wait(q_empty, (issued_q - 1) & 1, abort_flag, p.budget)))) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(q_full, uint32_t(L::kChunks * 128 * p.chunk * p.box_rows));
          const int across = at.tile / p.chunks, h0 = (at.tile - across * p.chunks) * p.chunk;
          for (int c = 0; c < L::kChunks; ++c)
            tma_load_3d(smem + L::q + c * kQBox, &map_q, q_full, c * 64, at.hk * p.group + h0, s.q0 + across * p.tokens, pol);
        }
        __syncwarp();
        ++issued_q;
      }
      const int t = at.tile / p.chunks * p.tokens, limit = limit_of(s, min(s.n, t + p.tokens) - 1);
      auto row_at = [&](int blk) {  // of the lane's box; -1: none of its rows is seen
        const int key = blk * kTK + lane * p.box;
        return lane < boxes && key < limit ? pool_row(p, s.seq, key) : -1;
      };
      int row = row_at(at.lo);
      for (int blk = at.lo; blk < at.hi && ok; ++blk, ++j) {
        const int here = row;
        if (blk + 1 < at.hi) row = row_at(blk + 1);  // a block ahead
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, here >= 0)) * p.box * 128u * L::kChunks;
        auto load = [&](uint64_t* full, uint64_t* empty, int stages, uint32_t to, int x0) -> bool {
          const int st = j % stages;
          if (j >= stages && !__all_sync(0xffffffffu, mbar_wait(&empty[st], (j / stages - 1) & 1, abort_flag, p.budget)))
            return false;
          if (lane == 0) mbar_arrive_expect_tx(&full[st], bytes);
          __syncwarp();
          if (here >= 0)
            for (int c = 0; c < L::kChunks; ++c)
              tma_load_2d(smem + to + (st * L::kChunks + c) * kKBox + lane * p.box * 128, &map_kv, &full[st], x0 + c * 64, here, pol);
          return true;
        };
        if (!(ok = load(k_full, k_empty, NS, L::k, at.hk * HD))) break;
        issued_k = j + 1;
        if (!(ok = load(v_full, v_empty, NV, L::v, (p.n_kv_heads + at.hk) * HD))) break;
        issued_v = j + 1;
      }
    } while (ok && at.next(p, sq));
    if (!ok && lane == 0) {
      *abort_flag = 1;
      set_status(p.status, SPD_ETIMEOUT);
    }
  } else if (warp == 5 || warp == 6) {
    // ---- MMA issuers, all lanes in step: warp 5 the scores, warp 6 the products with V ----
    // Their loops are short because a block's instructions here are on its critical path: even lanes watch one of the two
    // barriers that a block waits for, odd lanes the other.
    const uint32_t base = smem_u32(smem), t_all = uniform(tmem);
    const int blocks = int(uniform(uint32_t(count)));
    const bool odd = lane & 1;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.budget)) != 0; };
    int stage = 0, buf = 0;              // of K or V, of S and P
    uint32_t round = 0, buf_round = 0;   // parity of their rounds
    int unit_end = at.hi - at.lo;        // the first block behind the unit
    bool ok = true, first = true;        // of the unit
    if (warp == 5) {
      constexpr uint32_t id_s = idesc_bf16_f32(128, kTK);
      uint32_t q_round = 0;
      for (int j = 0; j < blocks; ++j) {
        if (first) {
          if (!(ok = wait(q_full, q_round))) break;
          q_round ^= 1;
          first = false;
        }
        // (the buffer's last P has been multiplied; none before the first round, whose parity a new barrier has completed)
        if (!(ok = wait(odd ? &o_done[buf] : &k_full[stage], odd ? buf_round ^ 1 : round))) break;
        tc_fence_after();
        const uint64_t dk = sdesc_k128(base + L::k + stage * L::kChunks * kKBox), dq = sdesc_k128(base + L::q);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk)
          issue_ss(t_all + kTK * buf, dq + (((kk >> 2) * kQBox + (kk & 3) * 32) >> 4),
                   dk + (((kk >> 2) * kKBox + (kk & 3) * 32) >> 4), id_s, kk > 0);
        issue_commit(&s_full[buf]);
        issue_commit(&k_empty[stage]);
        if (++stage == NS) stage = 0, round ^= 1;
        if (++buf == NB) buf = 0, buf_round ^= 1;
        if (j + 1 == unit_end) {
          issue_commit(q_empty);
          at.next(p, sq);
          unit_end += at.hi - at.lo;
          first = true;
        }
      }
    } else {
      constexpr uint32_t id_o = idesc_bf16_f32(128, HD) | (1u << 16);  // V is MN-major
      for (int j = 0; j < blocks; ++j) {
        if (!(ok = wait(odd ? &p_full[buf] : &v_full[stage], odd ? buf_round : round))) break;
        tc_fence_after();
        const uint32_t t_o_all = t_all + NB * kTK, t_p = t_all + kTK * buf;
        const uint64_t dv = sdesc_mn128(base + L::v + stage * L::kChunks * kKBox, kKBox);
#pragma unroll
        for (int kk = 0; kk < 2 * (kTK / 16); ++kk) {  // the weights' first terms, then their second
          const int k = kk % (kTK / 16), term = kk / (kTK / 16);
          issue_ts(t_o_all, t_p + 16 * k + 8 * term, dv + ((k * 2048) >> 4), id_o, !first || kk > 0);
        }
        issue_commit(&o_done[buf]);
        issue_commit(&v_empty[stage]);
        first = false;
        if (++stage == NV) stage = 0, round ^= 1;
        if (++buf == NB) buf = 0, buf_round ^= 1;
        if (j + 1 == unit_end) {
          at.next(p, sq);
          unit_end += at.hi - at.lo;
          first = true;
        }
      }
    }
    if (!ok) {
      *abort_flag = 1;
      set_status(p.status, SPD_ETIMEOUT);
    }
    issue_commit(drain);  // arrives once every MMA issued above has completed
    volatile int no_abort = 0;
    if (!mbar_wait(drain, 0, &no_abort, p.budget)) set_status(p.status, SPD_ETIMEOUT);
  } else if (warp < nw) {
    // ---- softmax: warp w has TMEM lanes [32 w, 32 w + 32) of S, P and O ----
    const int r = threadIdx.x, T = nw * 32;
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    const uint32_t t_oh = t_o + lanes;
    auto any = [](bool mine) { return __any_sync(0xffffffffu, mine) != 0; };
    // a unit's rows: the thread's token, head and query row
    struct Row {
      int token;
      bool valid;
      size_t row;  // token of the call times n_heads + head
    };
    auto row_of = [&](const Place& u) {
      const PagedSeq& s = sq.s[u.e];
      const int t = u.tile / p.chunks, h0 = (u.tile - t * p.chunks) * p.chunk, n0 = t * p.tokens;
      const int tokens = min(p.tokens, s.n - n0), heads = min(p.chunk, p.group - h0), hc = r % p.chunk;
      Row w;
      w.token = n0 + min(r / p.chunk, tokens - 1);  // rows without a token repeat the last one's, and are not stored
      w.valid = r < tokens * p.chunk && hc < heads;
      w.row = (size_t(s.q0) + w.token) * p.n_heads + u.hk * p.group + h0 + min(hc, heads - 1);
      return w;
    };
    bool ok = true;
    int j = 0;  // block of the CTA
    for (int unit = 0;; ++unit) {
      const PagedSeq& s = sq.s[at.e];
      const Row now = row_of(at);
      const int n0 = at.tile / p.chunks * p.tokens;
      const int lim = limit_of(s, now.token);                            // what the row sees,
      const int lim_all = limit_of(s, n0), lim_any = limit_of(s, min(s.n, n0 + p.tokens) - 1);  // every row, some row
      float m_run = -INFINITY, l_run = 0.0f;  // the row's reference (raw scores); the thread's sum of weights
      for (int blk = at.lo; blk < at.hi; ++blk, ++j) {
        const uint32_t t_s = tmem + kTK * (j % NB) + lanes;
        const int kb = blk * kTK;
        const bool partly = kb + kTK > lim_all;  // the block holds keys that not every row sees, or none at all
        if (partly) {
          ok = ok && mbar_wait(&v_full[j % NV], (j / NV) & 1, abort_flag, p.budget);
          bool odd = false;
          for (int x = r; x < kTK * L::kChunks * 8; x += T) {  // 16 bytes each
            const int key = kb + (x >> 3) % kTK;
            if (key < lim_all) continue;
            uint4* at_v = reinterpret_cast<uint4*>(smem + L::v + (j % NV) * L::kChunks * kKBox) + x;
            const uint4 w = *at_v;
            if (not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w)) {
              *at_v = make_uint4(finite_of(w.x), finite_of(w.y), finite_of(w.z), finite_of(w.w));
              odd |= key < lim_any;
            }
          }
          if (odd) atomicMax(odd_v, unit + 1);
          fence_proxy_async_smem();
          // (every softmax warp arrives on p_full after its share, so the products see all of them)
        }
        ok = ok && mbar_wait(&s_full[j % NB], (j / NB) & 1, abort_flag, p.budget);
        __syncwarp();
        tc_fence_after();
        float v[kTK];
        tmem_ld64(t_s, v);
        if (partly) {
          const int sees = lim - kb;
#pragma unroll
          for (int i = 0; i < kTK; ++i)
            if (i >= sees) v[i] = -INFINITY;
        }
        float m4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int i = 4; i < kTK; ++i) m4[i & 3] = fmaxf(m4[i & 3], v[i]);
        const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
        if (any(blk == at.lo || (mx - m_run) * p.scale_log2 > kGrown || !ok)) {
          // the references are taken anew. O can be rescaled once the products before have completed
          if (blk > at.lo) ok = ok && mbar_wait(&o_done[(j - 1) % NB], ((j - 1) / NB) & 1, abort_flag, p.budget);
          if (any(!ok)) {
            ok = false;
            break;
          }
          // (a row whose maximum has not grown keeps its reference: its bits do not hang on its neighbours' values)
          const float m_new = blk == at.lo || (mx - m_run) * p.scale_log2 > kGrown ? fmaxf(m_run, mx) : m_run;
          const float corr = m_new == m_run ? 1.0f : ex2((m_run - m_new) * p.scale_log2);
          m_run = m_new;
          l_run *= corr;
          if (blk > at.lo) {
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < HD; c += 8) {
              float ov[8];
              tmem_ld8(t_oh + c, ov);
#pragma unroll
              for (int i = 0; i < 8; ++i) ov[i] *= corr;
              tmem_st8(t_oh + c, ov);
            }
            tmem_st_wait();
          }
        }
        const float off = m_run == -INFINITY ? 0.0f : m_run * p.scale_log2;  // nothing seen yet: all weights are 0
        const Two scale{p.scale_log2, p.scale_log2}, less{-off, -off}, minus{-1.0f, -1.0f};
        Two sum[2] = {Two{0.0f, 0.0f}, Two{0.0f, 0.0f}};
#pragma unroll
        for (int x = 0; x < kTK / 16; ++x) {
          float first_t[8], second_t[8];  // the terms of keys 16 x + 2 i and 16 x + 2 i + 1 in word i
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int k = 16 * x + 2 * i;
            Two w = fma2(Two{v[k], v[k + 1]}, scale, less);
            w = Two{ex2(w.lo), ex2(w.hi)};
            sum[i & 1] = add2(sum[i & 1], w);
            const uint32_t hi = pack_bf16(w.lo, w.hi);
            w = fma2(two_of(hi), minus, w);  // what is left
            const uint32_t mid = pack_bf16(w.lo, w.hi);
            first_t[i] = __uint_as_float(hi);
            second_t[i] = __uint_as_float(mid);
          }
          tmem_st8(t_s + 16 * x, first_t);  // over the scores
          tmem_st8(t_s + 16 * x + 8, second_t);
        }
        l_run += (sum[0].lo + sum[0].hi) + (sum[1].lo + sum[1].hi);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[j % NB]);
      }
      if (!ok) break;
      ok = mbar_wait(&o_done[(j - 1) % NB], ((j - 1) / NB) & 1, abort_flag, p.budget);
      if (any(!ok)) {
        ok = false;
        break;
      }
      __syncwarp();
      tc_fence_after();
      // A V that every row sees and that is infinite: the products of a weight's terms, which can be 0 or negative, are NaN
      // together. Which infinity a column has is the same for every row (each has a weight above 0 for it).
      float sick = 0.0f;  // NaN where a column is not finite
#pragma unroll 1
      for (int c = 0; c < HD; c += 32) {
        float v[32];
        tmem_ld32(t_oh + c, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) sick = fmaf(v[i], 0.0f, sick);
      }
      const int key0 = at.lo * kTK, key1 = min(at.hi * kTK, lim_any);
      const __nv_bfloat16* vcol = p.pool + (size_t(p.n_kv_heads) + at.hk) * HD;
      const size_t ld = 2 * size_t(p.n_kv_heads) * HD;
      const int rows_all = p.n_pages * p.page_size;
      const bool mend = now.valid && isnan(sick) && !isnan(l_run);  // (scores that are NaN leave the row NaN)
      if (__any_sync(0xffffffffu, mend)) {
        constexpr int E = HD / 32;  // columns a lane looks through
        uint32_t has = 0;  // of column e in bits 4 e: +inf, -inf, NaN
        for (int k = key0; k < min(lim_all, key1); ++k) {
          const int at_row = pool_row(p, s.seq, k);
          if (at_row >= rows_all) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float x = __bfloat162float(vcol[at_row * ld + E * lane + e]);
            has |= (isnan(x) ? 4u : x == INFINITY ? 1u : x == -INFINITY ? 2u : 0u) << (4 * e);
          }
        }
#pragma unroll 1
        for (int c = 0; c < HD; c += 8) {
          float ov[8];
          tmem_ld8(t_oh + c, ov);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t h = (__shfl_sync(0xffffffffu, has, (c + i) / E) >> (4 * ((c + i) % E))) & 15u;
            if (mend && isnan(ov[i]) && (h == 1u || h == 2u)) ov[i] = h == 1u ? INFINITY : -INFINITY;
          }
          tmem_st8(t_oh + c, ov);
        }
        tmem_st_wait();
      }
      // (a warp that is a unit ahead may raise it meanwhile: the lanes, which work together below, decide together)
      if (any(*reinterpret_cast<volatile int*>(odd_v) > unit)) {
        // values of V that were cleared: rows that see one add p v in fp32 (the score again from q and k)
        const float off = m_run == -INFINITY ? 0.0f : m_run * p.scale_log2;
        const __nv_bfloat16* qsrc = p.q + now.row * HD;
        for (int k = max(lim_all, key0); k < key1; ++k) {
          const int at_row = pool_row(p, s.seq, k);
          if (at_row >= rows_all) continue;
          const bool sees = now.valid && k < lim;
          const __nv_bfloat16* kr = p.pool + at_row * ld + at.hk * HD;
          const __nv_bfloat16* vr = vcol + at_row * ld;
          bool some = false;
          for (int x = lane; x < HD; x += 32) some |= !isfinite(__bfloat162float(vr[x]));
          if (!__any_sync(0xffffffffu, some)) continue;
          float d = 0.0f;
          if (sees)
            for (int x = 0; x < HD; ++x) d = fmaf(__bfloat162float(qsrc[x]), __bfloat162float(kr[x]), d);
          const float w = ex2(fmaf(d, p.scale_log2, -off));
          __syncwarp();
#pragma unroll 1
          for (int c = 0; c < HD; c += 8) {
            float ov[8];
            tmem_ld8(t_oh + c, ov);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x = __bfloat162float(vr[c + i]);
              if (sees && !isfinite(x)) ov[i] = fmaf(w, x, ov[i]);
            }
            tmem_st8(t_oh + c, ov);
          }
          tmem_st_wait();
        }
      }
      // the outputs, or the part's state
      const bool part = at.hi - at.lo < at.blocks;
      const size_t slot = (2 * size_t(blockIdx.x) + (at.lo == 0)) * p.rows_part + r;
      const float m2 = m_run * p.scale_log2, inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
      if (now.valid) {
        if (part) p.part_ml[slot] = make_float2(m2, l_run);
        else if (p.lse) p.lse[now.row] = fmaf(m2, 0.6931471805599453f, logf(l_run));
      }
#pragma unroll 1
      for (int c = 0; c < HD; c += 32) {
        float v[32];
        __syncwarp();
        tmem_ld32(t_oh + c, v);
        if (!now.valid) continue;
        if (part) {
          // [HD / 4][rows_part][4]: the rows of a warp side by side; few rows: [rows_part][HD]
          float4* po = reinterpret_cast<float4*>(p.part_o) + (p.by_row ? slot * (HD / 4) : (slot - r) * (HD / 4) + r);
          const int step = p.by_row ? 1 : p.rows_part;
#pragma unroll
          for (int y = 0; y < 8; ++y)
            po[((c) / 4 + y) * step] = make_float4(v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
        } else {
          uint4* to = reinterpret_cast<uint4*>(p.o + now.row * HD + c);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            to[y] = make_uint4(pack_bf16(v[8 * y] * inv, v[8 * y + 1] * inv), pack_bf16(v[8 * y + 2] * inv, v[8 * y + 3] * inv),
                               pack_bf16(v[8 * y + 4] * inv, v[8 * y + 5] * inv), pack_bf16(v[8 * y + 6] * inv, v[8 * y + 7] * inv));
        }
      }
      tc_fence_before();  // (O is written again by products that wait for this warp's next arrival)
      if (!at.next(p, sq)) break;
    }
    if (!ok) {
      *abort_flag = 1;
      set_status(p.status, SPD_ETIMEOUT);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 128 && *abort_flag) {
    // loads issued but never consumed land before the CTA exits
    volatile int no_abort = 0;
    if (issued_q > 0) mbar_wait(q_full, (issued_q - 1) & 1, &no_abort, p.budget);
    for (int j = max(0, issued_k - NS); j < issued_k; ++j) mbar_wait(&k_full[j % NS], (j / NS) & 1, &no_abort, p.budget);
    for (int j = max(0, issued_v - NV); j < issued_v; ++j) mbar_wait(&v_full[j % NV], (j / NV) & 1, &no_abort, p.budget);
  }
  __syncwarp();
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, kTmemCols);
  if (threadIdx.x == 0) stamp_end(p.stamp);
}

// ---- single tokens --------------------------------------------------------------------------------
// A sequence's one new token with up to 16 query heads a K/V head: too few rows to fill an MMA's 128, so keys and dims are its
// rows: S^T = K Q^T (128 keys x 16 heads), O^T += V^T P^T (128 dims x 64; of heads of 64 the other half is what lies behind V,
// and is not read), V in place as an MN-major operand, P^T through shared memory. P^T's columns are the three bf16 terms of every
// head's weights, side by side (48 of 64), all 24 bits of them (the tensor pipe has the time): V is read once for all of them
// and a term that is zero or negative does not meet an infinite V in another's sum. One CTA an SM, 192 KB of K and V on their way.
// What bounds it: the stream of K and V. 48 sequences over 301 to 8432 rows, 28 heads on 4: 0.43 GB in 75 us, 5.7 TB/s; a token
// over 322 rows of 32 heads 7.5 us, a chain of launch, first loads, product, exponentials, product, output.
//   warp 4     TMA producer          warp 5     MMA issuer          warp 6     the units' Q, a unit ahead
//   warps 0-3  a thread a key: exponentials against a reference a head, renewed for all of them once a score has
//              outgrown one by kGrown; sums a thread, added up at the end. In the end a thread a dim: O out of TMEM.
constexpr int kTokenKeys = 128, kTokenHeads = 16;
constexpr int kTokenThreads = 224;
template <int HD>
struct TokenSmem {
  static constexpr int kStages = 384 / HD, kChunks = HD / 64;
  static constexpr uint32_t box = kTokenKeys * 128;        // 64 columns of a block of K or V
  static constexpr uint32_t qbox = kTokenHeads * 128;      // 64 columns of Q
  static constexpr uint32_t k = 0;
  static constexpr uint32_t v = k + kStages * kChunks * box;
  static constexpr uint32_t p = v + kStages * kChunks * box;  // [128 keys][64]
  static constexpr uint32_t q = p + box;                      // two units'
  static constexpr uint32_t bars = q + 2 * kChunks * qbox;
  static constexpr uint32_t red = bars + 320;                 // [4 warps][16]
  static constexpr uint32_t bytes = red + 256;
  static_assert(bytes <= 227 * 1024, "one CTA an SM");
  static_assert(8 * (4 * kStages + 9) + 8 <= red - bars, "room for the barriers");
};
__device__ __forceinline__ void sync_softmax() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool any_softmax(bool mine) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred a, b;\n\tsetp.ne.u32 a, %1, 0;\n\tbarrier.cta.red.or.pred b, 2, 128, a;\n\tselp.u32 %0, 1, 0, b;\n\t}"
      : "=r"(all)
      : "r"(uint32_t(mine))
      : "memory");
  return all != 0;
}
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t u) { return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u); }

// R: heads a thread works on, 8 or 16 (those past the group's are of zeros and are not stored).
template <int HD, int R>
__global__ void __launch_bounds__(kTokenThreads, 1)
    paged_token_kernel(const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap,
                       const __grid_constant__ PagedArgs p, const __grid_constant__ PagedSeqs sq) {
  using L = TokenSmem<HD>;
  constexpr int NS = L::kStages, NC = L::kChunks;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + L::bars);  // [NS] K block landed
  uint64_t* k_empty = k_full + NS;                                 // [NS] its product has completed
  uint64_t* v_full = k_empty + NS;
  uint64_t* v_empty = v_full + NS;
  uint64_t* q_full = v_empty + NS;   // [2] unit u's Q is in buffer u % 2
  uint64_t* q_empty = q_full + 2;    // [2] its products have completed
  uint64_t* s_full = q_empty + 2;    // [2] S of block j is in TMEM buffer j % 2
  uint64_t* p_full = s_full + 2;     // P of the block written and O rescaled
  uint64_t* o_done = p_full + 1;     // PV product of the block completed
  uint64_t* drain = o_done + 1;      // every MMA completed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* red = reinterpret_cast<float*>(smem + L::red);

  if (smem_u32(smem) & 1023) {  // every CTA alike
    pdl_wait();
    if (threadIdx.x == 0) set_status(p.status, SPD_ECUDA);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Place at;
  const int count = at.begin(p, sq, int(blockIdx.x));
  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_full[s], 1);
      mbar_init(&v_empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&q_full[s], 1);
      mbar_init(&q_empty[s], 1);
      mbar_init(&s_full[s], 1);
    }
    mbar_init(p_full, 4);  // one arrival per softmax warp
    mbar_init(o_done, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&map_kv);
  }
  for (uint32_t i = threadIdx.x; i < L::box / 16; i += kTokenThreads)  // the columns that nobody writes are zero
    reinterpret_cast<uint4*>(smem + L::p)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  if (warp == 4) {
    tmem_alloc(tmem_slot, 128);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t t_o = tmem + 64;  // S: two buffers of 16 columns

  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x == 0) stamp_start(p.stamp);

  int issued_k = 0, issued_v = 0;
  bool ok = true;
  if (warp == 4) {
    // ---- TMA producer ----
    const uint64_t pol = policy_evict_first();
    const int boxes = kTokenKeys / p.box;
    int j = 0;  // block of the CTA
    do {
      const PagedSeq& s = sq.s[at.e];
      auto row_at = [&](int blk) {  // of the lane's box; -1: none of its rows is there
        const int key = blk * kTokenKeys + lane * p.box;
        return lane < boxes && key < s.len ? pool_row(p, s.seq, key) : -1;
      };
      int row = row_at(at.lo);
      for (int blk = at.lo; blk < at.hi && ok; ++blk, ++j) {
        const int here = row;
        if (blk + 1 < at.hi) row = row_at(blk + 1);  // a block ahead
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, here >= 0)) * p.box * 128u * NC;
        const int st = j % NS;
        auto load = [&](uint64_t* full, uint64_t* empty, uint32_t to, int x0) -> bool {
          if (j >= NS && !__all_sync(0xffffffffu, mbar_wait(&empty[st], (j / NS - 1) & 1, abort_flag, p.budget))) return false;
          if (lane == 0) mbar_arrive_expect_tx(&full[st], bytes);
          __syncwarp();
          if (here >= 0)
            for (int c = 0; c < NC; ++c)
              tma_load_2d(smem + to + (st * NC + c) * L::box + lane * p.box * 128, &map_kv, &full[st], x0 + c * 64, here, pol);
          return true;
        };
        if (!(ok = load(k_full, k_empty, L::k, at.hk * HD))) break;
        issued_k = j + 1;
        if (!(ok = load(v_full, v_empty, L::v, (p.n_kv_heads + at.hk) * HD))) break;
        issued_v = j + 1;
      }
    } while (ok && at.next(p, sq));
  } else if (warp == 5) {
    // ---- MMA issuer (all lanes in step) ----
    const uint32_t id_s = idesc_bf16_f32(128, kTokenHeads);
    const uint32_t id_o = idesc_bf16_f32(128, 64) | (3u << 15);  // V and P are MN-major
    const uint32_t base = smem_u32(smem), t_all = uniform(tmem);
    auto wait = [&](uint64_t* bar, int phase) { return __all_sync(0xffffffffu, mbar_wait(bar, phase & 1, abort_flag, p.budget)) != 0; };
    auto issue_s = [&](int j, int unit) -> bool {
      const int s = j % NS;
      if (!wait(&k_full[s], j / NS)) return false;
      // (the scores of block j - 2 have been read: its weights have arrived)
      tc_fence_after();
      const uint64_t dk = sdesc_k128(base + L::k + s * NC * L::box), dq = sdesc_k128(base + L::q + (unit & 1) * NC * L::qbox);
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk)
        issue_ss(t_all + kTokenHeads * (j & 1), dk + (((kk >> 2) * L::box + (kk & 3) * 32) >> 4),
                 dq + (((kk >> 2) * L::qbox + (kk & 3) * 32) >> 4), id_s, kk > 0);
      issue_commit(&s_full[j & 1]);
      issue_commit(&k_empty[s]);
      return true;
    };
    int j = 0, unit = 0;
    int n = at.hi - at.lo;  // blocks of the unit
    ok = wait(&q_full[0], 0) && issue_s(0, 0);
    while (ok) {
      Place then = at;
      const bool more = then.next(p, sq);
      for (int u = 0; u < n && ok; ++u, ++j) {
        const int s = j % NS;
        if (u + 1 < n) {
          if (!(ok = issue_s(j + 1, unit))) break;
        } else {
          issue_commit(&q_empty[unit & 1]);
          // the next unit's first block
          if (more && !(ok = wait(&q_full[(unit + 1) & 1], (unit + 1) >> 1) && issue_s(j + 1, unit + 1))) break;
        }
        if (!(ok = wait(&v_full[s], j / NS))) break;
        if (!(ok = wait(p_full, j))) break;
        tc_fence_after();
        const uint64_t dv = sdesc_mn128(base + L::v + s * NC * L::box, L::box), dp = sdesc_mn128(base + L::p, L::box);
#pragma unroll
        for (int x = 0; x < kTokenKeys / 16; ++x)
          issue_ss(t_all + 64, dv + ((x * 2048) >> 4), dp + ((x * 2048) >> 4), id_o, u > 0 || x > 0);
        issue_commit(o_done);
        issue_commit(&v_empty[s]);
      }
      if (!ok || !more) break;
      at = then;
      n = at.hi - at.lo;
      ++unit;
    }
    issue_commit(drain);  // arrives once every MMA issued above has completed
    volatile int no_abort = 0;
    if (!ok) {
      *abort_flag = 1;
      set_status(p.status, SPD_ETIMEOUT);
    }
    if (!mbar_wait(drain, 0, &no_abort, p.budget)) set_status(p.status, SPD_ETIMEOUT);
  } else if (warp == 6) {
    // ---- Q: 16 rows, those past the group's zero, in the 128-byte swizzle ----
    constexpr int P = HD / 8, N = 16 * P / 32;  // 16-byte pieces a row, a lane
    int unit = 0;
    do {
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (size_t(sq.s[at.e].q0) * p.n_heads + at.hk * p.group) * HD);
      uint4 v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (32 * i + lane) / P, piece = lane % P;
        v[i] = row < p.group ? src[row * P + piece] : make_uint4(0u, 0u, 0u, 0u);
      }
      const int b = unit & 1;
      if (unit >= 2 && !(ok = __all_sync(0xffffffffu, mbar_wait(&q_empty[b], ((unit >> 1) - 1) & 1, abort_flag, p.budget)))) break;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (32 * i + lane) / P, piece = lane % P;
        *reinterpret_cast<uint4*>(smem + L::q + (b * NC + (piece >> 3)) * L::qbox + row * 128 + (((piece & 7) ^ (row & 7)) << 4)) = v[i];
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[b]);
      ++unit;
    } while (at.next(p, sq));
  } else {
    // A wait that gives up must not part the four warps, which meet at barriers: it ends the loop for all of them at the next.
    const int t = threadIdx.x;  // key of the block; dim of the output
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    int j = 0;  // block of the CTA
    for (;;) {
      const PagedSeq& s = sq.s[at.e];
      float m[R], l[R];  // the heads' references (raw scores); the thread's sums of weights
#pragma unroll
      for (int r = 0; r < R; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.0f;
      }
      for (int blk = at.lo; blk < at.hi; ++blk, ++j) {
        const bool there = blk * kTokenKeys + t < s.len;
        if ((blk + 1) * kTokenKeys > s.len) {  // behind the last row: values that a weight of zero would turn into NaN
          ok = ok && mbar_wait(&v_full[j % NS], (j / NS) & 1, abort_flag, p.budget);
          if (!there) {
            uint4* vr = reinterpret_cast<uint4*>(smem + L::v + (j % NS) * NC * L::box + t * 128);
#pragma unroll
            for (int y = 0; y < 8 * NC; ++y) vr[(y >> 3) * (L::box / 16) + ((y + t) & 7)] = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
        }
        ok = ok && mbar_wait(&s_full[j & 1], (j >> 1) & 1, abort_flag, p.budget);
        __syncwarp();
        tc_fence_after();
        float v[R];
        {
          const uint32_t t_s = tmem + kTokenHeads * (j & 1) + lanes;
          float a[8];
          if constexpr (R == 8) {
            tmem_ld8(t_s, a);
          } else {
            float b[8];
            tmem_ld8x2(t_s, a, t_s + 8, b);
#pragma unroll
            for (int r = 0; r < 8; ++r) v[8 + r] = b[r];
          }
#pragma unroll
          for (int r = 0; r < 8; ++r) v[r] = a[r];
        }
        bool over = false;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (!there) v[r] = -INFINITY;
          over |= (v[r] - m[r]) * p.scale_log2 > kGrown;
        }
        // the product before has read P and O is whole; every warp has read its scores
        if (j > 0) ok = ok && mbar_wait(o_done, (j - 1) & 1, abort_flag, p.budget);
        if (any_softmax(over || !ok)) {
          if (any_softmax(!ok)) {  // (all of them leave together)
            ok = false;
            break;
          }
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const uint32_t top = __reduce_max_sync(0xffffffffu, order_of(fmaxf(v[r], -INFINITY)));
            if (lane == 0) red[warp * kTokenHeads + r] = order_value(top);
          }
          sync_softmax();
          float corr[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float n = fmaxf(m[r], fmaxf(fmaxf(red[r], red[kTokenHeads + r]), fmaxf(red[2 * kTokenHeads + r], red[3 * kTokenHeads + r])));
            corr[r] = n == m[r] ? 1.0f : ex2((m[r] - n) * p.scale_log2);
            m[r] = n;
            l[r] *= corr[r];
          }
          if (blk > at.lo) {
            __syncwarp();
            tc_fence_after();
#pragma unroll
            for (int x = 0; x < 3 * (R / 8); ++x) {
              const uint32_t col = t_o + lanes + (x / (R / 8)) * kTokenHeads + (x % (R / 8)) * 8;
              float o[8];
              tmem_ld8(col, o);
#pragma unroll
              for (int r = 0; r < 8; ++r) o[r] *= corr[(x % (R / 8)) * 8 + r];
              tmem_st8(col, o);
            }
            tmem_st_wait();
          }
          sync_softmax();  // red is free
        }
        uint32_t term[3][R / 2];
#pragma unroll
        for (int r = 0; r < R; r += 2) {
          const float f0 = m[r] == -INFINITY ? 0.0f : m[r] * p.scale_log2, f1 = m[r + 1] == -INFINITY ? 0.0f : m[r + 1] * p.scale_log2;
          const float p0 = ex2(fmaf(v[r], p.scale_log2, -f0)), p1 = ex2(fmaf(v[r + 1], p.scale_log2, -f1));
          l[r] += p0;
          l[r + 1] += p1;
          const uint32_t hi = pack_bf16(p0, p1);
          const float a = p0 - __uint_as_float(hi << 16), b = p1 - __uint_as_float(hi & 0xffff0000u);
          const uint32_t mid = pack_bf16(a, b);
          term[0][r / 2] = hi;
          term[1][r / 2] = mid;
          term[2][r / 2] = pack_bf16(a - __uint_as_float(mid << 16), b - __uint_as_float(mid & 0xffff0000u));
        }
#pragma unroll
        for (int x = 0; x < 3; ++x)
#pragma unroll
          for (int y = 0; y < R / 8; ++y)
            *reinterpret_cast<uint4*>(smem + L::p + t * 128 + (((2 * x + y) ^ (t & 7)) << 4)) =
                make_uint4(term[x][4 * y], term[x][4 * y + 1], term[x][4 * y + 2], term[x][4 * y + 3]);
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
      }
      if (!ok) break;
      // the sums of all keys, then the outputs
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int off = 16; off; off >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], off);
      if (lane == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) red[warp * kTokenHeads + r] = l[r];
      }
      sync_softmax();
#pragma unroll
      for (int r = 0; r < R; ++r) l[r] = (red[r] + red[kTokenHeads + r]) + (red[2 * kTokenHeads + r] + red[3 * kTokenHeads + r]);
      ok = mbar_wait(o_done, (j - 1) & 1, abort_flag, p.budget);
      if (any_softmax(!ok)) {
        ok = false;
        break;
      }
      __syncwarp();
      tc_fence_after();
      const size_t row = size_t(s.q0) * p.n_heads + at.hk * p.group;
      const bool whole = at.hi - at.lo == at.blocks;
      const size_t slot = (2 * size_t(blockIdx.x) + (at.lo == 0)) * p.rows_part;
#pragma unroll
      for (int y = 0; y < R / 8; ++y) {
        float o[8], mid[8], lo[8];
        __syncwarp();
        tmem_ld8(t_o + lanes + 8 * y, o);
        tmem_ld8x2(t_o + lanes + kTokenHeads + 8 * y, mid, t_o + lanes + 2 * kTokenHeads + 8 * y, lo);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = 8 * y + i;
          if (r >= p.group || t >= HD) continue;
          if (isfinite(o[i])) o[i] += mid[i] + lo[i];  // (an infinite V meets lower terms that are 0 or negative)
          if (whole) p.o[(row + r) * HD + t] = __float2bfloat16(l[r] == 0.0f ? 0.0f : o[i] * (1.0f / l[r]));
          else p.part_o[(slot + r) * HD + t] = o[i];
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (t != r || r >= p.group) continue;
        const float m2 = m[r] * p.scale_log2;
        if (!whole) p.part_ml[slot + r] = make_float2(m2, l[r]);
        else if (p.lse) p.lse[row + r] = fmaf(m2, 0.6931471805599453f, logf(l[r]));
      }
      sync_softmax();  // red is free
      tc_fence_before();
      if (!at.next(p, sq)) break;
    }
  }
  if (!ok) {
    *abort_flag = 1;
    set_status(p.status, SPD_ETIMEOUT);
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
  if (warp == 4) tmem_dealloc(tmem, 128);
  if (threadIdx.x == 0) stamp_end(p.stamp);
}

// Units whose blocks several CTAs had: states (m_i, l_i, O_i) joined in key order, m = max m_i, l = sum l_i 2^(m_i - m),
// O = sum O_i 2^(m_i - m). A part in which a row sees nothing has l_i = 0. (Its maximum does not tell: fmaxf passes over those of
// parts whose scores are all NaN, whose sums are NaN and stay so.) blockIdx.x stands for the border between two CTAs; the first
// border inside a unit has it.
struct Split {
  Place u;
  int c, parts;  // the CTA that begins the unit; CTAs that have a part of it
  bool mine;     // this border is the first inside the unit (all threads alike)
  __device__ __forceinline__ void find(const PagedArgs& p, const PagedSeqs& sq) {
    const int border = first_block(p, int(blockIdx.x) + 1);
    c = int(blockIdx.x);
    u.seek(p, sq, border, 1);
    const int start = border - u.lo;
    mine = u.lo > 0 && first_block(p, c) <= start;
    parts = ctas_before(p, start + u.blocks) - c;
  }
  __device__ __forceinline__ size_t slot(int part) const { return 2 * size_t(c + part) + (part == 0); }
};
struct State {
  float m = -INFINITY, l = 0.0f;
};
// A part's state joined to a row's: what both sums are multiplied by.
__device__ __forceinline__ float2 join(State& s, float2 ml) {
  if (ml.y == 0.0f) return make_float2(1.0f, 0.0f);
  const float m = fmaxf(s.m, ml.x), keep = exp2f(s.m - m), f = exp2f(ml.x - m);
  s.l = fmaf(ml.y, f, s.l * keep);
  s.m = m;
  return make_float2(keep, f);
}

// Tiles: a thread a row and eight columns, so that the rows of a warp lie side by side in every load; three parts in flight.
constexpr int kMergeThreads = 256;
template <int HD>
__global__ void __launch_bounds__(kMergeThreads)
    paged_merge_kernel(const __grid_constant__ PagedArgs p, const __grid_constant__ PagedSeqs sq) {
  constexpr int A = 3;
  pdl_launch_dependents();
  Split x;
  x.find(p, sq);
  const PagedSeq& s = sq.s[x.u.e];
  const int t = x.u.tile / p.chunks, h0 = (x.u.tile - t * p.chunks) * p.chunk, n0 = t * p.tokens;
  const int at = int(blockIdx.y) * kMergeThreads + int(threadIdx.x), col = at / p.rows_part, r = at - col * p.rows_part;
  const int hc = r % p.chunk, token = r / p.chunk;
  pdl_wait();
  if (!x.mine || col >= HD / 8 || token >= min(p.tokens, s.n - n0) || hc >= min(p.chunk, p.group - h0)) return;
  State st;
  float o[8] = {};
  for (int k0 = 0; k0 < x.parts; k0 += A) {
    float2 ml[A];
    float4 v[A][2];
#pragma unroll
    for (int k = 0; k < A; ++k) {
      ml[k] = make_float2(-INFINITY, 0.0f);
      if (k0 + k >= x.parts) continue;
      const size_t slot = x.slot(k0 + k) * p.rows_part;
      const float4* po = reinterpret_cast<const float4*>(p.part_o) + slot * (HD / 4) + 2 * col * p.rows_part + r;
      ml[k] = p.part_ml[slot + r];
      v[k][0] = po[0];
      v[k][1] = po[p.rows_part];
    }
#pragma unroll
    for (int k = 0; k < A; ++k) {
      if (ml[k].y == 0.0f) continue;  // a part in which the row sees nothing
      const float2 f = join(st, ml[k]);
      const float w[8] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w, v[k][1].x, v[k][1].y, v[k][1].z, v[k][1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = fmaf(w[i], f.y, o[i] * f.x);
    }
  }
  const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
  const size_t row = (size_t(s.q0) + n0 + token) * p.n_heads + x.u.hk * p.group + h0 + hc;
  *reinterpret_cast<uint4*>(p.o + row * HD + 8 * col) = make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv),
                                                                  pack_bf16(o[4] * inv, o[5] * inv), pack_bf16(o[6] * inv, o[7] * inv));
  if (p.lse && col == 0) p.lse[row] = fmaf(st.m, 0.6931471805599453f, logf(st.l));
}

// Few rows of many parts: W warps a row, a lane HD / 32 columns, each warp a range of the parts, four in flight.
constexpr int kMergeWarps = 8, kMergeAhead = 4, kMergeRows = 32;
template <int HD>
__global__ void __launch_bounds__(kMergeWarps * 32)
    row_merge_kernel(const __grid_constant__ PagedArgs p, const __grid_constant__ PagedSeqs sq, int W) {
  constexpr int A = kMergeAhead, D = HD / 32;
  __shared__ float2 wml[kMergeWarps];
  __shared__ float wo[kMergeWarps][HD];
  pdl_launch_dependents();
  Split x;
  x.find(p, sq);
  const PagedSeq& s = sq.s[x.u.e];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = warp & (W - 1);
  const int r = (int(blockIdx.y) * kMergeWarps + warp) / W;
  const int t = x.u.tile / p.chunks, h0 = (x.u.tile - t * p.chunks) * p.chunk, n0 = t * p.tokens;
  const int hc = r % p.chunk, token = r / p.chunk;
  const bool have = token < min(p.tokens, s.n - n0) && hc < min(p.chunk, p.group - h0);
  pdl_wait();
  if (!x.mine) return;
  State st;
  float o[D] = {};
  auto add = [&](float2 ml, const float* v) {
    if (ml.y == 0.0f) return;  // nothing was seen
    const float2 f = join(st, ml);
#pragma unroll
    for (int i = 0; i < D; ++i) o[i] = fmaf(v[i], f.y, o[i] * f.x);
  };
  if (have) {
    const int k1 = (w + 1) * x.parts / W;
    for (int k0 = w * x.parts / W; k0 < k1; k0 += A) {
      float2 ml[A];
      float v[A][D];
#pragma unroll
      for (int k = 0; k < A; ++k) {
        ml[k] = make_float2(-INFINITY, 0.0f);
        if (k0 + k >= k1) continue;
        const size_t slot = x.slot(k0 + k) * p.rows_part + r;
        ml[k] = p.part_ml[slot];
        const float* po = p.part_o + slot * HD + D * lane;
        if constexpr (D == 4) {
          const float4 f = *reinterpret_cast<const float4*>(po);
          v[k][0] = f.x, v[k][1] = f.y, v[k][2] = f.z, v[k][3] = f.w;
        } else {
          const float2 f = *reinterpret_cast<const float2*>(po);
          v[k][0] = f.x, v[k][1] = f.y;
        }
      }
#pragma unroll
      for (int k = 0; k < A; ++k) add(ml[k], v[k]);
    }
  }
  if (W > 1) {
    if (lane == 0) wml[warp] = make_float2(st.m, st.l);
#pragma unroll
    for (int i = 0; i < D; ++i) wo[warp][D * lane + i] = o[i];
    __syncthreads();
    if (w > 0) return;
    for (int k = 1; k < W; ++k) add(wml[warp + k], &wo[warp + k][D * lane]);
  }
  if (!have) return;
  const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
  const size_t row = (size_t(s.q0) + n0 + token) * p.n_heads + x.u.hk * p.group + h0 + hc;
  uint32_t* to = reinterpret_cast<uint32_t*>(p.o + row * HD + D * lane);
#pragma unroll
  for (int i = 0; i < D / 2; ++i) to[i] = pack_bf16(o[2 * i] * inv, o[2 * i + 1] * inv);
  if (p.lse && lane == 0) p.lse[row] = fmaf(st.m, 0.6931471805599453f, logf(st.l));
}

// Rows of a state: a tile's, or as many as the call has.
int rows_of_part(int n_q, int n_heads, int n_kv_heads) {
  const int chunk = std::min(n_heads / n_kv_heads, 128);
  return std::min(128 / chunk, n_q) * chunk;
}

// Tensor map of rows of heads, bf16 [rows][heads][head_dim], in boxes of 64 columns x box_heads x box_rows (16-byte aligned).
int make_heads_map(CUtensorMap* map, const void* ptr, int head_dim, int heads, int rows, int box_heads, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) == cudaSuccess &&
                    found == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<Encode>(f) : nullptr;
  }();
  if (!encode) return fail(SPD_ECUDA, "cuTensorMapEncodeTiled unavailable");
  const cuuint64_t dims[3] = {cuuint64_t(head_dim), cuuint64_t(heads), cuuint64_t(rows)};
  const cuuint64_t strides[2] = {cuuint64_t(head_dim) * 2, cuuint64_t(heads) * head_dim * 2};
  const cuuint32_t box[3] = {64, cuuint32_t(box_heads), cuuint32_t(box_rows)}, every[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, every,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SPD_OK : fail(SPD_ECUDA, "cuTensorMapEncodeTiled failed (%d)", int(r));
}

}  // namespace

size_t paged_attention_bytes(int n_q, int n_heads, int n_kv_heads, int head_dim) {
  const size_t rows = 2 * size_t(kCtas) * rows_of_part(n_q, n_heads, n_kv_heads);
  Carve cv(nullptr, ~size_t(0));
  cv.take<float>(rows * head_dim);
  cv.take<float2>(rows);
  return cv.used;
}

int paged_attention_run(const void* q, const int32_t* q_cu, const int32_t* len, const int32_t* prefix, int n_seqs,
                        const int32_t* table, int max_pages, const void* pool, int n_pages, int page_size, int n_heads,
                        int n_kv_heads, int head_dim, void* o, float* lse, void* ws, size_t ws_bytes, int* status,
                        cudaStream_t st) {
  const int kvd = n_kv_heads * head_dim, n_q = q_cu[n_seqs];
  PagedArgs p{};
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.pool = static_cast<const __nv_bfloat16*>(pool);
  p.table = table;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  p.page_size = page_size;
  p.n_heads = n_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_heads / n_kv_heads;
  p.scale_log2 = float(1.4426950408889634 / sqrt(double(head_dim)));
  p.o = static_cast<__nv_bfloat16*>(o);
  p.lse = lse;
  Carve cv(ws, ws_bytes);
  p.rows_part = rows_of_part(n_q, n_heads, n_kv_heads);
  const size_t rows = 2 * size_t(kCtas) * p.rows_part;
  p.part_o = cv.take<float>(rows * head_dim);
  p.part_ml = cv.take<float2>(rows);
  p.status = status;
  p.budget = kWaitBudget;
  const bool tokens_apart = p.group <= kTokenHeads;
  const int sms = std::min(kCtas / 2, num_sms());
  // sequences of one new token on their own where the token kernel takes them; up to kMaxSeqs a launch
  for (int form = 0; form < 2; ++form) {
    const bool token = form == 0;
    if (token && !tokens_apart) continue;
    p.keys = token ? kTokenKeys : kTK;
    p.chunk = token ? p.group : std::min(p.group, 128);
    p.chunks = token ? 1 : (p.group + 127) / 128;
    p.tokens = token ? 1 : 128 / p.chunk;
    p.box = p.keys;
    while (page_size % p.box) p.box /= 2;  // (pages are multiples of 16 rows)
    p.box_rows = std::min(p.tokens, n_q);
    CUtensorMap map_kv, map_q;
    bool mapped = false;
    for (int next = 0; next < n_seqs;) {
      PagedSeqs sq;
      sq.n = 0;
      long long total = 0, units = 0;
      int most = 0, longest = 0;
      int sizes[256] = {};  // tiles of as many blocks, from 128 on of 128 times (the index - 128) or more
      double pairs = 0.0, keys = 0.0, tokens = 0.0;
      for (; next < n_seqs && sq.n < kMaxSeqs; ++next) {
        const int b = next, n = q_cu[b + 1] - q_cu[b];
        if (n == 0 || (tokens_apart && (n == 1) != token)) continue;
        PagedSeq& s = sq.s[sq.n++];
        s = {int(total), q_cu[b], n, len[b], prefix ? prefix[b] : 0, b, 0, (n + p.tokens - 1) / p.tokens * p.chunks};
        long long blocks = 0;
        for (int i = 0; i < n; i += p.tokens) {
          const int here = blocks_at(s, i, p.tokens, p.keys);
          longest = std::max(longest, here);
          sizes[here < 128 ? here : 128 + std::min(127, here >> 7)] += p.chunks;
          blocks += (long long)here * p.chunks;
        }
        total += blocks * n_kv_heads;
        if (total > 0x3fffffff) return fail(SPD_EUNSUPPORTED, "paged attention of more than 2^30 blocks of keys");
        s.head_blocks = int(blocks);
        units += (long long)s.tiles * n_kv_heads;
        most = std::max(most, n);
        keys += len[b];
        tokens += n;
        pairs += double(n) * len[b] - 0.5 * double(n) * (n - 1);
      }
      if (sq.n == 0) continue;
      if (!mapped) {
        if (int rc = make_operand_map(&map_kv, pool, 2 * kvd, n_pages * page_size, p.box)) return rc;
        if (token) map_q = map_kv;  // (not used)
        else if (int rc = make_heads_map(&map_q, q, head_dim, n_heads, n_q, p.chunk, p.box_rows)) return rc;
        mapped = true;
      }
      p.total = int(total);
      const int places = token ? sms : 2 * sms;
      p.ctas = int(std::min<long long>(places, total));
      // Parts of units are written, read and joined, at the price of a launch and some blocks a CTA, of more the more CTAs do so
      // at once; a CTA that goes on from one unit to the next does nothing for some 4 us. One unit a CTA, the longest first, and equal
      // stretches, us. 28 heads of 128 on 4: 1500 fresh tokens (336 units of 1 to 24 blocks, 13.8 a place) 33 and 65, 2000 (448, 24.5)
      // 42 and 91, 19 prompts of 2 to 1079 (612) 34 and 85, 1500 behind 1500 (336 of 24 to 47, 40) 73 and 75, 2048 behind 4000 (456
      // of 63 to 95, 120) 177 and 166, 18 behind 400 (4 of 7, 1) 11.9 and 10.0. 32 heads of 128: 500 behind 700 (128 of 13 to 19, 6.9)
      // 27.6 and 31.4, 300 behind 1500 (96 of 25 to 29, 8.7) 36.9 and 33.0. 16 heads of 64 on 8: 700 fresh (88 of 1 to 11, 1.7) 13.0
      // and 15.8, 3000 (376, 29) 44 and 53, 2048 behind 2000 (256 of 32 to 64, 40) 58 and 53. Few rows a unit, whose parts are small: 32
      // sequences of 4 behind 1500 (128 of 24, 10.1) 33.4 and 32.0, 31 of 2 behind 50, 32 heads (992 of 1, 3.3) 33 and 27.
      // Single tokens: over 200 rows of 32 heads (32 units of 2) 6.4 and 7.2, 350 (of 3) 7.9 and 7.6 and 3 us less for the host,
      // 700 (of 6) 12.4 and 9.0; 4 sequences over 1100 (128 units of 9, 7.6 a CTA) 17.8 and 19.7, of 2000 (of 16, 13.5) 29.3 and
      // 29.1. (Their form has the next unit's scores under way; the tiles' form takes 33 us for 31 tokens over 50 rows of 32 heads,
      // theirs 24.)
      const bool few = std::min(most, p.tokens) * p.chunk <= kMergeRows;
      if (token) {
        p.whole = units <= places && (longest <= 3 || 2 * longest <= 2 * total / p.ctas + 3);
      } else {
        long long load = longest;  // blocks of the fullest place
        if (units > places) {
          int size = 0;  // of the units that begin last
          for (long long left = units % places; left > 0; ++size) left -= (long long)sizes[size] * n_kv_heads;
          load = std::max(load, total / places + (size <= 128 ? size : (size - 128) * 128));
        }
        const long long price = std::min<long long>(27 * units * p.ctas / places, (few ? 10ll : head_dim == 64 ? 16ll : 27ll) * p.ctas);
        p.whole = (units <= places || !few) && (load - 2) * p.ctas <= total + price;
      }
      if (p.whole) {
        if (units > places)
          std::sort(sq.s, sq.s + sq.n, [&](const PagedSeq& a, const PagedSeq& b) {
            return limit_of(a, a.n - 1) > limit_of(b, b.n - 1);
          });
        p.ctas = int(units);
        int first = 0;
        for (int e = 0; e < sq.n; ++e) {
          sq.s[e].block0 = first;
          first += sq.s[e].tiles * n_kv_heads;
        }
      }
      p.share = p.total / p.ctas;
      p.more = p.total - p.share * p.ctas;
      p.by_row = token || few;
      p.warps = (std::min(most, p.tokens) * p.chunk + 31) / 32;
      const double fl = 4.0 * head_dim * n_heads * pairs;
      const double by = 4.0 * kvd * keys + 4.0 * n_heads * head_dim * tokens;
      p.stamp = stamp_slot(TR_ATTN, fl, by);
      const int slot = trace_begin(st);
      using Kernel = void (*)(CUtensorMap, CUtensorMap, PagedArgs, PagedSeqs);
      static constexpr Kernel kernels[6] = {paged_token_kernel<64, 8>,   paged_token_kernel<128, 8>, paged_token_kernel<64, 16>,
                                            paged_token_kernel<128, 16>, paged_attn_kernel<64>,      paged_attn_kernel<128>};
      static constexpr uint32_t bytes[6] = {TokenSmem<64>::bytes,  TokenSmem<128>::bytes, TokenSmem<64>::bytes,
                                            TokenSmem<128>::bytes, PagedSmem<64>::bytes,  PagedSmem<128>::bytes};
      const int which = (token ? 2 * (p.group > 8) : 4) + (head_dim == 128);
      const Kernel kernel = kernels[which];
      const uint32_t smem = bytes[which];
      static DeviceOnce attr[6];
      SPD_CUDA_TRY(once_per_device(attr[which], [&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
      }));
      SPD_CUDA_TRY(launch_pdl(kernel, dim3(p.ctas), dim3(token ? kTokenThreads : kThreads), smem, st, map_kv, map_q, p, sq));
      if (p.ctas > 1 && !p.whole) {
        if (p.by_row) {
          const int parts = int((long long)longest * p.ctas / total) + 2;  // of a unit, at most
          const int rows_unit = std::min(most, p.tokens) * p.chunk;
          int W = 1;
          while (W < kMergeWarps && parts > kMergeAhead * W) W *= 2;
          SPD_CUDA_TRY(launch_pdl(head_dim == 128 ? row_merge_kernel<128> : row_merge_kernel<64>,
                                  dim3(p.ctas - 1, (rows_unit * W + kMergeWarps - 1) / kMergeWarps), dim3(kMergeWarps * 32), 0, st, p,
                                  sq, W));
        } else {
          const int threads = p.rows_part * (head_dim / 8);
          SPD_CUDA_TRY(launch_pdl(head_dim == 128 ? paged_merge_kernel<128> : paged_merge_kernel<64>,
                                  dim3(p.ctas - 1, (threads + kMergeThreads - 1) / kMergeThreads), dim3(kMergeThreads), 0, st, p, sq));
        }
      }
      trace_end(slot, st, TR_ATTN, fl, by);
    }
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
