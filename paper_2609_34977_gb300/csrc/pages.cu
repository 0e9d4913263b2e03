// The paged KV cache: new rows rotated and appended to pages, page tables that fork, grow, end and are compacted.
//
// A pool is bf16 [layer][page][row of the page][K of every K/V head | V of every K/V head]; row r of a sequence lies in page
// table[r / page_size], row r % page_size. ref counts the tables that list a page; 0 is free.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "ptx.cuh"
#include "trace.h"

namespace spd {
namespace {

// ---- rotary positions with several axes, K/V into pages -------------------------------------------
// Pair (j, j + d/2) of a head turns by pos[axis_j] theta^(-2j/d). An angle is kept in turns: theta^(-2j/d) / 2 pi as a 64-bit
// fraction times the integer position, modulo 2^64, is exact but for the fraction's own error (below 2^-54 a position where
// theta is 1 or more: 2^-23 of a turn at a position of 2^31); its upper 32 bits go through sincospi.
// A thread has 8 pairs of a token (16 bytes of either half) for one, four or eight heads (eight: four and four), so that it works
// its angles out once for them where there are threads enough. Heads of 128, 36 of 64 / 256 / 1024 / 4096 tokens with one and with
// four: 3.5 and 4.8 / 6.7 and 5.0 / 10.6 and 8.8 / 34.9 and 19.9 us; 96 of 64 / 4096: 5.1 and 4.9 / 73 and 39. With four and with
// eight: 36 of 2000 / 2600 / 4096 / 8000 tokens 9.2 and 10.9 / 11.3 and 11.3 / 15.8 and 13.7 / 30.8 and 27.2, 96 of 500 / 800 / 2000 /
// 4048 8.8 and 8.9 / 9.2 and 8.8 / 20.3 and 16.4 / 38.0 and 33.8 (199 MB, 5.9 TB/s); heads of 64, 32 of 4096 / 8000 / 16000 7.8 and
// 9.8 / 11.9 and 11.5 / 24.8 and 23.1.
constexpr int kRopeThreads = 256;
constexpr long long kRopeSingle = 40000;  // threads of a head each up to which it is one,
constexpr long long kRopeEight = 800000;  // beyond which it is eight
constexpr int kRopeSeqs = 384;  // sequences whose places fit in a launch's parameters

struct RopeSeq {
  int q0, slot0;  // first new token, and the cache row that it gets
};
struct RopeArgs {
  const uint16_t *q, *kv;
  int ldq, ldkv, tok0, n_tok, n_pos, n_axes;  // tokens [tok0, tok0 + n_tok) of the n_pos of the call
  const int32_t* pos;
  const int32_t* table;  // of the launch's first sequence
  int max_pages, n_pages, page_size, n_heads, n_kv_heads, n_seqs;
  uint16_t *pool, *q_out;
  int* status;
  uint64_t turns[64];  // theta^(-2j/d) / 2 pi, 64 bits behind the point
  uint8_t axis[64];    // n_axes: the pair does not turn
  RopeSeq seq[kRopeSeqs];
};

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int HD, int U, int R>
__global__ void __launch_bounds__(kRopeThreads, 4) rope_pages_kernel(const __grid_constant__ RopeArgs p) {
  constexpr int P = HD / 16;  // threads a head
  const int heads = p.n_heads + 2 * p.n_kv_heads, slots = (heads + U * R - 1) / (U * R);  // a thread's heads are `slots` apart
  const unsigned at = blockIdx.x * kRopeThreads + threadIdx.x;
  const unsigned tok = at / unsigned(slots * P), rest = at - tok * unsigned(slots * P);
  const int piece = int(rest % P), h0 = int(rest / P);
  pdl_launch_dependents();
  pdl_wait();
  if (tok >= unsigned(p.n_tok)) return;
  const int t = p.tok0 + int(tok);
  uint4 a[U], b[U];
  auto load = [&](int r) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + (r * U + u) * slots;
      if (h >= heads) continue;
      const uint16_t* src = h < p.n_heads ? p.q + size_t(t) * p.ldq + h * HD : p.kv + size_t(t) * p.ldkv + (h - p.n_heads) * HD;
      a[u] = *reinterpret_cast<const uint4*>(src + 8 * piece);
      b[u] = *reinterpret_cast<const uint4*>(src + HD / 2 + 8 * piece);
    }
  };
  load(0);
  float c[8], s[8];
  if (h0 < p.n_heads + p.n_kv_heads) {
    int32_t at_axis[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int x = p.axis[8 * piece + i];
      at_axis[i] = x < p.n_axes ? p.pos[size_t(x) * p.n_pos + t] : 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t turn = uint64_t(int64_t(at_axis[i])) * p.turns[8 * piece + i];
      sincospif(float(int32_t(turn >> 32)) * 0x1p-31f, &s[i], &c[i]);
    }
  }
  uint16_t* row = nullptr;  // the token's row in the pool
  if (h0 + (U * R - 1) * slots >= p.n_heads) {
    int e = 0;
    for (int hi = p.n_seqs; hi - e > 1;) {
      const int mid = (e + hi) >> 1;
      if (p.seq[mid].q0 <= t) e = mid;
      else hi = mid;
    }
    const int slot = p.seq[e].slot0 + t - p.seq[e].q0, k = slot / p.page_size;
    const int page = p.table[size_t(e) * p.max_pages + k];
    if (unsigned(page) < unsigned(p.n_pages))
      row = p.pool + (size_t(page) * p.page_size + (slot - k * p.page_size)) * (2 * size_t(p.n_kv_heads) * HD);
    else set_status(p.status, SPD_EINVAL);
  }
#pragma unroll 1
  for (int r = 0; r < R; ++r) {
    if (r > 0) load(r);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + (r * U + u) * slots;
      if (h >= heads) continue;
      uint16_t* dst = h < p.n_heads ? p.q_out + (size_t(t) * p.n_heads + h) * HD : row ? row + (h - p.n_heads) * HD : nullptr;
      if (!dst) continue;
      uint32_t x[4] = {a[u].x, a[u].y, a[u].z, a[u].w}, y[4] = {b[u].x, b[u].y, b[u].z, b[u].w};
      if (h < p.n_heads + p.n_kv_heads) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = __uint_as_float(x[i] << 16), x1 = __uint_as_float(x[i] & 0xffff0000u);
          const float y0 = __uint_as_float(y[i] << 16), y1 = __uint_as_float(y[i] & 0xffff0000u);
          x[i] = bf16_pair(x0 * c[2 * i] - y0 * s[2 * i], x1 * c[2 * i + 1] - y1 * s[2 * i + 1]);
          y[i] = bf16_pair(x0 * s[2 * i] + y0 * c[2 * i], x1 * s[2 * i + 1] + y1 * c[2 * i + 1]);
        }
      }
      *reinterpret_cast<uint4*>(dst + 8 * piece) = make_uint4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<uint4*>(dst + HD / 2 + 8 * piece) = make_uint4(y[0], y[1], y[2], y[3]);
    }
  }
}

// ---- page tables ------------------------------------------------------------------------------------
// Output b takes over the table of input parent[b] (its held = len_in rows) and gets room for grow[b] more. The order of
// things: how many outputs every input has; ref of every listed page by that number less one; the last pages, if not full,
// that an output would write behind its rows: the sequence that holds most of one (the first of them) keeps it, unless the page
// is listed anywhere else too, the others that grow get copies; then free pages, the lowest first, by output: its copy, its
// new ones. Integer additions and maxima in any order: the same result in every run.
constexpr int kPageThreads = 1024, kPageWarps = kPageThreads / 32;

struct PageCopy {
  int from, to, rows;
};
struct UpdateArgs {
  int n_pages, page_size, n_in, n_out, max_pages;
  const int32_t *ref_in, *table_in, *len_in, *parent, *grow;
  int32_t *ref_out, *table_out, *len_out;
  int32_t *count, *free_list;                                  // counters and lists in the workspace
  unsigned long long* owner;
  int32_t *kids, *rows, *from, *more, *tail, *first, *copy_at;
  PageCopy* copies;                                            // [n_out]
  int* n_copies;
  int* status;
};

// Exclusive prefix sum over the block; *total the block's sum.
__device__ int page_prefix(int v, int* tmp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
  if (lane == 31) tmp[warp] = x;
  __syncthreads();
  int w = tmp[lane];
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

// ceil(rows / page)
__device__ __forceinline__ int pages_for(int rows, int page) { return int((unsigned(rows) + unsigned(page) - 1u) / unsigned(page)); }

// What bounds it: a chain of dependent loads, phases that wait for each other. So the counters live in shared memory where they fit
// (kPageShared: about 8000 pages and 1000 sequences), in the workspace beyond; the lists are read once, side by side. 64 beams of
// 16 requests with their copies: 13 us in all.
constexpr size_t kPageShared = 200 * 1024;
__host__ __device__ inline size_t page_bytes(int n_pages, int n_in, int n_out) {
  return 20 * size_t(n_pages) + 8 * size_t(n_in) + 20 * size_t(n_out);
}

__global__ void __launch_bounds__(kPageThreads, 1) pages_update_kernel(const __grid_constant__ UpdateArgs p, bool shared) {
  __shared__ int tmp[kPageWarps];
  extern __shared__ unsigned long long mem[];
  const int tid = threadIdx.x, room = int(min(0x7fffffffLL, (long long)p.max_pages * p.page_size));
  unsigned long long* owner = shared ? mem : p.owner;                                         // [n_pages]
  int* count = shared ? reinterpret_cast<int*>(mem + p.n_pages) : p.count;                    // [n_pages]
  int* ref = shared ? count + p.n_pages : p.ref_out;                                          // [n_pages]
  int* free_list = shared ? ref + p.n_pages : p.free_list;                                    // [n_pages]
  int* listed = free_list;  // until the free pages are looked for: entries of the outputs' tables that list a page, before copies
  int* kids = shared ? free_list + p.n_pages : p.kids;                                        // [n_in]
  int* rows = shared ? kids + p.n_in : p.rows;                                                // [n_in] rows that it holds
  int* from = shared ? rows + p.n_in : p.from;                                                // [n_out] parent, or -1
  int* more = shared ? from + p.n_out : p.more;                                               // [n_out] rows that it grows by
  int* tail = shared ? more + p.n_out : p.tail;                                               // [n_out] its last page if not full, or -1
  int* first = shared ? tail + p.n_out : p.first;                                             // [n_out] its first new page among all
  int* copy_at = shared ? first + p.n_out : p.copy_at;                                        // [n_out] its copy, or -1
  pdl_launch_dependents();
  pdl_wait();
  auto page_of = [&](int q) { return unsigned(q) < unsigned(p.n_pages) ? q : -1; };
  // this thread's first entry of the tables, on its way while the lengths are read
  const unsigned width = unsigned(p.max_pages), entries = unsigned(p.n_in) * width, entries_out = unsigned(p.n_out) * width;
  const int entry = unsigned(tid) < entries ? p.table_in[tid] : -1;
  for (int i = tid; i < p.n_in; i += kPageThreads) {
    const int n = p.len_in[i];
    if (n < 0 || n > room) set_status(p.status, SPD_EINVAL);
    rows[i] = min(max(n, 0), room);
    kids[i] = 0;
  }
  for (int b = tid; b < p.n_out; b += kPageThreads) {
    const int i = p.parent ? p.parent[b] : b;
    from[b] = unsigned(i) < unsigned(p.n_in) ? i : -1;
    more[b] = p.grow ? p.grow[b] : 0;
  }
  for (int i = tid; i < p.n_pages; i += kPageThreads) {
    ref[i] = p.ref_in[i];
    count[i] = 0;
    listed[i] = 0;
    owner[i] = 0;
  }
  __syncthreads();
  auto held_by = [&](int b) { return from[b] < 0 ? 0 : rows[from[b]]; };
  for (int b = tid; b < p.n_out; b += kPageThreads) {
    const int i = from[b], held = held_by(b), part = held % p.page_size, n = more[b];
    if (n < 0 || n > room - held) set_status(p.status, SPD_EINVAL);
    more[b] = min(max(n, 0), room - held);
    tail[b] = -1;
    if (i < 0) continue;
    atomicAdd(&kids[i], 1);
    if (part == 0) continue;
    const int q = tail[b] = page_of(p.table_in[size_t(i) * p.max_pages + held / p.page_size]);
    if (q < 0) continue;
    atomicAdd(&count[q], 1);
    atomicMax(&owner[q], (static_cast<unsigned long long>(part) << 32) | (0xffffffffu - unsigned(b)));
  }
  __syncthreads();
  for (unsigned x = tid; x < entries; x += kPageThreads) {
    const int i = int(x / width), k = int(x - i * width);
    if (k >= pages_for(rows[i], p.page_size)) continue;
    const int q = page_of(x == unsigned(tid) ? entry : p.table_in[x]), change = kids[i] - 1;
    if (q < 0) {
      set_status(p.status, SPD_EINVAL);
      continue;
    }
    if (change >= 0) atomicAdd(&listed[q], change + 1);
    if (change != 0 && atomicAdd(&ref[q], change) + change < 0) set_status(p.status, SPD_EINVAL);
  }
  __syncthreads();
  // A count below the tables' entries shows here (where none of the inputs goes on: above, as a negative one). Taken for their number, no
  // page that a table lists counts as free, and no copy's source is another's target.
  for (int i = tid; i < p.n_pages; i += kPageThreads) {
    const int n = listed[i];
    if (n > 0 && n > ref[i]) {
      set_status(p.status, SPD_EINVAL);
      ref[i] = n;
    }
  }
  __syncthreads();
  int need = 0, copies = 0;
  for (int b0 = 0; b0 < p.n_out; b0 += kPageThreads) {
    const int b = b0 + tid;
    int fresh = 0, copy = 0;
    if (b < p.n_out) {
      const int held = held_by(b), q = more[b] > 0 ? tail[b] : -1;
      if (q >= 0) copy = !(uint32_t(owner[q]) == 0xffffffffu - unsigned(b) && ref[q] == count[q]);
      fresh = pages_for(held + more[b], p.page_size) - pages_for(held, p.page_size) + copy;
      p.len_out[b] = held + more[b];
    }
    int all, all_copies;
    const int at = page_prefix(fresh, tmp, &all), c = page_prefix(copy, tmp, &all_copies);
    if (b < p.n_out) {
      first[b] = need + at;
      copy_at[b] = copy ? copies + c : -1;
    }
    need += all;
    copies += all_copies;
  }
  if (tid == 0) *p.n_copies = copies;
  __syncthreads();
  for (int b = tid; b < p.n_out; b += kPageThreads)
    if (copy_at[b] >= 0) atomicSub(&ref[tail[b]], 1);
  __syncthreads();
  int found = 0;
  for (int q0 = 0; q0 < p.n_pages && found < need; q0 += kPageThreads) {
    const int q = q0 + tid;
    const int is = q < p.n_pages && ref[q] <= 0;
    int all;
    const int at = page_prefix(is, tmp, &all);
    if (is && found + at < need) free_list[found + at] = q;
    found += all;
  }
  const int got = min(found, need);
  if (found < need && tid == 0) set_status(p.status, SPD_ENOSPC);
  __syncthreads();
  for (unsigned x = tid; x < entries_out; x += kPageThreads) {
    const int b = int(x / width), k = int(x - b * width);
    const int held = held_by(b), copy = copy_at[b];
    const int have = pages_for(held, p.page_size), at = have - (copy >= 0);
    int q = -1;
    if (k < at) {
      q = page_of(p.table_in[size_t(from[b]) * p.max_pages + k]);
    } else if (k < pages_for(held + more[b], p.page_size)) {
      const int f = first[b] + k - at;
      if (f < got) {
        q = free_list[f];
        ref[q] = 1;
      }
      if (k < have) p.copies[copy] = {tail[b], q, held % p.page_size};
    }
    p.table_out[x] = q;
  }
  if (shared) {
    __syncthreads();
    for (int i = tid; i < p.n_pages; i += kPageThreads) p.ref_out[i] = ref[i];
  }
}

struct CompactArgs {
  int n_pages, page_size, n_seqs, max_pages;
  const int32_t *ref_in, *table_in;
  int32_t *ref_out, *table_out, *used;
  int32_t* goes;     // [n_pages] where a page moves, or -1
  int32_t* holes;    // [n_pages]
  PageCopy* copies;  // [n_pages]
  int* n_copies;
  int* status;
};

// The j-th page in use at or behind `used`, their number, moves into the j-th free page before it.
__global__ void __launch_bounds__(kPageThreads, 1) pages_compact_kernel(const __grid_constant__ CompactArgs p) {
  __shared__ int tmp[kPageWarps];
  const int tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  int used = 0;
  for (int q0 = 0; q0 < p.n_pages; q0 += kPageThreads)
    used += __syncthreads_count(q0 + tid < p.n_pages && p.ref_in[q0 + tid] > 0);
  int holes = 0, fills = 0;
  for (int q0 = 0; q0 < p.n_pages; q0 += kPageThreads) {
    const int q = q0 + tid;
    const bool in = q < p.n_pages, live = in && p.ref_in[q] > 0;
    const int hole = in && !live && q < used, fill = live && q >= used;
    int all_h, all_f;
    const int h = page_prefix(hole, tmp, &all_h), f = page_prefix(fill, tmp, &all_f);
    if (hole) p.holes[holes + h] = q;
    if (fill) p.copies[fills + f].from = q;
    if (in) p.goes[q] = live && q < used ? q : -1;
    holes += all_h;
    fills += all_f;
  }
  if (tid == 0) {
    *p.used = used;
    *p.n_copies = fills;
  }
  __syncthreads();
  for (int j = tid; j < fills; j += kPageThreads) {
    const int from = p.copies[j].from, to = p.holes[j];
    p.copies[j] = {from, to, p.page_size};
    p.goes[from] = to;
    p.ref_out[to] = p.ref_in[from];
  }
  __syncthreads();
  for (int q = tid; q < p.n_pages; q += kPageThreads) {
    if (q >= used) p.ref_out[q] = 0;
    else if (p.goes[q] == q) p.ref_out[q] = p.ref_in[q];
  }
  for (size_t x = tid; x < size_t(p.n_seqs) * p.max_pages; x += kPageThreads) {
    int q = p.table_in[x];
    if (unsigned(q) < unsigned(p.n_pages)) {
      if (p.goes[q] >= 0) q = p.goes[q];
      else set_status(p.status, SPD_EINVAL);  // a page that nobody counts
    }
    p.table_out[x] = q;
  }
}

// The rows of the copies of a list, in every layer. A page's rows lie side by side, so a copy is one stretch of bytes. Bound by HBM:
// 28 layers of a pool compacted, 0.63 GB read and written in 99 us (0.94 of a plain copy's rate), four 16-byte pieces a thread in
// flight and as many CTAs as there can be work for, at most two waves.
constexpr int kCopyThreads = 256, kCopyDepth = 4, kCopyChunk = kCopyThreads * kCopyDepth;  // 16-byte pieces
constexpr int kCopyCtas = 16;  // an SM, two waves
__global__ void __launch_bounds__(kCopyThreads)
    pages_copy_kernel(uint4* pool, const PageCopy* copies, const int* n_copies, int n_layers, size_t layer16, size_t page16, int row16,
                      int chunks) {
  pdl_launch_dependents();
  pdl_wait();
  const long long all = (long long)*n_copies * n_layers * chunks;
  for (long long w = blockIdx.x; w < all; w += gridDim.x) {
    // (division of 64 bits is a hundred instructions)
    const bool narrow = all <= 0xffffffffll;
    const long long rest = narrow ? uint32_t(w) / uint32_t(chunks) : w / chunks;
    const int chunk = int(w - rest * chunks);
    const long long copy = narrow ? uint32_t(rest) / uint32_t(n_layers) : rest / n_layers;
    const int layer = int(rest - copy * n_layers);
    const PageCopy c = copies[copy];
    const size_t n = size_t(c.rows) * row16, at = size_t(chunk) * kCopyChunk + threadIdx.x;
    if (c.from < 0 || c.to < 0) continue;
    const uint4* from = pool + layer * layer16 + c.from * page16;
    uint4* to = pool + layer * layer16 + c.to * page16;
    uint4 v[kCopyDepth];
#pragma unroll
    for (int u = 0; u < kCopyDepth; ++u)
      if (at + u * kCopyThreads < n) v[u] = from[at + u * kCopyThreads];
#pragma unroll
    for (int u = 0; u < kCopyDepth; ++u)
      if (at + u * kCopyThreads < n) to[at + u * kCopyThreads] = v[u];
  }
}

// most: copies at most.
int copy_pages(uint16_t* pool, const PageCopy* copies, const int* n, int most, int n_layers, int n_pages, int page_size, int row16,
               cudaStream_t st) {
  const size_t page16 = size_t(page_size) * row16;
  const int chunks = int((page16 + kCopyChunk - 1) / kCopyChunk);
  const long long ctas = std::min((long long)kCopyCtas * num_sms(), (long long)most * n_layers * chunks);
  SPD_CUDA_TRY(launch_pdl(pages_copy_kernel, dim3(unsigned(ctas)), dim3(kCopyThreads), 0, st, reinterpret_cast<uint4*>(pool), copies, n,
                          n_layers, page16 * n_pages, page16, row16, chunks));
  return SPD_OK;
}

struct PagesWs {
  int32_t *count, *free_list, *kids, *rows, *from, *more, *tail, *first, *copy_at;
  unsigned long long* owner;
  PageCopy* copies;
  int* n_copies;
};
PagesWs carve_pages(Carve& cv, int n_pages, int n_seqs) {
  PagesWs w;
  const size_t most = size_t(std::max(n_pages, n_seqs));
  w.owner = cv.take<unsigned long long>(n_pages);
  w.count = cv.take<int32_t>(n_pages);
  w.free_list = cv.take<int32_t>(n_pages);
  for (int32_t** list : {&w.kids, &w.rows, &w.from, &w.more, &w.tail, &w.first, &w.copy_at}) *list = cv.take<int32_t>(n_seqs);
  w.copies = cv.take<PageCopy>(most);
  w.n_copies = cv.take<int>(1);
  return w;
}

bool misaligned(const void* p, int to) { return reinterpret_cast<uintptr_t>(p) & uintptr_t(to - 1); }

}  // namespace

int pool_check(const void* pool, int n_layers, int n_pages, int page_size, int n_kv_heads, int head_dim, int max_pages) {
  if (!pool || n_layers < 1 || n_pages < 1 || page_size < 1 || n_kv_heads < 1 || max_pages < 1)
    return fail(SPD_EINVAL, "bad pool arguments");
  if (head_dim != 64 && head_dim != 128) return fail(SPD_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (page_size % 16) return fail(SPD_EUNSUPPORTED, "page_size must be a multiple of 16");
  if ((long long)n_pages * page_size > 0x7fffffffLL) return fail(SPD_EUNSUPPORTED, "more than 2^31 - 1 rows in a layer of the pool");
  if (misaligned(pool, 16)) return fail(SPD_EINVAL, "the pool must be 16-byte aligned");
  return SPD_OK;
}

int paged_check(const int32_t* q_cu, int n_q, const int32_t* len, const int32_t* prefix, int n_seqs, int max_pages, int page_size) {
  if (q_cu[0] != 0 || q_cu[n_seqs] != n_q) return fail(SPD_EINVAL, "q_cu must run from 0 to the number of tokens");
  for (int b = 0; b < n_seqs; ++b) {
    if (q_cu[b + 1] < q_cu[b]) return fail(SPD_EINVAL, "q_cu decreases at sequence %d", b);
    const int n = q_cu[b + 1] - q_cu[b];  // (at most n_q)
    if (len[b] < n || len[b] > (long long)max_pages * page_size)
      return fail(SPD_EINVAL, "sequence %d: %d rows do not hold its new ones, or exceed its table", b, len[b]);
    if (prefix && (prefix[b] < 0 || prefix[b] > len[b])) return fail(SPD_EINVAL, "prefix of sequence %d outside [0, its rows]", b);
  }
  return SPD_OK;
}

int rope_pages_run(const void* q, int ldq, const void* kv, int ldkv, const int32_t* pos, int n_axes, const uint8_t* axis,
                   double theta, const int32_t* q_cu, const int32_t* len, int n_seqs, const int32_t* table, int max_pages,
                   void* pool, int n_pages, int page_size, int n_heads, int n_kv_heads, int head_dim, void* q_out, int* status,
                   cudaStream_t st) {
  RopeArgs p;
  p.q = static_cast<const uint16_t*>(q);
  p.kv = static_cast<const uint16_t*>(kv);
  p.ldq = ldq;
  p.ldkv = ldkv;
  p.n_pos = q_cu[n_seqs];
  p.n_axes = n_axes;
  p.pos = pos;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  p.page_size = page_size;
  p.n_heads = n_heads;
  p.n_kv_heads = n_kv_heads;
  p.pool = static_cast<uint16_t*>(pool);
  p.q_out = static_cast<uint16_t*>(q_out);
  p.status = status;
  // (64 powers take 3 us: a thread keeps those of the base that it used last)
  static thread_local struct {
    double theta = 0.0;
    int head_dim = 0;
    uint64_t turns[64];
  } kept;
  if (kept.theta != theta || kept.head_dim != head_dim) {
    kept.theta = theta;
    kept.head_dim = head_dim;
    for (int j = 0; j < head_dim / 2; ++j) {
      const double f = pow(theta, -2.0 * j / head_dim) / 6.283185307179586476925;
      kept.turns[j] = uint64_t((f - floor(f)) * 18446744073709551616.0);
    }
  }
  for (int j = 0; j < head_dim / 2; ++j) {
    p.turns[j] = kept.turns[j];
    p.axis[j] = !axis ? 0 : axis[j] < n_axes ? axis[j] : uint8_t(n_axes);
  }
  const int heads = n_heads + 2 * n_kv_heads, P = head_dim / 16;
  for (int s0 = 0; s0 < n_seqs; s0 += kRopeSeqs) {
    p.n_seqs = std::min(kRopeSeqs, n_seqs - s0);
    p.tok0 = q_cu[s0];
    p.n_tok = q_cu[s0 + p.n_seqs] - p.tok0;
    if (p.n_tok == 0) continue;
    p.table = table + size_t(s0) * max_pages;
    for (int b = 0; b < p.n_seqs; ++b)
      p.seq[b] = {q_cu[s0 + b], len[s0 + b] - (q_cu[s0 + b + 1] - q_cu[s0 + b])};
    const long long single = (long long)p.n_tok * heads * P;
    if (single > 0x7fffffffLL) return fail(SPD_EUNSUPPORTED, "%d tokens of %d heads in one call", p.n_tok, heads);
    const int each = single > kRopeEight ? 8 : single > kRopeSingle ? 4 : 1;
    const long long threads = (long long)p.n_tok * ((heads + each - 1) / each) * P;
    using Kernel = void (*)(RopeArgs);
    static constexpr Kernel kernels[2][3] = {{rope_pages_kernel<64, 1, 1>, rope_pages_kernel<64, 4, 1>, rope_pages_kernel<64, 4, 2>},
                                             {rope_pages_kernel<128, 1, 1>, rope_pages_kernel<128, 4, 1>, rope_pages_kernel<128, 4, 2>}};
    const Kernel kernel = kernels[head_dim == 128][each == 8 ? 2 : each == 4];
    const int slot = trace_begin(st);
    SPD_CUDA_TRY(launch_pdl(kernel, dim3(unsigned((threads + kRopeThreads - 1) / kRopeThreads)), dim3(kRopeThreads), 0, st, p));
    trace_end(slot, st, TR_ROWS, 0.0, 4.0 * p.n_tok * heads * head_dim);
  }
  return SPD_OK;
}

}  // namespace spd

using namespace spd;

extern "C" int spd_rope_pages(const uint16_t* q, int ldq, const uint16_t* kv, int ldkv, int n_tok, const int32_t* pos, int n_axes,
                              const uint8_t* axis, float theta, const int32_t* q_cu, const int32_t* len, int n_seqs,
                              const int32_t* table, int max_pages, uint16_t* pool, int n_pages, int page_size, int n_heads,
                              int n_kv_heads, int head_dim, uint16_t* q_out, void* ws, void* stream) {
  if (!q || !kv || !pos || !q_cu || !len || !table || !q_out || n_tok < 0 || n_seqs < 1 || n_axes < 1 || n_axes > 255 ||
      n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads)
    return fail(SPD_EINVAL, "bad rotary arguments");
  if (!(theta > 0.0f) || !isfinite(theta)) return fail(SPD_EINVAL, "theta must be positive and finite");
  if (int rc = pool_check(pool, 1, n_pages, page_size, n_kv_heads, head_dim, max_pages)) return rc;
  if (ldq < n_heads * head_dim || ldkv < 2 * n_kv_heads * head_dim || ldq % 8 || ldkv % 8)
    return fail(SPD_EINVAL, "row strides must hold a row and be multiples of 8");
  if (misaligned(q, 16) || misaligned(kv, 16) || misaligned(q_out, 16)) return fail(SPD_EINVAL, "q, kv and q_out must be 16-byte aligned");
  if (q == q_out && ldq != n_heads * head_dim) return fail(SPD_EINVAL, "in place, rows of q must lie side by side");
  if (int rc = paged_check(q_cu, n_tok, len, nullptr, n_seqs, max_pages, page_size)) return rc;
  return rope_pages_run(q, ldq, kv, ldkv, pos, n_axes, axis, theta, q_cu, len, n_seqs, table, max_pages, pool, n_pages, page_size,
                        n_heads, n_kv_heads, head_dim, q_out, static_cast<int*>(ws), static_cast<cudaStream_t>(stream));
}

extern "C" size_t spd_pages_workspace_size(int n_pages, int n_seqs) {
  if (n_pages < 1 || n_seqs < 1) return 0;
  Carve cv(nullptr, ~size_t(0));
  carve_pages(cv, n_pages, n_seqs);
  return cv.used;
}

extern "C" int spd_pages_update(uint16_t* pool, int n_layers, int n_pages, int page_size, int n_kv_heads, int head_dim,
                                const int32_t* ref_in, const int32_t* table_in, const int32_t* len_in, int n_in,
                                const int32_t* parent, const int32_t* grow, int n_out, int max_pages, int32_t* ref_out,
                                int32_t* table_out, int32_t* len_out, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = pool_check(pool, n_layers, n_pages, page_size, n_kv_heads, head_dim, max_pages)) return rc;
  if (!ref_in || !table_in || !len_in || !ref_out || !table_out || !len_out || !ws || n_in < 1 || n_out < 1)
    return fail(SPD_EINVAL, "bad page table arguments");
  if (!parent && n_in != n_out) return fail(SPD_EINVAL, "without parents there are as many sequences after as before");
  if ((long long)std::max(n_in, n_out) * max_pages > 0x7fffffffLL) return fail(SPD_EUNSUPPORTED, "more than 2^31 - 1 table entries");
  if (table_out == table_in || len_out == len_in) return fail(SPD_EINVAL, "tables and lengths are not updated in place");
  if (misaligned(ws, 16)) return fail(SPD_EINVAL, "ws must be 16-byte aligned");
  Carve cv(ws, ws_bytes);
  const PagesWs w = carve_pages(cv, n_pages, std::max(n_in, n_out));
  if (!cv.fits()) return fail(SPD_ENOSPC, "page workspace too small (%zu < %zu)", ws_bytes, cv.used);
  UpdateArgs p{};
  p.n_pages = n_pages;
  p.page_size = page_size;
  p.n_in = n_in;
  p.n_out = n_out;
  p.max_pages = max_pages;
  p.ref_in = ref_in;
  p.table_in = table_in;
  p.len_in = len_in;
  p.parent = parent;
  p.grow = grow;
  p.ref_out = ref_out;
  p.table_out = table_out;
  p.len_out = len_out;
  p.count = w.count;
  p.free_list = w.free_list;
  p.owner = w.owner;
  p.kids = w.kids;
  p.rows = w.rows;
  p.from = w.from;
  p.more = w.more;
  p.tail = w.tail;
  p.first = w.first;
  p.copy_at = w.copy_at;
  p.copies = w.copies;
  p.n_copies = w.n_copies;
  p.status = cv.status();
  const size_t smem = page_bytes(n_pages, n_in, n_out);
  const bool shared = smem <= kPageShared;
  static DeviceOnce once;
  SPD_CUDA_TRY(once_per_device(once, [] {
    return cudaFuncSetAttribute(pages_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kPageShared));
  }));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int slot = trace_begin(st);
  SPD_CUDA_TRY(launch_pdl(pages_update_kernel, dim3(1), dim3(kPageThreads), shared ? smem : 0, st, p, shared));
  const int rc = copy_pages(pool, w.copies, w.n_copies, n_out, n_layers, n_pages, page_size, n_kv_heads * head_dim / 4, st);
  trace_end(slot, st, TR_ROWS, 0.0, 8.0 * n_pages + 4.0 * (double(n_in) + n_out) * max_pages);
  return rc;
}

extern "C" int spd_pages_compact(uint16_t* pool, int n_layers, int n_pages, int page_size, int n_kv_heads, int head_dim,
                                 const int32_t* ref_in, const int32_t* table_in, int n_seqs, int max_pages, int32_t* ref_out,
                                 int32_t* table_out, int32_t* used, void* ws, size_t ws_bytes, void* stream) {
  if (int rc = pool_check(pool, n_layers, n_pages, page_size, n_kv_heads, head_dim, max_pages)) return rc;
  if (!ref_in || !table_in || !ref_out || !table_out || !used || !ws || n_seqs < 1)
    return fail(SPD_EINVAL, "bad compaction arguments");
  if (misaligned(ws, 16)) return fail(SPD_EINVAL, "ws must be 16-byte aligned");
  Carve cv(ws, ws_bytes);
  const PagesWs w = carve_pages(cv, n_pages, n_seqs);
  if (!cv.fits()) return fail(SPD_ENOSPC, "page workspace too small (%zu < %zu)", ws_bytes, cv.used);
  CompactArgs p{n_pages, page_size, n_seqs,  max_pages,   ref_in,   table_in,   ref_out,
                table_out, used,    w.count, w.free_list, w.copies, w.n_copies, cv.status()};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int slot = trace_begin(st);
  SPD_CUDA_TRY(launch_pdl(pages_compact_kernel, dim3(1), dim3(kPageThreads), 0, st, p));
  const int rc = copy_pages(pool, w.copies, w.n_copies, (n_pages + 1) / 2, n_layers, n_pages, page_size, n_kv_heads * head_dim / 4, st);
  trace_end(slot, st, TR_ROWS, 0.0, 8.0 * n_pages + 8.0 * double(n_seqs) * max_pages);
  return rc;
}
