// Paged token memory: which pages sequences have, copies of pages, and new tokens
// rounded into them.
//
// fork, extend and compact work on tables and reference counts alone:
//   fork      table'[s][i] = table[parent_s][i] where i page_rows < length'_s,
//             length'_s = min(length[parent_s], keep_s), without pages that lie past the
//             sinks and behind the window; refs[p] = number of entries naming p;
//   extend    the k-th wanted page (by sequence, then place) is the k-th page p with
//             refs[p] = 0;
//   compact   the k-th page with refs > 0 at or past L, the number of pages in use,
//             moves to the k-th page below L with refs = 0.
// They read and write a few hundred kilobytes, so the launch and a chain of dependent
// steps bound them, not the memory.  The numberings of extend and compact are prefix sums
// over the pages and the sequences: one launch of a cluster of eight blocks, whose sums
// meet in shared memory, instead of a launch per step.  fork has no sum, but counts have to
// be cleared before entries are counted: a barrier of the same cluster, or two launches.
//
// Measured: 2048 sequences of up to 13 pages out of 16,384, fork 7 us and extend 10; compact
// over 8192 pages and 16,384 entries 11, over 500 pages and 427 entries 5.  fork in two
// launches over all SMs, which it takes above 65,536 entries, 4 (1,000 entries 3.8 for 3.5,
// 9,000 3.7 for 4.7, 60,000 4.4 for 10.6): from some 5,000 entries on that is the faster one.
//
// copy and write move every byte once and are bound by HBM: 2048 pages of 2 x 64 KB, 537 MB
// read and written, 76 us, 7.0 TB/s; 54,700 tokens of 8 key heads of 112, 294 MB, 50 us,
// 5.9 TB/s.
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "pages.cuh"
#include "rtcc.h"

namespace rtcc {

bool page_shape(const rtcc_page_config* c, PageShape* s) {
  if (!c) return false;
  if (c->kv_heads < 1 || c->kv_heads > 4096 || c->head_dim < 16 || c->head_dim > 128 || c->head_dim % 16) return false;
  if (c->page_rows != 32 && c->page_rows != 64 && c->page_rows != 128) return false;
  if (c->n_pages < 0 || c->n_pages > (1 << 26) || c->n_seqs < 0 || c->table_row < 0) return false;
  constexpr long long kMost = 1LL << 30;
  if ((long long)c->table_row * c->page_rows > kMost || (long long)c->n_seqs * c->table_row > kMost) return false;
  const long long dense = (long long)c->kv_heads * c->page_rows * c->head_dim;
  const long long scales = (long long)c->kv_heads * (c->page_rows / kPageBlock) * 2;
  if (c->page_bytes % 16 || c->scale_bytes % 4) return false;
  if ((c->page_bytes && c->page_bytes < dense) || (c->scale_bytes && c->scale_bytes < scales)) return false;
  if (c->page_bytes > (1LL << 40) || c->scale_bytes > (1LL << 40)) return false;
  s->page_bytes = c->page_bytes ? c->page_bytes : dense;
  s->scale_bytes = c->scale_bytes ? c->scale_bytes : scales;
  s->kv_heads = c->kv_heads; s->dim = c->head_dim; s->page_rows = c->page_rows;
  s->shift = c->page_rows == 32 ? 5 : c->page_rows == 64 ? 6 : 7;
  s->n_pages = c->n_pages; s->n_seqs = c->n_seqs; s->table_row = c->table_row;
  return true;
}

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kBlocks = 8;                       // of the cluster

// Exclusive sum over the block of one value per thread; *total = the sum of all.
__device__ __forceinline__ int block_sum(int v, int* warp_sum, int* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) warp_sum[w] = x;
  __syncthreads();
  const int s = warp_sum[lane];                  // kWarps = 32
  int before = s;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, before, d);
    if (lane >= d) before += y;
  }
  *total = __shfl_sync(0xFFFFFFFFu, before, 31);
  before = __shfl_sync(0xFFFFFFFFu, before - s, w);
  __syncthreads();
  return before + x - v;
}

// The cluster's sums of two values per block: before this block, and of all.  Peers'
// shared memory is read before the next barrier of the cluster, which there has to be.
__device__ __forceinline__ int2 cluster_sum(int2 mine, int2* slot, int rank, int blocks, int2* all) {
  if (threadIdx.x == 0) *slot = mine;
  __syncthreads();
  cluster_sync_all();
  int2 before = make_int2(0, 0), sum = make_int2(0, 0);
  for (int i = 0; i < blocks; ++i) {
    int2 v;
    asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];"
                 : "=r"(v.x), "=r"(v.y)
                 : "r"(mapa_shared(smem_u32(slot), i))
                 : "memory");
    if (i < rank) {
      before.x += v.x;
      before.y += v.y;
    }
    sum.x += v.x;
    sum.y += v.y;
  }
  *all = sum;
  return before;
}

// ---------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------

struct ForkArgs {
  const int *parent, *keep, *length, *table;
  int *length_out, *table_out, *refs;
  int n_from, window, sinks;
  PageShape s;
};

__device__ __forceinline__ int fork_length(const ForkArgs& A, int seq, int* from) {
  const int p = A.parent[seq];
  *from = p;
  if (p < 0 || p >= A.n_from) return 0;
  int n = min(A.length[p], A.s.table_row << A.s.shift);
  if (A.keep) n = min(n, A.keep[seq]);
  return max(n, 0);
}

__device__ __forceinline__ int fork_entry(const ForkArgs& A, int seq, int i) {
  int p;
  const int n = fork_length(A, seq, &p);
  const int place = i << A.s.shift;
  if (place >= n) return -1;
  if (A.window > 0 && place >= A.sinks && (long long)place + A.s.page_rows - 1 + A.window <= n) return -1;
  const int page = A.table[(long long)p * A.s.table_row + i];
  return (unsigned)page < (unsigned)A.s.n_pages ? page : -1;
}

// Four entries at a time, step apart: their chains of loads (parent, length, entry) run
// beside one another.
__device__ __forceinline__ void fork_cells(const ForkArgs& A, long long first, long long step, bool count) {
  const long long cells = (long long)A.s.n_seqs * A.s.table_row;
  for (long long c0 = first; c0 < cells; c0 += 4 * step) {
    int page[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long c = c0 + u * step;
      page[u] = c < cells ? fork_entry(A, (int)(c / A.s.table_row), (int)(c % A.s.table_row)) : -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (c0 + u * step < cells) {
        A.table_out[c0 + u * step] = page[u];
        if (count && page[u] >= 0) atomicAdd(&A.refs[page[u]], 1);       // whole numbers: the order does not matter
      }
  }
  for (long long s = first; s < A.s.n_seqs; s += step) {
    int p;
    A.length_out[s] = fork_length(A, (int)s, &p);
  }
}

// Small tables in one launch of a cluster: counts are cleared, then entries counted.
__global__ void __launch_bounds__(kThreads) k_fork(const __grid_constant__ ForkArgs A) {
  const int rank = (int)cluster_ctarank(), blocks = (int)cluster_nctarank();
  for (int p = rank * kThreads + threadIdx.x; p < A.s.n_pages; p += blocks * kThreads) A.refs[p] = 0;
  __threadfence();
  cluster_sync_all();
  fork_cells(A, rank * kThreads + threadIdx.x, blocks * kThreads, true);
}

// Larger ones in two: entries are written and counts cleared, then counted.
__global__ void __launch_bounds__(256) k_fork_table(const __grid_constant__ ForkArgs A) {
  pdl_trigger();
  const long long step = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  for (long long p = first; p < A.s.n_pages; p += step) A.refs[p] = 0;
  fork_cells(A, first, step, false);
}
__global__ void __launch_bounds__(256) k_fork_count(const int* table, int* refs, long long cells) {
  pdl_wait();
  const long long step = (long long)gridDim.x * blockDim.x;
  for (long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x; c < cells; c += step) {
    const int page = table[c];
    if (page >= 0) atomicAdd(&refs[page], 1);
  }
}

// ---------------------------------------------------------------------------
// extend
// ---------------------------------------------------------------------------

struct ExtendArgs {
  const int *fresh, *length;
  int *table, *refs, *length_out, *src, *dst, *rows, *missing;
  int *free_list, *offset;                       // workspace: [n_pages], [n_seqs]
  PageShape s;
};

// What a sequence asks for: `own` 1 if its last held page needs a substitute (src: the
// page it shares, -1 if there is none), then entries [first, last).
struct Want {
  int held, end, first, last, own, src;
  __device__ __forceinline__ int count() const { return own + last - first; }
};
__device__ __forceinline__ Want want_of(const ExtendArgs& A, int seq) {
  Want w;
  const int cap = A.s.table_row << A.s.shift, pr = A.s.page_rows;
  w.held = min(max(A.length[seq], 0), cap);
  w.end = (int)min((long long)cap, (long long)w.held + max(A.fresh[seq], 0));
  w.first = (w.held + pr - 1) >> A.s.shift;
  w.last = max(w.first, (w.end + pr - 1) >> A.s.shift);
  w.own = 0;
  w.src = -1;
  if (w.end > w.held && (w.held & (pr - 1))) {
    const int page = A.table[(long long)seq * A.s.table_row + (w.held >> A.s.shift)];
    if ((unsigned)page >= (unsigned)A.s.n_pages) {
      w.own = 1;
    } else if (A.refs[page] > 1) {
      w.own = 1;
      w.src = page;
    }
  }
  return w;
}

__global__ void __launch_bounds__(kThreads) k_extend(const __grid_constant__ ExtendArgs A) {
  __shared__ int warp_sum[kWarps];
  __shared__ int2 slot;
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = (int)cluster_ctarank(), blocks = (int)cluster_nctarank();
  // ---- what is wanted, and which pages are free, each block over its share
  const int s0 = (int)((long long)A.s.n_seqs * rank / blocks), s1 = (int)((long long)A.s.n_seqs * (rank + 1) / blocks);
  const int p0 = (int)((long long)A.s.n_pages * rank / blocks), p1 = (int)((long long)A.s.n_pages * (rank + 1) / blocks);
  int n_free = 0, wanted = 0, total;
#pragma unroll 4
  for (int p = p0 + tid; p < p1; p += kThreads) n_free += A.refs[p] == 0;
  for (int s = s0; s < s1; s += kThreads) {
    int n = 0;
    Want w{};
    if (s + tid < s1) {
      w = want_of(A, s + tid);
      n = w.count();
      A.src[s + tid] = w.src;                    // the counts as the call began: kept for later
    }
    const int at = wanted + block_sum(n, warp_sum, &total);
    // whether its own last page is asked for rides along in the sign
    if (s + tid < s1) A.offset[s + tid] = w.own ? ~at : at;
    wanted += total;
  }
  block_sum(n_free, warp_sum, &total);
  int2 all;
  const int2 base = cluster_sum(make_int2(wanted, total), &slot, rank, blocks, &all);
  // ---- the free pages that will be given, in order
  int at_free = base.y;
  for (int p = p0; p < p1 && at_free < all.x; p += kThreads) {
    const bool is = p + tid < p1 && A.refs[p + tid] == 0;
    const int k = at_free + block_sum(is, warp_sum, &total);
    if (is && k < all.x) A.free_list[k] = p + tid;
    at_free += total;
  }
  __threadfence();
  cluster_sync_all();
  // ---- given out: a thread per sequence for its own page and the first few, its warp
  // for what is left of long ones
  const int given = min(all.x, all.y);
  constexpr int kFew = 4;
  for (int s = s0 + tid; s - lane < s1; s += kThreads) {
    int k0 = 0, i0 = 0, i1 = 0;                  // wanted page i0 + n is number k0 + n
    if (s < s1) {
      const int off = A.offset[s], own = off < 0, src = A.src[s];
      const int cap = A.s.table_row << A.s.shift, pr = A.s.page_rows;
      const int held = min(max(A.length[s], 0), cap);
      const int end = (int)min((long long)cap, (long long)held + max(A.fresh[s], 0));
      const int first = (held + pr - 1) >> A.s.shift, last = max(first, (end + pr - 1) >> A.s.shift);
      const int k = base.x + (own ? ~off : off);
      int* row = A.table + (long long)s * A.s.table_row;
      k0 = k + own;
      i0 = first;
      i1 = last;
      int page[kFew + 1];
#pragma unroll
      for (int u = 0; u <= kFew; ++u) page[u] = u < own + last - first && k + u < given ? A.free_list[k + u] : -1;
      // places that have pages: up to the first one that was not given
      const int got = min(max(given - k, 0), own + last - first);
      int n = end;
      if (got < own + last - first) n = got < own ? held : max(held, (first + got - own) << A.s.shift);
      int from = -1, to = -1, rows = 0;
      if (own) {
        if (page[0] >= 0) {
          row[held >> A.s.shift] = page[0];
          A.refs[page[0]] = 1;
          if (src >= 0) {
            atomicSub(&A.refs[src], 1);
            from = src;
            to = page[0];
            rows = held & (pr - 1);
          }
        } else if (src < 0) {
          row[held >> A.s.shift] = -1;
        }
      }
      A.src[s] = from;
      A.dst[s] = to;
      A.rows[s] = rows;
      A.length_out[s] = n;
#pragma unroll
      for (int u = 0; u < kFew; ++u) {
        if (i0 >= i1) break;
        const int p = own ? page[u + 1] : page[u];
        row[i0++] = p;
        ++k0;
        if (p >= 0) A.refs[p] = 1;
      }
    }
    for (unsigned left = __ballot_sync(0xFFFFFFFFu, i0 < i1); left; left &= left - 1) {
      const int l = __ffs(left) - 1;
      const int k = __shfl_sync(0xFFFFFFFFu, k0, l), a = __shfl_sync(0xFFFFFFFFu, i0, l), b = __shfl_sync(0xFFFFFFFFu, i1, l);
      int* row = A.table + (long long)(s - lane + l) * A.s.table_row;
      for (int i = a + lane; i < b; i += 32) {
        const int p = k + i - a < given ? A.free_list[k + i - a] : -1;
        row[i] = p;
        if (p >= 0) A.refs[p] = 1;
      }
    }
  }
  if (rank == 0 && tid == 0 && A.missing) *A.missing = all.x - given;
}

// ---------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------

struct CompactArgs {
  const int *table, *refs;
  int *table_out, *refs_out, *src, *dst, *count;
  int *to, *n_live;                              // workspace: [n_pages], [2]
  int remap;                                     // 1: the table is written here too
  PageShape s;
};

// refs > 0 and number at or past n_live: `to` has the page's number among those in use.
__device__ __forceinline__ int new_number(const CompactArgs& A, int page, int n_live, int below) {
  if ((unsigned)page >= (unsigned)A.s.n_pages || A.refs[page] <= 0) return -1;
  return page < n_live ? page : A.dst[A.to[page] - below];
}

// Four entries at a time, as in fork_cells.
__device__ __forceinline__ void compact_cells(const CompactArgs& A, int n_live, int below, long long first, long long step) {
  const long long cells = (long long)A.s.n_seqs * A.s.table_row;
  for (long long c0 = first; c0 < cells; c0 += 4 * step) {
    int page[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) page[u] = c0 + u * step < cells ? A.table[c0 + u * step] : -1;
#pragma unroll
    for (int u = 0; u < 4; ++u) page[u] = new_number(A, page[u], n_live, below);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (c0 + u * step < cells) A.table_out[c0 + u * step] = page[u];
  }
}

__global__ void __launch_bounds__(kThreads) k_compact(const __grid_constant__ CompactArgs A) {
  __shared__ int warp_sum[kWarps];
  __shared__ int2 slot, slot_below;
  const int tid = threadIdx.x;
  const int rank = (int)cluster_ctarank(), blocks = (int)cluster_nctarank(), n = A.s.n_pages;
  pdl_trigger();
  const int p0 = (int)((long long)n * rank / blocks), p1 = (int)((long long)n * (rank + 1) / blocks);
  int v = 0, total;
#pragma unroll 4
  for (int p = p0 + tid; p < p1; p += kThreads) v += A.refs[p] > 0;
  block_sum(v, warp_sum, &total);
  int2 all;
  const int base = cluster_sum(make_int2(total, 0), &slot, rank, blocks, &all).x, live = all.x;
  // page p is the at-th in use: a free one below `live` is hole p - at, one in use past
  // it the at-th of all, that is number at - below among those that move, where `below`
  // pages in use stay
  int at0 = base, stay = 0;
  for (int p = p0; p < p1; p += kThreads) {
    const int i = p + tid, count = i < p1 ? A.refs[i] : 0;
    const int at = at0 + block_sum(count > 0, warp_sum, &total);
    at0 += total;
    if (i >= p1) continue;
    if (count > 0) {
      A.to[i] = at;
      stay += i < live;
    }
    if (count <= 0 && i < live) A.dst[i - at] = i;
    if (count > 0 || i >= live) A.refs_out[i] = i < live ? count : 0;    // holes get theirs below
  }
  block_sum(stay, warp_sum, &total);
  __threadfence();
  const int below = (cluster_sum(make_int2(total, 0), &slot_below, rank, blocks, &all), all.x), moves = live - below;
  for (int i = p0 + tid; i < p1; i += kThreads) {
    if (i >= live && A.refs[i] > 0) {
      const int k = A.to[i] - below, hole = A.dst[k];
      A.src[k] = i;
      A.refs_out[hole] = A.refs[i];
    }
    if (i >= moves) A.src[i] = A.dst[i] = -1;    // no hole's number: those are below `moves`
  }
  if (rank == 0 && tid == 0) {
    *A.count = moves;
    A.n_live[0] = live;
    A.n_live[1] = below;
  }
  if (A.remap) compact_cells(A, live, below, rank * kThreads + tid, blocks * kThreads);
  cluster_sync_all();                            // no block's sums go while another reads them
}

__global__ void __launch_bounds__(256) k_compact_table(const __grid_constant__ CompactArgs A) {
  pdl_wait();
  compact_cells(A, A.n_live[0], A.n_live[1], (long long)blockIdx.x * blockDim.x + threadIdx.x, (long long)gridDim.x * blockDim.x);
}

// ---------------------------------------------------------------------------
// copy
// ---------------------------------------------------------------------------

struct CopyArgs {
  const int *count, *src, *dst, *rows;
  const unsigned char *k_src, *v_src, *s_src;
  unsigned char *k_dst, *v_dst, *s_dst;
  int n, n_dst, tiles;                           // tiles of a pair
  PageShape s;
};

constexpr int kCopyThreads = 256;

// A tile is kCopyVecs 16-byte vectors of every thread, of a page's keys or values: up to 32 KB,
// eight loads under way before the first store.  The listed pages' bytes bound it.
template <int kCopyVecs>
__global__ void __launch_bounds__(kCopyThreads) k_pages_copy(const __grid_constant__ CopyArgs A) {
  const int n = A.count ? min(A.n, *A.count) : A.n;
  const int head = A.s.page_rows * A.s.dim / 16, vecs = A.s.kv_heads * head;   // of a head, of a page's keys
  // block b takes tile b % tiles of pairs b / tiles, ...: gridDim.x is a multiple of the tiles
  const int part = (int)blockIdx.x % A.tiles;
  const bool values = part >= A.tiles / 2;
  const unsigned char* k_src = values ? A.v_src : A.k_src;
  unsigned char* k_dst = values ? A.v_dst : A.k_dst;
  const int v0 = (values ? part - A.tiles / 2 : part) * kCopyThreads * kCopyVecs + (int)threadIdx.x;
  const int step = (int)gridDim.x / A.tiles;
  for (int pair = (int)blockIdx.x / A.tiles; pair < n; pair += step) {
    const int from = A.src[pair], to = A.dst[pair];
    if ((unsigned)from >= (unsigned)A.s.n_pages || (unsigned)to >= (unsigned)A.n_dst) continue;
    const int rows = A.rows ? min(max(A.rows[pair], 0), A.s.page_rows) : A.s.page_rows;
    const uint4* a = reinterpret_cast<const uint4*>(k_src + from * A.s.page_bytes) + v0;
    uint4* b = reinterpret_cast<uint4*>(k_dst + to * A.s.page_bytes) + v0;
    uint4 x[kCopyVecs];
    if (rows == A.s.page_rows && v0 + (kCopyVecs - 1) * kCopyThreads < vecs) {
#pragma unroll
      for (int u = 0; u < kCopyVecs; ++u) x[u] = __ldcs(a + u * kCopyThreads);
#pragma unroll
      for (int u = 0; u < kCopyVecs; ++u) __stcs(b + u * kCopyThreads, x[u]);
    } else {
      const int keep = rows * A.s.dim / 16;      // vectors of a head that are copied
      bool on[kCopyVecs];
#pragma unroll
      for (int u = 0; u < kCopyVecs; ++u) {
        const int v = v0 + u * kCopyThreads;
        on[u] = v < vecs && v % head < keep;
        if (on[u]) x[u] = __ldcs(a + u * kCopyThreads);
      }
#pragma unroll
      for (int u = 0; u < kCopyVecs; ++u)
        if (on[u]) __stcs(b + u * kCopyThreads, x[u]);
    }
    if (part == 0) {
      const int blocks = A.s.page_rows / kPageBlock, live = (rows + kPageBlock - 1) / kPageBlock;
      const uint16_t* sa = reinterpret_cast<const uint16_t*>(A.s_src + from * A.s.scale_bytes);
      uint16_t* sb = reinterpret_cast<uint16_t*>(A.s_dst + to * A.s.scale_bytes);
      for (int i = threadIdx.x; i < A.s.kv_heads * blocks; i += kCopyThreads)
        if (i % blocks < live) sb[i] = sa[i];
    }
  }
}

// ---------------------------------------------------------------------------
// write
// ---------------------------------------------------------------------------

struct WriteArgs {
  const void *k, *v;
  const int *offsets, *held, *length, *table;
  unsigned char *k_pages, *v_pages;
  signed char* scales;
  long long k_row, k_head, v_row, v_head;
  int n_tokens, blocks;                          // blocks of a sequence that the launch has warps for
  PageShape s;
};

constexpr int kWriteThreads = 256;

// Least e in range with top <= 448 * 2^e.  top = m 2^x with m in [1, 2), 448 = 1.75 * 2^8.
__device__ __forceinline__ int least_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  if ((u >> 23) == 0) return kExpMin;            // 0, or below 2^-126
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return min(max(e, kExpMin), kExpMax);
}

// To e4m3, nearest even; |x| at most 448 (or NaN).
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t v) { return Store<__half>::unpack2(widen_e4m3x2(v)); }

// Eight numbers x of type T, finite, as 8 bits each of x 2^-e.
template <typename T> struct Narrow;
// fp16 all the way: a power of two changes no digits where the product is at least 2^-14,
// and what is smaller rounds to 0 in 8 bits anyway.  2^-e is two factors, since fp16 ends
// at 2^15: e from kLeast on; larger e than 40 leave 0 as 40 does.
template <> struct Narrow<__half> {
  static constexpr int kLeast = -30;
  __half2 f, g;
  __device__ __forceinline__ explicit Narrow(int e) {
    const int n = max(-e, -40), a = n / 2;
    f = __float2half2_rn(pow2(a));
    g = __float2half2_rn(pow2(n - a));
  }
  __device__ __forceinline__ uint32_t two(uint32_t x) const {
    __half2 h = __hmul2(__hmul2(*reinterpret_cast<__half2*>(&x), f), g);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<uint32_t*>(&h)));
    return r;
  }
};
template <> struct Narrow<__nv_bfloat16> {
  static constexpr int kLeast = kExpMin;
  float2 f;
  __device__ __forceinline__ explicit Narrow(int e) { f = make_float2(pow2(-e), pow2(-e)); }
  __device__ __forceinline__ uint32_t two(uint32_t x) const {
    const float2 y = mul2(Store<__nv_bfloat16>::unpack2(x), f);
    return to_e4m3x2(y.x, y.y);
  }
};
// The larger magnitudes of two pairs (signs are anything), NaN where there is one.
template <typename T> __device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t larger2<__half>(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <> __device__ __forceinline__ uint32_t larger2<__nv_bfloat16>(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <typename T> constexpr uint32_t kInfBits = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;

// A warp per block of 16 places, key head, and keys or values (and then the next block of
// the same, fetched while this one is rounded: without that, 58 us for 50): 16 x dim
// numbers stay in registers between the search for the largest and the rounding.
// Lane l has the 8-number units l, l + 32, ... of the block, row by row, so loads and stores of
// neighbouring lanes are neighbours.  Keys and values of neighbouring heads are
// neighbouring warps' work, as they are neighbours in a packed projection.  The largest
// is found two at a time; a block with an infinity or a NaN in it looks again.
template <typename T, int J>                     // J = dim / 16 units of a lane
__global__ void __launch_bounds__(kWriteThreads, 2) k_pages_write(const __grid_constant__ WriteArgs A) {
  constexpr int U = 2 * J;                       // units of a row
  const int lane = threadIdx.x & 31;
  const unsigned item = blockIdx.x * (kWriteThreads / 32) + (threadIdx.x >> 5);
  const int head = (int)(item % (unsigned)A.s.kv_heads), rest = (int)(item / (unsigned)A.s.kv_heads);
  const bool values = rest & 1;
  const int b0 = rest >> 1;
  if (b0 >= A.blocks) return;
  for (long long seq = blockIdx.y; seq < A.s.n_seqs; seq += gridDim.y) {
    const int t0 = min(max(A.offsets[seq], 0), A.n_tokens), t1 = min(max(A.offsets[seq + 1], t0), A.n_tokens);
    const int cap = A.s.table_row << A.s.shift;
    const int held = min(max(A.held[seq], 0), cap);
    int end = (int)min((long long)held + (t1 - t0), (long long)cap);
    if (A.length) end = min(end, max(A.length[seq], 0));
    const T* x0 = static_cast<const T*>(values ? A.v : A.k) + head * (values ? A.v_head : A.k_head);
    const long long row = values ? A.v_row : A.k_row;
    const unsigned row_bytes = (unsigned)row * 2u;
    unsigned char* pages = values ? A.v_pages : A.k_pages;
    // the numbers of block b's new rows, on their way
    auto fetch = [&](long long b, uint4 (&x)[J]) {
      const int place = (int)b * kPageBlock, lo = max(held - place, 0), hi = min(end - place, kPageBlock);
      const char* src = reinterpret_cast<const char*>(x0 + (long long)(t0 + place - held) * row);   // row 0's
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int i = j * 32 + lane, r = i / U, c = i % U;
        x[j] = make_uint4(0u, 0u, 0u, 0u);
        if (r >= lo && r < hi)
          x[j] = __ldcs(reinterpret_cast<const uint4*>(src + (unsigned long long)(unsigned)r * row_bytes + c * 16));
      }
    };
    auto page_at = [&](long long b) -> int { return A.table[seq * A.s.table_row + (b * kPageBlock >> A.s.shift)]; };
    auto store = [&](long long b, int page, const uint4 (&x)[J]) {
      if ((unsigned)page >= (unsigned)A.s.n_pages) return;
      const int place = (int)b * kPageBlock, r0 = place & (A.s.page_rows - 1);
      const int lo = max(held - place, 0), hi = min(end - place, kPageBlock);      // rows [0, lo) are old, [lo, hi) new
      unsigned char* block = pages + page * A.s.page_bytes + ((long long)head * A.s.page_rows + r0) * A.s.dim;
      signed char* scale = A.scales + page * A.s.scale_bytes +
                           ((long long)head * (A.s.page_rows / kPageBlock) + r0 / kPageBlock) * 2 + values;
      const int was = lo > 0 ? min(max((int)*scale, kExpMin), kExpMax) : kExpMin;
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t u[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int h = 0; h < 4; ++h) most = larger2<T>(most, u[h]);
      }
      most = __reduce_max_sync(0xFFFFFFFFu, max(most & 0x7FFFu, most >> 16 & 0x7FFFu));
      const bool finite = most < kInfBits<T>;
      if (!finite) {
        most = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint32_t u[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const uint32_t p = u[h] & 0x7FFFu, q = u[h] >> 16 & 0x7FFFu;
            most = max(most, max(p < kInfBits<T> ? p : 0u, q < kInfBits<T> ? q : 0u));
          }
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
      }
      const int e = max(least_exponent(Store<T>::unpack2(most).x), was);
      if (lane == 0) *scale = (signed char)e;
      const Narrow<T> narrow(e);
      if (finite && e >= Narrow<T>::kLeast) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int i = j * 32 + lane, r = i / U;
          if (r >= lo && r < hi)                   // unit i of the block
            *reinterpret_cast<uint2*>(block + i * 8) =
                make_uint2(__byte_perm(narrow.two(x[j].x), narrow.two(x[j].y), 0x5410),
                           __byte_perm(narrow.two(x[j].z), narrow.two(x[j].w), 0x5410));
        }
      } else {
        const float down = pow2(-e);
#pragma unroll 1
        for (int j = 0; j < J; ++j) {
          const int i = j * 32 + lane, r = i / U;
          if (r < lo || r >= hi) continue;
          uint4 z = x[0];
#pragma unroll
          for (int k = 1; k < J; ++k)
            if (k == j) z = x[k];
          const uint32_t u[4] = {z.x, z.y, z.z, z.w};
          uint32_t y[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            float2 f = Store<T>::unpack2(u[h]);
            f.x = fabsf(f.x) < INFINITY ? f.x * down : NAN;
            f.y = fabsf(f.y) < INFINITY ? f.y * down : NAN;
            y[h] = to_e4m3x2(f.x, f.y);
          }
          *reinterpret_cast<uint2*>(block + i * 8) = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
        }
      }
      if (lo > 0 && e > was) {
        // numbers of before, whose exponent rose: 2^-60 leaves 0 as what is smaller does
        const float f = pow2(max(was - e, -60));
        for (int i = lane; i < lo * U; i += 32) {
          uint2* dst = reinterpret_cast<uint2*>(block + i * 8);
          const uint2 z = *dst;
          const uint32_t u[2] = {z.x, z.y};
          uint32_t y[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 p = from_e4m3x2(u[h] & 0xFFFFu), q = from_e4m3x2(u[h] >> 16);
            y[h] = to_e4m3x2(p.x * f, p.y * f) | to_e4m3x2(q.x * f, q.y * f) << 16;
          }
          *dst = make_uint2(y[0], y[1]);
        }
      }
    };
    uint4 x[J], y[J];
    long long b = held / kPageBlock + b0;
    int page = 0, page_y = 0;
    if (b * kPageBlock < end) {
      fetch(b, x);
      page = page_at(b);
    }
    // two blocks a round, each one's numbers fetched while the other's are rounded
    while (b * kPageBlock < end) {
      const long long next = b + A.blocks;
      const bool more = next * kPageBlock < end;
      if (more) {
        fetch(next, y);
        page_y = page_at(next);
      }
      store(b, page, x);
      b = next;
      if (!more) break;
      b = next + A.blocks;
      if (b * kPageBlock < end) {
        fetch(b, x);
        page = page_at(b);
      }
      store(next, page_y, y);
    }
  }
}

template <typename T>
cudaError_t launch_write(const WriteArgs& a, long long grid, cudaStream_t st) {
  const dim3 g((unsigned)grid, (unsigned)(a.s.n_seqs < 65535 ? a.s.n_seqs : 65535)), b(kWriteThreads);
  switch (a.s.dim / 16) {
    case 1: k_pages_write<T, 1><<<g, b, 0, st>>>(a); break;
    case 2: k_pages_write<T, 2><<<g, b, 0, st>>>(a); break;
    case 3: k_pages_write<T, 3><<<g, b, 0, st>>>(a); break;
    case 4: k_pages_write<T, 4><<<g, b, 0, st>>>(a); break;
    case 5: k_pages_write<T, 5><<<g, b, 0, st>>>(a); break;
    case 6: k_pages_write<T, 6><<<g, b, 0, st>>>(a); break;
    case 7: k_pages_write<T, 7><<<g, b, 0, st>>>(a); break;
    default: k_pages_write<T, 8><<<g, b, 0, st>>>(a); break;
  }
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool overlap(const void* a, long long na, const void* b, long long nb) {
  if (!a || !b || na <= 0 || nb <= 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

template <typename Args>
cudaError_t launch_cluster(void (*kern)(Args), const Args& a, long long work, cudaStream_t st) {
  cudaLaunchConfig_t lc = {};
  lc.blockDim = dim3(kThreads);
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  // one block where it has no more than a thread's worth of work; and where a part of a
  // GPU has no room for eight neighbours
  for (int blocks = work <= kThreads ? 1 : kBlocks;; blocks = 1) {
    lc.gridDim = dim3(blocks);
    at[0].val.clusterDim.x = blocks;
    const cudaError_t e = cudaLaunchKernelEx(&lc, kern, a);
    if (e == cudaSuccess || blocks == 1) return e;
    cudaGetLastError();
  }
}

}  // namespace
}  // namespace rtcc

using namespace rtcc;

extern "C" rtcc_status rtcc_pages_fork(const rtcc_page_config* cfg, int32_t n_from, const int32_t* d_parent,
                                       const int32_t* d_keep, int32_t window, int32_t sinks, const int32_t* d_length,
                                       const int32_t* d_table, int32_t* d_length_out, int32_t* d_table_out,
                                       int32_t* d_refs, void* stream) {
  ForkArgs a{};
  if (!page_shape(cfg, &a.s)) return RTCC_E_ARG;
  const long long n = a.s.n_seqs, cells = n * a.s.table_row, from = (long long)n_from * a.s.table_row;
  if (n_from < 0 || from > (1LL << 30) || window < 0 || sinks < 0) return RTCC_E_ARG;
  if (n > 0 && (!d_parent || !d_length_out)) return RTCC_E_ARG;
  if (n > 0 && n_from > 0 && !d_length) return RTCC_E_ARG;
  if (cells > 0 && (!d_table_out || (n_from > 0 && !d_table))) return RTCC_E_ARG;
  if (a.s.n_pages > 0 && !d_refs) return RTCC_E_ARG;
  const void* all[] = {d_parent, d_keep, d_length, d_table, d_length_out, d_table_out, d_refs};
  for (const void* p : all)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  const struct { const void* p; long long n; } in[] = {{d_parent, 4 * n}, {d_keep, 4 * n}, {d_length, 4LL * n_from}, {d_table, 4 * from}},
      out[] = {{d_length_out, 4 * n}, {d_table_out, 4 * cells}, {d_refs, 4LL * a.s.n_pages}};
  for (const auto& o : out)
    for (const auto& i : in)
      if (overlap(o.p, o.n, i.p, i.n)) return RTCC_E_ARG;
  if (n == 0 && a.s.n_pages == 0) return RTCC_OK;
  a.parent = d_parent; a.keep = d_keep; a.length = d_length; a.table = d_table;
  a.length_out = d_length_out; a.table_out = d_table_out; a.refs = d_refs;
  a.n_from = n_from; a.window = window; a.sinks = sinks;
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const long long work = cells > a.s.n_pages ? (cells > n ? cells : n) : (a.s.n_pages > n ? a.s.n_pages : n);
  if (work <= 8LL * kBlocks * kThreads)
    return launch_cluster(k_fork, a, work, st) == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
  long long grid = (work + 255) / 256;
  if (grid > sms * 8LL) grid = sms * 8LL;
  k_fork_table<<<(unsigned)grid, 256, 0, st>>>(a);
  if (cudaGetLastError() != cudaSuccess) return RTCC_E_CUDA;
  if (cells == 0) return RTCC_OK;
  return launch_pdl(k_fork_count, dim3((unsigned)grid), dim3(256), 0, st, d_table_out, d_refs, cells) == cudaSuccess
             ? RTCC_OK : RTCC_E_CUDA;
}

extern "C" size_t rtcc_pages_workspace(const rtcc_page_config* cfg) {
  PageShape s;
  if (!page_shape(cfg, &s)) return 0;
  return ((size_t)s.n_pages + (size_t)s.n_seqs + 4) * sizeof(int);
}

extern "C" rtcc_status rtcc_pages_extend(const rtcc_page_config* cfg, const int32_t* d_new, const int32_t* d_length,
                                         int32_t* d_table, int32_t* d_refs, int32_t* d_length_out, int32_t* d_copy_src,
                                         int32_t* d_copy_dst, int32_t* d_copy_rows, int32_t* d_short,
                                         void* d_workspace, size_t workspace_bytes, void* stream) {
  ExtendArgs a{};
  if (!page_shape(cfg, &a.s)) return RTCC_E_ARG;
  const long long n = a.s.n_seqs, cells = n * a.s.table_row;
  if (n > 0 && (!d_new || !d_length || !d_length_out || !d_copy_src || !d_copy_dst || !d_copy_rows)) return RTCC_E_ARG;
  if ((cells > 0 && !d_table) || (a.s.n_pages > 0 && !d_refs)) return RTCC_E_ARG;
  if (!d_workspace || workspace_bytes < rtcc_pages_workspace(cfg) || misaligned(d_workspace, 16)) return RTCC_E_ARG;
  const void* all[] = {d_new, d_length, d_table, d_refs, d_length_out, d_copy_src, d_copy_dst, d_copy_rows, d_short};
  for (const void* p : all)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  const struct { const void* p; long long n; } arrays[] = {
      {d_length_out, 4 * n}, {d_copy_src, 4 * n}, {d_copy_dst, 4 * n}, {d_copy_rows, 4 * n}, {d_short, 4},
      {d_table, 4 * cells}, {d_refs, 4LL * a.s.n_pages}, {d_workspace, (long long)rtcc_pages_workspace(cfg)},
      {d_new, 4 * n}, {d_length, 4 * n}};
  for (int i = 0; i < 8; ++i)                    // of the two inputs only d_length may be an output's array
    for (int j = i + 1; j < 10; ++j)
      if (!(i == 0 && j == 9 && d_length_out == d_length) && overlap(arrays[i].p, arrays[i].n, arrays[j].p, arrays[j].n))
        return RTCC_E_ARG;
  a.fresh = d_new; a.length = d_length; a.table = d_table; a.refs = d_refs; a.length_out = d_length_out;
  a.src = d_copy_src; a.dst = d_copy_dst; a.rows = d_copy_rows; a.missing = d_short;
  a.free_list = static_cast<int*>(d_workspace);
  a.offset = a.free_list + a.s.n_pages;
  const long long work = n > a.s.n_pages ? n : a.s.n_pages;
  return launch_cluster(k_extend, a, work, static_cast<cudaStream_t>(stream)) == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}

extern "C" rtcc_status rtcc_pages_compact(const rtcc_page_config* cfg, const int32_t* d_table, const int32_t* d_refs,
                                          int32_t* d_table_out, int32_t* d_refs_out, int32_t* d_move_src,
                                          int32_t* d_move_dst, int32_t* d_count, void* d_workspace,
                                          size_t workspace_bytes, void* stream) {
  CompactArgs a{};
  if (!page_shape(cfg, &a.s)) return RTCC_E_ARG;
  const long long cells = (long long)a.s.n_seqs * a.s.table_row, pages = a.s.n_pages;
  if (cells > 0 && (!d_table || !d_table_out)) return RTCC_E_ARG;
  if (pages > 0 && (!d_refs || !d_refs_out || !d_move_src || !d_move_dst)) return RTCC_E_ARG;
  if (!d_count || !d_workspace || workspace_bytes < rtcc_pages_workspace(cfg) || misaligned(d_workspace, 16))
    return RTCC_E_ARG;
  const void* all[] = {d_table, d_refs, d_table_out, d_refs_out, d_move_src, d_move_dst, d_count};
  for (const void* p : all)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  const struct { const void* p; long long n; } arrays[] = {
      {d_table_out, 4 * cells}, {d_refs_out, 4 * pages}, {d_move_src, 4 * pages}, {d_move_dst, 4 * pages}, {d_count, 4},
      {d_workspace, (long long)rtcc_pages_workspace(cfg)}, {d_refs, 4 * pages}, {d_table, 4 * cells}};
  for (int i = 0; i < 6; ++i)
    for (int j = i + 1; j < 8; ++j)
      if (!(i == 0 && j == 7 && d_table_out == d_table) && overlap(arrays[i].p, arrays[i].n, arrays[j].p, arrays[j].n))
        return RTCC_E_ARG;
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
  a.table = d_table; a.refs = d_refs; a.table_out = d_table_out; a.refs_out = d_refs_out;
  a.src = d_move_src; a.dst = d_move_dst; a.count = d_count;
  a.to = static_cast<int*>(d_workspace);
  a.n_live = a.to + a.s.n_pages;
  a.remap = cells <= 4LL * kBlocks * kThreads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const long long work = a.remap && cells > pages ? cells : pages;
  if (launch_cluster(k_compact, a, work, st) != cudaSuccess) return RTCC_E_CUDA;
  if (a.remap) return RTCC_OK;
  long long grid = (cells + 255) / 256;
  if (grid > sms * 8LL) grid = sms * 8LL;
  return launch_pdl(k_compact_table, dim3((unsigned)grid), dim3(256), 0, st, a) == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}

extern "C" rtcc_status rtcc_pages_copy(const rtcc_page_config* cfg, int32_t n, const int32_t* d_count,
                                       const int32_t* d_src, const int32_t* d_dst, const int32_t* d_rows,
                                       const void* d_k_src, const void* d_v_src, const void* d_scales_src,
                                       int32_t n_pages_dst, void* d_k_dst, void* d_v_dst, void* d_scales_dst,
                                       void* stream) {
  CopyArgs a{};
  if (!page_shape(cfg, &a.s)) return RTCC_E_ARG;
  if (n < 0 || n_pages_dst < 0 || n_pages_dst > (1 << 26)) return RTCC_E_ARG;
  if (n > 0 && (!d_src || !d_dst)) return RTCC_E_ARG;
  if (n > 0 && a.s.n_pages > 0 && n_pages_dst > 0 &&
      (!d_k_src || !d_v_src || !d_scales_src || !d_k_dst || !d_v_dst || !d_scales_dst))
    return RTCC_E_ARG;
  const void* by16[] = {d_k_src, d_v_src, d_k_dst, d_v_dst};
  for (const void* p : by16)
    if (misaligned(p, 16)) return RTCC_E_ARG;
  const void* by4[] = {d_count, d_src, d_dst, d_rows, d_scales_src, d_scales_dst};
  for (const void* p : by4)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  if (n == 0 || a.s.n_pages == 0 || n_pages_dst == 0) return RTCC_OK;
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
  a.count = d_count; a.src = d_src; a.dst = d_dst; a.rows = d_rows;
  a.k_src = static_cast<const unsigned char*>(d_k_src); a.v_src = static_cast<const unsigned char*>(d_v_src);
  a.s_src = static_cast<const unsigned char*>(d_scales_src);
  a.k_dst = static_cast<unsigned char*>(d_k_dst); a.v_dst = static_cast<unsigned char*>(d_v_dst);
  a.s_dst = static_cast<unsigned char*>(d_scales_dst);
  a.n = n; a.n_dst = n_pages_dst;
  const int vecs = a.s.kv_heads * a.s.page_rows * a.s.dim / 16;
  const int per = vecs >= 8 * kCopyThreads ? 8 : vecs >= 4 * kCopyThreads ? 4 : vecs >= 2 * kCopyThreads ? 2 : 1;
  a.tiles = 2 * ((vecs + kCopyThreads * per - 1) / (kCopyThreads * per));
  long long at_once = sms * 32LL / a.tiles;      // pairs
  if (at_once > n) at_once = n;
  if (at_once < 1) at_once = 1;
  const dim3 grid((unsigned)(at_once * a.tiles)), block(kCopyThreads);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (per == 8) k_pages_copy<8><<<grid, block, 0, st>>>(a);
  else if (per == 4) k_pages_copy<4><<<grid, block, 0, st>>>(a);
  else if (per == 2) k_pages_copy<2><<<grid, block, 0, st>>>(a);
  else k_pages_copy<1><<<grid, block, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}

extern "C" rtcc_status rtcc_pages_write(const rtcc_page_config* cfg, const rtcc_write_config* t, const void* d_k,
                                        const void* d_v, const int32_t* d_offsets, const int32_t* d_held,
                                        const int32_t* d_length, const int32_t* d_table, void* d_k_pages,
                                        void* d_v_pages, void* d_scales, void* stream) {
  WriteArgs a{};
  if (!page_shape(cfg, &a.s) || !t) return RTCC_E_ARG;
  if ((t->dtype != RTCC_FP16 && t->dtype != RTCC_BF16) || t->n_tokens < 0 || t->max_new < 0 || t->reserved) return RTCC_E_ARG;
  const int64_t strides[] = {t->k_row, t->k_head, t->v_row, t->v_head};
  for (int64_t s : strides)
    if (s < 0 || s % 8 || s >= (1LL << 31)) return RTCC_E_ARG;
  const long long cells = (long long)a.s.n_seqs * a.s.table_row;
  if (a.s.n_seqs > 0 && (!d_offsets || !d_held || (cells > 0 && !d_table))) return RTCC_E_ARG;
  if (t->n_tokens > 0 && (!d_k || !d_v)) return RTCC_E_ARG;
  if (a.s.n_pages > 0 && (!d_k_pages || !d_v_pages || !d_scales)) return RTCC_E_ARG;
  const void* by16[] = {d_k, d_v, d_k_pages, d_v_pages};
  for (const void* p : by16)
    if (misaligned(p, 16)) return RTCC_E_ARG;
  const void* by4[] = {d_offsets, d_held, d_length, d_table, d_scales};
  for (const void* p : by4)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  if (t->n_tokens == 0 || a.s.n_pages == 0 || cells == 0) return RTCC_OK;
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
  a.k = d_k; a.v = d_v; a.offsets = d_offsets; a.held = d_held; a.length = d_length; a.table = d_table;
  a.k_pages = static_cast<unsigned char*>(d_k_pages); a.v_pages = static_cast<unsigned char*>(d_v_pages);
  a.scales = static_cast<signed char*>(d_scales);
  a.k_row = t->k_row; a.k_head = t->k_head; a.v_row = t->v_row; a.v_head = t->v_head;
  a.n_tokens = t->n_tokens;
  const int most = t->max_new < 1 ? 1 : t->max_new > t->n_tokens ? t->n_tokens : t->max_new;
  long long blocks = (most + 14LL) / kPageBlock + 1;       // that they touch at most, wherever they begin
  const long long each = a.s.kv_heads * 2LL;
  while (each * blocks > 0x3FFFFFFF) blocks = (blocks + 1) / 2;     // warps then loop
  // so do they where there are more than three times as many as run at once, and no more
  // than eight to a block that there is: one long sequence among many short ones
  const long long most_blocks = t->n_tokens / kPageBlock + 2LL * a.s.n_seqs;
  const long long live = blocks * a.s.n_seqs < most_blocks ? blocks * a.s.n_seqs : most_blocks;
  const long long rounds = each * live / (48LL * sms);
  if (rounds > 1) blocks = (blocks + rounds - 1) / rounds;
  if (blocks > 8 * most_blocks / a.s.n_seqs) blocks = 8 * most_blocks / a.s.n_seqs;
  a.blocks = (int)blocks;
  const long long grid = (each * blocks + kWriteThreads / 32 - 1) / (kWriteThreads / 32);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = t->dtype == RTCC_BF16 ? launch_write<__nv_bfloat16>(a, grid, st) : launch_write<__half>(a, grid, st);
  return e == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}
