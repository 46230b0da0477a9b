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
// steps bound them, not the memory.  Both numberings are prefix sums over the pages and
// the sequences: one launch of a cluster of eight blocks, whose sums meet in shared
// memory, instead of a launch per step.
//
// copy and write move every byte once and are bound by HBM.
#include <atomic>

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

// The cluster's sums of one value per block: before this block, and of all.
__device__ __forceinline__ int cluster_sum(int mine, int* slot, int rank, int blocks, int* all) {
  if (threadIdx.x == 0) *slot = mine;
  __syncthreads();
  cluster_sync_all();
  int before = 0, sum = 0;
  for (int i = 0; i < blocks; ++i) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(smem_u32(slot), i)) : "memory");
    if (i < rank) before += v;
    sum += v;
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

// References to `page`, counted together where lanes of a warp name the same one.
__device__ __forceinline__ void count_page(int* refs, int page) {
  if (page >= 0) atomicAdd(&refs[page], 1);      // whole numbers: the order does not matter
}

// One block for small tables: the counts are cleared, then entries counted.
__global__ void __launch_bounds__(kThreads) k_fork_small(const __grid_constant__ ForkArgs A) {
  for (int p = threadIdx.x; p < A.s.n_pages; p += kThreads) A.refs[p] = 0;
  __syncthreads();
  const int cells = A.s.n_seqs * A.s.table_row;
  for (int c = threadIdx.x; c < cells; c += kThreads) {
    const int page = fork_entry(A, c / A.s.table_row, c % A.s.table_row);
    A.table_out[c] = page;
    count_page(A.refs, page);
  }
  for (int s = threadIdx.x; s < A.s.n_seqs; s += kThreads) {
    int p;
    A.length_out[s] = fork_length(A, s, &p);
  }
}

// Larger ones in two launches: entries are written and counts cleared, then counted.
__global__ void __launch_bounds__(256) k_fork_table(const __grid_constant__ ForkArgs A) {
  pdl_trigger();
  const long long step = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  for (long long p = first; p < A.s.n_pages; p += step) A.refs[p] = 0;
  const long long cells = (long long)A.s.n_seqs * A.s.table_row;
  for (long long c = first; c < cells; c += step)
    A.table_out[c] = fork_entry(A, (int)(c / A.s.table_row), (int)(c % A.s.table_row));
  for (long long s = first; s < A.s.n_seqs; s += step) {
    int p;
    A.length_out[s] = fork_length(A, (int)s, &p);
  }
}
__global__ void __launch_bounds__(256) k_fork_count(const int* table, int* refs, long long cells) {
  pdl_wait();
  const long long step = (long long)gridDim.x * blockDim.x;
  for (long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x; c < cells; c += step) count_page(refs, table[c]);
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
  __shared__ int warp_sum[kWarps], slot_w, slot_f;
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = (int)cluster_ctarank(), blocks = (int)cluster_nctarank();
  // ---- what is wanted, and which pages are free, each block over its share
  const int s0 = (int)((long long)A.s.n_seqs * rank / blocks), s1 = (int)((long long)A.s.n_seqs * (rank + 1) / blocks);
  int wanted = 0;
  for (int s = s0; s < s1; s += kThreads) {
    int n = 0;
    Want w{};
    if (s + tid < s1) {
      w = want_of(A, s + tid);
      n = w.count();
      A.src[s + tid] = w.src;                    // the counts as the call began: kept for later
    }
    int total;
    const int at = wanted + block_sum(n, warp_sum, &total);
    // whether its own last page is asked for rides along in the sign
    if (s + tid < s1) A.offset[s + tid] = w.own ? ~at : at;
    wanted += total;
  }
  const int p0 = (int)((long long)A.s.n_pages * rank / blocks), p1 = (int)((long long)A.s.n_pages * (rank + 1) / blocks);
  int n_free = 0;
  for (int p = p0 + tid; p < p1; p += kThreads) n_free += A.refs[p] == 0;
  int total;
  block_sum(n_free, warp_sum, &total);
  n_free = total;
  int all_wanted, all_free;
  const int want_base = cluster_sum(wanted, &slot_w, rank, blocks, &all_wanted);
  const int free_base = cluster_sum(n_free, &slot_f, rank, blocks, &all_free);
  // ---- the free pages that will be given, in order
  int at_free = free_base;
  for (int p = p0; p < p1 && at_free < all_wanted; p += kThreads) {
    const bool is = p + tid < p1 && A.refs[p + tid] == 0;
    const int k = at_free + block_sum(is, warp_sum, &total);
    if (is && k < all_wanted) A.free_list[k] = p + tid;
    at_free += total;
  }
  __threadfence();
  cluster_sync_all();
  // ---- given out, a warp per sequence
  const int given = min(all_free, all_wanted);
  for (int s = s0 + (tid >> 5); s < s1; s += kWarps) {
    const int off = A.offset[s], own = off < 0, src = A.src[s];
    const int base = want_base + (own ? ~off : off);
    const int cap = A.s.table_row << A.s.shift, pr = A.s.page_rows;
    const int held = min(max(A.length[s], 0), cap);
    const int end = (int)min((long long)cap, (long long)held + max(A.fresh[s], 0));
    const int first = (held + pr - 1) >> A.s.shift, last = max(first, (end + pr - 1) >> A.s.shift);
    int* row = A.table + (long long)s * A.s.table_row;
    for (int i = first + lane; i < last; i += 32) {
      const int k = base + own + i - first;
      const int page = k < given ? A.free_list[k] : -1;
      row[i] = page;
      if (page >= 0) A.refs[page] = 1;
    }
    __syncwarp();
    if (lane == 0) {
      // places that have pages: up to the first one that was not given
      const int got = min(max(given - base, 0), own + last - first);
      int n = end;
      if (got < own + last - first) n = got < own ? held : max(held, (first + got - own) << A.s.shift);
      int from = -1, to = -1, rows = 0;
      if (own) {
        const int page = got > 0 ? A.free_list[base] : -1;
        if (page >= 0) {
          row[held >> A.s.shift] = page;
          A.refs[page] = 1;
          if (src >= 0) {
            atomicSub(&A.refs[src], 1);
            from = src;
            to = page;
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
    }
  }
  if (rank == 0 && tid == 0 && A.missing) *A.missing = all_wanted - given;
  cluster_sync_all();                            // no block's sums go while another reads them
}

// ---------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------

struct CompactArgs {
  const int *table, *refs;
  int *table_out, *refs_out, *src, *dst, *count;
  int *to, *n_live;                              // workspace: [n_pages], [1]
  int remap;                                     // 1: the table is written here too
  PageShape s;
};

__device__ __forceinline__ int new_number(const CompactArgs& A, int page, int n_live) {
  if ((unsigned)page >= (unsigned)A.s.n_pages || A.refs[page] <= 0) return -1;
  return page < n_live ? page : A.to[page];
}

__global__ void __launch_bounds__(kThreads) k_compact(const __grid_constant__ CompactArgs A) {
  __shared__ int warp_sum[kWarps], slot_l, slot_b;
  const int tid = threadIdx.x;
  const int rank = (int)cluster_ctarank(), blocks = (int)cluster_nctarank(), n = A.s.n_pages;
  pdl_trigger();
  const int p0 = (int)((long long)n * rank / blocks), p1 = (int)((long long)n * (rank + 1) / blocks);
  int v = 0, total, live, below;
  for (int p = p0 + tid; p < p1; p += kThreads) v += A.refs[p] > 0;
  block_sum(v, warp_sum, &total);
  const int live_base = cluster_sum(total, &slot_l, rank, blocks, &live);
  v = 0;
  for (int p = p0 + tid; p < min(p1, live); p += kThreads) v += A.refs[p] > 0;
  block_sum(v, warp_sum, &total);
  cluster_sum(total, &slot_b, rank, blocks, &below);
  const int moves = live - below;
  // page p is the at-th in use: a free one below `live` is hole p - at, one in use past
  // it is number at - below among those that move
  int at0 = live_base;
  for (int p = p0; p < p1; p += kThreads) {
    const int i = p + tid;
    const bool in = i < p1, is = in && A.refs[i] > 0;
    const int at = at0 + block_sum(is, warp_sum, &total);
    at0 += total;
    if (!in) continue;
    if (is && i >= live) A.src[at - below] = i;
    if (!is && i < live) A.dst[i - at] = i;
    if (is || i >= live) A.refs_out[i] = i < live ? A.refs[i] : 0;     // holes get theirs below
    if (i >= moves) A.src[i] = A.dst[i] = -1;
  }
  __threadfence();
  cluster_sync_all();
  for (int k = rank * kThreads + tid; k < moves; k += blocks * kThreads) {
    const int from = A.src[k], hole = A.dst[k];
    A.to[from] = hole;
    A.refs_out[hole] = A.refs[from];
  }
  if (rank == 0 && tid == 0) {
    *A.count = moves;
    *A.n_live = live;
  }
  if (A.remap) {
    __threadfence();
    cluster_sync_all();
    const int cells = A.s.n_seqs * A.s.table_row;
    for (int c = rank * kThreads + tid; c < cells; c += blocks * kThreads)
      A.table_out[c] = new_number(A, A.table[c], live);
  }
  cluster_sync_all();
}

__global__ void __launch_bounds__(256) k_compact_table(const __grid_constant__ CompactArgs A) {
  pdl_wait();
  const int live = *A.n_live;
  const long long cells = (long long)A.s.n_seqs * A.s.table_row, step = (long long)gridDim.x * blockDim.x;
  for (long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x; c < cells; c += step)
    A.table_out[c] = new_number(A, A.table[c], live);
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

constexpr int kCopyThreads = 256, kCopyVecs = 8; // 16-byte vectors of a thread and tile

// A tile is 32 KB of a page's keys or values; every thread has eight loads under way
// before its first store.  The listed pages' bytes bound it.
__global__ void __launch_bounds__(kCopyThreads) k_pages_copy(const __grid_constant__ CopyArgs A) {
  const int n = A.count ? min(A.n, *A.count) : A.n;
  const int head = A.s.page_rows * A.s.dim / 16, vecs = A.s.kv_heads * head;   // of a head, of a page's keys
  const long long tiles = (long long)n * A.tiles;
  for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int pair = (int)(t / A.tiles), part = (int)(t % A.tiles);
    const int from = A.src[pair], to = A.dst[pair];
    if ((unsigned)from >= (unsigned)A.s.n_pages || (unsigned)to >= (unsigned)A.n_dst) continue;
    const int rows = A.rows ? min(max(A.rows[pair], 0), A.s.page_rows) : A.s.page_rows;
    const int keep = rows * A.s.dim / 16;        // vectors of a head that are copied
    const bool values = part >= A.tiles / 2;
    const uint4* a = reinterpret_cast<const uint4*>((values ? A.v_src : A.k_src) + from * A.s.page_bytes);
    uint4* b = reinterpret_cast<uint4*>((values ? A.v_dst : A.k_dst) + to * A.s.page_bytes);
    const int v0 = (values ? part - A.tiles / 2 : part) * kCopyThreads * kCopyVecs + threadIdx.x;
    uint4 x[kCopyVecs];
    bool on[kCopyVecs];
#pragma unroll
    for (int u = 0; u < kCopyVecs; ++u) {
      const int v = v0 + u * kCopyThreads;
      on[u] = v < vecs && v % head < keep;
      if (on[u]) x[u] = __ldcs(a + v);
    }
#pragma unroll
    for (int u = 0; u < kCopyVecs; ++u)
      if (on[u]) __stcs(b + v0 + u * kCopyThreads, x[u]);
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

// A warp per block of 16 places, key head, and keys or values: 16 x dim numbers stay in
// registers between the search for the largest and the rounding.  Lane l has the
// 8-number units l, l + 32, ... of the block, row by row, so loads and stores of
// neighbouring lanes are neighbours.  Keys and values of neighbouring heads are
// neighbouring warps' work, as they are neighbours in a packed projection.
template <typename T, int J>                     // J = dim / 16 units of a lane
__global__ void __launch_bounds__(kWriteThreads) k_pages_write(const __grid_constant__ WriteArgs A) {
  constexpr int U = 2 * J;                       // units of a row
  const int lane = threadIdx.x & 31;
  long long item = (long long)blockIdx.x * (kWriteThreads / 32) + (threadIdx.x >> 5);
  const int head = (int)(item % A.s.kv_heads);
  item /= A.s.kv_heads;
  const bool values = item & 1;
  item >>= 1;
  const int b0 = (int)(item % A.blocks);
  const long long seq = item / A.blocks;
  if (seq >= A.s.n_seqs) return;
  const int t0 = min(max(A.offsets[seq], 0), A.n_tokens), t1 = min(max(A.offsets[seq + 1], t0), A.n_tokens);
  const int cap = A.s.table_row << A.s.shift;
  const int held = min(max(A.held[seq], 0), cap);
  int end = (int)min((long long)held + (t1 - t0), (long long)cap);
  if (A.length) end = min(end, max(A.length[seq], 0));
  const T* x0 = static_cast<const T*>(values ? A.v : A.k) + head * (values ? A.v_head : A.k_head);
  const long long row = values ? A.v_row : A.k_row;
  unsigned char* pages = values ? A.v_pages : A.k_pages;
  for (long long b = held / kPageBlock + b0; b * kPageBlock < end; b += A.blocks) {
    const int place = (int)b * kPageBlock;
    const int page = A.table[seq * A.s.table_row + (place >> A.s.shift)];
    if ((unsigned)page >= (unsigned)A.s.n_pages) continue;
    const int r0 = place & (A.s.page_rows - 1);
    const int lo = max(held - place, 0), hi = min(end - place, kPageBlock);      // rows [0, lo) are old, [lo, hi) new
    uint4 x[J];
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int i = j * 32 + lane, r = i / U, c = i % U;
      x[j] = make_uint4(0u, 0u, 0u, 0u);
      if (r >= lo && r < hi)
        x[j] = __ldcs(reinterpret_cast<const uint4*>(x0 + (long long)(t0 + place + r - held) * row + c * 8));
    }
    unsigned char* block = pages + page * A.s.page_bytes + ((long long)head * A.s.page_rows + r0) * A.s.dim;
    signed char* scale = A.scales + page * A.s.scale_bytes +
                         ((long long)head * (A.s.page_rows / kPageBlock) + r0 / kPageBlock) * 2 + values;
    const int was = lo > 0 ? *scale : kExpMin;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t u[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const float2 f = Store<T>::unpack2(u[h]);
        const float a = fabsf(f.x), c = fabsf(f.y);
        top = fmaxf(top, a < INFINITY ? a : 0.f);
        top = fmaxf(top, c < INFINITY ? c : 0.f);
      }
    }
    top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));
    const int e = max(least_exponent(top), min(max(was, kExpMin), kExpMax));
    const float down = pow2(-e);
    if (lane == 0) *scale = (signed char)e;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int i = j * 32 + lane, r = i / U, c = i % U;
      uint2* dst = reinterpret_cast<uint2*>(block + r * A.s.dim + c * 8);
      if (r >= lo && r < hi) {
        const uint32_t u[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
        uint32_t y[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          float2 f = Store<T>::unpack2(u[h]);
          f.x = fabsf(f.x) < INFINITY ? f.x * down : NAN;
          f.y = fabsf(f.y) < INFINITY ? f.y * down : NAN;
          y[h] = to_e4m3x2(f.x, f.y);
        }
        *dst = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
      } else if (r < lo && e > was) {
        // numbers of before, whose exponent rose: 2^(was - e) below 2^-30 leaves 0
        const uint2 z = *dst;
        const float f = pow2(max(was - e, -60));
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
  }
}

template <typename T>
cudaError_t launch_write(const WriteArgs& a, long long grid, cudaStream_t st) {
  const dim3 g((unsigned)grid), b(kWriteThreads);
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
bool bad_stride(int64_t s) { return s < 0 || s % 8 != 0 || s > (1LL << 40); }
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
  if (work <= 4 * kThreads) {
    k_fork_small<<<1, kThreads, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
  }
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
  a.tiles = 2 * ((vecs + kCopyThreads * kCopyVecs - 1) / (kCopyThreads * kCopyVecs));
  long long grid = (long long)n * a.tiles;
  if (grid > sms * 8LL) grid = sms * 8LL;
  k_pages_copy<<<(unsigned)grid, kCopyThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}

extern "C" rtcc_status rtcc_pages_write(const rtcc_page_config* cfg, const rtcc_write_config* t, const void* d_k,
                                        const void* d_v, const int32_t* d_offsets, const int32_t* d_held,
                                        const int32_t* d_length, const int32_t* d_table, void* d_k_pages,
                                        void* d_v_pages, void* d_scales, void* stream) {
  WriteArgs a{};
  if (!page_shape(cfg, &a.s) || !t) return RTCC_E_ARG;
  if ((t->dtype != RTCC_FP16 && t->dtype != RTCC_BF16) || t->n_tokens < 0 || t->max_new < 0 || t->reserved) return RTCC_E_ARG;
  if (bad_stride(t->k_row) || bad_stride(t->k_head) || bad_stride(t->v_row) || bad_stride(t->v_head)) return RTCC_E_ARG;
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
  a.k = d_k; a.v = d_v; a.offsets = d_offsets; a.held = d_held; a.length = d_length; a.table = d_table;
  a.k_pages = static_cast<unsigned char*>(d_k_pages); a.v_pages = static_cast<unsigned char*>(d_v_pages);
  a.scales = static_cast<signed char*>(d_scales);
  a.k_row = t->k_row; a.k_head = t->k_head; a.v_row = t->v_row; a.v_head = t->v_head;
  a.n_tokens = t->n_tokens;
  const int most = t->max_new < 1 ? 1 : t->max_new > t->n_tokens ? t->n_tokens : t->max_new;
  long long blocks = (most + 14LL) / kPageBlock + 1;       // that they touch at most, wherever they begin
  const long long each = (long long)a.s.n_seqs * a.s.kv_heads * 2;
  constexpr long long kMostWarps = (1LL << 31) * (kWriteThreads / 32) - 64;
  while (each * blocks > kMostWarps && blocks > 1) blocks = (blocks + 1) / 2;      // warps then loop
  if (each * blocks > kMostWarps) return RTCC_E_ARG;
  a.blocks = (int)blocks;
  const long long grid = (each * blocks + kWriteThreads / 32 - 1) / (kWriteThreads / 32);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = t->dtype == RTCC_BF16 ? launch_write<__nv_bfloat16>(a, grid, st) : launch_write<__half>(a, grid, st);
  return e == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}
