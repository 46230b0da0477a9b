// Host side of the attention over the token memory: argument checks, the
// choice of kernel and of the split of long spans.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <map>
#include <mutex>
#include <utility>

#include "attn.cuh"
#include "kernels.h"
#include "pages.cuh"
#include "rtcc.h"

namespace rtcc {
namespace {

// The tensor-core kernel takes over from this many (token, head) rows of a key head
// on: 33 rows over 9 ragged histories of 5001 keys, heads of 80, take 24 us there
// and 27 in blocks of 16 rows, 30 rows over 50,000 keys, heads of 64, 25 and 23.
constexpr int kTcRows = 32;
// Over pages, whose keys and values are widened first, from this many on: 4 key heads of
// 128 over 9 ragged histories of 5001 keys take 42 us in blocks of 16 rows and 53 there at
// 68 rows, 59 and 61 at 132, 95 and 74 at 200.
constexpr int kTcPageRows = 128;
// With a window also from this many (block of 16 rows, key) pairs on: 9 histories over
// windows of 2000 and 4 key heads take 18 us in blocks of 16 rows and 22 there at 20 rows
// (150,000 pairs), 25 and 25 at 36, 29 and 25 at 52; one history over 1000 keys and 6
// heads 9 and 18 at 100 rows (50,000).
constexpr double kTcWindowWork = 200000;
// Over pages from this many on: 14 histories of 689 keys, 196 rows of one head of 32 (125,000)
// take 15 us in blocks of 16 rows and 26 there, 2 of 615 keys, 1230 rows of 3 heads of 48
// (284,000) 20 and 26, 6 of 389 keys, 482 rows of 5 heads of 80 (361,000) 24 and 30.
constexpr double kTcPageWork = 300000;

// The tensor cores cut what does not fit the float32 sum off whenever they add the products
// of four keys (a unit in the last place at most), so a sum over n keys of equal weight and
// values of one sign comes out smaller by up to 3 n 2^-28: measured at 65,536, 2^18 and 10^6
// keys 0.03 %, 0.16 % and 0.6 % with random values, 0.05 %, 0.26 % and 1.04 % with the worst
// (fp16's rounding is 0.05 %).  Parts of a span are no longer than this where the
// workspace has room: kSumKeys per sum, a block of the few-rows kernel has a sum in each
// of its four warps.  A call of the tensor-core kernel without room, whose parts would be
// longer than kLongSum, goes to the few-rows kernel instead: slower, but a cluster of its
// blocks has up to 64 sums.
constexpr long long kSumKeys = 1 << 16, kLongSum = 1 << 20;

// Chunks of the span for the few-rows kernels, `resident` blocks of which run on an SM
// (2, or 3 over pages where a key head has up to 8 rows).  A block costs about `begin` to
// begin and end, and a step of its four warps (32 KB of keys and values) about kStep, the
// memory's share of it when all blocks run.
// One sequence: whole rounds of blocks; 110,537 keys of 2 heads take 30 us in one
// round, 38 in two, 55 in four.  Several sequences are taken to be ragged: blocks of
// unlike lengths run into one another, so the number weighs what they cost to begin
// against the last one's length; 61 sequences of up to 16,384 keys and 8 heads take
// 323 us in 3 chunks, 297 in 5 (the rule's) and 299 in 8; 8 sequences of up to
// 20,000 keys and 4 heads 60, 23 (the rule's 22) and 32 us in 3, 22 and 8; over pages
// the 61 take 163 us in 4 chunks, 157 in 5 (the rule's) and 156 in 8.  Behind a window
// most are as long as one another (`equal`): rounds again, the last one of which may
// overhang by a quarter, since some are shorter; the 61 over windows of 5000 take 206,
// 175 (the rule's 2 chunks), 190 and 197 us in 1, 2, 3 and 8, 30 of them over windows of
// 2000 47, 57 and 59 in 1 (the rule's), 2 and 3.
long long rows_chunks(long long units, bool several, bool equal, long long steps, long long least_chunks, long long most,
                      int sms, int resident, double begin) {
  constexpr double kStep = 1.5;
  const long long slots = (long long)resident * sms;
  long long best = 1;
  double least = 0;
  if (several && equal) {
    for (long long c = 1; c <= std::min(most, 64LL); ++c) {
      const double rounds = std::max(1.0, ceil((double)(units * c) / slots - 0.25));
      const double cost = rounds * (6.0 + kStep * ((steps + c - 1) / c));
      if (c == 1 || cost < least) {
        least = cost;
        best = c;
      }
    }
  } else if (several) {
    best = (long long)(sqrt((double)steps * kStep * slots / (units * begin)) + 0.5);
  } else {
    for (long long k = 1; k <= 8; ++k) {
      const long long c = std::max(1LL, std::min(most, slots * k / units));
      const double cost = (double)((units * c + slots - 1) / slots) * (begin + kStep * ((steps + c - 1) / c)) + 0.02 * c;
      if (k == 1 || cost < least) {
        least = cost;
        best = c;
      }
    }
  }
  return std::max(1LL, std::min(std::max(best, least_chunks), most));
}

// Chunks that a cluster of blocks joins by itself through shared memory (1: none),
// which saves the second launch: taken where a chunk then has at most kJoin steps
// more than in the split, about a join's time, if all blocks are resident (clusters
// of more than 8 find room in few places).  One token, 6 heads of 64 over 2000 keys:
// 6.0 us against 7.2, 4097 8.1 against 8.9, 8000 9.5 and 9.2, and 12,000 would be
// 11.5 against 10.1; every call from the host is 2.5 us shorter.  Four ragged
// sequences of up to 4000 keys and 8 heads 10.1 against 13.0.
// Also taken, with blocks resident or not, where it gives more chunks than the
// workspace has room for and the least number is not reached.
long long rows_cluster(long long units, long long steps, long long split, long long least_chunks, int sms, int dim) {
  const long long kJoin = dim <= 64 ? 2 : 1;
  const long long wide = attn_rows_cluster();
  const long long most = std::min(least_chunks, units * wide <= sms ? wide : 8LL);
  if (split < most && units * most <= 0x7FFFFFFF) return most;
  const long long limit = units * wide <= sms ? wide : std::min(8LL, 2LL * sms / units);
  if (limit < 2) return 1;
  const long long per = (steps + limit - 1) / limit;
  return per <= (steps + split - 1) / split + kJoin ? (steps + per - 1) / per : 1;
}

// Chunks of the span for the tensor-core kernel, which has one block on an SM: the
// number of least cost, in steps of 64 keys.  Rounds of blocks over the SMs, each
// with its share of the steps and about four steps' time to begin and end, and for
// the merge two steps' time and the traffic of the partial results (a step takes
// about 1.2 us).  With 384 units of 768 steps, one chunk leaves the third round half
// empty and five would fill 13 rounds, if the workspace has room for them: at 16,384
// tokens of 6 heads of 64 a part takes 26 MB.
// Over pages and behind windows, whose steps are shorter, the merge's own time counts too:
// a few steps, and one for 5,000 rows.
long long tc_chunks(long long units, long long steps, long long least_chunks, long long most, int sms, int streams,
                    long long n_q, int heads, int dim, bool merge_counts) {
  const long long first = std::max(1LL, std::min(least_chunks, most));
  long long best = first;
  double least = 0;
  for (long long c = first; c <= std::max(first, std::min(most, 64LL)); ++c) {
    const double rounds = (double)((units * c + sms - 1) / sms);
    double cost = rounds * ((double)((steps + c - 1) / c) + 4);
    if (c * streams > 1) cost += 2 + 8e-6 * (double)(c * streams * n_q * heads) * dim / (6.8 * 1.2);
    if (c * streams > 1 && merge_counts) cost += 4 + (double)(n_q * heads) / 5000;
    if (c == first || cost < least) {
      least = cost;
      best = c;
    }
  }
  return best;
}

// Whether the two chains of a block share a tile (see attn_tc.cuh), where the number of tiles
// is odd: half the steps to a block, but as many blocks as tiles, and a merge.  In steps'
// time (1 us): a block has 8 besides its steps, a merge 6 and the partial results' traffic.
// 3 sequences of up to 926 tokens and as many keys, 12 query and 4 key heads of 128 on pages
// (23 tiles) take 70 us with shared tiles and 44 without.
int tc_streams(const AttnArgs& a, int max_q, long long most_k, int sms) {
  const long long tokens = 128 / a.group, tiles = (max_q + tokens - 1) / tokens;
  long long keys = most_k;
  if (a.window > 0 && !a.prefix) keys = std::min(keys, (long long)a.window + a.sinks + 2 * tokens + 128);
  const double steps = (double)(keys + 63) / 64, units = (double)a.n_seqs * a.kv_heads;
  const double one = ceil(units * ((tiles + 1) / 2) / sms) * (steps + 8);
  const double two = ceil(units * tiles / sms) * (steps / 2 + 8) + 6 + 16.0 * a.n_q * a.heads * a.dim / 6.8e6;
  return two < one ? 2 : 1;
}

std::atomic<int> g_test{0};                      // bits of rtcc_test_attention

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool bad_stride(int64_t s) { return s < 0 || s % 8 != 0; }

}  // namespace
}  // namespace rtcc

namespace rtcc {
namespace {

// Shapes and scores that 16-bit rows and pages have in common.
bool bad_scores(int dtype, int heads, int kv_heads, float scale, float cap) {
  if (dtype != RTCC_FP16 && dtype != RTCC_BF16) return true;
  if (heads < 1 || heads > 4096 || kv_heads < 1 || heads % kv_heads) return true;
  if (!isfinite(scale) || !isfinite(cap) || cap < 0.f) return true;
  if (cap > 0.f) {
    const float ratio = fabsf(scale / cap);
    if (cap > 1e38f || !isfinite(ratio) || (ratio < FLT_MIN && scale != 0.f)) return true;
  }
  return false;
}

// Bytes of the workspace for keys and values widened from pages: both, then the steps' halves on no page.
size_t widened_bytes(long long rows, const AttnArgs& a) {
  return (size_t)rows * a.kv_heads * a.dim * 4 + ((size_t)rows / 64 + 255) / 256 * 256;
}

// Chooses kernel and split, and launches.  max_q, max_k size the launch; `pages`: the
// keys and values are on pages (else NULL).
rtcc_status run_attention(AttnArgs& a, const PagesArgs* pages, int max_q, int max_k, bool bf16, void* d_workspace,
                          size_t workspace_bytes, cudaStream_t st) {
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
  const int test = g_test.load(std::memory_order_relaxed);
  a.stall = (test & RTCC_TEST_UNREACHABLE_WAIT) != 0;
  a.budget = a.stall ? kWaitBudgetCycles / 100 : kWaitBudgetCycles;
  const long long most_k = attn_most_keys(a, max_q, max_k);
  // the tensor-core kernel from kTcRows (token, head) rows per key head on
  const long long rows = (long long)max_q * a.group;
  bool tc = rows > (pages ? kTcPageRows : kTcRows) && a.group <= 128 && a.n_rows > 0;
  // behind short windows its blocks hardly begin before they end, and over pages there is the
  // widening: not for little work
  const double work = (double)((rows + attn_rows_per_block() - 1) / attn_rows_per_block()) * a.n_seqs * a.kv_heads * most_k;
  if (pages) tc = tc && work > kTcPageWork;
  else if (a.window > 0) tc = tc && work > kTcWindowWork;
  const size_t part = (size_t)a.n_q * a.heads * (a.dim * sizeof(float) + sizeof(float2));
  const long long span = (most_k + 63) / 64 * 64, span_rows = span * a.n_seqs;
  size_t wide = pages ? widened_bytes(span_rows, a) : 0;
  if (pages && (wide > workspace_bytes || !d_workspace || span_rows > kMaxRows)) tc = false;
  bool clusters = true, widened = false;
  for (;; tc = false) {
    AttnArgs w = a;                              // as the kernel gets it
    char* space = static_cast<char*>(d_workspace);
    size_t left = d_workspace ? workspace_bytes : 0;
    if (pages && tc) {
      w.k = space;
      w.v = space + (size_t)span_rows * a.kv_heads * a.dim * 2;
      w.hidden = reinterpret_cast<unsigned char*>(space) + (size_t)span_rows * a.kv_heads * a.dim * 4;
      w.k_row = w.v_row = (long long)a.kv_heads * a.dim;
      w.k_head = w.v_head = a.dim;
      w.span_rows = (int)span;
      w.n_rows = (int)span_rows;
      space += wide;
      left -= wide;
    }
    const long long room = (long long)(left / part);
    w.streams = tc ? attn_tc_streams(w.group, max_q) : 1;
    if (w.streams > 1 && (pages || a.window > 0)) w.streams = tc_streams(a, max_q, most_k, sms);
    if (w.streams > room) w.streams = 1;
    w.unit = tc ? attn_tc_unit(w.streams) : pages ? attn_pages_unit() : attn_rows_unit(w.dim);
    const long long step = tc ? attn_tc_tokens_per_block(w.group, w.streams) : 1;
    long long groups = tc ? (max_q + step - 1) / step
                          : ((long long)max_q * w.group + attn_rows_per_block() - 1) / attn_rows_per_block();
    long long units = (long long)w.n_seqs * w.kv_heads;
    if (units > 0x3FFFFFFF) return RTCC_E_ARG;
    while (units * groups > 0x3FFFFFFF && groups > 1) groups = (groups + 1) / 2;   // blocks then loop
    units *= groups;
    w.row_groups = (int)groups;
    const long long steps = (most_k + w.unit - 1LL) / w.unit;
    long long most = tc ? (steps + 3) / 4 : steps;
    const long long sums = tc ? w.streams : 4;     // of a block
    const long long least = (most_k + sums * kSumKeys - 1) / (sums * kSumKeys);
    // keys of a token: tokens that see mostly other keys than one another's leave nothing to
    // split but long sums, over a prefix, sinks or a window of their own
    const long long sees = w.window > 0 && !w.prefix ? std::min(most_k, (long long)w.sinks + w.window) : most_k;
    if (tc && w.window > 0 && max_q > w.window) most = std::min(most, sees > sums * kSumKeys ? least : 1);
    if (most > room / w.streams) most = room / w.streams;
    if (most > 0x7FFFFFFF / units) most = 0x7FFFFFFF / units;
    long long chunks = tc ? tc_chunks(units, steps, least, most, sms, w.streams, w.n_q, w.heads, w.dim,
                                      pages || w.window > 0)
                          : rows_chunks(units, w.n_seqs > 1, most_k < max_k, steps, least, most, sms,
                                        pages && (long long)max_q * w.group <= 8 ? 3 : 2, pages ? 8.0 : 10.0);
    if (tc && std::min(sees, most_k / chunks) / sums > kLongSum) continue;
    const long long joined = tc || !clusters ? 1 : rows_cluster(units, steps, chunks, least, sms, w.dim);
    w.cluster = joined > 1;
    if (w.cluster) chunks = joined;
    w.n_chunks = (int)chunks;
    w.chunk = (int)((most_k + chunks - 1) / chunks);
    w.part_o = reinterpret_cast<float*>(space);
    w.part_ml = reinterpret_cast<float2*>(w.part_o + (size_t)chunks * w.streams * w.n_q * w.heads * w.dim);
    if (pages && tc && !widened) {
      const cudaError_t e = launch_pages_widen(a, *pages, const_cast<void*>(w.k), const_cast<void*>(w.v),
                                               const_cast<unsigned char*>(w.hidden), (int)span, bf16, st);
      if (e == cudaErrorNotSupported) continue;
      if (e != cudaSuccess) return RTCC_E_CUDA;
      widened = true;
    }
    cudaError_t e = w.cluster && (test & RTCC_TEST_NO_CLUSTERS) ? cudaErrorInvalidClusterSize
                    : tc ? launch_attn_tc(w, bf16, st)
                    : pages ? launch_attn_pages(w, *pages, bf16, st) : launch_attn_rows(w, bf16, st);
    if (tc && e == cudaErrorNotSupported) continue;
    if (w.cluster && e != cudaSuccess) {           // no room for such clusters (a part of a GPU): two launches
      cudaGetLastError();
      clusters = false;
      continue;
    }
    if (e != cudaSuccess) return RTCC_E_CUDA;
    if (!w.cluster && chunks * w.streams > 1 && launch_attn_join(w, bf16, st) != cudaSuccess) return RTCC_E_CUDA;
    return RTCC_OK;
  }
}

rtcc_status memory_attention(const rtcc_attn_config* c, int window, int sinks, const void* d_q, const void* d_k,
                             const void* d_v, const int32_t* d_q_offsets, const int32_t* d_k_begin,
                             const int32_t* d_k_end, const int32_t* d_prefix, const int32_t* d_present,
                             const float* d_slopes, const float* d_q_pos, const float* d_k_pos, void* d_out,
                             float* d_lse, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (!c) return RTCC_E_ARG;
  if (bad_scores(c->dtype, c->heads, c->kv_heads, c->scale, c->cap)) return RTCC_E_ARG;
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return RTCC_E_ARG;
  if (c->n_q < 0 || c->n_rows < 0 || c->n_seqs < 0 || c->max_q < 0 || c->max_k < 0) return RTCC_E_ARG;
  if ((long long)c->n_q * c->heads > kMaxRows || c->n_rows > kMaxRows) return RTCC_E_ARG;
  const int64_t strides[] = {c->q_row, c->q_head, c->k_row, c->k_head, c->v_row, c->v_head, c->out_row, c->out_head};
  for (int64_t s : strides)
    if (bad_stride(s)) return RTCC_E_ARG;
  if (c->n_slots < 0 || c->n_slots > kMaxSlots || (c->n_slots > 0) != (d_present != nullptr)) return RTCC_E_ARG;
  if (c->n_slots > 0 && (c->slot_rows < 1 || (long long)c->n_slots * c->slot_rows < c->n_rows)) return RTCC_E_ARG;
  if ((d_slopes != nullptr) != (d_q_pos != nullptr) || (d_slopes != nullptr) != (d_k_pos != nullptr)) return RTCC_E_ARG;
  if (d_slopes && c->q_pos_row < 2) return RTCC_E_ARG;
  if (c->n_seqs > 0 && (!d_q_offsets || !d_k_begin || !d_k_end)) return RTCC_E_ARG;
  if (c->n_q > 0 && (!d_q || !d_out)) return RTCC_E_ARG;
  if (c->n_rows > 0 && (!d_k || !d_v)) return RTCC_E_ARG;
  const void* by16[] = {d_q, d_k, d_v, d_out, d_workspace};
  for (const void* p : by16)
    if (misaligned(p, 16)) return RTCC_E_ARG;
  const void* by4[] = {d_q_offsets, d_k_begin, d_k_end, d_prefix, d_present, d_slopes, d_q_pos, d_lse, c->d_q_start};
  for (const void* p : by4)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  if (misaligned(d_k_pos, 8)) return RTCC_E_ARG;
  if (c->n_q == 0 || c->n_seqs == 0) return RTCC_OK;

  AttnArgs a{};
  a.q = d_q; a.k = d_k; a.v = d_v; a.out = d_out; a.lse = d_lse;
  a.q_offsets = d_q_offsets; a.k_begin = d_k_begin; a.k_end = d_k_end;
  a.prefix = d_prefix; a.present = d_present; a.q_start = c->d_q_start;
  a.slopes = d_slopes; a.q_pos = d_q_pos; a.k_pos = d_k_pos;
  a.q_row = c->q_row; a.q_head = c->q_head; a.k_row = c->k_row; a.k_head = c->k_head;
  a.v_row = c->v_row; a.v_head = c->v_head; a.out_row = c->out_row; a.out_head = c->out_head;
  a.n_q = c->n_q; a.n_rows = c->n_rows; a.heads = c->heads; a.kv_heads = c->kv_heads;
  a.group = c->heads / c->kv_heads; a.dim = c->head_dim; a.n_seqs = c->n_seqs; a.causal = c->causal != 0;
  a.n_slots = c->n_slots; a.slot_rows = c->n_slots ? c->slot_rows : 1; a.q_pos_row = c->q_pos_row;
  // with l = ceil(log2(d)), ceil(2^(31 + l) / d) is a 32-bit multiplier that divides
  // every row number (below 2^31) exactly
  int l = 0;
  while ((1LL << l) < a.slot_rows) ++l;
  a.slot_mul = (uint32_t)(((1ull << (31 + l)) + a.slot_rows - 1) / a.slot_rows);
  a.slot_shift = 31 + l;
  a.cap_log2 = c->cap * kLog2e;
  a.scale_log2 = c->cap > 0.f ? c->scale / c->cap : c->scale * kLog2e;

  a.window = window; a.sinks = sinks;
  const int max_q = c->max_q < 1 ? 1 : c->max_q > c->n_q ? c->n_q : c->max_q;
  const int max_k = c->max_k < 1 ? 1 : c->max_k > c->n_rows ? (c->n_rows < 1 ? 1 : c->n_rows) : c->max_k;
  return run_attention(a, nullptr, max_q, max_k, c->dtype == RTCC_BF16, d_workspace, workspace_bytes,
                       static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace rtcc

using namespace rtcc;

extern "C" rtcc_status rtcc_memory_attention(const rtcc_attn_config* c, const void* d_q, const void* d_k,
                                             const void* d_v, const int32_t* d_q_offsets,
                                             const int32_t* d_k_begin, const int32_t* d_k_end,
                                             const int32_t* d_prefix, const int32_t* d_present,
                                             const float* d_slopes, const float* d_q_pos,
                                             const float* d_k_pos, void* d_out, float* d_lse,
                                             void* d_workspace, size_t workspace_bytes, void* stream) {
  return memory_attention(c, 0, 0, d_q, d_k, d_v, d_q_offsets, d_k_begin, d_k_end, d_prefix, d_present, d_slopes,
                          d_q_pos, d_k_pos, d_out, d_lse, d_workspace, workspace_bytes, stream);
}

extern "C" rtcc_status rtcc_memory_window_attention(const rtcc_attn_config* c, int32_t window, int32_t sinks,
                                                    const void* d_q, const void* d_k, const void* d_v,
                                                    const int32_t* d_q_offsets, const int32_t* d_k_begin,
                                                    const int32_t* d_k_end, const int32_t* d_prefix,
                                                    const int32_t* d_present, const float* d_slopes,
                                                    const float* d_q_pos, const float* d_k_pos, void* d_out,
                                                    float* d_lse, void* d_workspace, size_t workspace_bytes,
                                                    void* stream) {
  if (!c || !c->causal || window < 1 || sinks < 0) return RTCC_E_ARG;
  return memory_attention(c, window, sinks, d_q, d_k, d_v, d_q_offsets, d_k_begin, d_k_end, d_prefix, d_present,
                          d_slopes, d_q_pos, d_k_pos, d_out, d_lse, d_workspace, workspace_bytes, stream);
}

extern "C" rtcc_status rtcc_pages_attention(const rtcc_page_config* cfg, const rtcc_page_attn_config* c, const void* d_q,
                                            const int32_t* d_q_offsets, const int32_t* d_start, const int32_t* d_length,
                                            const int32_t* d_prefix, const int32_t* d_table, const void* d_k_pages,
                                            const void* d_v_pages, const void* d_scales, void* d_out, float* d_lse,
                                            void* d_workspace, size_t workspace_bytes, void* stream) {
  PagesArgs p{};
  if (!page_shape(cfg, &p.s) || !c) return RTCC_E_ARG;
  if (bad_scores(c->dtype, c->heads, p.s.kv_heads, c->scale, c->cap)) return RTCC_E_ARG;
  if (c->n_q < 0 || c->max_q < 0 || c->max_k < 0 || (long long)c->n_q * c->heads > kMaxRows) return RTCC_E_ARG;
  const int64_t strides[] = {c->q_row, c->q_head, c->out_row, c->out_head};
  for (int64_t s : strides)
    if (bad_stride(s)) return RTCC_E_ARG;
  if (c->window < 0 || c->sinks < 0 || (c->window > 0 && !c->causal)) return RTCC_E_ARG;
  const long long cells = (long long)p.s.n_seqs * p.s.table_row;
  if (p.s.n_seqs > 0 && (!d_q_offsets || !d_length || (cells > 0 && !d_table))) return RTCC_E_ARG;
  if (c->n_q > 0 && (!d_q || !d_out)) return RTCC_E_ARG;
  if (p.s.n_pages > 0 && (!d_k_pages || !d_v_pages || !d_scales)) return RTCC_E_ARG;
  const void* by16[] = {d_q, d_k_pages, d_v_pages, d_out, d_workspace};
  for (const void* x : by16)
    if (misaligned(x, 16)) return RTCC_E_ARG;
  const void* by4[] = {d_q_offsets, d_start, d_length, d_prefix, d_table, d_scales, d_lse};
  for (const void* x : by4)
    if (misaligned(x, 4)) return RTCC_E_ARG;
  if (c->n_q == 0 || p.s.n_seqs == 0) return RTCC_OK;

  p.table = d_table;
  p.k = static_cast<const unsigned char*>(d_k_pages);
  p.v = static_cast<const unsigned char*>(d_v_pages);
  p.scales = static_cast<const signed char*>(d_scales);
  const int places = p.s.table_row << p.s.shift;
  const int max_q = c->max_q > c->n_q ? c->n_q : c->max_q, max_k = c->max_k > places ? places : c->max_k;
  AttnArgs a{};
  a.q = d_q; a.out = d_out; a.lse = d_lse;
  a.q_offsets = d_q_offsets; a.k_end = d_length; a.prefix = d_prefix; a.q_start = d_start;
  a.q_row = c->q_row; a.q_head = c->q_head; a.out_row = c->out_row; a.out_head = c->out_head;
  a.n_q = c->n_q; a.n_rows = places; a.heads = c->heads; a.kv_heads = p.s.kv_heads;
  a.group = c->heads / p.s.kv_heads; a.dim = p.s.dim; a.n_seqs = p.s.n_seqs; a.causal = c->causal != 0;
  a.slot_rows = 1;
  a.cap_log2 = c->cap * kLog2e;
  a.scale_log2 = c->cap > 0.f ? c->scale / c->cap : c->scale * kLog2e;
  a.window = c->window; a.sinks = c->sinks;
  a.most_q = max_q; a.most_k = max_k;
  return run_attention(a, &p, max_q < 1 ? 1 : max_q, max_k < 1 ? 1 : max_k, c->dtype == RTCC_BF16, d_workspace,
                       workspace_bytes, static_cast<cudaStream_t>(stream));
}

// The device counts and nothing clears the count, so no failure is lost between a read
// and a clear; each stream remembers the count of its last report.
extern "C" rtcc_status rtcc_memory_attention_status(void* stream) try {
  static std::mutex mu;
  static std::map<std::pair<int, void*>, unsigned> reported;
  unsigned count = 0;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return RTCC_E_CUDA;
  if (attn_tc_errors(&count, static_cast<cudaStream_t>(stream)) != cudaSuccess) return RTCC_E_CUDA;
  std::lock_guard<std::mutex> lk(mu);
  unsigned& last = reported[{dev, stream}];
  if ((int)(count - last) <= 0) return RTCC_OK;
  last = count;
  return RTCC_E_DEVICE;
} catch (...) {
  return RTCC_E_NOMEM;
}

extern "C" rtcc_status rtcc_test_attention(int32_t what) {
  if (what & ~(RTCC_TEST_UNREACHABLE_WAIT | RTCC_TEST_NO_CLUSTERS)) return RTCC_E_ARG;
  g_test.store(what, std::memory_order_relaxed);
  return RTCC_OK;
}
