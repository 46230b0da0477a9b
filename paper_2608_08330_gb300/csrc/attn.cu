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
#include "rtcc.h"

namespace rtcc {
namespace {

// The tensor-core kernel takes over from this many (token, head) rows of a key head
// on: 33 rows over 9 ragged histories of 5001 keys, heads of 80, take 24 us there
// and 27 in blocks of 16 rows, 30 rows over 50,000 keys, heads of 64, 25 and 23.
constexpr int kTcRows = 32;

// The tensor cores cut what does not fit the float32 sum off at every 16 keys' addition
// (a unit in the last place at most), so a sum over n keys of equal weight comes out
// smaller by up to (n / 32) 2^-23: 2^-12 at 65,536 keys, half of fp16's rounding; measured
// 0.1 % at 2^18 keys, 0.6 % at 2^20.  Parts of a span are no longer than this where the
// workspace has room: kSumKeys per sum, a block of the few-rows kernel has a sum in each
// of its four warps.  A call of the tensor-core kernel without room, whose parts would be
// longer than kLongSum, goes to the few-rows kernel instead: slower, but a cluster of its
// blocks has up to 64 sums.
constexpr long long kSumKeys = 1 << 16, kLongSum = 1 << 20;

// Chunks of the span for the few-rows kernel, two blocks of which run on an SM.  A
// block costs about kBegin to begin and end, and a step of its four warps (32 KB of
// keys and values) about kStep, the memory's share of it when all blocks run.
// One sequence: whole rounds of blocks; 110,537 keys of 2 heads take 30 us in one
// round, 38 in two, 55 in four.  Several sequences are taken to be ragged: blocks of
// unlike lengths run into one another, so the number weighs what they cost to begin
// against the last one's length; 61 sequences of up to 16,384 keys and 8 heads take
// 323 us in 3 chunks, 297 in 5 (the rule's) and 299 in 8; 8 sequences of up to
// 20,000 keys and 4 heads 60, 23 (the rule's 22) and 32 us in 3, 22 and 8.
long long rows_chunks(long long units, int n_seqs, long long steps, long long least_chunks, long long most, int sms) {
  constexpr double kBegin = 10.0, kStep = 1.5;
  const long long slots = 2LL * sms;
  long long best = 1;
  if (n_seqs > 1) {
    best = (long long)(sqrt((double)steps * kStep * slots / (units * kBegin)) + 0.5);
  } else {
    double least = 0;
    for (long long k = 1; k <= 8; ++k) {
      const long long c = std::max(1LL, std::min(most, slots * k / units));
      const double cost = (double)((units * c + slots - 1) / slots) * (kBegin + kStep * ((steps + c - 1) / c)) + 0.02 * c;
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
long long tc_chunks(long long units, long long steps, long long least_chunks, long long most, int sms, int streams,
                    long long n_q, int heads, int dim) {
  const long long first = std::max(1LL, std::min(least_chunks, most));
  long long best = first;
  double least = 0;
  for (long long c = first; c <= std::max(first, std::min(most, 64LL)); ++c) {
    const double rounds = (double)((units * c + sms - 1) / sms);
    double cost = rounds * ((double)((steps + c - 1) / c) + 4);
    if (c * streams > 1) cost += 2 + 8e-6 * (double)(c * streams * n_q * heads) * dim / (6.8 * 1.2);
    if (c == first || cost < least) {
      least = cost;
      best = c;
    }
  }
  return best;
}

std::atomic<int> g_test{0};                      // bits of rtcc_test_attention

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool bad_stride(int64_t s) { return s < 0 || s % 8 != 0; }

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
  if (!c) return RTCC_E_ARG;
  if (c->dtype != RTCC_FP16 && c->dtype != RTCC_BF16) return RTCC_E_ARG;
  if (c->heads < 1 || c->heads > 4096 || c->kv_heads < 1 || c->heads % c->kv_heads) return RTCC_E_ARG;
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return RTCC_E_ARG;
  if (c->n_q < 0 || c->n_rows < 0 || c->n_seqs < 0 || c->max_q < 0 || c->max_k < 0) return RTCC_E_ARG;
  if ((long long)c->n_q * c->heads > kMaxRows || c->n_rows > kMaxRows) return RTCC_E_ARG;
  const int64_t strides[] = {c->q_row, c->q_head, c->k_row, c->k_head, c->v_row, c->v_head, c->out_row, c->out_head};
  for (int64_t s : strides)
    if (bad_stride(s)) return RTCC_E_ARG;
  if (!isfinite(c->scale) || !isfinite(c->cap) || c->cap < 0.f) return RTCC_E_ARG;
  if (c->cap > 0.f) {
    const float ratio = fabsf(c->scale / c->cap);
    if (c->cap > 1e38f || !isfinite(ratio) || (ratio < FLT_MIN && c->scale != 0.f)) return RTCC_E_ARG;
  }
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

  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
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

  const int test = g_test.load(std::memory_order_relaxed);
  a.stall = (test & RTCC_TEST_UNREACHABLE_WAIT) != 0;
  a.budget = a.stall ? kWaitBudgetCycles / 100 : kWaitBudgetCycles;
  const int max_q = c->max_q < 1 ? 1 : c->max_q > c->n_q ? c->n_q : c->max_q;
  const int max_k = c->max_k < 1 ? 1 : c->max_k > c->n_rows ? (c->n_rows < 1 ? 1 : c->n_rows) : c->max_k;
  const bool bf16 = c->dtype == RTCC_BF16;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // the tensor-core kernel from kTcRows (token, head) rows per key head on
  bool tc = (long long)max_q * a.group > kTcRows && a.group <= 128 && c->n_rows > 0;
  const size_t part = (size_t)c->n_q * c->heads * (c->head_dim * sizeof(float) + sizeof(float2));
  const long long room = d_workspace ? (long long)(workspace_bytes / part) : 0;
  bool clusters = true;
  for (;; tc = false) {
    a.streams = tc ? attn_tc_streams(a.group, max_q) : 1;
    if (a.streams > room) a.streams = 1;
    a.unit = tc ? attn_tc_unit(a.streams) : attn_rows_unit(c->head_dim);
    const long long step = tc ? attn_tc_tokens_per_block(a.group, a.streams) : 1;
    long long groups = tc ? (max_q + step - 1) / step
                          : ((long long)max_q * a.group + attn_rows_per_block() - 1) / attn_rows_per_block();
    long long units = (long long)c->n_seqs * a.kv_heads;
    if (units > 0x3FFFFFFF) return RTCC_E_ARG;
    while (units * groups > 0x3FFFFFFF && groups > 1) groups = (groups + 1) / 2;   // blocks then loop
    units *= groups;
    a.row_groups = (int)groups;
    const long long steps = (max_k + a.unit - 1LL) / a.unit;
    long long most = tc ? (steps + 3) / 4 : steps;
    if (most > room / a.streams) most = room / a.streams;
    if (most > 0x7FFFFFFF / units) most = 0x7FFFFFFF / units;
    const long long sums = tc ? a.streams : 4;     // of a block
    const long long least = (max_k + sums * kSumKeys - 1) / (sums * kSumKeys);
    long long chunks = tc ? tc_chunks(units, steps, least, most, sms, a.streams, a.n_q, a.heads, a.dim)
                          : rows_chunks(units, c->n_seqs, steps, least, most, sms);
    if (tc && max_k / (chunks * sums) > kLongSum) continue;
    const long long joined = tc || !clusters ? 1 : rows_cluster(units, steps, chunks, least, sms, a.dim);
    a.cluster = joined > 1;
    if (a.cluster) chunks = joined;
    a.n_chunks = (int)chunks;
    a.chunk = (int)((max_k + chunks - 1) / chunks);
    a.part_o = static_cast<float*>(d_workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + (size_t)chunks * a.streams * c->n_q * c->heads * c->head_dim);
    cudaError_t e = a.cluster && (test & RTCC_TEST_NO_CLUSTERS) ? cudaErrorInvalidClusterSize
                    : tc ? launch_attn_tc(a, bf16, st) : launch_attn_rows(a, bf16, st);
    if (tc && e == cudaErrorNotSupported) continue;
    if (a.cluster && e != cudaSuccess) {           // no room for such clusters (a part of a GPU): two launches
      cudaGetLastError();
      clusters = false;
      continue;
    }
    if (e != cudaSuccess) return RTCC_E_CUDA;
    if (!a.cluster && chunks * a.streams > 1 && launch_attn_join(a, max_q, bf16, st) != cudaSuccess) return RTCC_E_CUDA;
    return RTCC_OK;
  }
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
