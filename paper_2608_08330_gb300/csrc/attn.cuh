// Shared by the attention kernels over the token memory: arguments, spans of
// the sequences, the absent slots' mask and the score's arithmetic.
#pragma once

#include "common.cuh"

namespace rtcc {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxSlots = 64;
// Largest row number, and number of (token, head) rows: 32-bit key and row numbers
// go past the last one by less than a step of a block or of its copies' ring.
constexpr long long kMaxRows = (1LL << 31) - (1 << 16);

struct AttnArgs {
  const void *q, *k, *v;
  void* out;
  float* lse;                    // [n_q][heads], may be null
  const int *q_offsets, *k_begin, *k_end;
  const int* prefix;             // may be null
  const int* q_start;            // may be null: the tokens are the span's last rows
  const int* present;            // [n_slots], may be null
  const float *slopes, *q_pos, *k_pos;
  float* part_o;                 // [n_chunks * streams][n_q * heads][dim] when there are several
  float2* part_ml;               // [n_chunks * streams][n_q * heads]: running maximum (log2) and sum
  long long q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head;
  int n_q, n_rows, heads, kv_heads, group, dim, n_seqs, causal;
  int n_slots, slot_rows, q_pos_row;
  uint32_t slot_mul, slot_shift; // row / slot_rows = row * slot_mul >> slot_shift
  int n_chunks, chunk, unit;     // key chunks per sequence at most, keys per chunk at least, a multiple of unit
  int streams;                   // partial results per chunk
  int cluster;                   // 1: the chunks are a cluster of blocks that joins them itself
  int row_groups;                // blocks along the rows of one sequence and key head
  float scale_log2;              // scale * log2(e); with a cap: scale / cap
  float cap_log2;                // cap * log2(e), 0 = no cap
  long long budget;              // cycles of a bounded wait
  int stall;                     // test hook: the queries are never loaded
};

// One sequence: its tokens [q0, q0 + nq) and memory rows [kb, kb + nk), the first
// token's place among the keys (a causal token i sees keys up to first + i; negative
// where there are more tokens than keys).  Offsets come from device memory, so they
// are cut to the arrays' extents; keys after the last token's are left out.
struct AttnSpan {
  int q0, nq, kb, nk, prefix, first;
};

__device__ __forceinline__ AttnSpan attn_span(const AttnArgs& A, int seq) {
  AttnSpan s;
  const int q0 = A.q_offsets[seq], q1 = A.q_offsets[seq + 1];
  const int kb = A.k_begin[seq], ke = A.k_end[seq];
  s.q0 = min(max(q0, 0), A.n_q);
  s.nq = min(max(q1, s.q0), A.n_q) - s.q0;
  s.kb = min(max(kb, 0), A.n_rows);
  s.nk = min(max(ke, s.kb), A.n_rows) - s.kb;
  s.prefix = A.prefix ? min(max(A.prefix[seq], 0), s.nk) : 0;
  s.first = s.nk - s.nq;
  if (A.causal && A.q_start) {
    s.first = min(max(A.q_start[seq], 0), s.nk);
    if (s.nk - s.first > s.nq) s.nk = max(s.prefix, s.first + s.nq);
  }
  return s;
}

// Keys [0, n) of the span that token i of the sequence sees (slots aside).
__device__ __forceinline__ int attn_visible(const AttnArgs& A, const AttnSpan& s, int first, int i) {
  if (!A.causal) return s.nk;
  const int own = i < s.nk - first ? first + i + 1 : s.nk;
  return max(0, max(s.prefix, own));
}

// Slot of a memory row (there are at most 64).
__device__ __forceinline__ int slot_of(const AttnArgs& A, int row) {
  return (int)min((uint32_t)(((unsigned long long)(uint32_t)row * A.slot_mul) >> A.slot_shift), 63u);
}

// Bit s set: slot s is present (all ones without slots).  Whole warp.
__device__ __forceinline__ unsigned long long attn_slot_mask(const AttnArgs& A, int lane) {
  if (!A.present) return ~0ull;
  const unsigned lo = __ballot_sync(0xFFFFFFFFu, lane < A.n_slots && A.present[min(lane, A.n_slots - 1)] != 0);
  const unsigned hi =
      __ballot_sync(0xFFFFFFFFu, lane + 32 < A.n_slots && A.present[min(lane + 32, A.n_slots - 1)] != 0);
  return (unsigned long long)hi << 32 | lo;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// tanh(u) = 1 - 2 / (1 + e^2u) to about 2e-7, for caps up to kAbsCap: the cap multiplies
// the error into a score, 5e-5 at most, a tenth of fp16's rounding of a probability.  An
// infinite e^2u gives 1, a NaN stays one (a minimum in its place would turn it into a
// score of the cap).
constexpr float kAbsCap = 256.0f;
__device__ __forceinline__ float tanh_abs(float u) {
  return 1.0f - __fdividef(2.0f, 1.0f + ex2(2.0f * kLog2e * u));
}

// For larger caps, tanh to 2^-20 of itself, NaN for NaN: near 0 it is u + u w q(w),
// w = u^2, with q of the least largest relative error (1.5e-8) on |u| <= 1/2.  (Used for
// all caps it cost 12,036 packed causal tokens under a cap 4 %.)
__device__ __forceinline__ float tanh_rel(float u) {
  const float w = u * u, a = fabsf(u);
  float q = fmaf(w, 0.01724149208652909f, -0.05304549457178399f);
  q = fmaf(w, q, 0.13325878962197332f);
  q = fmaf(w, q, -0.33333143896473094f);
  const float far = copysignf(1.0f - __fdividef(2.0f, 1.0f + ex2(2.0f * kLog2e * a)), u);
  return a < 0.5f ? fmaf(u * w, q, u) : far;
}

// Keys per chunk of a sequence: the launch's, or more where the sequence is
// longer than the launch was told; the chunks in use follow.
__device__ __forceinline__ int attn_chunk(const AttnArgs& A, int nk, int unit) {
  const int need = (int)(((long long)nk + A.n_chunks - 1) / A.n_chunks);
  const int c = max(A.chunk, need);
  return (c + unit - 1) / unit * unit;
}

}  // namespace rtcc
