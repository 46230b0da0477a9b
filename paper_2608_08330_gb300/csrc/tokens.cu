// Token memory: rows for new tokens, and queries/keys made ready for attention.
//
// A token memory is a set of fixed slots of `capacity` rows in device memory
// that the caller owns; a row holds the key and value vectors of one token (a
// BEV cell of one agent's map, an object, a step of a sequence).  Two
// operators fill it:
//
// rtcc_memory_append: from the number of new tokens of each sequence,
//   offsets[s] = sum of new over the sequences before s,
//   row(token i of s) = slot_s * capacity + held_s + i   (-1 past the slot),
//   and the span and length of every sequence afterwards.  One launch: the
//   scan is short (at most 16,384 sequences, 64 KB), so every block repeats it
//   in shared memory instead of waiting for another block, then fills its own
//   share of the tokens.
//
// rtcc_qkv_prepare: for every token and head of q and k
//   x^ = x * rsqrt(mean(x^2) + eps) * gain,
//   and pair m of axis a of x^ turned by pos_a * theta^(-m / pairs_a);
//   q goes to a dense output, k, v and the (y, x) coordinates to the token's
//   memory row.  It reads and writes every vector once, so HBM bounds it.  A
//   thread keeps one place (a head's 8 channels: one 16-byte load and store) for
//   all the tokens it sees, so pointers, gains and the place's kind are set up
//   once; it has up to four tokens' vectors in flight, and a block computes the
//   angles of its batch of tokens once for all heads in the meantime.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "rtcc.h"

namespace rtcc {
namespace {

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------

constexpr int kMaxSeqs = 16384;
constexpr int kAppendThreads = 512;

struct AppendArgs {
  const int *fresh, *held, *slot;
  int *offsets, *rows, *seq, *pos, *begin, *end, *length;
  int n_seqs, capacity, n_tokens;
};

// Exclusive sum over the block of one value per thread; *total = the sum of all.
__device__ __forceinline__ long long block_exclusive(long long v, long long* warp_sum, long long* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xFFFFFFFFu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) warp_sum[w] = x;
  __syncthreads();
  long long before = 0, all = 0;
  for (int i = 0; i < kAppendThreads / 32; ++i) {
    if (i < w) before += warp_sum[i];
    all += warp_sum[i];
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

__global__ void __launch_bounds__(kAppendThreads) k_memory_append(const AppendArgs A) {
  extern __shared__ int off[];                   // [n_seqs + 1]
  __shared__ long long warp_sum[kAppendThreads / 32];
  const int tid = threadIdx.x;
  // sums in 64 bits, cut at the token buffer's length: a token that has no
  // place in the buffer gets no row and does not count towards its sequence
  const long long cap = A.n_tokens;
  long long carry = 0;
  for (int s0 = 0; s0 < A.n_seqs; s0 += kAppendThreads) {
    const int s = s0 + tid;
    const long long v = s < A.n_seqs ? max(A.fresh[s], 0) : 0;
    long long total;
    const long long at = carry + block_exclusive(v, warp_sum, &total);
    if (s < A.n_seqs) off[s] = (int)min(at, cap);
    carry += total;
  }
  if (tid == 0) off[A.n_seqs] = (int)min(carry, cap);
  __syncthreads();
  const int stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + tid;
  for (int s = first; s <= A.n_seqs; s += stride) {
    A.offsets[s] = off[s];
    if (s == A.n_seqs) break;
    const int slot = A.slot ? A.slot[s] : s;
    const int held = min(max(A.held[s], 0), A.capacity);
    const int len = (int)min((long long)A.capacity, (long long)held + (off[s + 1] - off[s]));
    const long long b = (long long)slot * A.capacity;
    const bool ok = slot >= 0 && b + A.capacity <= 0x7FFFFFFFLL;
    A.begin[s] = ok ? (int)b : 0;
    A.end[s] = ok ? (int)b + len : 0;
    A.length[s] = len;
  }
  const int live = off[A.n_seqs];
  for (int i = first; i < A.n_tokens; i += stride) {
    int row = -1, seq = -1, pos = -1;
    if (i < live) {
      int lo = 0, hi = A.n_seqs;                 // the last sequence with off <= i
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= i) lo = mid; else hi = mid;
      }
      seq = lo;
      const int slot = A.slot ? A.slot[seq] : seq;
      const int held = min(max(A.held[seq], 0), A.capacity);
      const long long p = (long long)held + (i - off[seq]);
      const long long b = (long long)slot * A.capacity;
      pos = (int)min(p, 0x7FFFFFFFLL);
      if (slot >= 0 && p < A.capacity && b + A.capacity <= 0x7FFFFFFFLL) row = (int)(b + p);
    }
    A.rows[i] = row;
    if (A.seq) A.seq[i] = seq;
    if (A.pos) A.pos[i] = pos;
  }
}

// ---------------------------------------------------------------------------
// prepare
// ---------------------------------------------------------------------------

constexpr int kPrepThreads = 256;                // at most, per block
constexpr int kPrepBatch = 4;                    // tokens in flight per thread
constexpr int kMaxPairs = 64;

struct PrepArgs {
  const void *q, *k, *v;
  const float *q_gain, *k_gain, *pos;
  const int* rows;
  void *q_out, *k_mem, *v_mem;
  float* coord;
  long long q_row, q_head, k_row, k_head, v_row, v_head;
  long long qo_row, qo_head, km_row, km_head, vm_row, vm_head;
  int n_tokens, n_rows, n_qh, n_kh, n_vh, dim;
  int n_rot;                   // pairs of all axes together
  int end_t, end_y;            // pairs [0, end_t) turn by t, [end_t, end_y) by y, the rest by x
  int norm;
  int places, side, batch;     // threads per token in a block, tokens side by side, tokens per thread
  float eps;
  // turns per unit of position, theta^(-m / n) / 2 pi, as the sum of two floats:
  // the product with a position stays exact to a small fraction of a turn at
  // positions where one float's rounding would be most of a turn
  float turn_hi[kMaxPairs], turn_lo[kMaxPairs];
};

// How pairs lie: none, (2m, 2m + 1), or (m, m + n_rot) with n_rot a multiple of
// 8 (the partner is another lane's whole vector) or not (read again, an L1 hit).
enum { kTurnNone, kTurnInterleaved, kTurnLanes, kTurnAny };

template <typename T>
__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8]) {
  const float2 a = Store<T>::unpack2(u.x), b = Store<T>::unpack2(u.y), c = Store<T>::unpack2(u.z),
               d = Store<T>::unpack2(u.w);
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(Store<T>::pack2(x[0], x[1]), Store<T>::pack2(x[2], x[3]), Store<T>::pack2(x[4], x[5]),
                    Store<T>::pack2(x[6], x[7]));
}

// LP lanes hold one head (8 channels each, LP * 8 >= dim).  blockIdx.y picks the
// block's heads, threads are [side][places].
template <typename T, int LP, int TURN>
__global__ void __launch_bounds__(kPrepThreads) k_qkv_prepare(const __grid_constant__ PrepArgs A) {
  extern __shared__ __align__(16) float2 cs[];   // [2][side * batch][n_rot]: cos, sin
  __shared__ float2 turn[kMaxPairs];
  const int tid = threadIdx.x;
  for (int i = tid; i < A.n_rot; i += blockDim.x) turn[i] = make_float2(A.turn_hi[i], A.turn_lo[i]);
  const int per_block = A.places * A.side;       // threads with a place; the rest help with the angles
  const int sub = tid / A.places, place = tid - sub * A.places;
  const int e0 = (place % LP) * 8;               // first channel
  const int h = blockIdx.y * (A.places / LP) + place / LP;
  const bool is_q = h < A.n_qh, is_k = !is_q && h < A.n_qh + A.n_kh;
  const bool turned = is_q || is_k;
  const bool live = tid < per_block && h < A.n_qh + A.n_kh + A.n_vh && e0 < A.dim;
  const T* src = nullptr;
  T* dst = nullptr;
  long long src_row = 0, dst_row = 0;
  if (live) {
    if (is_q) {
      src = static_cast<const T*>(A.q) + h * A.q_head;
      dst = static_cast<T*>(A.q_out) + h * A.qo_head;
      src_row = A.q_row;
      dst_row = A.qo_row;
    } else if (is_k) {
      src = static_cast<const T*>(A.k) + (h - A.n_qh) * A.k_head;
      dst = static_cast<T*>(A.k_mem) + (h - A.n_qh) * A.km_head;
      src_row = A.k_row;
      dst_row = A.km_row;
    } else {
      src = static_cast<const T*>(A.v) + (h - A.n_qh - A.n_kh) * A.v_head;
      dst = static_cast<T*>(A.v_mem) + (h - A.n_qh - A.n_kh) * A.vm_head;
      src_row = A.v_row;
      dst_row = A.vm_row;
    }
  }
  const float* gain = is_q ? A.q_gain : A.k_gain;
  float gn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) gn[i] = live && turned && gain ? gain[e0 + i] : 1.0f;
  // the partner's place, for pairs that lie n_rot channels apart
  const int apart = A.n_rot / 8;
  const bool low = e0 < A.n_rot, in_rot = e0 < 2 * A.n_rot;
  float go[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    go[i] = TURN == kTurnLanes && live && turned && gain && in_rot ? gain[e0 + i + (low ? A.n_rot : -A.n_rot)] : 1.0f;
  const float inv_dim = 1.0f / A.dim;
  const int per_batch = A.side * A.batch;
  int buf = 0;
  __syncthreads();
  for (long long t0 = (long long)blockIdx.x * per_batch; t0 < A.n_tokens; t0 += (long long)gridDim.x * per_batch) {
    uint4 raw[kPrepBatch];
    long long to[kPrepBatch];                    // the output row, -1 = none
#pragma unroll
    for (int u = 0; u < kPrepBatch; ++u) {
      const long long tok = t0 + u * A.side + sub;
      const bool on = live && u < A.batch && tok < A.n_tokens;
      raw[u] = on ? *reinterpret_cast<const uint4*>(src + tok * src_row + e0) : make_uint4(0u, 0u, 0u, 0u);
      long long row = on ? tok : -1;
      if (on && !is_q) {
        row = A.rows ? A.rows[tok] : tok;
        if (row >= A.n_rows) row = -1;
      }
      to[u] = row;
    }
    float2* c = cs + buf * per_batch * A.n_rot;
    if (TURN != kTurnNone || A.coord) {
      // the batch's angles, one (token, pair) a thread at a time
      const int n = (int)min((long long)per_batch, A.n_tokens - t0);
      if (TURN != kTurnNone)
        for (int i = tid; i < n * A.n_rot; i += blockDim.x) {
          const int tk = i / A.n_rot, m = i - tk * A.n_rot;
          const float p = A.pos[3 * (t0 + tk) + (m < A.end_t ? 0 : m < A.end_y ? 1 : 2)];
          const float2 f = turn[m];
          const float t = p * f.x;
          const float frac = (t - rintf(t)) + fmaf(p, f.y, fmaf(p, f.x, -t));
          float2 v;
          sincospif(2.0f * frac, &v.y, &v.x);
          c[i] = v;
        }
      if (A.coord && blockIdx.y == 0)
        for (int i = tid; i < n; i += blockDim.x) {
          const long long row = A.rows ? A.rows[t0 + i] : t0 + i;
          if (row >= 0 && row < A.n_rows)
            *reinterpret_cast<float2*>(A.coord + 2 * row) =
                make_float2(A.pos[3 * (t0 + i) + 1], A.pos[3 * (t0 + i) + 2]);
        }
      if (TURN != kTurnNone) __syncthreads();    // the other buffer's readers are past it
    }
    buf ^= 1;
#pragma unroll
    for (int u = 0; u < kPrepBatch; ++u) {
      if (u >= A.batch) break;
      float x[8], y[8];
      unpack8<T>(raw[u], x);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
      for (int d = 1; d < LP; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
      const float r = A.norm ? rsqrtf(fmaf(sum, inv_dim, A.eps)) : 1.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i] * (r * gn[i]);
      const float2* ct = c + (u * A.side + sub) * A.n_rot;
      if (TURN == kTurnInterleaved) {
        const int m0 = e0 >> 1;
        if (live && turned) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (m0 + i < A.n_rot) {
              const float2 v = ct[m0 + i];
              const float a = y[2 * i], b = y[2 * i + 1];
              y[2 * i] = a * v.x - b * v.y;
              y[2 * i + 1] = a * v.y + b * v.x;
            }
          }
        }
      } else if (TURN == kTurnLanes) {
        const int from = low ? (place % LP) + apart : (place % LP) - apart;
        uint4 o;
        o.x = __shfl_sync(0xFFFFFFFFu, raw[u].x, from, LP);
        o.y = __shfl_sync(0xFFFFFFFFu, raw[u].y, from, LP);
        o.z = __shfl_sync(0xFFFFFFFFu, raw[u].z, from, LP);
        o.w = __shfl_sync(0xFFFFFFFFu, raw[u].w, from, LP);
        if (live && turned && in_rot) {
          float z[8];
          unpack8<T>(o, z);
          const float4* cv = reinterpret_cast<const float4*>(ct + (low ? e0 : e0 - A.n_rot));
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float4 v = cv[i / 2];          // cos, sin of two pairs
            const float o0 = z[i] * (r * go[i]), o1 = z[i + 1] * (r * go[i + 1]);
            y[i] = y[i] * v.x + (low ? -o0 : o0) * v.y;
            y[i + 1] = y[i + 1] * v.z + (low ? -o1 : o1) * v.w;
          }
        }
      } else if (TURN == kTurnAny) {
        const long long tok = t0 + u * A.side + sub;
        if (live && turned && tok < A.n_tokens) {
          const T* head = src + tok * src_row;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = e0 + i;
            if (e < 2 * A.n_rot) {
              const bool lo = e < A.n_rot;
              const int o = lo ? e + A.n_rot : e - A.n_rot;
              const float other = Store<T>::to_f(head[o]) * (r * (gain ? gain[o] : 1.0f));
              const float2 v = ct[lo ? e : o];
              y[i] = y[i] * v.x + (lo ? -other : other) * v.y;
            }
          }
        }
        __syncwarp();                            // every lane has read: q_out may be q
      }
      if (to[u] >= 0) *reinterpret_cast<uint4*>(dst + to[u] * dst_row + e0) = turned ? pack8<T>(y) : raw[u];
    }
  }
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool bad_stride(int64_t s) { return s < 0 || s % 8 != 0; }

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return sms;
}

template <typename T, int LP>
cudaError_t launch_prepare_t(const PrepArgs& a, int turn, const cudaLaunchConfig_t& lc) {
  switch (turn) {
    case kTurnNone: return cudaLaunchKernelEx(&lc, k_qkv_prepare<T, LP, kTurnNone>, a);
    case kTurnInterleaved: return cudaLaunchKernelEx(&lc, k_qkv_prepare<T, LP, kTurnInterleaved>, a);
    case kTurnLanes: return cudaLaunchKernelEx(&lc, k_qkv_prepare<T, LP, kTurnLanes>, a);
    default: return cudaLaunchKernelEx(&lc, k_qkv_prepare<T, LP, kTurnAny>, a);
  }
}

template <typename T>
cudaError_t launch_prepare(const PrepArgs& a, int lp, int turn, const cudaLaunchConfig_t& lc) {
  if (lp == 2) return launch_prepare_t<T, 2>(a, turn, lc);
  if (lp == 4) return launch_prepare_t<T, 4>(a, turn, lc);
  if (lp == 8) return launch_prepare_t<T, 8>(a, turn, lc);
  return launch_prepare_t<T, 16>(a, turn, lc);
}

}  // namespace
}  // namespace rtcc

using namespace rtcc;

extern "C" rtcc_status rtcc_memory_append(int32_t n_seqs, int32_t capacity, int32_t n_tokens,
                                          const int32_t* d_new, const int32_t* d_held,
                                          const int32_t* d_slot, int32_t* d_offsets, int32_t* d_rows,
                                          int32_t* d_seq, int32_t* d_pos, int32_t* d_begin,
                                          int32_t* d_end, int32_t* d_length, void* stream) {
  if (n_seqs < 0 || n_seqs > kMaxSeqs || capacity < 1 || n_tokens < 0) return RTCC_E_ARG;
  if (!d_offsets || (n_seqs > 0 && (!d_new || !d_held || !d_begin || !d_end || !d_length)) ||
      (n_tokens > 0 && !d_rows))
    return RTCC_E_ARG;
  const void* all[] = {d_new, d_held, d_slot, d_offsets, d_rows, d_seq, d_pos, d_begin, d_end, d_length};
  for (const void* p : all)
    if (misaligned(p, 4)) return RTCC_E_ARG;
  // the inputs are read by every block while others write: no output over an input
  if (n_seqs > 0 && (d_length == d_held || d_length == d_new)) return RTCC_E_ARG;
  AppendArgs a{d_new, d_held, d_slot, d_offsets, d_rows, d_seq, d_pos, d_begin, d_end, d_length,
               n_seqs, capacity, n_tokens};
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;
  const long long work = n_tokens > n_seqs ? n_tokens : n_seqs;
  long long blocks = (work + kAppendThreads * 4 - 1) / (kAppendThreads * 4);
  if (blocks > sms) blocks = sms;
  if (blocks < 1) blocks = 1;
  const size_t smem = sizeof(int) * ((size_t)n_seqs + 1);
  if (smem > 48 * 1024 &&
      cudaFuncSetAttribute(k_memory_append, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           (int)(sizeof(int) * (kMaxSeqs + 1))) != cudaSuccess)
    return RTCC_E_CUDA;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)blocks);
  lc.blockDim = dim3(kAppendThreads);
  lc.dynamicSmemBytes = smem;
  lc.stream = static_cast<cudaStream_t>(stream);
  return cudaLaunchKernelEx(&lc, k_memory_append, a) == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}

extern "C" rtcc_status rtcc_qkv_prepare(const rtcc_prepare_config* c, const void* d_q, const void* d_k,
                                        const void* d_v, const float* d_q_gain, const float* d_k_gain,
                                        const float* d_pos, const int32_t* d_rows, void* d_q_out,
                                        void* d_k_mem, void* d_v_mem, float* d_coord, void* stream) {
  if (!c) return RTCC_E_ARG;
  if (c->dtype != RTCC_FP16 && c->dtype != RTCC_BF16) return RTCC_E_ARG;
  if (c->n_tokens < 0 || c->n_rows < 0 || c->heads < 0 || c->heads > 4096 || c->kv_heads < 0 ||
      c->kv_heads > 4096)
    return RTCC_E_ARG;
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return RTCC_E_ARG;
  long long pairs = 0;
  for (int i = 0; i < 3; ++i) {
    if (c->axis_pairs[i] < 0 || c->axis_pairs[i] > c->head_dim / 2) return RTCC_E_ARG;
    pairs += c->axis_pairs[i];
  }
  if (pairs > c->head_dim / 2) return RTCC_E_ARG;
  if (!(c->theta >= 1.0f) || !isfinite(c->theta) || !(c->eps >= 0.0f) || !isfinite(c->eps)) return RTCC_E_ARG;
  if ((d_q != nullptr) != (d_q_out != nullptr) || (d_k != nullptr) != (d_k_mem != nullptr) ||
      (d_v != nullptr) != (d_v_mem != nullptr))
    return RTCC_E_ARG;
  if (c->n_tokens > 0 && !d_pos) return RTCC_E_ARG;
  if (d_q && (c->heads < 1 || bad_stride(c->q_row) || bad_stride(c->q_head) || bad_stride(c->qo_row) ||
              bad_stride(c->qo_head)))
    return RTCC_E_ARG;
  if (d_k && (c->kv_heads < 1 || bad_stride(c->k_row) || bad_stride(c->k_head) || bad_stride(c->km_row) ||
              bad_stride(c->km_head)))
    return RTCC_E_ARG;
  if (d_v && (c->kv_heads < 1 || bad_stride(c->v_row) || bad_stride(c->v_head) || bad_stride(c->vm_row) ||
              bad_stride(c->vm_head)))
    return RTCC_E_ARG;
  if (misaligned(d_q, 16) || misaligned(d_k, 16) || misaligned(d_v, 16) || misaligned(d_q_out, 16) ||
      misaligned(d_k_mem, 16) || misaligned(d_v_mem, 16) || misaligned(d_coord, 8) || misaligned(d_pos, 4) ||
      misaligned(d_rows, 4) || misaligned(d_q_gain, 4) || misaligned(d_k_gain, 4))
    return RTCC_E_ARG;
  if (c->n_tokens == 0 || (!d_q && !d_k && !d_v)) return RTCC_OK;
  const int sms = sm_count();
  if (sms < 1) return RTCC_E_CUDA;

  PrepArgs a{};
  a.q = d_q; a.k = d_k; a.v = d_v;
  a.q_gain = d_q_gain; a.k_gain = d_k_gain; a.pos = d_pos; a.rows = d_rows;
  a.q_out = d_q_out; a.k_mem = d_k_mem; a.v_mem = d_v_mem; a.coord = d_coord;
  a.q_row = c->q_row; a.q_head = c->q_head; a.k_row = c->k_row; a.k_head = c->k_head;
  a.v_row = c->v_row; a.v_head = c->v_head; a.qo_row = c->qo_row; a.qo_head = c->qo_head;
  a.km_row = c->km_row; a.km_head = c->km_head; a.vm_row = c->vm_row; a.vm_head = c->vm_head;
  a.n_tokens = c->n_tokens; a.n_rows = c->n_rows;
  a.n_qh = d_q ? c->heads : 0; a.n_kh = d_k ? c->kv_heads : 0; a.n_vh = d_v ? c->kv_heads : 0;
  a.dim = c->head_dim; a.n_rot = (int)pairs;
  a.end_t = c->axis_pairs[0]; a.end_y = c->axis_pairs[0] + c->axis_pairs[1];
  a.norm = c->norm != 0; a.eps = c->eps;
  int at = 0;
  for (int ax = 0; ax < 3; ++ax) {
    const int n = c->axis_pairs[ax];
    if (n == 0) continue;
    const double step = pow((double)c->theta, -1.0 / n);
    double f = 0.15915494309189533577;           // 1 / (2 pi)
    for (int m = 0; m < n; ++m, ++at, f *= step) {
      a.turn_hi[at] = (float)f;
      a.turn_lo[at] = (float)(f - (double)a.turn_hi[at]);
    }
  }
  // Threads: a place per head and 8 channels, heads over blockIdx.y where they do
  // not fit a block, several tokens side by side where they are few.
  const int lp = a.dim <= 16 ? 2 : a.dim <= 32 ? 4 : a.dim <= 64 ? 8 : 16;
  const int turn = pairs == 0 ? kTurnNone : c->interleaved ? kTurnInterleaved
                   : pairs % 8 == 0 ? kTurnLanes : kTurnAny;
  const int heads = a.n_qh + a.n_kh + a.n_vh;
  const int fit = kPrepThreads / lp;              // heads in a block at most
  const int ys = (heads + fit - 1) / fit, per = (heads + ys - 1) / ys;
  a.places = per * lp;
  a.side = kPrepThreads / a.places;
  while (a.side > 1 && sizeof(float2) * 2 * a.side * kPrepBatch * a.n_rot > 48 * 1024) a.side /= 2;
  // four tokens a thread, fewer while that leaves SMs without a block
  const long long columns = (a.n_tokens + a.side - 1LL) / a.side;
  a.batch = kPrepBatch;
  while (a.batch > 1 && (columns + a.batch - 1) / a.batch * ys < 2LL * sms) a.batch /= 2;
  while (a.side > 1 && (a.n_tokens + a.side * a.batch - 1LL) / (a.side * a.batch) * ys < sms) a.side /= 2;
  long long blocks = (a.n_tokens + (long long)a.side * a.batch - 1) / ((long long)a.side * a.batch);
  const long long most = (8LL * sms + ys - 1) / ys;
  if (blocks > most) blocks = most;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)blocks, (unsigned)ys);
  lc.blockDim = dim3((a.places * a.side + 31) / 32 * 32);
  lc.dynamicSmemBytes = sizeof(float2) * 2 * a.side * a.batch * a.n_rot;
  lc.stream = static_cast<cudaStream_t>(stream);
  const cudaError_t e = c->dtype == RTCC_BF16 ? launch_prepare<__nv_bfloat16>(a, lp, turn, lc)
                                              : launch_prepare<__half>(a, lp, turn, lc);
  return e == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}
