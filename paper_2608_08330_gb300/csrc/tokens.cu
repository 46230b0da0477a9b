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
//   share of the tokens.  The launch and the scan's latency bound it:
//   61 sequences take 2.6 us, 2048 with 409,000 token places (5 MB) 7.0 us.
//
// rtcc_qkv_prepare: for every token and head of q and k
//   x^ = x * rsqrt(mean(x^2) + eps) * gain,
//   and pair m of axis a of x^ turned by pos_a * theta^(-m / pairs_a);
//   q goes to a dense output, k, v and the (y, x) coordinates to the token's
//   memory row.  It reads and writes every vector once, so HBM bounds it.  2 to 16
//   lanes hold one token (8 channels, one 16-byte copy in and one store out each)
//   and go through its heads: a lane's angles are computed once and stay in
//   registers for all heads.  Eight heads' vectors are on their way to a ring in
//   shared memory, every thread's own places, so nothing is waited for but the
//   copy itself.  With few tokens a token's heads are divided among several groups
//   of lanes.  Measured: 176,000 tokens of 18 heads of 64, 815 MB, 121.5 us: 6.7 TB/s,
//   99 % of a plain copy's; 16,384 of them 16.9 us, 66 %, or 14.6 us, 77 %, where pairs
//   are neighbours and no lane needs another's vector; 12,345 tokens of 20 heads of 80
//   (10 of 16 lanes have channels) 19.7 us, 59 %; 61 tokens 3.7 us.
#include <math.h>

#include <atomic>

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
  for (int s = first; s <= A.n_seqs; s += stride) {   // at most kMaxSeqs + stride
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
  for (long long t = first; t < A.n_tokens; t += stride) {   // in 64 bits: n_tokens + stride may pass 2^31
    const int i = (int)t;
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

constexpr int kPrepThreads = 128;
constexpr int kPrepPairs = 4;                    // pairs of heads on their way per lane
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
  float eps;
  // turns per unit of position, theta^(-m / n) / 2 pi, as the sum of two floats:
  // the product with a position stays exact to a small fraction of a turn at
  // positions where one float's rounding would be most of a turn
  float turn_hi[kMaxPairs], turn_lo[kMaxPairs];
};

// How pairs lie: none, (2m, 2m + 1), or (m, m + n_rot) with n_rot a multiple of
// 8 (the partner is another lane's whole vector) or not (read again, an L1 hit).
enum { kTurnNone, kTurnInterleaved, kTurnLanes, kTurnAny };

// cos and sin of p * 2 pi * (hi + lo).  The turns are reduced to [-1/2, 1/2]
// exactly enough before the hardware's sine and cosine (absolute error below 2^-21,
// against 2^-11 or 2^-8 of the result's rounding).
__device__ __forceinline__ float2 cos_sin(float p, float2 f) {
  const float t = p * f.x;
  const float frac = (t - rintf(t)) + fmaf(p, f.y, fmaf(p, f.x, -t));
  float2 c;
  __sincosf(6.283185307f * frac, &c.y, &c.x);
  return c;
}

// LP lanes hold one token's channels (8 each, LP * 8 >= dim); blockIdx.y of
// gridDim.y takes its share of the q, k and v heads.
template <typename T, int LP, int TURN>
__global__ void __launch_bounds__(kPrepThreads, 6) k_qkv_prepare(const __grid_constant__ PrepArgs A) {
  __shared__ float2 turn[kMaxPairs];
  __shared__ uint4 ring[kPrepPairs][2][kPrepThreads];
  const int tid = threadIdx.x;
  for (int i = tid; i < A.n_rot; i += kPrepThreads) turn[i] = make_float2(A.turn_hi[i], A.turn_lo[i]);
  const long long id = (long long)blockIdx.x * kPrepThreads + tid;
  const int lane = (int)(id % LP), e0 = lane * 8;
  const bool live = id / LP < A.n_tokens && e0 < A.dim;
  const long long tok = min(id / LP, (long long)A.n_tokens - 1);
  // this block's heads of q, k and v, in pairs
  const int all = A.n_qh + A.n_kh + A.n_vh;
  const int h0 = (int)((long long)all * blockIdx.y / gridDim.y), h1 = (int)((long long)all * (blockIdx.y + 1) / gridDim.y);
  const int q0 = min(h0, A.n_qh), q1 = min(h1, A.n_qh);
  const int k0 = min(max(h0 - A.n_qh, 0), A.n_kh), k1 = min(max(h1 - A.n_qh, 0), A.n_kh);
  const int v0 = max(h0 - A.n_qh - A.n_kh, 0), v1 = max(h1 - A.n_qh - A.n_kh, 0);
  const int qp = (q1 - q0 + 1) / 2, kp = qp + (k1 - k0 + 1) / 2, vp = kp + (v1 - v0 + 1) / 2;
  const T* qs = static_cast<const T*>(A.q) + tok * A.q_row + e0;
  const T* ks = static_cast<const T*>(A.k) + tok * A.k_row + e0;
  const T* vs = static_cast<const T*>(A.v) + tok * A.v_row + e0;
  auto issue = [&](int j) {                      // pair j on its way
    if (live && j < vp) {
      const T* src;
      long long step;
      int n;
      if (j < qp) {
        src = qs + (q0 + 2 * j) * A.q_head, step = A.q_head, n = q1 - q0 - 2 * j;
      } else if (j < kp) {
        src = ks + (k0 + 2 * (j - qp)) * A.k_head, step = A.k_head, n = k1 - k0 - 2 * (j - qp);
      } else {
        src = vs + (v0 + 2 * (j - kp)) * A.v_head, step = A.v_head, n = v1 - v0 - 2 * (j - kp);
      }
      uint4(*slot)[kPrepThreads] = ring[j % kPrepPairs];
      cp_async16(&slot[0][tid], src);
      if (n > 1) cp_async16(&slot[1][tid], src + step);
    }
    cp_async_commit();
  };
#pragma unroll
  for (int j = 0; j < kPrepPairs; ++j) issue(j);
  const long long row = A.rows ? A.rows[tok] : tok;
  const bool stored = live && row >= 0 && row < A.n_rows;
  float pos[3] = {0.f, 0.f, 0.f};
  if (TURN != kTurnNone || A.coord) {            // else d_pos may be null
#pragma unroll
    for (int i = 0; i < 3; ++i) pos[i] = A.pos[3 * tok + i];
  }
  if (A.coord && blockIdx.y == 0 && stored && lane == 0)
    *reinterpret_cast<float2*>(A.coord + 2 * row) = make_float2(pos[1], pos[2]);
  __syncthreads();                               // the table of turns

  // This lane's cosines and sines: channel e of a pair becomes x_e cs + x_other sn,
  // the sine's sign with it (1 and 0 where nothing turns).  The two channels of
  // an interleaved pair share theirs.
  constexpr int P = TURN == kTurnInterleaved ? 2 : 4;
  float2 cs[P], sn[P];
  const bool low = e0 < A.n_rot, in_rot = e0 < 2 * A.n_rot;
  auto angle = [&](int m) -> float2 {            // pair m's cosine and sine
    if (m >= A.n_rot) return make_float2(1.0f, 0.0f);
    return cos_sin(m < A.end_t ? pos[0] : m < A.end_y ? pos[1] : pos[2], turn[m]);
  };
  if (TURN == kTurnLanes && kp > 0) {
    // the partner's lane has the same eight pairs: four each, and an exchange
    const int from = lane + (low ? A.n_rot / 8 : -(A.n_rot / 8)), base = low ? e0 : e0 - A.n_rot + 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 own = angle(in_rot ? base + i : A.n_rot);
      const float ox = __shfl_sync(0xFFFFFFFFu, own.x, from, LP), oy = __shfl_sync(0xFFFFFFFFu, own.y, from, LP);
      const float2 c0 = low ? own : make_float2(ox, oy), c1 = low ? make_float2(ox, oy) : own;   // pairs i, i + 4
      const float sign = low ? -1.0f : 1.0f;
      (i & 1 ? cs[i / 2].y : cs[i / 2].x) = in_rot ? c0.x : 1.0f;
      (i & 1 ? cs[i / 2 + 2].y : cs[i / 2 + 2].x) = in_rot ? c1.x : 1.0f;
      (i & 1 ? sn[i / 2].y : sn[i / 2].x) = in_rot ? sign * c0.y : 0.0f;
      (i & 1 ? sn[i / 2 + 2].y : sn[i / 2 + 2].x) = in_rot ? sign * c1.y : 0.0f;
    }
  } else if (TURN != kTurnNone && kp > 0) {
#pragma unroll
    for (int i = 0; i < 2 * P; ++i) {
      const int e = e0 + i;
      const float2 c = angle(TURN == kTurnInterleaved ? e0 / 2 + i : e < A.n_rot ? e : e - A.n_rot);
      (i & 1 ? cs[i / 2].y : cs[i / 2].x) = c.x;
      (i & 1 ? sn[i / 2].y : sn[i / 2].x) = TURN != kTurnInterleaved && e < A.n_rot ? -c.y : c.y;
    }
  }
  const float inv_dim = 1.0f / A.dim;

  // pairs [j0, j1) are heads [0, n) of q or k, at src and dst
  auto heads = [&](int j0, int j1, int n, const T* src, long long src_step, T* dst, long long dst_step, bool write,
                   const float* gain) {
    float2 gn[4], go[4];                         // gains: own, and the partner's, for all heads
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      gn[i] = gain && live ? make_float2(gain[e0 + 2 * i], gain[e0 + 2 * i + 1]) : make_float2(1.f, 1.f);
      if (TURN == kTurnLanes) {                  // with the cosine and the sine
        const int o = e0 + 2 * i + (low ? A.n_rot : -A.n_rot);
        go[i] = gain && live && in_rot ? mul2(make_float2(gain[o], gain[o + 1]), sn[i]) : sn[i];
        gn[i] = mul2(gn[i], cs[i]);
      }
    }
    for (int j = j0; j < j1; ++j, n -= 2, src += 2 * src_step, dst += 2 * dst_step) {
      cp_async_wait<kPrepPairs - 1>();
      uint4 raw[2];
      raw[0] = live ? ring[j % kPrepPairs][0][tid] : make_uint4(0u, 0u, 0u, 0u);
      raw[1] = live && n > 1 ? ring[j % kPrepPairs][1][tid] : make_uint4(0u, 0u, 0u, 0u);
      issue(j + kPrepPairs);
      float rs[2] = {1.f, 1.f};
      if (A.norm) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float2 x = Store<T>::unpack2(raw[u].x);
          float2 q = mul2(x, x);
          x = Store<T>::unpack2(raw[u].y);
          q = fma2(x, x, q);
          x = Store<T>::unpack2(raw[u].z);
          q = fma2(x, x, q);
          x = Store<T>::unpack2(raw[u].w);
          q = fma2(x, x, q);
          rs[u] = q.x + q.y;
        }
#pragma unroll
        for (int d = 1; d < LP; d <<= 1)
#pragma unroll
          for (int u = 0; u < 2; ++u) rs[u] += __shfl_xor_sync(0xFFFFFFFFu, rs[u], d);
#pragma unroll
        for (int u = 0; u < 2; ++u) rs[u] = rsqrtf(fmaf(rs[u], inv_dim, A.eps));
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (u >= n) continue;                    // the same for the whole block
        const float2 rr = make_float2(rs[u], rs[u]);
        float2 y[4];
        y[0] = mul2(Store<T>::unpack2(raw[u].x), rr);
        y[1] = mul2(Store<T>::unpack2(raw[u].y), rr);
        y[2] = mul2(Store<T>::unpack2(raw[u].z), rr);
        y[3] = mul2(Store<T>::unpack2(raw[u].w), rr);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], gn[i]);
        if (TURN == kTurnInterleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float c = i & 1 ? cs[i / 2].y : cs[i / 2].x, s = i & 1 ? sn[i / 2].y : sn[i / 2].x;
            // a pair that is not turned (1 and 0) keeps its channels, whatever the other holds
            if (s != 0.f || c < 0.f) y[i] = make_float2(y[i].x * c - y[i].y * s, y[i].x * s + y[i].y * c);
          }
        } else if (TURN == kTurnLanes) {
          const int from = lane + (low ? A.n_rot / 8 : -(A.n_rot / 8));
          float2 z[4];
          z[0] = Store<T>::unpack2(__shfl_sync(0xFFFFFFFFu, raw[u].x, from, LP));
          z[1] = Store<T>::unpack2(__shfl_sync(0xFFFFFFFFu, raw[u].y, from, LP));
          z[2] = Store<T>::unpack2(__shfl_sync(0xFFFFFFFFu, raw[u].z, from, LP));
          z[3] = Store<T>::unpack2(__shfl_sync(0xFFFFFFFFu, raw[u].w, from, LP));
          if (in_rot) {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fma2(mul2(z[i], rr), go[i], y[i]);
          }
        } else if (TURN == kTurnAny) {
          if (live) {
            const T* head = src + u * src_step - e0;
            auto other = [&](int e) {
              if (e >= 2 * A.n_rot) return 0.f;
              const int o = e < A.n_rot ? e + A.n_rot : e - A.n_rot;
              return Store<T>::to_f(head[o]) * rs[u] * (gain ? gain[o] : 1.0f);
            };
#pragma unroll
            for (int i = 0; i < 4; ++i)
              y[i] = fma2(y[i], cs[i], mul2(make_float2(other(e0 + 2 * i), other(e0 + 2 * i + 1)), sn[i]));
          }
          __syncwarp();                          // every lane has read: q_out may be q
        }
        if (write)
          *reinterpret_cast<uint4*>(dst + u * dst_step) =
              make_uint4(Store<T>::pack2(y[0].x, y[0].y), Store<T>::pack2(y[1].x, y[1].y),
                         Store<T>::pack2(y[2].x, y[2].y), Store<T>::pack2(y[3].x, y[3].y));
      }
    }
  };
  if (qp > 0)
    heads(0, qp, q1 - q0, qs + q0 * A.q_head, A.q_head,
          static_cast<T*>(A.q_out) + tok * A.qo_row + q0 * A.qo_head + e0, A.qo_head, live, A.q_gain);
  const long long to = stored ? row : 0;
  if (kp > qp)
    heads(qp, kp, k1 - k0, ks + k0 * A.k_head, A.k_head, static_cast<T*>(A.k_mem) + to * A.km_row + k0 * A.km_head + e0,
          A.km_head, stored, A.k_gain);
  T* vd = static_cast<T*>(A.v_mem) + to * A.vm_row + v0 * A.vm_head + e0;
  for (int j = kp, n = v1 - v0; j < vp; ++j, n -= 2, vd += 2 * A.vm_head) {
    cp_async_wait<kPrepPairs - 1>();
    if (stored) {
      *reinterpret_cast<uint4*>(vd) = ring[j % kPrepPairs][0][tid];
      if (n > 1) *reinterpret_cast<uint4*>(vd + A.vm_head) = ring[j % kPrepPairs][1][tid];
    }
    issue(j + kPrepPairs);
  }
  cp_async_wait<0>();
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool bad_stride(int64_t s) { return s < 0 || s % 8 != 0; }

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

constexpr int kMaxDevices = 64;
std::atomic<int> g_sms[kMaxDevices];             // 0: not asked yet

}  // namespace

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  n = g_sms[dev].load(std::memory_order_relaxed);
  if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
    g_sms[dev].store(n, std::memory_order_relaxed);
  return n;
}

cudaError_t allow_smem(const void* kernel, int bytes, std::atomic<uint64_t>* devices, bool wide_clusters) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (devices->load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && wide_clusters) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess && dev < 64) devices->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

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
  static std::atomic<uint64_t> allowed{0};
  if (smem > 48 * 1024 && allow_smem(reinterpret_cast<const void*>(k_memory_append), (int)(sizeof(int) * (kMaxSeqs + 1)),
                                     &allowed) != cudaSuccess)
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
  if (c->n_tokens > 0 && !d_pos && (pairs > 0 || d_coord)) return RTCC_E_ARG;
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
  if (c->n_tokens == 0 || (!d_q && !d_k && !d_v && !d_coord)) return RTCC_OK;
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
  const int lp = a.dim <= 16 ? 2 : a.dim <= 32 ? 4 : a.dim <= 64 ? 8 : 16;
  const int turn = pairs == 0 ? kTurnNone : c->interleaved ? kTurnInterleaved
                   : pairs % 8 == 0 ? kTurnLanes : kTurnAny;
  // a token's heads stay together unless that leaves threads for less than half
  // of what the GPU holds (1024 a SM; twice and four times that many took up to
  // 13 and 40 % longer on 3000 to 20,000 tokens)
  const int heads = a.n_qh + a.n_kh + a.n_vh;
  const long long threads = (long long)a.n_tokens * lp;
  long long parts = (512LL * sms + threads - 1) / threads;
  if (parts > heads) parts = heads;
  if (parts < 1) parts = 1;                      // coordinates alone
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)((threads + kPrepThreads - 1) / kPrepThreads), (unsigned)parts);
  lc.blockDim = dim3(kPrepThreads);
  lc.stream = static_cast<cudaStream_t>(stream);
  const cudaError_t e = c->dtype == RTCC_BF16 ? launch_prepare<__nv_bfloat16>(a, lp, turn, lc)
                                              : launch_prepare<__half>(a, lp, turn, lc);
  return e == cudaSuccess ? RTCC_OK : RTCC_E_CUDA;
}
