// Attention of a few rows over long spans of the token memory, and the join of
// partial results.
//
//   s_ij = cap tanh(scale q_i.k_j / cap) - slope_h |r_i - r_j|_1   (cap 0: no tanh)
//   out_i = sum_j softmax_j(s_ij) v_j,  lse_i = ln sum_j exp(s_ij)
//   j over the visible keys; no visible key: out_i = 0, lse_i = -inf
//
// A row is a (token, head) pair; the heads that share a key head are rows of
// the same block, so every key and value is read once per 16 rows.  A block has
// 16 rows (the M of mma.m16n8k16), one key head and one chunk of the span; its
// four warps take key tiles in turn, each with a running maximum, sum and
// 16 x dim accumulator in registers and a ring of three tiles of its own in
// shared memory filled by 16-byte asynchronous copies (no block barrier in the
// loop).  Rows of the memory that no query may see are never read: their place
// in the tile is zero-filled, so stale or non-finite contents do not matter.
// The probabilities go to the second product as the sum of two numbers of the
// storage type: the tensor pipe has room for the second product, and a single
// token's error then is the output's rounding alone.  fp16 ends at 2^-24, so there
// the largest probability is 2^15 instead of 1: what is lost of a key is 2^-40 of
// the largest, not 2^-25, which over 280,000 keys would be up to 0.8 % of the weight.
//
// With few rows the memory's bytes bound it, and splitting the span into chunks
// fills the GPU; k_attn_join merges the chunks in index order, or, where the chunks
// are few, the blocks of a cluster do it from one another's shared memory.
// Measured: 61 tokens over ragged histories of up to 16,384 keys, 8 key heads of
// 128, 1.9 GB: 300 us, 6.4 TB/s, 94 % of a plain copy's; one token over 4097 keys of
// 6 heads of 64 takes 8.2 us, most of which is the launch, a block's first copies
// and three steps.  WIN: with a window; keys between the sinks and the window of a
// sequence's first token are numbered away (attn_span), so that chunks are of what is
// read.  The 61 tokens over windows of 5000 keys, 1.1 GB: 177 us, 6.2 TB/s; one token over
// 1000 keys of 4 key heads of 80: 7.6 us.
#include "attn_rows.cuh"
#include "kernels.h"

namespace rtcc {
namespace {

constexpr int kStages = 3;

// log2 of the largest probability (a row's m is its largest score less this)
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 15.0f : 0.0f;

template <int DP> struct RowsCfg {               // DP: head size padded to 64 or 128
  static constexpr int KT = DP == 64 ? 32 : 16;  // keys per tile: 4 KB of keys, 4 KB of values
  static constexpr int kTileBytes = KT * DP * 2;
  static constexpr int kPosBytes = KT * 8;
  static constexpr int kStageBytes = 2 * kTileBytes + kPosBytes;
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  // at the end the warps' accumulators, then the block's for its cluster: [row][DP + 4]
  static constexpr int kState = kRows * (DP + 4);
  static_assert((kWarps + 1) * kState * 4 <= kRing, "states at the end lie in the ring");
  static constexpr int kSmem = kRing;
};

// Byte offset of 16-byte unit c of row r in a tile of DP-channel rows; units
// are permuted within 128-byte lines so that ldmatrix reads 8 rows without
// bank conflicts.
template <int DP>
__device__ __forceinline__ uint32_t tile_off(int r, int c) {
  return (uint32_t)(r * DP * 2 + (c & ~7) * 16 + (((c ^ r) & 7) * 16));
}

// CLUSTER: the chunks are the cluster's blocks, which join them (a kernel of its own:
// the join's registers cost the long split 2 %).
template <typename T, int DP, bool CLUSTER, bool WIN>
__global__ void __launch_bounds__(kWarps * 32, 2) k_attn_rows(const __grid_constant__ AttnArgs A) {
  using C = RowsCfg<DP>;
  constexpr int KT = C::KT;
  extern __shared__ __align__(128) unsigned char smem[];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  // block -> (sequence, key head, first row group, chunk), chunks fastest
  int b = blockIdx.x;
  const int chunk = b % A.n_chunks;
  b /= A.n_chunks;
  const int rg0 = b % A.row_groups;
  b /= A.row_groups;
  const int kvh = b % A.kv_heads;
  const int seq = b / A.kv_heads;
  const AttnSpan S = attn_span<WIN>(A, seq);
  const int rows_all = S.nq * A.group;
  const int per = attn_chunk(A, S.nk, A.unit);
  const int c0 = (int)min((long long)per * chunk, (long long)S.nk), c1 = min(S.nk - c0, per) + c0;
  if (!CLUSTER && chunk > 0 && c0 >= S.nk) return;   // not in use; chunk 0 always answers
  const unsigned long long slots = attn_slot_mask(A, lane);
  const uint32_t ring = smem_u32(smem) + w * kStages * C::kStageBytes;
  const unsigned char* ring_g = smem + w * kStages * C::kStageBytes;
  const bool dist = A.slopes != nullptr, far_cap = WIN || A.cap_log2 > kAbsCap * kLog2e;   // windows: few keys, whose lse is a score
  const T* kbase = static_cast<const T*>(A.k) + (long long)kvh * A.k_head;
  const T* vbase = static_cast<const T*>(A.v) + (long long)kvh * A.v_head;

  for (int rg = rg0; (long long)rg * kRows < rows_all; rg += A.row_groups) {
    const int r0 = rg * kRows;
    // this lane's two rows: lane / 4 and 8 further
    int hi[2], head[2];
    AttnView view[2];
    bool row_ok[2];
    long long tok[2];
    float slope[2], qy[2], qx[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = r0 + lane / 4 + 8 * i;
      row_ok[i] = r < rows_all;
      const int ql = row_ok[i] ? r / A.group : 0;
      head[i] = kvh * A.group + (row_ok[i] ? r % A.group : 0);
      tok[i] = S.q0 + ql;
      hi[i] = row_ok[i] ? attn_visible(A, S, S.first, ql) : 0;
      if (WIN) view[i] = attn_view(A, S, S.first, ql);
      slope[i] = dist ? A.slopes[head[i]] * kLog2e : 0.f;
      qy[i] = dist && row_ok[i] ? A.q_pos[tok[i] * A.q_pos_row] : 0.f;
      qx[i] = dist && row_ok[i] ? A.q_pos[tok[i] * A.q_pos_row + 1] : 0.f;
    }
    // the rows' reach: keys past it are not read
    int reach = max(hi[0], hi[1]), least = min(row_ok[0] ? hi[0] : S.nk, row_ok[1] ? hi[1] : S.nk);
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      reach = max(reach, __shfl_xor_sync(0xFFFFFFFFu, reach, d));
      least = min(least, __shfl_xor_sync(0xFFFFFFFFu, least, d));
    }
    const int end = min(c1, reach);
    // with a window: keys [seen, low) are seen by no row, keys before seen_all and from low_all on by all
    int seen = 0, low = 0, seen_all = 0, low_all = 0;
    if (WIN) {
      const AttnView f = attn_view(A, S, S.first, r0 / A.group);
      const AttnView l = attn_view(A, S, S.first, (min(r0 + kRows, rows_all) - 1) / A.group);
      seen = l.seen; low = f.low; seen_all = f.seen; low_all = l.low;
    }
    // A fragments of Q
    uint32_t qa[DP / 16][4];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = s * 16 + (lane % 4) * 2 + (i >> 1) * 8;
        const int rr = i & 1;
        qa[s][i] = row_ok[rr] && col < A.dim
                       ? *reinterpret_cast<const uint32_t*>(static_cast<const T*>(A.q) + tok[rr] * A.q_row +
                                                            (long long)head[rr] * A.q_head + col)
                       : 0u;
      }
    float o[DP / 8][4];
#pragma unroll
    for (int n = 0; n < DP / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    const int n_tiles = end > c0 ? (end - c0 + KT - 1) / KT : 0;
    // bits of the tile's keys that may be read: in the span's reach, slot present
    auto key_bits = [&](int t) -> unsigned {
      const int j = c0 + t * KT + lane;
      bool ok = t < n_tiles && lane < KT && j < end;
      if (WIN) ok = ok && (j < seen || j >= low);
      if (ok && A.present) ok = (slots >> slot_of(A, WIN ? attn_row(S, j) : S.kb + j)) & 1;
      return __ballot_sync(0xFFFFFFFFu, ok);
    };
    auto load = [&](int t, int stage) {
      const unsigned bits = key_bits(t);
      if (bits) {
        const long long at_row = WIN ? attn_row(S, c0 + t * KT) : S.kb + c0 + t * KT;   // a tile lies on one side of a gap
        const uint32_t ks = ring + stage * C::kStageBytes, vs = ks + C::kTileBytes, ps = vs + C::kTileBytes;
        constexpr int U = DP / 8;                // 16-byte units of a row
#pragma unroll
        for (int i = 0; i < KT * U / 32; ++i) {
          const int idx = i * 32 + lane, r = idx / U, c = idx % U;
          const bool live = (bits >> r) & 1 && c * 8 < A.dim;
          const long long row = live ? at_row + r : 0;
          const int col = live ? c * 8 : 0;
          const uint32_t at = tile_off<DP>(r, c);
          cp16(ks + at, kbase + row * A.k_row + col, live);
          cp16(vs + at, vbase + row * A.v_row + col, live);
        }
        if (dist && lane < KT) {
          const bool live = (bits >> lane) & 1;
          const long long row = live ? at_row + lane : 0;
          cp8(ps + lane * 8, A.k_pos + 2 * row, live);
        }
      }
      cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) load(w + s * kWarps, s);
    int stage = 0;
    for (int t = w; t < n_tiles; t += kWarps) {
      cp_async_wait<kStages - 2>();
      __syncwarp();
      load(t + (kStages - 1) * kWarps, (stage + kStages - 1) % kStages);
      const unsigned bits = key_bits(t);
      if (bits) {
        const uint32_t ks = ring + stage * C::kStageBytes, vs = ks + C::kTileBytes;
        const float2* ps = reinterpret_cast<const float2*>(ring_g + stage * C::kStageBytes + 2 * C::kTileBytes);
        float s[KT / 8][4];
#pragma unroll
        for (int n = 0; n < KT / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)        // 32 channels: two k16 steps, one ldmatrix.x4 per 8 keys
#pragma unroll
          for (int n = 0; n < KT / 8; ++n) {
            uint32_t kb4[4];
            ldm4(ks + tile_off<DP>(n * 8 + (lane & 7), d * 4 + (lane >> 3)), kb4);
            mma16816<T>(s[n], qa[2 * d], kb4[0], kb4[1]);
            mma16816<T>(s[n], qa[2 * d + 1], kb4[2], kb4[3]);
          }
        const int j0 = c0 + t * KT;
        const unsigned full = KT == 32 ? 0xFFFFFFFFu : (1u << KT) - 1u;
        const bool edge = bits != full || j0 + KT > least || (WIN && j0 < low_all && j0 + KT > seen_all);
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < KT / 8; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = n * 8 + (lane & 3) * 2 + (i & 1), rr = i >> 1;
            float x = s[n][i] * A.scale_log2;
            if (A.cap_log2 > 0.f) x = A.cap_log2 * (far_cap ? tanh_rel(x) : tanh_abs(x));
            if (dist) {
              const float2 p = ps[key];
              x = fmaf(-slope[rr], fabsf(qy[rr] - p.x) + fabsf(qx[rr] - p.y), x);
            }
            if (edge && !(((bits >> key) & 1) && j0 + key < hi[rr])) x = -INFINITY;
            if (WIN && edge && j0 + key >= view[rr].seen && j0 + key < view[rr].low) x = -INFINITY;
            s[n][i] = x;
            top[rr] = fmaxf(top[rr], x);
          }
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          top[rr] = fmaxf(top[rr], __shfl_xor_sync(0xFFFFFFFFu, top[rr], 1));
          top[rr] = fmaxf(top[rr], __shfl_xor_sync(0xFFFFFFFFu, top[rr], 2));
          const float mn = fmaxf(m[rr], top[rr] - kLift<T>);
          const float base = mn == -INFINITY ? 0.f : mn;
          const float f = exp2f(m[rr] - base);   // m = -inf: 0
          m[rr] = mn;
          l[rr] *= f;
          top[rr] = base;
          if (__any_sync(0xFFFFFFFFu, f != 1.0f)) {
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
              o[n][2 * rr] *= f;
              o[n][2 * rr + 1] *= f;
            }
          }
        }
        // a tile's sum first: one by one, small probabilities behind a large one would
        // round to nothing (2^-25 of it each)
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < KT / 8; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[n][i] = exp2f(s[n][i] - top[i >> 1]);
            sum[i >> 1] += s[n][i];
          }
        l[0] += sum[0];
        l[1] += sum[1];
#pragma unroll
        for (int kk = 0; kk < KT / 16; ++kk) {
          // probabilities as two terms of the storage type, so that their rounding
          // (2^-22 or 2^-16) adds nothing to the result's; the memory leaves time for it
          uint32_t pa[4], pl[4];
          split2<T>(s[2 * kk][0], s[2 * kk][1], pa[0], pl[0]);
          split2<T>(s[2 * kk][2], s[2 * kk][3], pa[1], pl[1]);
          split2<T>(s[2 * kk + 1][0], s[2 * kk + 1][1], pa[2], pl[2]);
          split2<T>(s[2 * kk + 1][2], s[2 * kk + 1][3], pa[3], pl[3]);
#pragma unroll
          for (int n = 0; n < DP / 16; ++n) {
            uint32_t vb[4];
            ldm4t(vs + tile_off<DP>(kk * 16 + (lane & 15), n * 2 + (lane >> 4)), vb);
            mma16816<T>(o[2 * n], pa, vb[0], vb[1]);
            mma16816<T>(o[2 * n + 1], pa, vb[2], vb[3]);
            mma16816<T>(o[2 * n], pl, vb[0], vb[1]);
            mma16816<T>(o[2 * n + 1], pl, vb[2], vb[3]);
          }
        }
      }
      stage = (stage + 1) % kStages;
    }
    cp_async_wait<0>();
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      l[rr] += __shfl_xor_sync(0xFFFFFFFFu, l[rr], 1);
      l[rr] += __shfl_xor_sync(0xFFFFFFFFu, l[rr], 2);
    }
    // merge the four warps' states through shared memory (the ring is done with)
    __syncthreads();
    float* mo = reinterpret_cast<float*>(smem);  // [warp][row][DP + 4]: accumulator, maximum, sum
    constexpr int P = DP + 4;
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      float* dst = mo + (w * kRows + lane / 4 + 8 * rr) * P;
#pragma unroll
      for (int n = 0; n < DP / 8; ++n)
        *reinterpret_cast<float2*>(dst + n * 8 + (lane & 3) * 2) = make_float2(o[n][2 * rr], o[n][2 * rr + 1]);
      if ((lane & 3) == 0) {
        dst[DP] = m[rr];
        dst[DP + 1] = l[rr];
      }
    }
    merge_states<T, DP, CLUSTER>(A, S, mo, r0, rows_all, kvh, chunk);
    __syncthreads();
  }
}

// The sequence that token t belongs to, q_offsets[s] <= t < q_offsets[s + 1]; -1: none.
// Whole warp, 32 offsets at a time.
__device__ __forceinline__ int seq_of(const AttnArgs& A, int t, int lane) {
  int lo = 0, hi = A.n_seqs;                     // q_offsets[lo] <= t < q_offsets[hi]
  if (A.q_offsets[lo] > t || A.q_offsets[hi] <= t) return -1;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const unsigned past = __ballot_sync(0xFFFFFFFFu, A.q_offsets[min(lo + (lane + 1) * step, hi)] > t);
    const int l = __ffs(past) - 1;               // lane 31 is at hi
    hi = min(lo + (l + 1) * step, hi);
    lo += l * step;
  }
  return lo;
}

// out_i = sum_c 2^(m_c - M) O_c / sum_c 2^(m_c - M) l_c over the partial results
// in use: W warps per row (4 where there are many partial results, which one warp
// would read one after another: 5 rows of 600 took 120 us), 4 channels per lane.
// Every warp sums its share in index order, then the shares are summed in order.
// A warp (or the block's W) takes `per` rows of the call one after another, whatever
// sequences they belong to: with blocks for every sequence, as many as the longest one
// wants, ragged calls spend their time on blocks without work or on a few with too much
// (100 sequences of 1 to 16,000 tokens, most of them short, 6 heads of 64: 3.52 ms the whole
// call, 2.20 so; one of 2,700 tokens and 400 of 5, 12 heads of 128: 2.82 and 1.10).
constexpr int kJoinWarps = 4;
template <typename T, int W, int U>              // U: loads in flight
__global__ void __launch_bounds__(kJoinWarps * 32) k_attn_join(const __grid_constant__ AttnArgs A, int per) {
  __shared__ float4 sum_o[kJoinWarps][32];
  __shared__ float2 sum_ml[kJoinWarps];
  pdl_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long rows = (long long)A.n_q * A.heads, stride = rows;
  constexpr int kTakers = kJoinWarps / W;        // of a block
  const int first = W == 1 ? 0 : w;              // this warp's partial results: first, first + W, ...
  const long long R0 = ((long long)blockIdx.x * kTakers + (W == 1 ? w : 0)) * per, R1 = min(R0 + per, rows);
  AttnSpan S{};                                  // of the row's sequence: rows below `end`
  long long end = 0;
  int used = 0;
  for (long long R = R0; R < R1; ++R) {
    const int t = (int)((uint32_t)R / (uint32_t)A.heads);
    if (R >= end) {
      const int seq = seq_of(A, t, lane);
      if (seq < 0) continue;
      S = attn_span<true>(A, seq);
      end = (long long)min(A.q_offsets[seq + 1], A.n_q) * A.heads;
      const int chunk = attn_chunk(A, S.nk, A.unit);
      used = max(1, (int)(((long long)S.nk + chunk - 1) / chunk)) * A.streams;
    }
    if (t - S.q0 >= S.nq) continue;              // left out
    float mm = -INFINITY;                        // the row's maximum
    for (int c = lane; c < used; c += 32) mm = fmaxf(mm, A.part_ml[c * stride + R].x);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) mm = fmaxf(mm, __shfl_xor_sync(0xFFFFFFFFu, mm, d));
    const float base = mm == -INFINITY ? 0.f : mm;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float ll = 0.f;
    const int c4 = lane * 4;
    const bool on = c4 < A.dim;
    for (int c0 = first; c0 < used; c0 += U * W) {
      float2 ml[U];
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * W;
        const bool in = c < used;
        ml[u] = in ? A.part_ml[c * stride + R] : make_float2(-INFINITY, 0.f);
        x[u] = in && on ? *reinterpret_cast<const float4*>(A.part_o + (c * stride + R) * A.dim + c4)
                        : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = exp2f(ml[u].x - base);
        ll = fmaf(f, ml[u].y, ll);
        acc.x = fmaf(f, x[u].x, acc.x);
        acc.y = fmaf(f, x[u].y, acc.y);
        acc.z = fmaf(f, x[u].z, acc.z);
        acc.w = fmaf(f, x[u].w, acc.w);
      }
    }
    if (W > 1) {
      sum_o[w][lane] = acc;
      if (lane == 0) sum_ml[w] = make_float2(0.f, ll);
      __syncthreads();
      if (w == 0) {
#pragma unroll
        for (int v = 1; v < W; ++v) {
          const float4 y = sum_o[v][lane];
          acc.x += y.x;
          acc.y += y.y;
          acc.z += y.z;
          acc.w += y.w;
          ll += sum_ml[v].y;
        }
      }
    }
    if (W == 1 || w == 0) {
      const int h = (int)(R - (long long)t * A.heads);
      if (on) store_row<T>(A, t, h, c4, acc, mm, ll);
    }
    if (W > 1) __syncthreads();                  // before the next row's sums
  }
}

template <typename T, int DP, bool CLUSTER, bool WIN>
cudaError_t launch_rows_t(const AttnArgs& a, cudaStream_t st) {
  using C = RowsCfg<DP>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(k_attn_rows<T, DP, CLUSTER, WIN>), C::kSmem, &allowed, CLUSTER && kCluster > 8);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)((long long)a.n_seqs * a.kv_heads * a.row_groups * a.n_chunks));
  lc.blockDim = dim3(kWarps * 32);
  lc.dynamicSmemBytes = C::kSmem;
  lc.stream = st;
  cudaLaunchAttribute at[1];
  if (CLUSTER) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = a.n_chunks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&lc, k_attn_rows<T, DP, CLUSTER, WIN>, a);
}

}  // namespace

int attn_rows_unit(int dim) { return kWarps * (dim <= 64 ? RowsCfg<64>::KT : RowsCfg<128>::KT); }
int attn_rows_per_block() { return kRows; }
int attn_rows_cluster() { return kCluster; }

template <bool CLUSTER, bool WIN>
static cudaError_t launch_rows(const AttnArgs& a, bool bf16, cudaStream_t st) {
  if (a.dim <= 64)
    return bf16 ? launch_rows_t<__nv_bfloat16, 64, CLUSTER, WIN>(a, st) : launch_rows_t<__half, 64, CLUSTER, WIN>(a, st);
  return bf16 ? launch_rows_t<__nv_bfloat16, 128, CLUSTER, WIN>(a, st) : launch_rows_t<__half, 128, CLUSTER, WIN>(a, st);
}
cudaError_t launch_attn_rows(const AttnArgs& a, bool bf16, cudaStream_t st) {
  if (a.window > 0) return a.cluster ? launch_rows<true, true>(a, bf16, st) : launch_rows<false, true>(a, bf16, st);
  return a.cluster ? launch_rows<true, false>(a, bf16, st) : launch_rows<false, false>(a, bf16, st);
}

cudaError_t launch_attn_join(const AttnArgs& a, bool bf16, cudaStream_t st) {
  const int parts = a.n_chunks * a.streams;
  const bool wide = parts > 8;
  const int takers = wide ? 1 : kJoinWarps;      // of a block
  const long long rows = (long long)a.n_q * a.heads;
  // no more blocks than are resident, each with several rows: 2,700 tokens of 12 heads, two
  // parts each, take 25 us in blocks of 4 rows.  With many parts a row is work enough.
  const long long most = (wide ? 64LL : 16LL) * sm_count();
  const long long want = (rows + takers - 1) / takers, blocks = want < most ? want : most;
  const long long per = (rows + blocks * takers - 1) / (blocks * takers);
  const dim3 grid((unsigned)((rows + per * takers - 1) / (per * takers))), block(kJoinWarps * 32);
  if (bf16) {
    const auto kern = wide ? k_attn_join<__nv_bfloat16, kJoinWarps, 8>
                      : parts > 2 ? k_attn_join<__nv_bfloat16, 1, 8> : k_attn_join<__nv_bfloat16, 1, 2>;
    return launch_pdl(kern, grid, block, 0, st, a, (int)per);
  }
  const auto kern = wide ? k_attn_join<__half, kJoinWarps, 8>
                    : parts > 2 ? k_attn_join<__half, 1, 8> : k_attn_join<__half, 1, 2>;
  return launch_pdl(kern, grid, block, 0, st, a, (int)per);
}

}  // namespace rtcc
