// Attention of a few rows over pages of 8-bit keys and values, and the widening of
// pages to 16 bits for the tensor-core kernel of many rows.
//
// The formula is attn_rows.cu's, with k = 2^e_k k8 and v = 2^e_v v8: e4m3 numbers and an
// exponent for every 16 places of a page and key head.  e4m3 numbers are fp16 numbers, so
// both products run on them exactly (mma.m16n8k16 fp16, float32 sums), for queries of
// either type, and the exponents go where they cost least: e_k into the factor of the
// scores x (in log2), e_v into the values' weights 2^(x - m + e_v), m the scores' running
// maximum.  The weights have a running maximum of their own, as a difference from m:
// large values that hardly count, as of a key with a low score, do not press the others'
// weights out of fp16's range, and large scores, whose float32 steps are whole numbers
// from 2^24 on, do not round the exponents away.  bf16 queries
// are scaled by a power of two per row so that the largest is below 2^15; what is more
// than 2^39 below it is lost.  Weights are rounded to fp16's 11 bits, seven more than the
// values have; the largest is 2^15 to 2^16, so that 2^-40 of it still counts.
//
// Keys and channels are the products' 16-wide side, query rows the 8-wide one,
//   S^T = K Q^T,   O^T = V^T P^T,
// so that a block with up to 8 (token, head) rows of a key head pays for 8; with more it
// has two such groups for each widened number.  What bounds it is instructions, not
// bytes alone: 4 KB of keys and values are 64 conversions, 32 shuffled bytes, 16 products
// of 16 x 8 x 16 and the softmax of 4 numbers a lane.  As in attn_rows.cu the block's
// four warps take tiles of 32 keys in turn through rings of their own, and rows of the
// memory that no query sees are not read.  A tile lies in one page, whose number is
// fetched a round ahead of the copies.  Channels are permuted within groups of 16 so
// that what ldmatrix gives a lane (4 bytes of a key; 2 bytes of two keys' values) is
// what its products need: no number crosses lanes but P, transposed once.
//
// Measured: 61 tokens over ragged histories of up to 16,384 keys, 8 key heads of 128 with
// a cap, 958 MB: 162 us, 5.9 TB/s, 87 % of a plain copy's (rows on the 16-wide side, with
// probabilities as two terms: 268 us; the weights' maximum relative to the scores': 1 %);
// one token over 4097 keys of 6 heads of 64: 7.3 us.
#include <type_traits>

#include "attn_rows.cuh"
#include "kernels.h"
#include "pages.cuh"

namespace rtcc {
namespace {

constexpr int KT = 32;                           // keys of a tile

template <int DP> struct PagesCfg {              // DP: head size padded to 64 or 128
  static constexpr int kStages = DP == 64 ? 4 : 2;
  static constexpr int kTileBytes = KT * DP;
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  static constexpr int kNotes = kWarps * kStages * 8;        // per stage: exponents, keys that may be read
  static constexpr int kSmem = kRing + kNotes;
  static_assert((kWarps + 1) * kRows * (DP + 4) * 4 <= kRing, "states at the end lie in the ring");
};

__device__ __forceinline__ void cp4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp16z(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

// Byte offset of 16-byte unit c of row r in a tile of DP-byte rows; units are permuted
// within 128-byte lines so that ldmatrix reads 8 rows without bank conflicts.
template <int DP>
__device__ __forceinline__ uint32_t tile8_off(int r, int c) {
  if (DP == 128) return (uint32_t)(r * 128 + ((c ^ (r & 7)) * 16));
  return (uint32_t)((r >> 1) * 128 + ((((r & 1) * 4 + c) ^ ((r >> 1) & 3)) * 16));
}

// Transposes an 8 x 8 matrix of 16-bit numbers, two of a row per lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// The whole power of two that a row's results are in units of, above 2^m, where h is its
// largest weight (log2): weights of at most 2^(16 - 1/256), below fp16's largest number.
__device__ __forceinline__ float weight_unit(float h) { return h == -INFINITY ? 0.f : ceilf(h + 0x1p-8f) - 16.0f; }

// NR: groups of 8 rows of a block.
template <typename T, int DP, int NR, bool CLUSTER>
__global__ void __launch_bounds__(kWarps * 32, NR == 1 ? 3 : 2)
    k_attn_pages(const __grid_constant__ AttnArgs A, const __grid_constant__ PagesArgs P) {
  using C = PagesCfg<DP>;
  constexpr int kStages = C::kStages;
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
  const AttnSpan S = attn_span<true>(A, seq);
  const int rows_all = S.nq * A.group;
  const int per = attn_chunk(A, S.nk, A.unit);
  const int c0 = (int)min((long long)per * chunk, (long long)S.nk), c1 = min(S.nk - c0, per) + c0;
  if (!CLUSTER && chunk > 0 && c0 >= S.nk) return;   // not in use; chunk 0 always answers
  const uint32_t ring = smem_u32(smem) + w * kStages * C::kStageBytes;
  const uint32_t notes = smem_u32(smem) + C::kRing + w * kStages * 8;
  uint32_t* notes_g = reinterpret_cast<uint32_t*>(smem + C::kRing + w * kStages * 8);
  const int* table = P.table + (long long)seq * P.s.table_row;
  const long long head_at = (long long)kvh * P.s.page_rows * A.dim;
  const long long scale_at = (long long)kvh * (P.s.page_rows / kPageBlock) * 2;

  for (int rg = rg0; (long long)rg * kRows < rows_all; rg += A.row_groups) {
    const int r0 = rg * kRows;
    // B fragments of Q: this lane's row is lane / 4 of a group, and step s has channels
    // 16 s + 4 (lane % 4) + {0, 1 | 2, 3}
    uint32_t qb[NR][DP / 16][2];
    float qscale[NR];                            // what the row's scores are multiplied by
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int r = r0 + i * 8 + lane / 4;
      const bool row_ok = r < rows_all;
      uint2 x[DP / 16];
      const T* q = static_cast<const T*>(A.q);
      if (row_ok) q += (long long)(S.q0 + r / A.group) * A.q_row + (long long)(kvh * A.group + r % A.group) * A.q_head;
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        const int col = s * 16 + (lane % 4) * 4;
        x[s] = row_ok && col < A.dim ? *reinterpret_cast<const uint2*>(q + col) : make_uint2(0u, 0u);
      }
      qscale[i] = A.scale_log2;
      if (std::is_same<T, __nv_bfloat16>::value) {
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          const float2 f = Store<T>::unpack2(x[s].x), g = Store<T>::unpack2(x[s].y);
          const float v[4] = {fabsf(f.x), fabsf(f.y), fabsf(g.x), fabsf(g.y)};
#pragma unroll
          for (int k = 0; k < 4; ++k) top = fmaxf(top, v[k] < INFINITY ? v[k] : 0.f);
        }
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const int e = max((int)(__float_as_uint(top) >> 23) - 127 - 14, -110);   // top 2^-e in [2^14, 2^15)
        const float down = pow2(-e);
        qscale[i] *= pow2(e);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          const float2 f = Store<T>::unpack2(x[s].x), g = Store<T>::unpack2(x[s].y);
          qb[i][s][0] = Store<__half>::pack2(f.x * down, f.y * down);
          qb[i][s][1] = Store<__half>::pack2(g.x * down, g.y * down);
        }
      } else {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          qb[i][s][0] = x[s].x;
          qb[i][s][1] = x[s].y;
        }
      }
    }
    // of scores and results a lane has two rows of each group: 2 (lane % 4) and the next
    constexpr int N = 2 * NR;
    int hi[N];
    AttnView view[N];
    float qs[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + (i >> 1) * 8 + (lane & 3) * 2 + (i & 1);
      const int ql = r < rows_all ? r / A.group : 0;
      hi[i] = r < rows_all ? attn_visible(A, S, S.first, ql) : 0;
      view[i] = attn_view(A, S, S.first, ql);
      qs[i] = __shfl_sync(0xFFFFFFFFu, qscale[i >> 1], ((lane & 3) * 2 + (i & 1)) * 4);
    }
    // the rows' reach, and what some or all of them see of keys behind their windows
    const int ql0 = r0 / A.group, ql1 = (min(r0 + 8 * NR, rows_all) - 1) / A.group;
    const int end = min(c1, attn_visible(A, S, S.first, ql1)), least = attn_visible(A, S, S.first, ql0);
    const AttnView first = attn_view(A, S, S.first, ql0), last = attn_view(A, S, S.first, ql1);
    float o[NR][DP / 16][4];                     // channels 16 u + 2 (lane / 4) + {0, 1} of two rows: 00 01 10 11
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int u = 0; u < DP / 16; ++u) o[i][u][0] = o[i][u][1] = o[i][u][2] = o[i][u][3] = 0.f;
    float m[N], l[N];                            // of the scores
    float wt[N];                                 // largest weight (log2, from m): o is in units of 2^(m + weight_unit)
#pragma unroll
    for (int i = 0; i < N; ++i) m[i] = wt[i] = -INFINITY, l[i] = 0.f;

    const int n_tiles = end > c0 ? (end - c0 + KT - 1) / KT : 0;
    auto page_of = [&](int t) -> int {           // of tile t, -1: none
      if (t >= n_tiles) return -1;
      const int page = table[attn_row(S, c0 + t * KT) >> P.s.shift];
      return (unsigned)page < (unsigned)P.s.n_pages ? page : -1;
    };
    constexpr int U = DP / 16;                   // 16-byte units of a row
    const int lr = lane / U, lc = lane % U;      // this lane's first unit of a tile
    auto load = [&](int t, int stage, int page) {
      const int j = c0 + t * KT + lane;
      const bool ok = page >= 0 && j < end && (j < last.seen || j >= first.low);
      const unsigned bits = __ballot_sync(0xFFFFFFFFu, ok);
      if (bits) {
        const uint32_t ks = ring + stage * C::kStageBytes, vs = ks + C::kTileBytes;
        const int row = attn_row(S, c0 + t * KT) & (P.s.page_rows - 1);
        const long long at = page * P.s.page_bytes + head_at + (long long)row * A.dim;
        if (bits == 0xFFFFFFFFu && A.dim == DP) {
          const unsigned char *kg = P.k + at + lane * 16, *vg = P.v + at + lane * 16;
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const uint32_t to = tile8_off<DP>(i * (32 / U) + lr, lc);
            cp16z(ks + to, kg + i * 512, true);
            cp16z(vs + to, vg + i * 512, true);
          }
        } else {
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int r = i * (32 / U) + lr;
            const bool live = (bits >> r) & 1 && lc * 16 < A.dim;
            const int off = live ? r * A.dim + lc * 16 : 0;
            const uint32_t to = tile8_off<DP>(r, lc);
            cp16z(ks + to, P.k + at + off, live);
            cp16z(vs + to, P.v + at + off, live);
          }
        }
        if (lane == 0)
          cp4(notes + stage * 8, P.scales + page * P.s.scale_bytes + scale_at + (row / kPageBlock) * 2);
      }
      if (lane == 0) notes_g[stage * 2 + 1] = bits;
      cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) load(w + s * kWarps, s, page_of(w + s * kWarps));
    int page = page_of(w + (kStages - 1) * kWarps);
    int stage = 0;
    for (int t = w; t < n_tiles; t += kWarps) {
      load(t + (kStages - 1) * kWarps, (stage + kStages - 1) % kStages, page);
      cp_async_wait<kStages - 1>();
      __syncwarp();
      page = page_of(t + kStages * kWarps);
      const unsigned bits = notes_g[stage * 2 + 1];
      if (bits) {
        const uint32_t ks = ring + stage * C::kStageBytes, vs = ks + C::kTileBytes;
        const uint32_t exps = notes_g[stage * 2];
        float s[NR][KT / 16][4];                 // keys lane / 4 and 8 further of 16, two rows: 00 01 10 11
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int n = 0; n < KT / 16; ++n) s[i][n][0] = s[i][n][1] = s[i][n][2] = s[i][n][3] = 0.f;
#pragma unroll
        for (int u = 0; u < DP / 16; u += 2)     // 32 channels: two k16 steps, one ldmatrix.x4 per 16 keys
#pragma unroll
          for (int n = 0; n < KT / 16; ++n) {
            uint32_t k4[4];                      // keys of unit u, 8 further, of unit u + 1, 8 further
            ldm4(ks + tile8_off<DP>(n * 16 + (lane & 15), u + (lane >> 4)), k4);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t a[4] = {widen_e4m3x2(k4[2 * h]), widen_e4m3x2(k4[2 * h + 1]), widen_e4m3x2(k4[2 * h] >> 16),
                                     widen_e4m3x2(k4[2 * h + 1] >> 16)};
#pragma unroll
              for (int i = 0; i < NR; ++i) mma16816<__half>(s[i][n], a, qb[i][u + h][0], qb[i][u + h][1]);
            }
          }
        const int j0 = c0 + t * KT;
        const bool edge = bits != 0xFFFFFFFFu || j0 + KT > least || (j0 < last.low && j0 + KT > first.seen);
        float top[N][KT / 16];                   // largest score of each exponent's keys
        float ve[KT / 16];
#pragma unroll
        for (int n = 0; n < KT / 16; ++n) {
          const float ke = pow2(max((int)(signed char)(exps >> (n * 16)), kExpMin));
          ve[n] = (float)(signed char)(exps >> (n * 16 + 8));
#pragma unroll
          for (int i = 0; i < N; ++i) {
            // finite: a score of 0 stays 0 whatever the factor
            const float f = fminf(fmaxf(qs[i] * ke, -3e38f), 3e38f);
            float t = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& y = s[i >> 1][n][2 * h + (i & 1)];
              float x = y * f;
              if (A.cap_log2 > 0.f) x = A.cap_log2 * tanh_rel(x);      // few keys' lse is a score: to 2^-20 of itself
              if (edge) {
                const int key = n * 16 + h * 8 + lane / 4, j = j0 + key;
                if (!((bits >> key) & 1) || j >= hi[i] || (j >= view[i].seen && j < view[i].low)) x = -INFINITY;
              }
              y = x;
              t = fmaxf(t, x);
            }
            top[i][n] = t;
          }
        }
        bool moved = false;
        float base[N], unit[N], f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float mn = m[i];
#pragma unroll
          for (int n = 0; n < KT / 16; ++n) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top[i][n] = fmaxf(top[i][n], __shfl_xor_sync(0xFFFFFFFFu, top[i][n], d));
            mn = fmaxf(mn, top[i][n]);
          }
          base[i] = mn == -INFINITY ? 0.f : mn;
          const float fall = m[i] - base[i];     // m = -inf: -inf
          float h = wt[i] + fall;
#pragma unroll
          for (int n = 0; n < KT / 16; ++n) h = fmaxf(h, (top[i][n] - base[i]) + ve[n]);
          unit[i] = weight_unit(h);
          l[i] *= exp2f(fall);
          f[i] = ex2(fall + (weight_unit(wt[i]) - unit[i]));
          moved = moved || f[i] != 1.0f;
          m[i] = mn;
          wt[i] = h;
        }
        if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
          for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int u = 0; u < DP / 16; ++u) {
              o[i][u][0] *= f[2 * i];
              o[i][u][1] *= f[2 * i + 1];
              o[i][u][2] *= f[2 * i];
              o[i][u][3] *= f[2 * i + 1];
            }
        }
        uint32_t pb[NR][KT / 16][2];             // B fragments of the weights, transposed
        float sum[N];                            // a tile's sum first, as in attn_rows.cu
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.f;
#pragma unroll
        for (int n = 0; n < KT / 16; ++n) {
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            const float w0 = ve[n] - unit[2 * i], w1 = ve[n] - unit[2 * i + 1];      // whole numbers
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float x0 = s[i][n][2 * h] - base[2 * i], x1 = s[i][n][2 * h + 1] - base[2 * i + 1];
              sum[2 * i] += exp2f(x0);
              sum[2 * i + 1] += exp2f(x1);
              pb[i][n][h] = transpose8(Store<__half>::pack2(ex2(x0 + w0), ex2(x1 + w1)));
            }
          }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) l[i] += sum[i];
#pragma unroll
        for (int n = 0; n < KT / 16; ++n)
#pragma unroll
          for (int u = 0; u < DP / 16; u += 2) {
            uint32_t v4[4];                      // units u, u + 1: keys 2c, 2c + 1 and 8 further, channels 2g, 2g + 1
            ldm4t(vs + tile8_off<DP>(n * 16 + (lane & 15), u + (lane >> 4)), v4);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t even = __byte_perm(v4[2 * h], v4[2 * h + 1], 0x6420);
              const uint32_t odd = __byte_perm(v4[2 * h], v4[2 * h + 1], 0x7531);
              const uint32_t a[4] = {widen_e4m3x2(even), widen_e4m3x2(odd), widen_e4m3x2(even >> 16), widen_e4m3x2(odd >> 16)};
#pragma unroll
              for (int i = 0; i < NR; ++i) mma16816<__half>(o[i][u + h], a, pb[i][n][0], pb[i][n][1]);
            }
          }
      }
      __syncwarp();                              // the tile is done with: the next round's copies take its place
      stage = (stage + 1) % kStages;
    }
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 4);
      l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 8);
      l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 16);
    }
    // the states leave in units of the scores' maximum
    __syncthreads();
    float* state = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float back = wt[i] == -INFINITY ? 0.f : exp2f(weight_unit(wt[i]));
      float* dst = state + (w * kRows + (i >> 1) * 8 + (lane & 3) * 2 + (i & 1)) * (DP + 4);
#pragma unroll
      for (int u = 0; u < DP / 16; ++u)
        *reinterpret_cast<float2*>(dst + u * 16 + (lane / 4) * 2) =
            make_float2(o[i >> 1][u][i & 1] * back, o[i >> 1][u][2 + (i & 1)] * back);
      if (lane / 4 == 0) {
        dst[DP] = m[i];
        dst[DP + 1] = l[i];
      }
    }
    merge_states<T, DP, CLUSTER>(A, S, state, r0, rows_all, kvh, chunk);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// widening
// ---------------------------------------------------------------------------

template <typename T> __device__ __forceinline__ float in_range(float x) { return x; }
template <> __device__ __forceinline__ float in_range<__half>(float x) {
  return fabsf(x) > 65504.f ? copysignf(65504.f, x) : x;     // NaN stays
}

constexpr int kWidenThreads = 256;

// Keys and values that a sequence's tokens see, as 16-bit rows [key without the gap]
// [kv_heads][dim] from row seq * span on: a warp per 16 keys and key head.  bf16 holds the
// numbers exactly, and fp16 those that came from fp16.  Read once by each of the
// tensor-core kernel's blocks along the tokens, which would convert them as often: 19 us
// before its 297 for 5 chunks of up to 2100 tokens over windows of 4000 keys.
template <typename T>
__global__ void __launch_bounds__(kWidenThreads)
    k_pages_widen(const __grid_constant__ AttnArgs A, const __grid_constant__ PagesArgs P, T* k, T* v,
                  unsigned char* hidden, int span) {
  const int lane = threadIdx.x & 31;
  const unsigned item = blockIdx.x * (kWidenThreads / 32) + (threadIdx.x >> 5);
  const int head = (int)(item % (unsigned)A.kv_heads), j0 = (int)(item / (unsigned)A.kv_heads) * kPageBlock;
  if (j0 >= span) return;
  for (int seq = blockIdx.y; seq < A.n_seqs; seq += gridDim.y) {
    const AttnSpan S = attn_span<true>(A, seq);
    if (S.nq == 0 || j0 >= S.nk) continue;
    auto page_at = [&](int j) -> int {
      const int page = P.table[(long long)seq * P.s.table_row + (attn_row(S, j) >> P.s.shift)];
      return (unsigned)page < (unsigned)P.s.n_pages ? page : -1;
    };
    const int page = page_at(j0);
    if (head == 0 && lane == 0 && j0 % 64 == 0)
      hidden[((long long)seq * span + j0) / 64] =
          (unsigned char)((page < 0) | (j0 + 32 < S.nk && page_at(j0 + 32) < 0 ? 2 : 0));
    if (page < 0) continue;
    const int row = attn_row(S, j0) & (P.s.page_rows - 1);
    const long long at = page * P.s.page_bytes + ((long long)head * P.s.page_rows + row) * A.dim;
    const char2 e = *reinterpret_cast<const char2*>(P.scales + page * P.s.scale_bytes +
                                                   ((long long)head * (P.s.page_rows / kPageBlock) + row / kPageBlock) * 2);
    const int units = A.dim / 16, all = kPageBlock * units;          // 16-byte units of a row, of the block
    constexpr int N = 4;                         // of a lane at most
    uint4 x[2][N];                               // all loads first
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = n * 32 + lane;
      if (i < all) {
        x[0][n] = __ldcs(reinterpret_cast<const uint4*>(P.k + at) + i);
        x[1][n] = __ldcs(reinterpret_cast<const uint4*>(P.v + at) + i);
      }
    }
    const float f[2] = {pow2(max((int)e.x, kExpMin)), pow2(max((int)e.y, kExpMin))};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = n * 32 + lane, r = i / units, c = i % units;
      if (i >= all) continue;
      const long long to = (((long long)seq * span + j0 + r) * A.kv_heads + head) * A.dim + c * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t u[4] = {x[h][n].x, x[h][n].y, x[h][n].z, x[h][n].w};
        uint32_t y[8];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const float2 p = Store<__half>::unpack2(widen_e4m3x2(u[m])), q = Store<__half>::unpack2(widen_e4m3x2(u[m] >> 16));
          y[2 * m] = Store<T>::pack2(in_range<T>(p.x * f[h]), in_range<T>(p.y * f[h]));
          y[2 * m + 1] = Store<T>::pack2(in_range<T>(q.x * f[h]), in_range<T>(q.y * f[h]));
        }
        uint4* dst = reinterpret_cast<uint4*>((h ? v : k) + to);
        dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
        dst[1] = make_uint4(y[4], y[5], y[6], y[7]);
      }
    }
  }
}

template <typename T, int DP, int NR, bool CLUSTER>
cudaError_t launch_pages_t(const AttnArgs& a, const PagesArgs& p, cudaStream_t st) {
  using C = PagesCfg<DP>;
  const auto kern = k_attn_pages<T, DP, NR, CLUSTER>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), C::kSmem, &allowed, CLUSTER && kCluster > 8);
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
  return cudaLaunchKernelEx(&lc, kern, a, p);
}

template <int DP, int NR, bool CLUSTER>
cudaError_t launch_pages(const AttnArgs& a, const PagesArgs& p, bool bf16, cudaStream_t st) {
  return bf16 ? launch_pages_t<__nv_bfloat16, DP, NR, CLUSTER>(a, p, st) : launch_pages_t<__half, DP, NR, CLUSTER>(a, p, st);
}
template <int DP, bool CLUSTER>
cudaError_t launch_pages(const AttnArgs& a, const PagesArgs& p, bool bf16, cudaStream_t st) {
  return (long long)a.most_q * a.group <= 8 ? launch_pages<DP, 1, CLUSTER>(a, p, bf16, st)
                                            : launch_pages<DP, 2, CLUSTER>(a, p, bf16, st);
}
template <bool CLUSTER>
cudaError_t launch_pages(const AttnArgs& a, const PagesArgs& p, bool bf16, cudaStream_t st) {
  return a.dim <= 64 ? launch_pages<64, CLUSTER>(a, p, bf16, st) : launch_pages<128, CLUSTER>(a, p, bf16, st);
}

}  // namespace

int attn_pages_unit() { return kWarps * KT; }

cudaError_t launch_attn_pages(const AttnArgs& a, const PagesArgs& p, bool bf16, cudaStream_t st) {
  return a.cluster ? launch_pages<true>(a, p, bf16, st) : launch_pages<false>(a, p, bf16, st);
}

cudaError_t launch_pages_widen(const AttnArgs& a, const PagesArgs& p, void* k, void* v, unsigned char* hidden, int span,
                               bool bf16, cudaStream_t st) {
  const long long warps = (long long)(span / kPageBlock) * a.kv_heads;
  if (warps > 0x7FFFFFFF) return cudaErrorNotSupported;
  const dim3 grid((unsigned)((warps + kWidenThreads / 32 - 1) / (kWidenThreads / 32)),
                  (unsigned)(a.n_seqs < 65535 ? a.n_seqs : 65535));
  if (bf16)
    k_pages_widen<__nv_bfloat16><<<grid, kWidenThreads, 0, st>>>(a, p, static_cast<__nv_bfloat16*>(k),
                                                               static_cast<__nv_bfloat16*>(v), hidden, span);
  else
    k_pages_widen<__half><<<grid, kWidenThreads, 0, st>>>(a, p, static_cast<__half*>(k), static_cast<__half*>(v), hidden,
                                                        span);
  return cudaGetLastError();
}

}  // namespace rtcc
