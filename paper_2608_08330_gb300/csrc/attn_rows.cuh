// Shared by the attention kernels for few rows (16-bit rows, pages): copies, matrix
// instructions, and the merge of the warps' and the cluster's results.
#pragma once

#include <type_traits>

#include "attn.cuh"

namespace rtcc {
namespace {

constexpr int kWarps = 4;
constexpr int kRows = 16;
constexpr int kCluster = 16;                     // blocks of a cluster at most

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp8(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(live ? 8 : 0) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}

template <typename T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Shared memory of the cluster's blocks.
__device__ __forceinline__ float4 cluster_ld4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(a)
               : "memory");
  return v;
}
__device__ __forceinline__ float2 cluster_ld2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}

// Two floats as hi + lo of the storage type.
template <typename T>
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = Store<T>::pack2(a, b);
  const float2 h = Store<T>::unpack2(hi);
  lo = Store<T>::pack2(a - h.x, b - h.y);
}

// Four channels of a row's result: accumulators over the sum, and the lse.
template <typename T>
__device__ __forceinline__ void store_row(const AttnArgs& A, long long t, int h, int c, float4 acc, float mm, float ll) {
  const float inv = ll > 0.f ? 1.0f / ll : (ll == 0.f ? 0.f : ll);
  uint2 u;
  u.x = Store<T>::pack2(acc.x * inv, acc.y * inv);
  u.y = Store<T>::pack2(acc.z * inv, acc.w * inv);
  *reinterpret_cast<uint2*>(static_cast<T*>(A.out) + t * A.out_row + (long long)h * A.out_head + c) = u;
  if (c == 0 && A.lse) A.lse[t * A.heads + h] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * kLn2;
}

// The warps' states, [warp][row][DP + 4] (accumulator, maximum, sum) at mo, merged into
// the 16 rows from r0 on: into out and lse, the chunk's partial results, or, for a
// cluster, the block's state behind the warps', which its blocks then join.  All threads.
template <typename T, int DP, bool CLUSTER>
__device__ __forceinline__ void merge_states(const AttnArgs& A, const AttnSpan& S, float* mo, int r0, int rows_all, int kvh,
                                             int chunk) {
  constexpr int P = DP + 4, kState = kRows * P;
  __syncthreads();
  for (int idx = threadIdx.x; idx < kRows * (DP / 4); idx += kWarps * 32) {
    const int r = idx / (DP / 4), c = (idx % (DP / 4)) * 4;
    if (r0 + r >= rows_all) continue;
    float mm = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) mm = fmaxf(mm, mo[(i * kRows + r) * P + DP]);
    const float base = mm == -INFINITY ? 0.f : mm;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float ll = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float* src = mo + (i * kRows + r) * P;
      const float f = exp2f(src[DP] - base);
      const float4 x = *reinterpret_cast<const float4*>(src + c);
      acc.x = fmaf(f, x.x, acc.x);
      acc.y = fmaf(f, x.y, acc.y);
      acc.z = fmaf(f, x.z, acc.z);
      acc.w = fmaf(f, x.w, acc.w);
      ll = fmaf(f, src[DP + 1], ll);
    }
    if (c >= A.dim) continue;
    const long long t = S.q0 + (r0 + r) / A.group;
    const int h = kvh * A.group + (r0 + r) % A.group;
    const long long R = t * A.heads + h;
    if (CLUSTER) {
      float* dst = mo + kWarps * kState + r * P;
      *reinterpret_cast<float4*>(dst + c) = acc;
      if (c == 0) *reinterpret_cast<float2*>(dst + DP) = make_float2(mm, ll);
    } else if (A.n_chunks > 1) {
      const long long at = (long long)chunk * A.n_q * A.heads + R;
      *reinterpret_cast<float4*>(A.part_o + at * A.dim + c) = acc;
      if (c == 0) A.part_ml[at] = make_float2(mm, ll);
    } else {
      store_row<T>(A, t, h, c, acc, mm, ll);
    }
  }
  if (CLUSTER) {
    // every block joins its share of the rows, from the blocks' states in chunk order
    __syncwarp();
    cluster_sync_all();
    const uint32_t state = smem_u32(mo + kWarps * kState);
    const int blocks = (int)cluster_nctarank();
    for (int idx = chunk * kWarps * 32 + threadIdx.x; idx < kRows * (DP / 4); idx += A.n_chunks * kWarps * 32) {
      const int r = idx / (DP / 4), c = (idx % (DP / 4)) * 4;
      if (r0 + r >= rows_all || c >= A.dim) continue;
      float2 ml[kCluster];
      float4 x[kCluster];
      float mm = -INFINITY;
#pragma unroll
      for (int i = 0; i < kCluster; ++i) {
        const bool in = i < blocks;
        const uint32_t at = mapa_shared(state + r * P * 4, in ? i : 0);
        ml[i] = in ? cluster_ld2(at + DP * 4) : make_float2(-INFINITY, 0.f);
        x[i] = in ? cluster_ld4(at + c * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < kCluster; ++i) mm = fmaxf(mm, ml[i].x);
      const float base = mm == -INFINITY ? 0.f : mm;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float ll = 0.f;
#pragma unroll
      for (int i = 0; i < kCluster; ++i) {
        const float f = exp2f(ml[i].x - base);
        acc.x = fmaf(f, x[i].x, acc.x);
        acc.y = fmaf(f, x[i].y, acc.y);
        acc.z = fmaf(f, x[i].z, acc.z);
        acc.w = fmaf(f, x[i].w, acc.w);
        ll = fmaf(f, ml[i].y, ll);
      }
      const long long t = S.q0 + (r0 + r) / A.group;
      const int h = kvh * A.group + (r0 + r) % A.group;
      store_row<T>(A, t, h, c, acc, mm, ll);
    }
    __syncwarp();
    cluster_sync_all();                        // before a block's state goes
  }
}

}  // namespace
}  // namespace rtcc
