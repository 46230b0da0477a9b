// Attention of many rows over the token memory on the 5th-generation tensor
// cores (the formula is in attn_rows.cu).
//
// A block has two tiles of up to 128 rows and one key head; the query heads
// that share it are rows of the same tile (row r: token r / group, head
// r % group), so keys and values are read once for all of them.  Per 128 keys
// and tile:  S = Q K^T (128 x 128 floats in tensor memory), the softmax warps
// turn S into P = exp2(x - m), rounded to the storage type and written over S in
// tensor memory, and O += P V takes P from there.  The softmax goes by halves of
// 64 keys, which keeps a row's scores in registers, and the product of the first
// half starts while the second is still at work.  While one tile's softmax
// runs, the tensor pipe works for the other tile.  S and O of both tiles fill
// tensor memory: 2 x 128 + 2 x head size columns of 512.
//
// Roles: warps 0-3 softmax and epilogue of tile 0, warps 4-7 of tile 1 (a thread
// owns a row: no shuffles), warp 8 loads (TMA, one thread), warp 9 issues the
// products (one thread).  Keys and values share one ring of 128-row slots in the
// order they are used: K0 V0 K1 V1 ...
//
// The running maximum m moves only when a row's new maximum exceeds it by more
// than 2^8 in P (kSlack): P stays below 2^8, far inside either storage type's
// range, and O is rescaled rarely, by the softmax threads themselves.
//
// Key rows nobody may see (past the span, in an absent slot) are skipped as
// whole tiles; in a tile at the edge their scores are replaced, not added to,
// and their value rows are zeroed in shared memory before the product, so their
// contents never reach a result.
#include <type_traits>

#include "attn.cuh"
#include "kernels.h"

namespace rtcc {
namespace {

constexpr int kThreads = 320;
constexpr int kKeys = 128;                       // keys per tile
constexpr int kHalf = 64;                        // keys per softmax step
constexpr int kChunkBytes = 128 * 128;           // 128 rows x 64 channels
constexpr float kSlack = 8.0f;

__device__ int g_attn_err;                       // bit b: a wait on barrier b ran out

template <int DP> struct TcCfg {
  static constexpr int NC = DP / 64;             // 64-channel chunks (one 128-byte swizzle line each)
  static constexpr int kTile = NC * kChunkBytes;
  static constexpr int kSlots = DP == 64 ? 8 : 4;
  static constexpr int kQ = 2 * kTile;
  static constexpr int kPos = 8 * 2 * 2 * kKeys * 4;        // [softmax warp][buffer][y | x][128]
  static constexpr int kSmem = kQ + kSlots * kTile + kPos + 1024;
};

struct TcMaps {
  CUtensorMap q, k, v;
};

// coefficients of cap tanh(x scale / cap) log2(e) = x (c0 + w (c1 + w (c2 + w c3))), w = x^2
struct TanhPoly {
  float c[4];
};

// Each half of P has a barrier of its own (BAR_PREADY + 2 w + h): a softmax warp
// may finish both halves before the first is waited for, and one barrier's
// parity would then have come round.
enum : int { BAR_QFULL, BAR_QFREE, BAR_SFULL, BAR_PREADY = BAR_SFULL + 2, BAR_ODONE = BAR_PREADY + 4,
             BAR_HALF = BAR_ODONE + 2, BAR_FULL = BAR_HALF + 2, BAR_EMPTY = BAR_FULL + 8, BAR_DRAIN = BAR_EMPTY + 8, BAR_N };

__device__ __forceinline__ void tmem_ld32_issue(uint32_t a, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32"
      " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22,"
      " %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(a));
}
// Ties 32 loaded registers to a point after tmem_ld_wait().
__device__ __forceinline__ void reg_fence32(float* x) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+f"(x[i]), "+f"(x[i + 1]), "+f"(x[i + 2]), "+f"(x[i + 3]), "+f"(x[i + 4]), "+f"(x[i + 5]),
                      "+f"(x[i + 6]), "+f"(x[i + 7]));
}
__device__ __forceinline__ void tmem_st32(uint32_t a, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0],"
      " {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23,"
      " %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(a),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D[tmem] (+)= A[tmem] * B[smem]: A is the 16-bit probabilities, two per column.
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
// Descriptor of V as the B operand [head size][keys], head size contiguous
// (MN-major): 64-channel lines of 128 bytes, 8 keys per 1024 bytes, the next 64
// channels a chunk further.
__device__ __forceinline__ uint64_t desc_v(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr >> 4) & 0x3FFFu);
  d |= static_cast<uint64_t>(kChunkBytes >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float tanh_abs(float u) {
  return 1.0f - __fdividef(2.0f, 1.0f + ex2(fminf(2.0f * kLog2e * u, 64.0f)));
}
// two floats at a time (one issue slot)
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
        "l"(reinterpret_cast<unsigned long long&>(c)));
  return r;
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// Slots that the rows [r0, r1] of the memory touch: first one and a mask of
// their number of bits.
__device__ __forceinline__ unsigned long long slot_bits(const AttnArgs& A, unsigned long long slots, int r0, int r1,
                                                        unsigned long long* want) {
  const int s0 = min(r0 / A.slot_rows, 63), s1 = min(r1 / A.slot_rows, 63);
  *want = ~0ull >> (63 - (s1 - s0));
  return (slots >> s0) & *want;
}

// A walk over the key tiles of a chunk that have a key in a present slot.  Every
// role walks; which tiles are skipped depends on the chunk's end c1 alone, so a
// tile that one role visits is visited by all that reach it.
struct Walk {
  int t, end_key, c1;                            // current tile; tiles that begin before end_key count
  __device__ __forceinline__ void settle(const AttnArgs& A, const AttnSpan& S, unsigned long long slots) {
    if (!A.present) return;
    while (t * kKeys < end_key) {
      unsigned long long want;
      if (slot_bits(A, slots, S.kb + t * kKeys, S.kb + min(t * kKeys + kKeys, c1) - 1, &want)) return;
      ++t;
    }
  }
  __device__ __forceinline__ bool live() const { return t * kKeys < end_key; }
};

// Bit c: key j0 + c, c < 64, lies before `lim` and in a present slot.
__device__ __forceinline__ unsigned long long key_mask(const AttnArgs& A, const AttnSpan& S, unsigned long long slots,
                                                       int j0, int lim) {
  const int n = min(max(lim - j0, 0), 64);
  if (n == 0) return 0;
  unsigned long long bits = ~0ull >> (64 - n);
  if (!A.present) return bits;
  const int r0 = S.kb + j0, s1 = min((r0 + n - 1) / A.slot_rows, 63);
  for (int s = min(r0 / A.slot_rows, 63); s <= s1; ++s) {
    if ((slots >> s) & 1) continue;
    const int a = (int)max((long long)s * A.slot_rows - r0, 0LL);
    const int b = (int)min((long long)(s + 1) * A.slot_rows - r0, 64LL);      // a < b
    bits &= ~((~0ull >> (64 - (b - a))) << a);
  }
  return bits;
}

template <typename T, int DP, bool CAP, bool DIST>
__global__ void __launch_bounds__(kThreads, 1)
    k_attn_tc(const __grid_constant__ AttnArgs A, const __grid_constant__ TcMaps M, const TanhPoly poly) {
  using C = TcCfg<DP>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bar[BAR_N];
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  unsigned char* sq = smem;
  unsigned char* ring = smem + C::kQ;
  float* spos = reinterpret_cast<float*>(ring + C::kSlots * C::kTile);

  // block -> (row group, chunk, key head, sequence); the last rows of a causal
  // sequence have the longest reach and go first
  int b = blockIdx.x;
  int rg0 = b % A.row_groups;
  b /= A.row_groups;
  const int chunk = b % A.n_chunks;
  b /= A.n_chunks;
  const int kvh = b % A.kv_heads;
  const int seq = b / A.kv_heads;
  const AttnSpan S = attn_span(A, seq);
  const int qpt = 128 / A.group;                 // tokens per tile
  const int groups = (S.nq + 2 * qpt - 1) / (2 * qpt);
  if (A.causal) rg0 = A.row_groups - 1 - rg0;
  const int per = attn_chunk(A, S.nk, kKeys);
  const int c0 = (int)min((long long)per * chunk, (long long)S.nk), c1 = min(S.nk - c0, per) + c0;
  if (rg0 >= groups || (chunk > 0 && c0 >= S.nk)) return;   // not in use; chunk 0 always answers

  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < BAR_N; ++i)
        if (i < BAR_PREADY || i >= BAR_PREADY + 4) mbar_init(&bar[i], 1);
      for (int i = 0; i < 4; ++i) mbar_init(&bar[BAR_PREADY + i], 4);
      fence_barrier_init();
      gave_up = 0;
      tma_prefetch_desc(&M.q);
      tma_prefetch_desc(&M.k);
      tma_prefetch_desc(&M.v);
    }
    __syncwarp();
  }
  if (warp == 9) {
    tmem_alloc(&tmem_base, 512);
    tmem_relinquish();
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  const unsigned long long slots = attn_slot_mask(A, lane);
  volatile int* stop = &gave_up;
  // a wait that runs out marks the block; every role then leaves its loops
  auto wait_one = [&](int i, uint32_t parity) -> bool {
    if (mbar_wait(&bar[i], parity)) return *stop == 0;
    *stop = 1;
    atomicOr(&g_attn_err, 1 << i);
    return false;
  };
  // the same by a whole warp, which goes on or leaves together
  auto wait = [&](int i, uint32_t parity) -> bool { return __all_sync(0xFFFFFFFFu, wait_one(i, parity)); };
  // keys that tile w of row group rg reaches within this chunk
  auto reach = [&](int rg, int w) -> int {
    const int i0 = (rg * 2 + w) * qpt;
    if (i0 >= S.nq) return c0;
    return max(c0, min(c1, attn_visible(A, S, min(i0 + qpt, S.nq) - 1)));
  };

  if (warp == 8) {
    // ---------------------------------------------------------------- loads
    if (lane == 0) {
      int slot = 0;
      uint32_t ph = 1, item = 0;                 // a fresh slot counts as empty
      long long issued = 0;
      bool ok = true;
      auto put = [&](const CUtensorMap* m, int row) {
        ok = wait_one(BAR_EMPTY + slot, ph);
        if (!ok) return;
        mbar_arrive_expect_tx(&bar[BAR_FULL + slot], C::kTile);
#pragma unroll
        for (int c = 0; c < C::NC; ++c)
          tma_load_3d(ring + slot * C::kTile + c * kChunkBytes, m, &bar[BAR_FULL + slot], c * 64, kvh, row);
        ++issued;
        if (++slot == C::kSlots) {
          slot = 0;
          ph ^= 1;
        }
      };
      for (int rg = rg0; rg < groups && ok; rg += A.row_groups, ++item) {
        if (item > 0 && !(ok = wait_one(BAR_QFREE, (item - 1) & 1))) break;
        mbar_arrive_expect_tx(&bar[BAR_QFULL], 2 * C::NC * qpt * A.group * 128);
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int c = 0; c < C::NC; ++c)
            tma_load_3d(sq + w * C::kTile + c * kChunkBytes, &M.q, &bar[BAR_QFULL], c * 64, kvh * A.group,
                        S.q0 + (rg * 2 + w) * qpt);
        Walk k{c0 / kKeys, max(reach(rg, 0), reach(rg, 1)), c1};
        for (k.settle(A, S, slots); k.live() && ok; ++k.t, k.settle(A, S, slots)) {
          put(&M.k, S.kb + k.t * kKeys);
          if (ok) put(&M.v, S.kb + k.t * kKeys);
        }
      }
      // leave no copy in flight behind (only a block that gave up has any)
      if (!ok) {
        mbar_wait(&bar[BAR_QFULL], item & 1);
        for (long long i = max(0LL, issued - C::kSlots); i < issued; ++i)
          mbar_wait(&bar[BAR_FULL + (int)(i % C::kSlots)], (uint32_t)((i / C::kSlots) & 1));
      }
    }
    __syncwarp();
  } else if (warp == 9) {
    // ------------------------------------------------------------- products
    constexpr uint32_t fmt = std::is_same<T, __nv_bfloat16>::value;
    constexpr uint32_t id_s = idesc_f16(128, kKeys, fmt);
    constexpr uint32_t id_o = idesc_f16(128, DP, fmt) | (1u << 16);      // B is MN-major
    int slot = 0;
    uint32_t ph = 0, item = 0, p_ph = 0;         // bit w of p_ph: tile w's P phase
    bool ok = true;
    auto advance = [&]() {
      if (++slot == C::kSlots) {
        slot = 0;
        ph ^= 1;
      }
    };
    auto score = [&](int w, int ks) {            // S_w = Q_w K^T
      if (lane == 0) {
        const uint32_t qa = smem_u32(sq + w * C::kTile), ka = smem_u32(ring + ks * C::kTile);
#pragma unroll
        for (int c = 0; c < C::NC; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_f16(tmem + w * 128, smem_desc(qa + c * kChunkBytes + k * 32, 1024, 2),
                     smem_desc(ka + c * kChunkBytes + k * 32, 1024, 2), id_s, c + k > 0);
        umma_commit(&bar[BAR_SFULL + w]);
      }
    };
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups, ++item) {
      const int e0 = reach(rg, 0), e1 = reach(rg, 1);
      Walk k{c0 / kKeys, max(e0, e1), c1};
      k.settle(A, S, slots);
      ok = wait(BAR_QFULL, item & 1);
      uint32_t first = 3;                        // bit w: tile w's accumulator is not begun
      if (ok && k.live()) {
        ok = wait(BAR_FULL + slot, ph);
        tc_fence_after();
        if (ok) {
          if (k.t * kKeys < e0) score(0, slot);
          if (k.t * kKeys < e1) score(1, slot);
          if (lane == 0) umma_commit(&bar[BAR_EMPTY + slot]);
          advance();
        }
        while (ok && k.live()) {
          const int vs = slot;
          ok = wait(BAR_FULL + vs, ph);
          if (!ok) break;
          advance();
          const int j0 = k.t * kKeys;
          // value rows past the span or in an absent slot: zero
          bool edge = j0 + kKeys > S.nk;
          if (A.present && !edge) {
            unsigned long long want;
            edge = slot_bits(A, slots, S.kb + j0, S.kb + j0 + kKeys - 1, &want) != want;
          }
          if (edge) {
            for (int h = 0; h < kKeys; h += 64) {
              const unsigned long long keep = key_mask(A, S, slots, j0 + h, S.nk);
              for (int i = lane; i < 64; i += 32)
                if (!((keep >> i) & 1))
                  for (int c = 0; c < C::NC; ++c)
                    for (int u = 0; u < 8; ++u)
                      *reinterpret_cast<uint4*>(ring + vs * C::kTile + c * kChunkBytes + (h + i) * 128 + u * 16) =
                          make_uint4(0u, 0u, 0u, 0u);
            }
            fence_async_smem();
            __syncwarp();
          }
          Walk nk = k;
          ++nk.t;
          nk.settle(A, S, slots);
          const int ks = slot;
          const uint32_t kph = ph;
          if (nk.live()) advance();
          bool k_in = false;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const int e = w ? e1 : e0;
            if (!ok || j0 >= e) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              ok = ok && wait(BAR_PREADY + 2 * w + h, (p_ph >> w) & 1);
              tc_fence_after();
              if (ok && lane == 0) {
                const uint32_t va = smem_u32(ring + vs * C::kTile) + h * (kHalf * 128);
#pragma unroll
                for (int kk = 0; kk < kHalf / 16; ++kk)
                  umma_ts(tmem + 256 + w * 128, tmem + w * 128 + h * 32 + kk * 8, desc_v(va + kk * 2048), id_o,
                          !((first >> w) & 1) || kk > 0);
                if (h == 0) umma_commit(&bar[BAR_HALF + w]);
              }
              first &= ~(1u << w);
            }
            p_ph ^= 1u << w;
            if (!ok) continue;
            if (nk.live() && nk.t * kKeys < e) {
              if (!k_in) {
                ok = wait(BAR_FULL + ks, kph);
                k_in = true;
                if (!ok) continue;
                tc_fence_after();
              }
              score(w, ks);
            } else if (lane == 0) {
              umma_commit(&bar[BAR_ODONE + w]);
            }
            __syncwarp();
          }
          if (ok && lane == 0) {
            umma_commit(&bar[BAR_EMPTY + vs]);
            if (nk.live()) umma_commit(&bar[BAR_EMPTY + ks]);
          }
          k = nk;
        }
      }
      if (ok && lane == 0) umma_commit(&bar[BAR_QFREE]);
      __syncwarp();
    }
    // no product may still run when tensor memory is freed
    if (lane == 0) {
      umma_commit(&bar[BAR_DRAIN]);
      if (!mbar_wait(&bar[BAR_DRAIN], 0)) atomicOr(&g_attn_err, 1 << BAR_DRAIN);
    }
    __syncwarp();
  } else {
    // -------------------------------------------------------------- softmax
    const int w = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + w * 128 + lanes, to = tmem + 256 + w * 128 + lanes;
    float* pbuf = spos + warp * (2 * 2 * kKeys);
    uint32_t s_ph = 0, o_ph = 0;
    bool ok = true;
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups) {
      const int i0 = (rg * 2 + w) * qpt;
      if (i0 >= S.nq) continue;
      const int ql = i0 + r / A.group;
      const bool valid = r < qpt * A.group && ql < S.nq;
      const int head = kvh * A.group + r % A.group;
      const long long tok = S.q0 + min(ql, S.nq - 1);
      const int hi = valid ? min(c1, attn_visible(A, S, ql)) : 0;
      const int all_see = attn_visible(A, S, i0);          // every row of the tile sees keys before this
      const int e = reach(rg, w);
      float qy = 0.f, qx = 0.f, slope = 0.f;
      if (DIST) {
        qy = -A.q_pos[tok * A.q_pos_row];
        qx = -A.q_pos[tok * A.q_pos_row + 1];
        slope = -A.slopes[head] * kLog2e;
      }
      float m = -INFINITY, l = 0.f;
      Walk k{c0 / kKeys, e, c1};
      k.settle(A, S, slots);
      const bool any = k.live();
      float2 pos_next[4];
      auto fetch = [&](int t) {                  // the tile's coordinates: four keys per lane
#pragma unroll
        for (int i = 0; i < 4; ++i)
          pos_next[i] = *reinterpret_cast<const float2*>(
              A.k_pos + 2 * (long long)min(S.kb + t * kKeys + i * 32 + lane, A.n_rows - 1));
      };
      if (DIST && any) fetch(k.t);
      int buf = 0;
      while (ok && k.live()) {
        const int j0 = k.t * kKeys;
        Walk nk = k;
        ++nk.t;
        nk.settle(A, S, slots);
        const float* py = pbuf + buf * 2 * kKeys;
        if (DIST) {
          float* d = pbuf + buf * 2 * kKeys + lane;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            d[i * 32] = pos_next[i].x;
            d[kKeys + i * 32] = pos_next[i].y;
          }
          __syncwarp();
          buf ^= 1;
          if (nk.live()) fetch(nk.t);
        }
        ok = wait(BAR_SFULL + w, s_ph);
        if (!ok) break;
        tc_fence_after();
        bool edge = !valid || j0 + kKeys > min(all_see, c1);
        if (A.present && !edge) {
          unsigned long long want;
          edge = slot_bits(A, slots, S.kb + j0, S.kb + j0 + kKeys - 1, &want) != want;
        }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          float2 x2[kHalf / 2];
          float* x = reinterpret_cast<float*>(x2);
          tmem_ld32_issue(ts + h * kHalf, x);
          tmem_ld32_issue(ts + h * kHalf + 32, x + 32);
          tmem_ld_wait();
          reg_fence32(x);
          reg_fence32(x + 32);
          // scores in log2 units
          if (CAP) {
            float big = 0.f;
#pragma unroll
            for (int i = 0; i < kHalf; ++i) big = fmaxf(big, fabsf(x[i]));
            if (__any_sync(0xFFFFFFFFu, valid && !(big * A.scale_log2 <= 0.5f))) {
#pragma unroll
              for (int i = 0; i < kHalf; ++i) x[i] = A.cap_log2 * tanh_abs(x[i] * A.scale_log2);
            } else {
              // an odd polynomial: |error| <= 1.5e-7 cap for |x| <= cap / 2
#pragma unroll
              for (int i = 0; i < kHalf / 2; ++i) {
                const float2 w2 = mul2(x2[i], x2[i]);
                float2 p = fma2(w2, both(poly.c[3]), both(poly.c[2]));
                p = fma2(w2, p, both(poly.c[1]));
                p = fma2(w2, p, both(poly.c[0]));
                x2[i] = mul2(x2[i], p);
              }
            }
          } else if (DIST) {
#pragma unroll
            for (int i = 0; i < kHalf / 2; ++i) x2[i] = mul2(x2[i], both(A.scale_log2));
          }
          if (DIST) {
            const float* ph = py + h * kHalf;
#pragma unroll
            for (int i = 0; i < kHalf; i += 4) {
              const float4 ky = *reinterpret_cast<const float4*>(ph + i);
              const float4 kx = *reinterpret_cast<const float4*>(ph + kKeys + i);
              const float2 y0 = add2(make_float2(ky.x, ky.y), both(qy)), y1 = add2(make_float2(ky.z, ky.w), both(qy));
              const float2 d0 = add2(make_float2(kx.x, kx.y), both(qx)), d1 = add2(make_float2(kx.z, kx.w), both(qx));
              const float2 t0 = make_float2(fabsf(y0.x) + fabsf(d0.x), fabsf(y0.y) + fabsf(d0.y));
              const float2 t1 = make_float2(fabsf(y1.x) + fabsf(d1.x), fabsf(y1.y) + fabsf(d1.y));
              x2[i / 2] = fma2(t0, both(slope), x2[i / 2]);
              x2[i / 2 + 1] = fma2(t1, both(slope), x2[i / 2 + 1]);
            }
          }
          if (edge) {
            const unsigned long long keep = key_mask(A, S, slots, j0 + h * kHalf, hi);
            const uint32_t k0 = (uint32_t)keep, k1 = (uint32_t)(keep >> 32);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              x[i] = (k0 >> i) & 1 ? x[i] : -INFINITY;
              x[i + 32] = (k1 >> i) & 1 ? x[i + 32] : -INFINITY;
            }
          }
          float t0 = x[0], t1 = x[1], t2 = x[2], t3 = x[3];
#pragma unroll
          for (int i = 4; i < kHalf; i += 4) {
            t0 = fmaxf(t0, x[i]);
            t1 = fmaxf(t1, x[i + 1]);
            t2 = fmaxf(t2, x[i + 2]);
            t3 = fmaxf(t3, x[i + 3]);
          }
          constexpr bool scaled = CAP || DIST;
          float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3));
          if (!scaled) top = top == -INFINITY ? top : top * A.scale_log2;
          // the maximum moves: at once from nothing, later only past the slack
          const bool move = m == -INFINITY ? top > m : top > m + kSlack;
          if (__any_sync(0xFFFFFFFFu, move && l > 0.f)) {
            // O as it stands: the previous tile's products ended before this S was
            // complete, the first half's are waited for
            if (h == 1) {
              ok = wait(BAR_HALF + w, s_ph);
              if (!ok) break;
              tc_fence_after();
            }
            const float f = move ? ex2(m - top) : 1.0f;    // m = -inf: 0
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
              float o[32];
              tmem_ld32_issue(to + c, o);
              tmem_ld_wait();
              reg_fence32(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] *= f;
              tmem_st32(to + c, reinterpret_cast<const uint32_t*>(o));
            }
            l *= f;
          }
          if (move) m = top;
          const float2 base = both(m == -INFINITY ? 0.f : -m);
          float2 s0 = both(0.f), s1 = both(0.f);
          uint32_t pk[kHalf / 2];
#pragma unroll
          for (int i = 0; i < kHalf / 2; i += 2) {
            float2 a, c;
            if (scaled) {
              a = add2(x2[i], base);
              c = add2(x2[i + 1], base);
            } else {
              a = fma2(x2[i], both(A.scale_log2), base);
              c = fma2(x2[i + 1], both(A.scale_log2), base);
            }
            a = make_float2(ex2(a.x), ex2(a.y));
            c = make_float2(ex2(c.x), ex2(c.y));
            s0 = add2(s0, a);
            s1 = add2(s1, c);
            pk[i] = Store<T>::pack2(a.x, a.y);   // the probabilities as the product takes them
            pk[i + 1] = Store<T>::pack2(c.x, c.y);
          }
          l += (s0.x + s0.y) + (s1.x + s1.y);
          tmem_st32(ts + h * 32, pk);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar[BAR_PREADY + 2 * w + h]);
        }
        if (!ok) break;
        s_ph ^= 1;
        k = nk;
      }
      if (!ok) break;
      // ---- out = O / l
      const long long R = tok * A.heads + head;
      if (any) {
        ok = wait(BAR_ODONE + w, o_ph);
        o_ph ^= 1;
        if (!ok) break;
        tc_fence_after();
      }
      const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
      const bool split = A.n_chunks > 1;
      const long long at = (long long)chunk * A.n_q * A.heads + R;
#pragma unroll
      for (int c = 0; c < DP; c += 32) {
        float o[32];
        if (any) {
          tmem_ld32_issue(to + c, o);
          tmem_ld_wait();
          reg_fence32(o);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0.f;
        }
        if (!valid) continue;
        if (split) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            if (c + i < A.dim)
              *reinterpret_cast<float4*>(A.part_o + at * A.dim + c + i) =
                  l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        } else {
          T* dst = static_cast<T*>(A.out) + tok * A.out_row + (long long)head * A.out_head + c;
#pragma unroll
          for (int i = 0; i < 32; i += 8)
            if (c + i < A.dim) {
              uint4 u;
              u.x = Store<T>::pack2(o[i] * inv, o[i + 1] * inv);
              u.y = Store<T>::pack2(o[i + 2] * inv, o[i + 3] * inv);
              u.z = Store<T>::pack2(o[i + 4] * inv, o[i + 5] * inv);
              u.w = Store<T>::pack2(o[i + 6] * inv, o[i + 7] * inv);
              *reinterpret_cast<uint4*>(dst + i) = u;
            }
        }
      }
      if (valid && split) A.part_ml[at] = make_float2(m, l);
      if (valid && !split && A.lse) A.lse[R] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <typename T, int DP>
cudaError_t launch_tc_t(const AttnArgs& a, const TcMaps& m, cudaStream_t st) {
  // tanh(u) / u on |u| <= 1/2 in w = u^2, least largest |error| of u p(w): 1.4e-7
  constexpr double kTanh[4] = {0.9999974621104636, -0.3331988899884361, 0.13138806507278963,
                                -0.04322690737438131};
  TanhPoly poly{};
  if (a.cap_log2 > 0.f) {
    double f = (double)a.cap_log2 * a.scale_log2;
    for (int i = 0; i < 4; ++i, f *= (double)a.scale_log2 * a.scale_log2) poly.c[i] = (float)(f * kTanh[i]);
  }
  auto kern = a.cap_log2 > 0.f ? (a.slopes ? k_attn_tc<T, DP, true, true> : k_attn_tc<T, DP, true, false>)
                               : (a.slopes ? k_attn_tc<T, DP, false, true> : k_attn_tc<T, DP, false, false>);
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, TcCfg<DP>::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)((long long)a.n_seqs * a.kv_heads * a.n_chunks * a.row_groups));
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = TcCfg<DP>::kSmem;
  lc.stream = st;
  return cudaLaunchKernelEx(&lc, kern, a, m, poly);
}

}  // namespace

int attn_tc_unit() { return kKeys; }
int attn_tc_tokens_per_block(int group) { return 2 * (128 / group); }

// cudaErrorNotSupported where the arrays cannot be described to the TMA unit
// (a zero stride over more than one head or row, or one of 2^40 bytes or more).
cudaError_t launch_attn_tc(const AttnArgs& a, bool bf16, cudaStream_t st) {
  TcMaps m;
  const int box_q = 128 / a.group;
  if (tmap_rows(&m.q, a.q, bf16, a.dim, a.heads, a.n_q, a.q_head, a.q_row, a.group, box_q) != cudaSuccess ||
      tmap_rows(&m.k, a.k, bf16, a.dim, a.kv_heads, a.n_rows, a.k_head, a.k_row, 1, kKeys) != cudaSuccess ||
      tmap_rows(&m.v, a.v, bf16, a.dim, a.kv_heads, a.n_rows, a.v_head, a.v_row, 1, kKeys) != cudaSuccess)
    return cudaErrorNotSupported;
  if (a.dim <= 64) return bf16 ? launch_tc_t<__nv_bfloat16, 64>(a, m, st) : launch_tc_t<__half, 64>(a, m, st);
  return bf16 ? launch_tc_t<__nv_bfloat16, 128>(a, m, st) : launch_tc_t<__half, 128>(a, m, st);
}

cudaError_t attn_tc_error(int* err, cudaStream_t st) {
  void* p = nullptr;
  cudaError_t e = cudaGetSymbolAddress(&p, g_attn_err);
  if (e == cudaSuccess) e = cudaMemcpyAsync(err, p, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && *err) e = cudaMemsetAsync(p, 0, sizeof(int), st);
  return e;
}

}  // namespace rtcc
