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
// owns a row: no shuffles), warp 8 loads (TMA, one thread), warps 9 and 10 issue
// the products of tile 0 and 1 (one thread issues an MMA in about 100 clocks, so
// two issue for one tensor pipe), warp 11 zeroes value rows at edges.  Keys and
// values share one ring of 128-row slots in the order they are used: K0 V0 K1 V1
// ..., so even slots hold keys and odd ones values.
//
// The running maximum m moves only when a row's new maximum exceeds it by more
// than 2^8 in P (kSlack): P stays below 2^8, far inside either storage type's
// range, O is rescaled rarely, by the softmax threads themselves, and x - m is
// formed with the m of the step before inside the score's last multiply-add.
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

constexpr int kThreads = 384;
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
  static constexpr int kPos = kSlots / 2 * 2 * kKeys * 4;   // [tile in the ring][y | x][128]
  // Tensor memory.  With 64-channel heads P has columns of its own, and the next
  // S may be made as soon as this one is in registers; with 128 it covers S.
  static constexpr bool kOwnP = DP == 64;
  static constexpr int kO = 256, kOStep = DP, kP = kOwnP ? 384 : 0, kPStep = kOwnP ? 64 : 128;
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
// parity would then have come round.  For the same reason every role that waits
// on a slot's barrier does so once for every use of the slot.
enum : int { BAR_QFULL, BAR_QFREE, BAR_SFULL, BAR_PREADY = BAR_SFULL + 2, BAR_ODONE = BAR_PREADY + 4,
             BAR_HALF = BAR_ODONE + 2, BAR_DONE = BAR_HALF + 2, BAR_SFREE = BAR_DONE + 2, BAR_DRAIN = BAR_SFREE + 2,
             BAR_FULL = BAR_DRAIN + 2, BAR_EMPTY = BAR_FULL + 8,
             BAR_VOK = BAR_EMPTY + 8, BAR_N = BAR_VOK + 8 };
__host__ __device__ constexpr int bar_count(int i, bool dist) {
  return (i >= BAR_PREADY && i < BAR_PREADY + 4) || i == BAR_SFREE || i == BAR_SFREE + 1 ? 4   // a tile's softmax warps
         : i == BAR_QFREE                      ? 2           // both product warps
         : dist && i >= BAR_FULL && i < BAR_FULL + 8 ? 2 - (i - BAR_FULL) % 2  // keys: and the coordinates
         : i >= BAR_EMPTY && i < BAR_EMPTY + 8 ? 2 + (i - BAR_EMPTY) % 2   // and, for values, warp 11
                                               : 1;
}

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
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0],"
      " {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(a),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Four MMAs of one 64-deep product by one elected lane of a converged warp; the
// descriptors advance inside (in 16-byte units), so they stay in uniform registers.
// S = Q K^T: both operands K-major in shared memory, 16 channels (32 bytes) a step.
__device__ __forceinline__ void umma4_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p, q;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, 0, 0;\n\t"
      "add.s64 a1, %1, 2;\n\tadd.s64 a2, %1, 4;\n\tadd.s64 a3, %1, 6;\n\t"
      "add.s64 b1, %2, 2;\n\tadd.s64 b2, %2, 4;\n\tadd.s64 b3, %2, 6;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, q;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, q;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, q;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
// O (+)= P V: P from tensor memory, two 16-bit probabilities per column; 16 keys
// (8 columns of P, 2048 bytes of V) a step.
__device__ __forceinline__ void umma4_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p, q;\n\t.reg .b32 a1, a2, a3;\n\t.reg .b64 b1, b2, b3;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, 0, 0;\n\t"
      "add.s32 a1, %1, 8;\n\tadd.s32 a2, %1, 16;\n\tadd.s32 a3, %1, 24;\n\t"
      "add.s64 b1, %2, 128;\n\tadd.s64 b2, %2, 256;\n\tadd.s64 b3, %2, 384;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, q;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, q;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, q;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
// umma_commit by the lane that elect.sync picks, the one that issued the MMAs.
__device__ __forceinline__ void umma_commit_elected(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
      : "memory");
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
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// A walk over the key tiles of a chunk that have a key in a present slot.  Every
// role walks; which tiles are skipped, and which are `partial` (some key in an
// absent slot), depends on the chunk's end c1 alone, so all roles agree.
struct Walk {
  int t, end_key, c1;                            // current tile; tiles that begin before end_key count
  bool partial;
  __device__ __forceinline__ void settle(const AttnArgs& A, const AttnSpan& S, unsigned long long slots, bool all) {
    partial = false;
    if (all) return;
    for (; live(); ++t) {
      const int r0 = S.kb + t * kKeys, r1 = S.kb + min(t * kKeys + kKeys, c1) - 1;
      const int s0 = slot_of(A, r0), s1 = slot_of(A, r1);
      const unsigned long long want = ~0ull >> (63 - (s1 - s0)), have = (slots >> s0) & want;
      partial = have != want;
      if (have) return;
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
  const int r0 = S.kb + j0, s1 = slot_of(A, r0 + n - 1);
  for (int s = slot_of(A, r0); s <= s1; ++s) {
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
      for (int i = 0; i < BAR_N; ++i) mbar_init(&bar[i], bar_count(i, DIST));
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
  bool all = true;                               // every slot of the chunk is present
  if (A.present && c1 > c0) {
    const int s0 = slot_of(A, S.kb + c0), s1 = slot_of(A, S.kb + c1 - 1);
    const unsigned long long want = ~0ull >> (63 - (s1 - s0));
    all = ((slots >> s0) & want) == want;
  }
  volatile int* stop = &gave_up;
  // a wait that runs out marks the block; every role then leaves its loops
  auto wait_one = [&](int i, uint32_t parity) -> bool {
    if (mbar_wait(&bar[i], parity)) return *stop == 0;
    *stop = 1;
    atomicOr(&g_attn_err, 1 << (i & 31));
    return false;
  };
  // the same by a whole warp, which goes on or leaves together
  auto wait = [&](int i, uint32_t parity) -> bool {
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(&bar[i], parity))) return true;
    return __all_sync(0xFFFFFFFFu, wait_one(i, parity));
  };
  // keys that tile w of row group rg reaches within this chunk
  auto reach = [&](int rg, int w) -> int {
    const int i0 = (rg * 2 + w) * qpt;
    if (i0 >= S.nq) return c0;
    return max(c0, min(c1, attn_visible(A, S, min(i0 + qpt, S.nq) - 1)));
  };
  // whether the tile has value rows to zero
  auto patched = [&](const Walk& k) -> bool { return k.partial || k.t * kKeys + kKeys > S.nk; };

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
        Walk k{c0 / kKeys, max(reach(rg, 0), reach(rg, 1)), c1, false};
        for (k.settle(A, S, slots, all); k.live() && ok; ++k.t, k.settle(A, S, slots, all)) {
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
  } else if (warp == 9 || warp == 10) {
    // ------------------------------------------------------ products of tile w
    const int w = __shfl_sync(0xFFFFFFFFu, warp - 9, 0);
    constexpr uint32_t fmt = std::is_same<T, __nv_bfloat16>::value;
    constexpr uint32_t id_s = idesc_f16(128, kKeys, fmt);
    constexpr uint32_t id_o = idesc_f16(128, DP, fmt) | (1u << 16);      // B is MN-major
    const uint32_t t_s = tmem + w * 128, t_o = tmem + C::kO + w * C::kOStep,
                   t_p = tmem + C::kP + w * C::kPStep;
    const uint64_t dq = smem_desc(smem_u32(sq + w * C::kTile), 1024, 2);
    const uint64_t dk = smem_desc(smem_u32(ring), 1024, 2), dv = desc_v(smem_u32(ring));
    constexpr uint64_t kSlotStep = C::kTile >> 4, kChunkStep = kChunkBytes >> 4, kHalfStep = (kHalf * 128) >> 4;
    int slot = 0;
    uint32_t ph = 0, item = 0, p_ph = 0, vok = 0;                        // bit s of vok: slot s's patch phase
    bool ok = true;
    auto advance = [&]() {
      if (++slot == C::kSlots) {
        slot = 0;
        ph ^= 1;
      }
    };
    auto score = [&](int ks) {                   // S = Q K^T; the slot is free when it is done
#pragma unroll
      for (int c = 0; c < C::NC; ++c)
        umma4_ss(t_s, dq + c * kChunkStep, dk + ks * kSlotStep + c * kChunkStep, id_s, c > 0);
      umma_commit_elected(&bar[BAR_SFULL + w]);
      umma_commit_elected(&bar[BAR_EMPTY + ks]);
    };
    auto skip = [&](int s) {                     // this tile does not use the slot
      if (lane == 0) mbar_arrive(&bar[BAR_EMPTY + s]);
    };
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups, ++item) {
      const int e = reach(rg, w);
      Walk k{c0 / kKeys, max(e, reach(rg, w ^ 1)), c1, false};
      k.settle(A, S, slots, all);
      ok = wait(BAR_QFULL, item & 1);
      if (ok && k.live()) {
        ok = wait(BAR_FULL + slot, ph);
        if (ok) {
          tc_fence_after();
          if (k.t * kKeys < e) score(slot); else skip(slot);
        }
        advance();
      }
      uint32_t begun = 0;
      while (ok && k.live()) {
        const int vs = slot;
        if (!(ok = wait(BAR_FULL + vs, ph))) break;
        advance();
        const bool mine = k.t * kKeys < e, zeroed = patched(k);
        Walk nk = k;
        ++nk.t;
        nk.settle(A, S, slots, all);
        const int ks = slot;
        const uint32_t kph = ph;
        if (nk.live()) advance();
        const bool more = nk.live() && nk.t * kKeys < e;
        if (mine) {
          if (zeroed && !(ok = wait(BAR_VOK + vs, (vok >> vs) & 1))) break;
          const uint64_t d = dv + vs * kSlotStep;
          if (!(ok = wait(BAR_PREADY + 2 * w, p_ph))) break;
          tc_fence_after();
          umma4_ts(t_o, t_p, d, id_o, begun);
          umma_commit_elected(&bar[BAR_HALF + w]);
          if (C::kOwnP && more) {
            if (!(ok = wait(BAR_FULL + ks, kph))) break;
            if (!(ok = wait(BAR_SFREE + w, p_ph))) break;
            tc_fence_after();
            score(ks);
          }
          if (!(ok = wait(BAR_PREADY + 2 * w + 1, p_ph))) break;
          tc_fence_after();
          umma4_ts(t_o, t_p + 32, d + kHalfStep, id_o, 1);
          umma_commit_elected(&bar[BAR_EMPTY + vs]);
          if (C::kOwnP) umma_commit_elected(&bar[BAR_DONE + w]);
          p_ph ^= 1;
          begun = 1;
        } else {
          skip(vs);
        }
        if (zeroed) vok ^= 1u << vs;
        if (mine && !more) umma_commit_elected(&bar[BAR_ODONE + w]);
        if (nk.live() && !(C::kOwnP && mine && more)) {
          if (!(ok = wait(BAR_FULL + ks, kph))) break;
          tc_fence_after();
          if (more) score(ks); else skip(ks);
        }
        k = nk;
      }
      if (ok) umma_commit_elected(&bar[BAR_QFREE]);
      __syncwarp();
    }
    // no product may still run when tensor memory is freed
    umma_commit_elected(&bar[BAR_DRAIN + w]);
    if (!mbar_wait(&bar[BAR_DRAIN + w], 0)) atomicOr(&g_attn_err, 1 << (BAR_DRAIN + w));
    __syncwarp();
  } else if (warp == 11) {
    // ------------ the keys' coordinates; value rows nobody sees: zero
    int tile = 0, last_tile = 0;                 // place in the ring: slots 2 tile and 2 tile + 1
    uint32_t ph = 0, last_ph = 0;
    bool ok = true, pending = false;
    Walk last{};
    // the values of the tile before, one step behind the coordinates
    auto patch = [&]() {
      const int slot = 2 * last_tile + 1;
      if (!(ok = wait(BAR_FULL + slot, last_ph))) return;
      if (patched(last)) {
        unsigned char* rows = ring + slot * C::kTile;
        for (int h = 0; h < kKeys; h += 64) {
          const unsigned long long keep = key_mask(A, S, slots, last.t * kKeys + h, S.nk);
          for (int i = lane; i < 64; i += 32)
            if (!((keep >> i) & 1))
              for (int c = 0; c < C::NC; ++c)
                for (int u = 0; u < 8; ++u)
                  *reinterpret_cast<uint4*>(rows + c * kChunkBytes + (h + i) * 128 + u * 16) =
                      make_uint4(0u, 0u, 0u, 0u);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[BAR_VOK + slot]);
      }
      if (lane == 0) mbar_arrive(&bar[BAR_EMPTY + slot]);
    };
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups) {
      Walk k{c0 / kKeys, max(reach(rg, 0), reach(rg, 1)), c1, false};
      for (k.settle(A, S, slots, all); k.live(); ++k.t, k.settle(A, S, slots, all)) {
        if (DIST) {
          float2 at[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            at[i] = *reinterpret_cast<const float2*>(
                A.k_pos + 2 * (long long)min(S.kb + k.t * kKeys + i * 32 + lane, A.n_rows - 1));
          // the ring's tile has been read when its values are released
          if (!(ok = wait(BAR_EMPTY + 2 * tile + 1, ph ^ 1))) break;
          float* d = spos + tile * 2 * kKeys + lane;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            d[i * 32] = at[i].x;
            d[kKeys + i * 32] = at[i].y;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar[BAR_FULL + 2 * tile]);
        }
        if (pending) {
          patch();
          if (!ok) break;
        }
        pending = true;
        last = k;
        last_tile = tile;
        last_ph = ph;
        if (++tile == C::kSlots / 2) {
          tile = 0;
          ph ^= 1;
        }
      }
    }
    if (ok && pending) patch();
  } else {
    // -------------------------------------------------------------- softmax
    const int w = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + w * 128 + lanes, to = tmem + C::kO + w * C::kOStep + lanes,
                   tp = tmem + C::kP + w * C::kPStep + lanes;
    uint32_t s_ph = 0, o_ph = 0, k_ph = 0, d_ph = 0;
    int tile = 0;                                // place in the ring, for the coordinates
    bool ok = true;
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups) {
      const int i0 = (rg * 2 + w) * qpt;
      const int e_all = max(reach(rg, w), reach(rg, w ^ 1));
      const int ql = i0 + r / A.group;
      const bool valid = r < qpt * A.group && ql < S.nq;
      const int head = kvh * A.group + r % A.group;
      const long long tok = S.q0 + min(ql, S.nq - 1);        // a row without a token computes nothing
      const int hi = valid ? min(c1, attn_visible(A, S, ql)) : 0;
      const int all_see = i0 < S.nq ? min(c1, attn_visible(A, S, i0)) : 0;   // every row sees the keys before this
      const int e = reach(rg, w);
      float qy = 0.f, qx = 0.f, slope = 0.f;
      if (DIST) {
        qy = -A.q_pos[tok * A.q_pos_row];
        qx = -A.q_pos[tok * A.q_pos_row + 1];
        slope = -A.slopes[head] * kLog2e;
      }
      float m = -INFINITY, l = 0.f;
      bool later = false;                      // a tile of this group came before
      Walk k{c0 / kKeys, e, c1, false};
      k.settle(A, S, slots, all);
      const bool any = k.live();
      while (ok && k.live()) {
        const int j0 = k.t * kKeys;
        const bool edge = k.partial || j0 + kKeys > all_see;
        const float* py = spos + tile * 2 * kKeys;
        ++k.t;
        k.settle(A, S, slots, all);
        ok = wait(BAR_SFULL + w, s_ph);
        if (DIST && ok) ok = wait(BAR_FULL + 2 * tile, k_ph);            // complete since before S
        if (!ok) break;
        tc_fence_after();
        if (++tile == C::kSlots / 2) {
          tile = 0;
          k_ph ^= 1;
        }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const float* pyh = py + h * kHalf;
          bool slow = edge || __any_sync(0xFFFFFFFFu, valid && m == -INFINITY);
          bool waited = !C::kOwnP || h == 1 || !later;
          // The previous tile's products are done with P and O before either changes
          // (with P over S they ended before this S was complete).
          auto settled = [&]() -> bool {
            if (waited) return true;
            waited = true;
            if (!wait(BAR_DONE + w, d_ph)) return false;
            d_ph ^= 1;
            tc_fence_after();
            return true;
          };
          // Rows' maxima go up by `up`: what they have summed so far is scaled down.
          auto rise = [&](float up) -> bool {
            if (__any_sync(0xFFFFFFFFu, up > 0.f && l > 0.f)) {
              if (h == 1) {                      // the first half's product into O
                if (!wait(BAR_HALF + w, s_ph)) return false;
                tc_fence_after();
              }
              const float f = l > 0.f ? ex2(-up) : 1.0f;
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
            return true;
          };
          bool again = !slow;
          while (again) {
            // One pass, with the maximum so far: z = score (log2 units) - m, p = exp2(z).
            // Only afterwards is it seen whether a maximum had to move, and then the pass
            // is repeated, or a score was too large for the polynomial (below).
            const float m0 = m;
            float2 x2[kHalf / 2];
            float* x = reinterpret_cast<float*>(x2);
            tmem_ld32_issue(ts + h * kHalf, x);
            tmem_ld32_issue(ts + h * kHalf + 32, x + 32);
            tmem_ld_wait();
            reg_fence32(x);
            reg_fence32(x + 32);
            float b0 = 0.f, b1 = 0.f, t0 = -INFINITY, t1 = -INFINITY;
            float2 s0 = both(0.f), s1 = both(0.f);
            uint32_t pk[kHalf / 2];
            constexpr int G = DIST ? 4 : 8;      // pairs abreast: a multiply-add's latency is several issue slots
#pragma unroll
            for (int i = 0; i < kHalf / 2; i += G) {
              float2 a[G];                       // what is added to the capped score
#pragma unroll
              for (int g = 0; g < G; ++g) a[g] = both(-m0);
              if (DIST) {
                float2 y[G], d[G];
#pragma unroll
                for (int g = 0; g < G; g += 2) {
                  const float4 ky = *reinterpret_cast<const float4*>(pyh + 2 * (i + g));
                  const float4 kx = *reinterpret_cast<const float4*>(pyh + kKeys + 2 * (i + g));
                  y[g] = make_float2(ky.x, ky.y);
                  y[g + 1] = make_float2(ky.z, ky.w);
                  d[g] = make_float2(kx.x, kx.y);
                  d[g + 1] = make_float2(kx.z, kx.w);
                }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                  y[g] = add2(y[g], both(qy));
                  d[g] = add2(d[g], both(qx));
                }
#pragma unroll
                for (int g = 0; g < G; ++g)
                  y[g] = make_float2(fabsf(y[g].x) + fabsf(d[g].x), fabsf(y[g].y) + fabsf(d[g].y));
#pragma unroll
                for (int g = 0; g < G; ++g) a[g] = fma2(y[g], both(slope), a[g]);
              }
              if (!CAP) {
#pragma unroll
                for (int g = 0; g < G; ++g) x2[i + g] = fma2(x2[i + g], both(A.scale_log2), a[g]);
              } else {
                // an odd polynomial: |error| <= 1.5e-7 cap for |x| <= cap / 2
                float2 w2[G], p[G];
#pragma unroll
                for (int g = 0; g < G; ++g) {
                  b0 = fmaxf(b0, fmaxf(fabsf(x2[i + g].x), fabsf(x2[i + g].y)));
                  w2[g] = mul2(x2[i + g], x2[i + g]);
                }
#pragma unroll
                for (int g = 0; g < G; ++g) p[g] = fma2(w2[g], both(poly.c[3]), both(poly.c[2]));
#pragma unroll
                for (int g = 0; g < G; ++g) p[g] = fma2(w2[g], p[g], both(poly.c[1]));
#pragma unroll
                for (int g = 0; g < G; ++g) p[g] = fma2(w2[g], p[g], both(poly.c[0]));
#pragma unroll
                for (int g = 0; g < G; ++g) x2[i + g] = fma2(x2[i + g], p[g], a[g]);
              }
#pragma unroll
              for (int g = 0; g < G; g += 2) {
                t0 = fmaxf(t0, fmaxf(x2[i + g].x, x2[i + g].y));
                t1 = fmaxf(t1, fmaxf(x2[i + g + 1].x, x2[i + g + 1].y));
                const float2 u = make_float2(ex2(x2[i + g].x), ex2(x2[i + g].y));
                const float2 v = make_float2(ex2(x2[i + g + 1].x), ex2(x2[i + g + 1].y));
                s0 = add2(s0, u);
                s1 = add2(s1, v);
                pk[i + g] = Store<T>::pack2(u.x, u.y);     // the probabilities as the product takes them
                pk[i + g + 1] = Store<T>::pack2(v.x, v.y);
              }
            }
            const float top = fmaxf(t0, t1);
            // without a distance bias a maximum hardly ever moves after the first tiles
            slow = __any_sync(0xFFFFFFFFu, valid && ((CAP && !(fmaxf(b0, b1) * A.scale_log2 <= 0.5f)) ||
                                                     (!DIST && top > kSlack)));
            if (slow || !(ok = settled())) break;
            again = DIST && __any_sync(0xFFFFFFFFu, valid && top > kSlack);
            if (again) {
              // one row has to move: all of the warp that can do
              const float up = valid ? fmaxf(top, 0.f) : 0.f;
              if (!(ok = rise(up))) break;
              m += up;
            } else {
              if (C::kOwnP && h == 1) {          // S is done with: the next one may come
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar[BAR_SFREE + w]);
              }
              l += (s0.x + s0.y) + (s1.x + s1.y);
              tmem_st32(tp + h * 32, pk);
            }
          }
          if (!ok) break;
          if (slow) {
            // In two passes over S, 32 keys at a time: scores with tanh itself, masked,
            // put back into S with their maximum; then the probabilities.
            const unsigned long long keep =
                edge ? key_mask(A, S, slots, j0 + h * kHalf, hi) : ~0ull;
            const float m0 = m == -INFINITY ? 0.f : m;
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < kHalf; c += 32) {
              float y[32];
              tmem_ld32_issue(ts + h * kHalf + c, y);
              tmem_ld_wait();
              reg_fence32(y);
              const uint32_t bits = (uint32_t)(keep >> c);
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                y[i] *= A.scale_log2;
                if (CAP) y[i] = A.cap_log2 * tanh_abs(y[i]);
                if (DIST) y[i] = fmaf(fabsf(pyh[c + i] + qy) + fabsf(pyh[kKeys + c + i] + qx), slope, y[i]);
                y[i] = (bits >> i) & 1 ? y[i] - m0 : -INFINITY;
                top = fmaxf(top, y[i]);
              }
              tmem_st32(ts + h * kHalf + c, reinterpret_cast<const uint32_t*>(y));
            }
            tmem_st_wait();
            if (!(ok = settled())) break;
            // the maximum moves at once from nothing, later only past the slack
            const bool move = m == -INFINITY ? top > -INFINITY : top > kSlack;
            const float up = move ? top : 0.f;
            if (!(ok = rise(m == -INFINITY ? 0.f : up))) break;
            if (move) m = m0 + up;
#pragma unroll 1
            for (int c = 0; c < kHalf; c += 32) {
              float y[32];
              tmem_ld32_issue(ts + h * kHalf + c, y);
              tmem_ld_wait();
              reg_fence32(y);
              uint32_t pk[16];
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float u = ex2(y[i] - up), v = ex2(y[i + 1] - up);
                l += u + v;
                pk[i / 2] = Store<T>::pack2(u, v);
              }
              tmem_st16(tp + h * 32 + c / 2, pk);
            }
            if (l != l && m == -INFINITY) m = 0.f;         // a NaN row never gets a maximum: it is done with
            if (C::kOwnP && h == 1) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&bar[BAR_SFREE + w]);
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar[BAR_PREADY + 2 * w + h]);
        }
        if (!ok) break;
        s_ph ^= 1;
        later = true;
      }
      if (!ok) break;
      // the tiles that only the other rows reach pass through the ring as well
      for (k.end_key = e_all; k.live(); ++k.t, k.settle(A, S, slots, all))
        if (++tile == C::kSlots / 2) {
          tile = 0;
          k_ph ^= 1;
        }
      // ---- out = O / l
      const long long R = tok * A.heads + head;
      if (any) {
        ok = wait(BAR_ODONE + w, o_ph);
        o_ph ^= 1;
        if (C::kOwnP && ok) {                    // the last tile's, so that none is left over
          ok = wait(BAR_DONE + w, d_ph);
          d_ph ^= 1;
        }
        if (!ok) break;
        tc_fence_after();
      }
      const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
      const bool split = A.n_chunks > 1;
      const long long at = (long long)chunk * A.n_q * A.heads + R;
#pragma unroll 1
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
        if (valid) {
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
        __syncwarp();
      }
      if (valid && split) A.part_ml[at] = make_float2(m, l);
      if (valid && !split && A.lse) A.lse[R] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      tc_fence_before();
      __syncwarp();
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
