// Attention of many rows over the token memory on the 5th-generation tensor
// cores (the formula is in attn_rows.cu).  Compiled twice: attn_tc.cu, and attn_win.cu with
// windows and keys widened from pages (WIN).
//
// A block has two tiles of 128 rows and one key head; the query heads that share it
// are rows of the same tile (row r: token r / group, head r % group), so keys and
// values are read once for all of them.  Keys come in steps of 64.  A "chain" is one
// tile's way through its steps:  S = Q K^T (128 x 64 floats in tensor memory), four
// softmax warps turn S into P = exp2(x - m), rounded to the storage type and written
// over S, and O += P V takes P from there.  The two chains run beside each other, so
// that one's softmax covers the other's products, and each has two S, so that the
// next scores are there when a softmax ends: 2 x (2 x 64 + head size) of 512 columns.
//
// An odd number of tiles would leave a chain idle in the last block.  Then both
// chains share a tile and take its steps in turn ("streams"): a stream writes a
// partial result as a chunk of the span does, and k_attn_join merges them.
//
// Roles: four softmax warps per chain (a thread owns a row: no shuffles), a warp
// that loads keys (TMA, one lane) and stages their coordinates, one that loads
// values and zeroes those of keys nobody sees, and one per chain that issues its
// products.  Steps run from the last key back: with a distance bias a causal row's
// nearest keys come last, and starting there its maximum hardly moves.
//
// A row's m moves late: P = exp2(x - m) is formed in one pass with the m of the step
// before.  When m is set it puts the largest P at 2^kLift; where a row's largest has
// passed 2^kSlack, m goes up, and O and the sum down, before the next step.  Up to
// 2^kHard, inside fp16's range, nothing is done again; beyond, and at masked steps and a
// row's first, a slower form of the step handles everything.  fp16 ends at 2^-24, and
// the lift keeps what is lost of a key at 2^-31 of the largest: without it 280,000 keys
// 2^-25 below one key, up to 0.8 % of the weight, were lost to the product while the sum
// had them.
//
// Key rows nobody may see (past the span, in an absent slot) are skipped as
// whole steps; in a step at the edge their scores are replaced, not added to, and
// their value rows are zeroed in shared memory before the product, so their
// contents never reach a result.
//
// With a window (WIN) a row group's steps are those of its rows' windows and of what
// they see from afar (the sinks, a prefix); the walk jumps from the one to the other, and
// a tile leaves out steps that only the other one sees.  A block then has few steps and
// several edges, which a form of the step of their own takes in one pass.
//
// What bounds it is the softmax warps' latency, no pipe alone.  Two of them share a
// scheduler.  Their 64 keys take 1,420 clocks bare, 1,890 with a cap, 1,950 with a bias
// and 2,630 with both, against 640 (heads of 64) or 1,280 of the tensor pipe.  A pair of
// keys costs 1 packed multiply-add bare or 5 with a cap, 3 and two single adds for a
// bias, and 1 for the sum: with both 1,280 clocks of the FMA pipe (packed ones take 2),
// and 512 for exp2 (4 a warp).  The rest is waiting for scores from tensor memory and for
// results.  Measured: 16,384 x 49,152 keys, 6 heads of 64: 1.54 ms bare (802 TFLOP/s),
// 2.17 with a cap, 2.16 with a bias, 3.00 with both (412), each with a sixth of the SMs'
// time lost to a half-empty third round of blocks; 12,036 packed causal tokens of 16
// heads of 128 with a cap: 127 us, 740 TFLOP/s (of a block's 22 us there, 1 goes to its
// set-up, 2 to its first scores, 2 to the masked step and 3 to its results).  Windows of
// 700 and 8 sinks, 20,900 packed tokens of 16 heads of 128: 197 us, 608 TFLOP/s; a block
// has 14 steps, of which an inner one takes 1.0 us (8.4 MFLOP, 0.68 us at a large GEMM's
// rate: in the rest no product runs), and 8 us besides, in which the SM has nothing else:
// 1.5 its set-up, 2.2 its first scores, 1.3 the first step, 3 its results.
// Tried and slower: four chains of one S each (four softmax warps a scheduler, 96
// registers: 10 to 30 %), the next S loaded while P is stored (spills: 5 to 15 %),
// scalar beside packed arithmetic (up to 30 %), a second form of the pass for steps
// whose keys share one y (8 % faster where all do, 8 % slower where two thirds do:
// the two forms push each other out of the instruction cache), blocks that take over
// the work of those not yet begun (up to 30 %: the roles change over one after the
// other; with queries released as soon as the last scores are under way, still 12 to
// 18 % on windows), results through shared memory to whole lines (4 %), keys and values
// released apart (6 % on windows: one wait and one commit more in the products' warp),
// one chain to a block and two blocks to an SM (50 %), more registers for the softmax
// warps at the others' cost (no spills, 2 %), and S released as soon as it is in
// registers, with a place of its own for P (the same time with heads of 128, 15 % more
// with 64).
#pragma once

#include <float.h>
#include <math.h>

#include <type_traits>

#include "attn.cuh"
#include "kernels.h"

namespace rtcc {
namespace {

constexpr int kKeys = 64;                        // keys per step
constexpr int kBox = 64 * 128;                   // 64 keys x 64 channels
constexpr int kQBox = 128 * 128;                 // 128 rows x 64 channels
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 6.0f : 0.0f;
template <typename T> constexpr float kSlack = std::is_same<T, __half>::value ? 11.0f : 8.0f;
constexpr float kHard = 15.9f;
// Measured on 300 queries over 281,600 keys with a bias, fp16, (lift, slack): (0, 8) 325 us,
// (6, 11) 325, (8, 11) 333, (8, 12) with kHard 15 367: what is short of kHard is done again.

__device__ unsigned g_attn_err;                  // threads whose waits ran out, since the start

constexpr int kChains = 2;
constexpr int kS = 2;                            // S per chain
constexpr int kWarps = 4 * kChains + 4;
constexpr int kLoadK = 4 * kChains, kLoadV = kLoadK + 1, kProduct = kLoadK + 2;       // warps

template <int DP> struct TcCfg {
  static constexpr int NC = DP / 64;             // 64-channel chunks (one 128-byte swizzle line each)
  static constexpr int kRing = DP == 64 ? 8 : 4; // steps of keys and of values in shared memory
  static constexpr int kStep = NC * kBox;
  static constexpr int kQ = kChains * NC * kQBox;
  static constexpr int kPos = kRing * 2 * kKeys * 4;         // [step in the ring][y | x][64]
  static constexpr int kSmem = kQ + 2 * kRing * kStep + kPos + 1024;
  // tensor memory: S of every chain, then O of every chain
  static constexpr int kO = kChains * kS * kKeys;
  static_assert(kO + kChains * DP <= 512, "tensor memory");
  // barriers
  static constexpr int FULL = 0, FREE = kRing, VOK = 2 * kRing, SFULL = 3 * kRing, PREADY = SFULL + kChains * kS,
                       DONE = PREADY + kChains * kS, QFULL = DONE + kChains * kS, QFREE = QFULL + 1,
                       DRAIN = QFREE + 1, kBars = DRAIN + kChains;
};

struct TcMaps {
  CUtensorMap q, k, v;
};

// coefficients of cap tanh(x scale / cap) log2(e) = x (c0 + w (c1 + w (c2 + w c3))), w = x^2,
// for |x| <= limit.  They work on scores before the scale, which saves a product, so
// with a small scale / cap (1e-5, say) they leave float32's range: the limit is 0 then,
// as for caps above kAbsCap, and every step takes the form with tanh itself.
struct TanhPoly {
  float c[4];
  float limit;
};

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
// 32 bytes to a 32-byte boundary of global memory.
__device__ __forceinline__ void st_global32(void* p, const uint32_t* r) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
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
// channels a box further.
__device__ __forceinline__ uint64_t desc_v(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr >> 4) & 0x3FFFu);
  d |= static_cast<uint64_t>(kBox >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}

__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// Which halves of step t (32 keys each) are on no page.
__device__ __forceinline__ int hidden_halves(const AttnArgs& A, const AttnSpan& S, int t) {
  return A.hidden[S.kb / kKeys + t];
}

// A view in whole steps: steps [seen, low) have no key that its rows see.
struct Steps {
  int seen, low;
  __device__ __forceinline__ Steps() {}
  __device__ __forceinline__ explicit Steps(AttnView v) : seen((v.seen + kKeys - 1) / kKeys), low(v.low / kKeys) {}
  __device__ __forceinline__ bool behind(int t) const { return t < low && t >= seen; }
};

// A walk over the steps of a chunk that have a key in a present slot, and their
// number, from the last key a row group reaches to the chunk's first: with a
// distance bias the nearest keys of a causal row come last, so going back the
// maxima are met first and hardly move.  Every role walks; which steps are skipped,
// and which are `partial` (some key in an absent slot), depends on the chunk's end
// c1 alone, so all roles agree.  With WIN it also jumps from the first step of the
// row group's windows to the last one that its rows see from afar (their view, the
// group's widest), and over steps of keys on no page.
template <bool WIN> struct Walk {
  int t, t0, c1;                                 // current step, the chunk's first
  int g;                                         // steps since the block began
  bool partial;
  Steps view;
  __device__ __forceinline__ Walk() {}
  __device__ __forceinline__ Walk(int c0, int end_key, int c1_, int g_, Steps view_)
      : t((end_key + kKeys - 1) / kKeys - 1), t0(c0 / kKeys), c1(c1_), g(g_), partial(false), view(view_) {
    if (end_key <= c0) t = t0 - 1;
  }
  __device__ __forceinline__ bool live() const { return t >= t0; }
  __device__ __forceinline__ void settle(const AttnArgs& A, const AttnSpan& S, unsigned long long slots, bool all) {
    partial = false;
    if (all) {
      if (WIN && view.behind(t)) t = view.seen - 1;
      return;
    }
    for (; live(); --t) {
      bool some = false;
      if (WIN) {
        if (view.behind(t)) {
          t = view.seen;                         // one past the step to go on with
          continue;
        }
        if (A.hidden) {
          const int h = hidden_halves(A, S, t);
          if (h == 3) continue;
          some = h != 0;
        }
        partial = some;
        if (!A.present) return;
      }
      const int base = WIN ? attn_row(S, t * kKeys) - t * kKeys : S.kb;
      const int r0 = base + t * kKeys, r1 = base + min(t * kKeys + kKeys, c1) - 1;
      const int s0 = slot_of(A, r0), s1 = slot_of(A, r1);
      const unsigned long long want = ~0ull >> (63 - (s1 - s0)), have = (slots >> s0) & want;
      partial = have != want || some;
      if (have) return;
    }
  }
  __device__ __forceinline__ void next(const AttnArgs& A, const AttnSpan& S, unsigned long long slots, bool all) {
    --t;
    ++g;
    settle(A, S, slots, all);
  }
  // to the next step of a stream: one whose number is `stream` in every `streams`
  __device__ __forceinline__ void seek(const AttnArgs& A, const AttnSpan& S, unsigned long long slots, bool all,
                                       int streams, int stream) {
    while (live() && (g & (streams - 1)) != stream) next(A, S, slots, all);
  }
  __device__ __forceinline__ void next_own(const AttnArgs& A, const AttnSpan& S, unsigned long long slots, bool all,
                                           int streams, int stream) {
    if (all) {                                   // nothing to skip, or the one gap
      if (!WIN) {
        t -= streams;
        g += streams;
        return;
      }
      for (int i = 0; i < streams; ++i) next(A, S, slots, true);
      return;
    }
    next(A, S, slots, all);
    seek(A, S, slots, all, streams, stream);
  }
};

// Bits below n.
__device__ __forceinline__ unsigned long long bits_below(int n) {
  return n <= 0 ? 0ull : n >= 64 ? ~0ull : ~0ull >> (64 - n);
}

// Bit c: key j0 + c, c < 64, lies before `lim`, in the view (with WIN), in a present
// slot and on a page.
template <bool WIN>
__device__ __forceinline__ unsigned long long key_mask(const AttnArgs& A, const AttnSpan& S, unsigned long long slots,
                                                       int j0, int lim, AttnView view) {
  const int n = min(max(lim - j0, 0), 64);
  if (n == 0) return 0;
  unsigned long long bits = ~0ull >> (64 - n);
  if (WIN) {
    bits &= bits_below(view.seen - j0) | ~bits_below(view.low - j0);
    if (A.hidden) {
      const int h = hidden_halves(A, S, j0 / kKeys);
      if (h & 1) bits &= ~0xFFFFFFFFull;
      if (h & 2) bits &= 0xFFFFFFFFull;
    }
  }
  if (!A.present) return bits;
  const int r0 = WIN ? attn_row(S, j0) : S.kb + j0, s1 = slot_of(A, r0 + n - 1);
  for (int s = slot_of(A, r0); s <= s1; ++s) {
    if ((slots >> s) & 1) continue;
    const int a = (int)max((long long)s * A.slot_rows - r0, 0LL);
    const int b = (int)min((long long)(s + 1) * A.slot_rows - r0, 64LL);      // a < b
    bits &= ~((~0ull >> (64 - (b - a))) << a);
  }
  return bits;
}

// A block that gave up stays for about 2 ms, so that no copy of its own (a few
// microseconds at most) is in flight when it ends.
__device__ __forceinline__ void outlast_copies() {
  const long long t0 = clock64();
  while (clock64() - t0 < kWaitBudgetCycles / 500) {
  }
}

template <typename T, int DP, bool CAP, bool DIST, bool WIN>
__global__ void __launch_bounds__(kWarps * 32, 1)
    k_attn_tc(const __grid_constant__ AttnArgs A, const __grid_constant__ TcMaps M, const TanhPoly poly) {
  using C = TcCfg<DP>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bar[C::kBars];
  __shared__ uint32_t tmem_base;
  __shared__ int gave_up, first_place;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  unsigned char* sq = smem;
  unsigned char* sk = smem + C::kQ;
  unsigned char* sv = sk + C::kRing * C::kStep;
  float* spos = reinterpret_cast<float*>(sv + C::kRing * C::kStep);

  // block -> (row group, chunk, key head, sequence); the last rows of causal
  // sequences have the longest reach and go first, those of all sequences together,
  // so that short work is left for the end
  const int streams = A.streams, tiles = kChains / streams;
  int b = blockIdx.x, rg0;
  if (A.causal) {
    const int each = gridDim.x / A.row_groups;
    rg0 = A.row_groups - 1 - b / each;
    b %= each;
  } else {
    rg0 = b % A.row_groups;
    b /= A.row_groups;
  }
  const int chunk = b % A.n_chunks;
  b /= A.n_chunks;
  const int kvh = b % A.kv_heads;
  const int seq = b / A.kv_heads;
  const AttnSpan S = attn_span<WIN>(A, seq);
  const int qpt = 128 / A.group;                 // tokens per tile
  const int groups = (S.nq + tiles * qpt - 1) / (tiles * qpt);
  const int per = attn_chunk(A, S.nk, A.unit);
  const int c0 = (int)min((long long)per * chunk, (long long)S.nk), c1 = min(S.nk - c0, per) + c0;
  if (rg0 >= groups || (chunk > 0 && c0 >= S.nk)) return;   // not in use; chunk 0 always answers

  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < C::kBars; ++i) {
        int n = 1;
        if (i < C::FREE) n = 2;                                                              // keys and values
        if (i >= C::FREE && i < C::VOK) n = tiles;                                           // the chains of a stream
        if (i >= C::PREADY && i < C::DONE) n = 4;                                            // a chain's softmax warps
        if (DIST && i >= C::SFULL && i < C::PREADY) n = 2;                                   // S, and its coordinates
        if (i == C::QFREE) n = 2;                                                            // the product warps
        mbar_init(&bar[i], n);
      }
      fence_barrier_init();
      gave_up = 0;
      first_place = S.first;
      tma_prefetch_desc(&M.q);
      tma_prefetch_desc(&M.k);
      tma_prefetch_desc(&M.v);
    }
    __syncwarp();
  }
  if (warp == kProduct) {
    tmem_alloc(&tmem_base, 512);
    tmem_relinquish();
  }
  // with pages: whether any of the chunk's keys is on none, as each step asks only then
  bool off_page = false;
  if (WIN && A.hidden)
    for (int t = c0 / kKeys + tid; t * kKeys < c1; t += kWarps * 32) off_page |= hidden_halves(A, S, t) != 0;
  if (WIN) off_page = __syncthreads_or(off_page);
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  const unsigned long long slots = attn_slot_mask(A, lane);
  bool all = !WIN || (!A.present && !off_page);  // every slot of the chunk is present, every key on a page
  if (!WIN && A.present && c1 > c0) {
    const int s0 = slot_of(A, S.kb + c0), s1 = slot_of(A, S.kb + c1 - 1);
    const unsigned long long want = ~0ull >> (63 - (s1 - s0));
    all = ((slots >> s0) & want) == want;
  }
  volatile int* stop = &gave_up;
  volatile int* first = &first_place;            // read once a group: registers are short
  // A wait by a whole warp; one that runs out marks the block, and every role then
  // leaves its loops.  A slot's barrier is waited for at every use by each role
  // that waits on it at all (a slot belongs to one stream), so parities suffice.
  const uint32_t bar0 = smem_u32(bar);
  auto wait = [&](int i, uint32_t parity) -> bool {
    uint32_t in;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(in)
        : "r"(bar0 + i * 8), "r"(parity)
        : "memory");
    if (__all_sync(0xFFFFFFFFu, in)) return true;
    bool ok = mbar_wait(&bar[i], parity, A.budget);
    if (!ok) {
      *stop = 1;
      atomicAdd(&g_attn_err, 1u);
    }
    return __all_sync(0xFFFFFFFFu, ok && *stop == 0);
  };
  // keys that tile w of row group rg reaches within this chunk
  auto reach = [&](int rg, int w) -> int {
    const int i0 = (rg * tiles + w) * qpt;
    if (i0 >= S.nq) return c0;
    return max(c0, min(c1, attn_visible(A, S, *first, min(i0 + qpt, S.nq) - 1)));
  };
  auto reach_all = [&](int rg) -> int {
    int e = reach(rg, 0);
    for (int w = 1; w < tiles; ++w) e = max(e, reach(rg, w));
    return e;
  };
  // what the tokens [i0, i0 + n) see of keys behind their windows, the widest of it
  auto view_of = [&](int i0, int n) -> AttnView {
    if (!WIN) return {0, 0};
    const AttnView a = attn_view(A, S, *first, min(i0, S.nq - 1)), b = attn_view(A, S, *first, min(i0 + n, S.nq) - 1);
    return {b.seen, a.low};
  };
  auto view_group = [&](int rg) -> Steps { return Steps(view_of(rg * tiles * qpt, tiles * qpt)); };
  const AttnView view_seq = WIN && S.nq > 0 ? view_of(0, S.nq) : AttnView{0, 0};
  // whether a tile whose reach is e and whose rows' widest view is v has step t
  auto mine = [&](int t, int e, Steps v) -> bool { return t * kKeys < e && !(WIN && v.behind(t)); };
  // whether the step has value rows to zero: rows that no token of the sequence sees
  auto patched = [&](const Walk<WIN>& k) -> bool {
    if (WIN && k.t * kKeys < view_seq.low && k.t * kKeys + kKeys > view_seq.seen) return true;
    return k.partial || k.t * kKeys + kKeys > S.nk;
  };
  auto step_row = [&](int t) -> int { return WIN ? attn_row(S, t * kKeys) : S.kb + t * kKeys; };
  auto place = [](int g) { return g & (C::kRing - 1); };
  auto phase = [](int g) { return (uint32_t)(g / C::kRing) & 1u; };

  if (warp == kLoadK) {
    // ------------------------------------------ queries, keys, coordinates
    bool ok = !A.stall;
    uint32_t item = 0;
    int g = 0;
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups, ++item) {
      if (item > 0 && !(ok = wait(C::QFREE, (item - 1) & 1))) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(&bar[C::QFULL], tiles * C::NC * qpt * A.group * 128);
        for (int w = 0; w < tiles; ++w)
#pragma unroll
          for (int c = 0; c < C::NC; ++c)
            tma_load_3d(sq + (w * C::NC + c) * kQBox, &M.q, &bar[C::QFULL], c * 64, kvh * A.group,
                        S.q0 + (rg * tiles + w) * qpt);
      }
      __syncwarp();
      Walk<WIN> k(c0, reach_all(rg), c1, g, view_group(rg));
      for (k.settle(A, S, slots, all); k.live(); k.next(A, S, slots, all)) {
        const int p = place(k.g);
        float2 at[2];
        if (DIST) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            at[i] = *reinterpret_cast<const float2*>(
                A.k_pos + 2 * (long long)min(step_row(k.t) + i * 32 + lane, A.n_rows - 1));
        }
        if (!(ok = wait(C::FREE + p, phase(k.g) ^ 1))) break;
        if (DIST) {
          float* d = spos + p * 2 * kKeys + lane;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            d[i * 32] = at[i].x;
            d[kKeys + i * 32] = at[i].y;
          }
          __syncwarp();
        }
        if (lane == 0) {
          mbar_arrive_expect_tx(&bar[C::FULL + p], C::kStep);
#pragma unroll
          for (int c = 0; c < C::NC; ++c)
            tma_load_3d(sk + p * C::kStep + c * kBox, &M.k, &bar[C::FULL + p], c * 64, kvh, step_row(k.t));
        }
        __syncwarp();
      }
      g = k.g;
    }
    if (!ok) outlast_copies();
  } else if (warp == kLoadV) {
    // ------------------------------------------ values, and zeroes at edges
    bool ok = true;
    int g = 0;
    Walk<WIN> last;
    bool pending = false;
    auto patch = [&]() -> bool {                 // the step before, one behind the loads
      if (!pending || !patched(last)) return true;
      const int p = place(last.g);
      if (!wait(C::FULL + p, phase(last.g))) return false;
      const unsigned long long keep = key_mask<WIN>(A, S, slots, last.t * kKeys, S.nk, view_seq);
      for (int i = lane; i < kKeys; i += 32)
        if (!((keep >> i) & 1))
          for (int c = 0; c < C::NC; ++c)
            for (int u = 0; u < 8; ++u)
              *reinterpret_cast<uint4*>(sv + p * C::kStep + c * kBox + i * 128 + u * 16) = make_uint4(0u, 0u, 0u, 0u);
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[C::VOK + p]);
      return true;
    };
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups) {
      Walk<WIN> k(c0, reach_all(rg), c1, g, view_group(rg));
      for (k.settle(A, S, slots, all); k.live(); k.next(A, S, slots, all)) {
        // with a ring of one stream's steps the patch of the step before must not
        // wait behind this step's slot
        if (!(ok = patch())) break;
        const int p = place(k.g);
        if (!(ok = wait(C::FREE + p, phase(k.g) ^ 1))) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&bar[C::FULL + p], C::kStep);
#pragma unroll
          for (int c = 0; c < C::NC; ++c)
            tma_load_3d(sv + p * C::kStep + c * kBox, &M.v, &bar[C::FULL + p], c * 64, kvh, step_row(k.t));
        }
        __syncwarp();
        pending = true;
        last = k;
      }
      g = k.g;
    }
    if (ok) ok = patch();
    if (!ok) outlast_copies();
  } else if (warp >= kProduct) {
    // ---------------------------------------------------- products of a chain
    const int chain = __shfl_sync(0xFFFFFFFFu, warp - kProduct, 0), w = chain / streams, stream = chain & (streams - 1);
    constexpr uint32_t fmt = std::is_same<T, __nv_bfloat16>::value;
    constexpr uint32_t id_s = idesc_f16(128, kKeys, fmt);
    constexpr uint32_t id_o = idesc_f16(128, DP, fmt) | (1u << 16);      // B is MN-major
    constexpr uint64_t kStepUnits = C::kStep >> 4, kBoxUnits = kBox >> 4, kQBoxUnits = kQBox >> 4;
    const uint64_t dk = smem_desc(smem_u32(sk), 1024, 2), dv = desc_v(smem_u32(sv));
    const uint64_t dq = smem_desc(smem_u32(sq), 1024, 2) + w * C::NC * kQBoxUnits;
    bool ok = true;
    uint32_t item = 0, vok = 0;                  // bit p of vok: the patch phase of place p
    uint32_t n_qk = 0, n_pv = 0;                 // products issued
    int g = 0;
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups, ++item) {
      const int end = reach_all(rg), e = reach(rg, w);
      const Steps tile(view_of((rg * tiles + w) * qpt, qpt));
      Walk<WIN> qk(c0, end, c1, g, view_group(rg));
      qk.settle(A, S, slots, all);
      qk.seek(A, S, slots, all, streams, stream);
      Walk<WIN> pv = qk;
      bool begun = false;
      // S = Q K^T of the next step (its values are there as well)
      auto score = [&]() -> bool {
        if (!qk.live()) return true;
        const int p = place(qk.g);
        if (!wait(C::FULL + p, phase(qk.g))) return false;
        if (mine(qk.t, e, tile)) {
          tc_fence_after();
          const uint32_t s = chain * kS + (n_qk & (kS - 1));
          const uint64_t kd = dk + p * kStepUnits;
#pragma unroll
          for (int i = 0; i < C::NC; ++i)
            umma4_ss(tmem + s * kKeys, dq + i * kQBoxUnits, kd + i * kBoxUnits, id_s, i > 0);
          umma_commit_elected(&bar[C::SFULL + s]);
          // this warp has seen the step's coordinates: its arrival passes them on
          if (DIST && lane == 0) mbar_arrive(&bar[C::SFULL + s]);
          ++n_qk;
        }
        if (!WIN) qk.next_own(A, S, slots, all, streams, stream);
        return true;
      };
      // O += P V of the next step; keys and values are released when it is done
      auto value = [&]() -> bool {
        const int p = place(pv.g);
        const bool zeroed = patched(pv);
        if (mine(pv.t, e, tile)) {
          if (zeroed && !wait(C::VOK + p, (vok >> p) & 1)) return false;
          const uint32_t s = chain * kS + (n_pv & (kS - 1));
          if (!wait(C::PREADY + s, (n_pv / kS) & 1)) return false;
          tc_fence_after();
          umma4_ts(tmem + C::kO + chain * DP, tmem + s * kKeys, dv + p * kStepUnits, id_o, begun);
          umma_commit_elected(&bar[C::FREE + p]);
          umma_commit_elected(&bar[C::DONE + s]);
          ++n_pv;
          begun = true;
        } else if (lane == 0) {
          mbar_arrive(&bar[C::FREE + p]);
        }
        if (zeroed) vok ^= 1u << p;
        if (!WIN) pv.next_own(A, S, slots, all, streams, stream);
        return true;
      };
      ok = wait(C::QFULL, item & 1);
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        ok = ok && score();
        if (WIN) qk.next_own(A, S, slots, all, streams, stream);
      }
      // with a window both walks go on while the softmax works, not between its end and the
      // next products (packed, windows of 700: 231 -> 211 us; without, where a walk is an
      // addition, 16,384 x 49,152 keys took 1.5 % longer)
      while (ok && pv.live()) {
        ok = value() && score();
        if (WIN) {
          pv.next_own(A, S, slots, all, streams, stream);
          qk.next_own(A, S, slots, all, streams, stream);
        }
      }
      // the steps of the whole group, for the next group's places
      Walk<WIN> k(c0, end, c1, g, view_group(rg));
      if (rg + A.row_groups < groups)
        for (k.settle(A, S, slots, all); k.live(); k.next(A, S, slots, all)) {
        }
      g = k.g;
      if (ok) umma_commit_elected(&bar[C::QFREE]);
      __syncwarp();
    }
    // no product may still run when tensor memory is freed
    umma_commit_elected(&bar[C::DRAIN + chain]);
    if (!mbar_wait(&bar[C::DRAIN + chain], 0, A.budget)) atomicAdd(&g_attn_err, 1u);
    __syncwarp();
  } else {
    // -------------------------------------------------------------- softmax
    const int chain = warp >> 2, r = tid & 127, w = chain / streams, stream = chain & (streams - 1);
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts0 = tmem + chain * kS * kKeys + lanes, to = tmem + C::kO + chain * DP + lanes;
    uint32_t n = 0;                              // steps of this chain since the block began
    int g = 0;
    bool ok = true;
    // The barrier of step i's product, and its phase: two by turns, since a product
    // may lag two steps.
    auto done = [&](uint32_t i) -> int { return C::DONE + chain * kS + (i & (kS - 1)); };
    auto phase_s = [](uint32_t i) -> uint32_t { return (i / kS) & 1; };
    for (int rg = rg0; rg < groups && ok; rg += A.row_groups) {
      const int i0 = (rg * tiles + w) * qpt;
      const int ql = i0 + r / A.group;
      const bool valid = r < qpt * A.group && ql < S.nq;
      const int head = kvh * A.group + r % A.group;
      const long long tok = S.q0 + min(ql, S.nq - 1);        // a row without a token computes nothing
      const int place0 = *first;
      const int hi = valid ? min(c1, attn_visible(A, S, place0, ql)) : 0;
      const AttnView view = WIN ? attn_view(A, S, place0, min(ql, S.nq - 1)) : AttnView{0, 0};
      const AttnView see_all = WIN ? AttnView{attn_view(A, S, place0, min(i0, S.nq - 1)).seen,
                                              attn_view(A, S, place0, min(i0 + qpt, S.nq) - 1).low}
                                   : AttnView{0, 0};
      const int all_see = i0 < S.nq ? min(c1, attn_visible(A, S, place0, i0)) : 0;   // every row sees the keys before this
      float qy = 0.f, qx = 0.f, slope = 0.f;
      if (DIST) {
        qy = -A.q_pos[tok * A.q_pos_row];
        qx = -A.q_pos[tok * A.q_pos_row + 1];
        slope = -A.slopes[head] * kLog2e;
      }
      float m = -INFINITY, l = 0.f, late = 0.f;  // late: what m has to go up by, if P passed the slack
      bool begun = false, lagging = false;       // for the warp: all its rows have an m; some row's `late` is not 0
      const int e = reach(rg, w);
      Walk<WIN> k(c0, reach_all(rg), c1, g, view_group(rg));
      k.settle(A, S, slots, all);
      k.seek(A, S, slots, all, streams, stream);
      const Steps tile(view_of(i0, qpt));
      auto skip = [&]() {                        // other tiles' steps
        while (k.live() && !mine(k.t, e, tile)) k.next_own(A, S, slots, all, streams, stream);
      };
      skip();
      const uint32_t n0 = n;
      // Rows' maxima go up by `up`: O and the sum so far are scaled down, once the
      // product before is done with O.
      auto rise = [&](float up) -> bool {
        if (n > n0) {
          if (!wait(done(n - 1), phase_s(n - 1))) return false;
          tc_fence_after();
          const float f = ex2(-up);
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
        }
        return true;
      };
      // S of the next step is there; maxima that lag behind are raised first
      auto begin = [&]() -> bool {
        if (!wait(C::SFULL + chain * kS + (n & (kS - 1)), phase_s(n))) return false;
        tc_fence_after();
        if (lagging) {
          if (!rise(late)) return false;
          l *= ex2(-late);
          m += late;
          late = 0.f;
          lagging = false;
        }
        return true;
      };
      // P of the step is complete
      auto publish = [&]() {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[C::PREADY + chain * kS + (n & (kS - 1))]);
        ++n;
        k.next_own(A, S, slots, all, streams, stream);
        if (WIN) skip();                         // else they are all ahead of the first own one
      };
      while (k.live()) {
        const bool edge = k.partial || k.t * kKeys + kKeys > all_see ||
                          (WIN && k.t * kKeys < see_all.low && k.t * kKeys + kKeys > see_all.seen);
        if (begun && !edge && (!CAP || poly.limit > 0.f)) {
          // going back, no further step is at the edge unless a slot is absent
          int run = all ? (k.t - (WIN && k.t * kKeys >= see_all.low ? max(k.t0, (see_all.low + kKeys - 1) / kKeys) : k.t0)) / streams + 1 : 1;
          bool slow = false;
          do {
            const uint32_t ts = ts0 + (n & (kS - 1)) * kKeys;
            const float* py = spos + place(k.g) * 2 * kKeys;
            if (!(ok = begin())) break;
            // one pass with the maximum as it is: z = score (log2 units) - m, p = exp2(z)
            float2 x2[kKeys / 2];
            float* x = reinterpret_cast<float*>(x2);
            // the second half comes while the first is worked on where that takes longest
            // (cap and bias: 4 % faster; the bias alone would be 4 % slower)
            constexpr bool kHalves = CAP && DIST;
            tmem_ld32_issue(ts, x);
            if (!kHalves) tmem_ld32_issue(ts + 32, x + 32);
            tmem_ld_wait();
            reg_fence32(x);
            if (!kHalves) reg_fence32(x + 32);
            if (kHalves) tmem_ld32_issue(ts + 32, x + 32);
            float b0 = 0.f, t0 = -INFINITY, t1 = -INFINITY;
            float2 s0 = both(0.f), s1 = both(0.f);
            uint32_t pk[kKeys / 2];
            constexpr int G = DIST ? 4 : 8;      // pairs abreast
#pragma unroll
            for (int ii = 0; ii < kKeys / 2 + 2 * G; ii += G) {
              // group ii's scores, the exponentials of the group before, and the sums
              // and packing of the one before that: each waits on nothing recent
              if (kHalves && ii == kKeys / 4) {
                tmem_ld_wait();
                reg_fence32(x + 32);
              }
              if (ii < kKeys / 2) {
                const int i = ii;
                float2 a[G];                       // what is added to the capped score
#pragma unroll
                for (int u = 0; u < G; ++u) a[u] = both(-m);
                if (DIST) {
                  float2 y[G], d[G];
#pragma unroll
                  for (int u = 0; u < G; u += 2) {
                    const float4 ky = *reinterpret_cast<const float4*>(py + 2 * (i + u));
                    const float4 kx = *reinterpret_cast<const float4*>(py + kKeys + 2 * (i + u));
                    y[u] = make_float2(ky.x, ky.y);
                    y[u + 1] = make_float2(ky.z, ky.w);
                    d[u] = make_float2(kx.x, kx.y);
                    d[u + 1] = make_float2(kx.z, kx.w);
                  }
#pragma unroll
                  for (int u = 0; u < G; ++u) {
                    y[u] = add2(y[u], both(qy));
                    d[u] = add2(d[u], both(qx));
                  }
#pragma unroll
                  for (int u = 0; u < G; ++u)
                    y[u] = make_float2(fabsf(y[u].x) + fabsf(d[u].x), fabsf(y[u].y) + fabsf(d[u].y));
#pragma unroll
                  for (int u = 0; u < G; ++u) a[u] = fma2(y[u], both(slope), a[u]);
                }
                if (!CAP) {
#pragma unroll
                  for (int u = 0; u < G; ++u) x2[i + u] = fma2(x2[i + u], both(A.scale_log2), a[u]);
                } else {
                  // an odd polynomial: |error| <= 2e-7 cap for scaled |x| <= cap / 2
                  float2 w2[G], p[G];
#pragma unroll
                  for (int u = 0; u < G; ++u) {
                    b0 = fmaxf(b0, fmaxf(fabsf(x2[i + u].x), fabsf(x2[i + u].y)));
                    w2[u] = mul2(x2[i + u], x2[i + u]);
                  }
#pragma unroll
                  for (int u = 0; u < G; ++u) p[u] = fma2(w2[u], both(poly.c[3]), both(poly.c[2]));
#pragma unroll
                  for (int u = 0; u < G; ++u) p[u] = fma2(w2[u], p[u], both(poly.c[1]));
#pragma unroll
                  for (int u = 0; u < G; ++u) p[u] = fma2(w2[u], p[u], both(poly.c[0]));
#pragma unroll
                  for (int u = 0; u < G; ++u) x2[i + u] = fma2(x2[i + u], p[u], a[u]);
                }
              }
              if (ii >= G && ii < kKeys / 2 + G) {
#pragma unroll
                for (int u = 0; u < G; ++u) {
                  float2& z = x2[ii - G + u];
                  (u & 1 ? t1 : t0) = fmaxf(u & 1 ? t1 : t0, fmaxf(z.x, z.y));
                  z = make_float2(ex2(z.x), ex2(z.y));
                }
              }
              if (ii >= 2 * G) {
#pragma unroll
                for (int u = 0; u < G; ++u) {
                  const float2 z = x2[ii - 2 * G + u];
                  if (u & 1) s1 = add2(s1, z);
                  else s0 = add2(s0, z);
                  pk[ii - 2 * G + u] = Store<T>::pack2(z.x, z.y);      // the probabilities as the product takes them
                }
              }
            }
            const float top = fmaxf(t0, t1);
            if (__any_sync(0xFFFFFFFFu, valid && ((CAP && !(b0 <= poly.limit)) || top > kSlack<T>))) {
              // too large for the polynomial, or for P; or m lags behind from here on
              slow = __any_sync(0xFFFFFFFFu, valid && ((CAP && !(b0 <= poly.limit)) || top > kHard));
              if (slow) break;
              if (valid && top > kSlack<T>) late = fmaxf(late, top - kLift<T>);
              lagging = true;
            }
            l += (s0.x + s0.y) + (s1.x + s1.y);
            tmem_st32(ts, pk);
            publish();
          } while (--run > 0);
          if (!ok) break;
          if (!slow) continue;
        } else if (!(ok = begin())) {
          break;
        } else if (WIN && !CAP && !DIST && begun) {
          // an edge of windows, which are many: one pass with the maximum as it is, as above,
          // without its order (the form below took 2 us longer a step)
          const uint32_t ts = ts0 + (n & (kS - 1)) * kKeys;
          const unsigned long long keep = key_mask<WIN>(A, S, slots, k.t * kKeys, hi, view);
          const uint32_t bits[2] = {(uint32_t)keep, (uint32_t)(keep >> 32)};
          float x[kKeys];
          tmem_ld32_issue(ts, x);
          tmem_ld32_issue(ts + 32, x + 32);
          tmem_ld_wait();
          reg_fence32(x);
          reg_fence32(x + 32);
          float t0 = -INFINITY, t1 = -INFINITY;
          float2 s0 = both(0.f);
          uint32_t pk[kKeys / 2];
#pragma unroll
          for (int i = 0; i < kKeys; i += 2) {
            float2 z = fma2(make_float2(x[i], x[i + 1]), both(A.scale_log2), both(-m));
            if (!(bits[i / 32] >> (i & 31) & 1)) z.x = -INFINITY;
            if (!(bits[i / 32] >> ((i + 1) & 31) & 1)) z.y = -INFINITY;
            t0 = fmaxf(t0, z.x);
            t1 = fmaxf(t1, z.y);
            z = make_float2(ex2(z.x), ex2(z.y));
            s0 = add2(s0, z);
            pk[i / 2] = Store<T>::pack2(z.x, z.y);
          }
          const float top = fmaxf(t0, t1);
          if (!__any_sync(0xFFFFFFFFu, valid && top > kHard)) {
            if (__any_sync(0xFFFFFFFFu, valid && top > kSlack<T>)) {
              if (valid && top > kSlack<T>) late = fmaxf(late, top - kLift<T>);
              lagging = true;
            }
            l += s0.x + s0.y;
            tmem_st32(ts, pk);
            publish();
            continue;
          }
        }
        const uint32_t ts = ts0 + (n & (kS - 1)) * kKeys;
        const float* py = spos + place(k.g) * 2 * kKeys;
        // 32 keys at a time, with tanh itself, masks, and maxima that move at once
        const unsigned long long keep = edge ? key_mask<WIN>(A, S, slots, k.t * kKeys, hi, view) : ~0ull;
#pragma unroll 1
        for (int c = 0; c < kKeys; c += 32) {
          const float m0 = m == -INFINITY ? 0.f : m;
          float y[32];
          tmem_ld32_issue(ts + c, y);
          tmem_ld_wait();
          reg_fence32(y);
          const uint32_t bits = (uint32_t)(keep >> c);
          float top = -INFINITY;
          // as in attn_rows.cu; behind windows of a few keys only, as it takes packed windows of
          // 700 keys 8 % longer
          const bool far_cap = CAP && (A.cap_log2 > kAbsCap * kLog2e || (WIN && A.window > 0 && A.window <= kKeys));
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            y[i] *= A.scale_log2;
            if (CAP) y[i] = A.cap_log2 * (far_cap ? tanh_rel(y[i]) : tanh_abs(y[i]));
            if (DIST) y[i] = fmaf(fabsf(py[c + i] + qy) + fabsf(py[kKeys + c + i] + qx), slope, y[i]);
            y[i] = (bits >> i) & 1 ? y[i] - m0 : -INFINITY;
            top = fmaxf(top, y[i]);
          }
          // from nothing at once, later past the slack and by whole powers of two: the
          // probabilities that this step has rounded already are scaled exactly
          const float rest = top - kLift<T>;
          const float up = m == -INFINITY ? (top > -INFINITY ? rest : 0.f) : top > kSlack<T> ? ceilf(rest) : 0.f;
          if (__any_sync(0xFFFFFFFFu, up != 0.f && l > 0.f)) {
            const float f = l > 0.f ? up : 0.f;
            if (!(ok = rise(f))) break;
            l *= ex2(-f);
            if (c > 0) {                     // this step's probabilities so far
              uint32_t u[16];
#pragma unroll 1
              for (int i = 0; i < c / 2; i += 16) {
                tmem_ld16_issue(ts + i, u);
                tmem_ld_wait();
                tmem_reg_fence(u);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  const float2 v = Store<T>::unpack2(u[j]);
                  u[j] = Store<T>::pack2(v.x * ex2(-f), v.y * ex2(-f));
                }
                tmem_st16(ts + i, u);
              }
            }
          }
          if (m != -INFINITY) {
            m += up;
            late = fmaxf(late - up, 0.f);
          } else if (top > -INFINITY) {
            m = up;
          }
          uint32_t pk[16];
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float v0 = ex2(y[i] - up), v1 = ex2(y[i + 1] - up);
            sum += v0 + v1;
            pk[i / 2] = Store<T>::pack2(v0, v1);
          }
          l += sum;
          tmem_st16(ts + c / 2, pk);
          tmem_st_wait();
          if (l != l && m == -INFINITY) m = 0.f;         // a NaN row never gets a maximum: it is done with
        }
        if (!ok) break;
        begun = !__any_sync(0xFFFFFFFFu, valid && m == -INFINITY);
        lagging = __any_sync(0xFFFFFFFFu, late > 0.f);
        publish();
      }
      if (!ok) break;
      // the steps of the whole group, for the next group's places
      if (rg + A.row_groups < groups) {
        Walk<WIN> a(c0, reach_all(rg), c1, g, view_group(rg));
        for (a.settle(A, S, slots, all); a.live(); a.next(A, S, slots, all)) {
        }
        g = a.g;
      }
      // ---- out = O / l
      const long long R = tok * A.heads + head;
      const bool any = n > n0;
      if (any) {
        if (!(ok = wait(done(n - 1), phase_s(n - 1)))) break;
        tc_fence_after();
      }
      const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
      const bool split = A.n_chunks * streams > 1;
      const long long at = (long long)(chunk * streams + stream) * A.n_q * A.heads + R;
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
            if (c + 32 <= A.dim && (reinterpret_cast<uintptr_t>(dst) & 31) == 0) {
              // whole sectors: a thread's row is far from its neighbours', so halves cost as much
              uint32_t u[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) u[i] = Store<T>::pack2(o[2 * i] * inv, o[2 * i + 1] * inv);
              st_global32(dst, u);
              st_global32(dst + 16, u + 8);
            } else
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
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kProduct) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <typename T, int DP, bool WIN>
cudaError_t launch_tc_t(const AttnArgs& a, const TcMaps& m, cudaStream_t st) {
  // tanh(u) / u on |u| <= 1/2 in w = u^2, least largest |error| of u p(w): 1.4e-7, and
  // up to 2e-7 as float32 computes it
  constexpr double kTanh[4] = {0.9999974621104636, -0.3331988899884361, 0.13138806507278963,
                                -0.04322690737438131};
  TanhPoly poly{};
  if (a.cap_log2 > 0.f) {
    double f = (double)a.cap_log2 * a.scale_log2;
    for (int i = 0; i < 4; ++i, f *= (double)a.scale_log2 * a.scale_log2) poly.c[i] = (float)(f * kTanh[i]);
    const float limit = fabsf(0.5f / a.scale_log2), c3 = fabsf(poly.c[3]);
    const bool range = c3 >= FLT_MIN && c3 <= FLT_MAX && limit * limit <= FLT_MAX;
    poly.limit = range && a.cap_log2 <= kAbsCap * kLog2e ? limit : 0.f;
  }
  const bool cap = a.cap_log2 > 0.f, dist = a.slopes != nullptr;
  auto kern = cap ? (dist ? k_attn_tc<T, DP, true, true, WIN> : k_attn_tc<T, DP, true, false, WIN>)
                  : (dist ? k_attn_tc<T, DP, false, true, WIN> : k_attn_tc<T, DP, false, false, WIN>);
  static std::atomic<uint64_t> allowed[4];
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), TcCfg<DP>::kSmem, &allowed[2 * cap + dist]);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)((long long)a.n_seqs * a.kv_heads * a.n_chunks * a.row_groups));
  lc.blockDim = dim3(kWarps * 32);
  lc.dynamicSmemBytes = TcCfg<DP>::kSmem;
  lc.stream = st;
  return cudaLaunchKernelEx(&lc, kern, a, m, poly);
}

// cudaErrorNotSupported where the arrays cannot be described to the TMA unit
// (a zero stride over more than one head or row, or one of 2^40 bytes or more).
template <bool WIN>
cudaError_t launch_tc(const AttnArgs& a, bool bf16, cudaStream_t st) {
  TcMaps m;
  const int box_q = 128 / a.group;
  if (tmap_rows(&m.q, a.q, bf16, a.dim, a.heads, a.n_q, a.q_head, a.q_row, a.group, box_q) != cudaSuccess ||
      tmap_rows(&m.k, a.k, bf16, a.dim, a.kv_heads, a.n_rows, a.k_head, a.k_row, 1, kKeys) != cudaSuccess ||
      tmap_rows(&m.v, a.v, bf16, a.dim, a.kv_heads, a.n_rows, a.v_head, a.v_row, 1, kKeys) != cudaSuccess)
    return cudaErrorNotSupported;
  if (a.dim <= 64) return bf16 ? launch_tc_t<__nv_bfloat16, 64, WIN>(a, m, st) : launch_tc_t<__half, 64, WIN>(a, m, st);
  return bf16 ? launch_tc_t<__nv_bfloat16, 128, WIN>(a, m, st) : launch_tc_t<__half, 128, WIN>(a, m, st);
}

cudaError_t tc_errors(unsigned* count, cudaStream_t st) {
  void* p = nullptr;
  cudaError_t e = cudaGetSymbolAddress(&p, g_attn_err);
  if (e == cudaSuccess) e = cudaMemcpyAsync(count, p, sizeof(*count), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  return e;
}

}  // namespace
}  // namespace rtcc
