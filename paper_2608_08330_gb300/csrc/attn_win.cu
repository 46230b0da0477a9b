// The tensor-core attention of attn_tc.cuh with sliding windows, and over keys that
// were widened from pages.
#include "attn_tc.cuh"

namespace rtcc {

cudaError_t launch_attn_win(const AttnArgs& a, bool bf16, cudaStream_t st) { return launch_tc<true>(a, bf16, st); }

cudaError_t attn_win_errors(unsigned* count, cudaStream_t st) { return tc_errors(count, st); }

}  // namespace rtcc
