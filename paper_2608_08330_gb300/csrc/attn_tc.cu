// The tensor-core attention of attn_tc.cuh without windows, and its host side.
#include "attn_tc.cuh"

namespace rtcc {

// Streams: two chains share a tile where that leaves fewer of them idle (300 rows
// are 3 tiles: 3 blocks of half the steps each instead of 2 of all).
int attn_tc_streams(int group, int max_q) { return (max_q + 128 / group - 1) / (128 / group) % 2 ? 2 : 1; }
int attn_tc_tokens_per_block(int group, int streams) { return kChains / streams * (128 / group); }
int attn_tc_unit(int streams) { return kKeys * streams; }

cudaError_t launch_attn_tc(const AttnArgs& a, bool bf16, cudaStream_t st) {
  return a.window > 0 || a.span_rows > 0 ? launch_attn_win(a, bf16, st) : launch_tc<false>(a, bf16, st);
}

cudaError_t attn_tc_errors(unsigned* count, cudaStream_t st) {
  unsigned more = 0;
  cudaError_t e = tc_errors(count, st);
  if (e == cudaSuccess) e = attn_win_errors(&more, st);
  *count += more;
  return e;
}

}  // namespace rtcc
