// Shared by the operators of the paged token memory: the shapes of pools and
// tables as the kernels take them.
#pragma once

#include "common.cuh"
#include "rtcc.h"

namespace rtcc {

constexpr int kPageBlock = 16;                   // places that share an exponent
constexpr int kExpMin = -120, kExpMax = 120;

struct PageShape {
  long long page_bytes, scale_bytes;             // from page to page
  int kv_heads, dim, page_rows, shift;           // page_rows = 1 << shift
  int n_pages, n_seqs, table_row;
};

// A pool as attention reads it.
struct PagesArgs {
  const int* table;
  const unsigned char *k, *v;
  const signed char* scales;
  PageShape s;
};

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Two e4m3 numbers (bits 0..15 of v) as two fp16 ones, exactly.
__device__ __forceinline__ uint32_t widen_e4m3x2(uint32_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)v));
  return h;
}

// Whether cfg is valid; if so, the shapes with strides filled in (pages.cu).
bool page_shape(const rtcc_page_config* cfg, PageShape* out);

}  // namespace rtcc
