// The paged cache as the kernels see it (layout and meaning: include/fathom.h).
#pragma once

#include "common.hpp"

namespace fathom {

constexpr int kMaxSeqs = FATHOM_MAX_SEQS;
// Positions of a request at most: those of some blocks behind the last are still 32-bit numbers.
constexpr int64_t kMaxTokens = 0x7fffffff - 1023;

// Pages with the block tables of a call's requests.  page = 1 << shift.
struct Paged {
  const uint16_t *K, *V;
  int H, shift;
  int32_t P;
  int64_t ld_page, ld_head, ld_tok;
  const int32_t* table;
  int64_t ld_table;
};

__device__ __forceinline__ float bf16_bits_to_float(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }

// Entry i of request s's table (every caller bounds i by the request's pages).
__device__ __forceinline__ int32_t page_of(const Paged& c, int s, int64_t i) {
  return ((const __attribute__((address_space(1))) int32_t*)c.table)[(int64_t)s * c.ld_table + i];
}

// Element offset of head h's row `tok` of request s; -1 for a page outside the pool.
__device__ __forceinline__ int64_t row_offset(const Paged& c, int s, int h, int64_t tok, uint32_t& flags) {
  const int32_t p = page_of(c, s, tok >> c.shift);
  if ((uint32_t)p >= (uint32_t)c.P) {
    flags |= FATHOM_DEV_BAD_PAGE;
    return -1;
  }
  return (int64_t)p * c.ld_page + (int64_t)h * c.ld_head + (tok & ((1 << c.shift) - 1)) * c.ld_tok;
}

}  // namespace fathom
