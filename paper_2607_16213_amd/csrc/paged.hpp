// A cache in pages as the kernels see it, and the lengths of its sequences.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace selkv {

// Length and number of new rows or nodes of sequence b; false: it takes no part.
__device__ __forceinline__ bool sequence_of(const Seqs& s, uint32_t b, int& len, int& count) {
  len = s.lens ? s.lens[b] : s.cache_len;
  count = s.counts ? s.counts[b] : s.n;
  return (uint32_t)len <= (uint32_t)s.cache_len && (uint32_t)count <= (uint32_t)s.n;
}

// Page of an entry, -1 where there is none.
__device__ __forceinline__ int page_of(const Paged& c, uint32_t b, int entry) {
  const int column = entry >> c.shift;
  if (column >= c.columns) return -1;
  const int page = c.table[(size_t)b * c.columns + column];
  return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

// Index of an entry's row in the pools (of its bias in theirs).
__device__ __forceinline__ size_t row_of(const Paged& c, int hkv, int page, int head, int entry) {
  return ((((size_t)page * hkv + head)) << c.shift) + (entry & ((1 << c.shift) - 1));
}

}  // namespace selkv
