// Addresses inside a paged cache (layouts in goose.h).  Device code only (included by .hip files).
#pragma once
#include "goose_internal.h"

// Element offsets inside one head's part of a page, slot s < 64: chunk ch = column / 8 of a key row (8 elements), one value element.
template <int D>
static __device__ __forceinline__ int page_k_chunk(int s, int ch) {
  const int kk = s & 31, i = (((kk >> 2) & 3) << 3) | ((kk >> 4) << 2) | (kk & 3);
  return (((s >> 5) * (D / 16) + (ch >> 1)) * 64 + i + 32 * (ch & 1)) * 8;
}
template <int D>
static __device__ __forceinline__ int page_v_elem(int s, int c) {
  const int kk = s & 31;
  return ((((s >> 5) * (D / 32) + (c >> 5)) * 2 + ((kk >> 3) & 1)) * 64 + (c & 31) + 32 * (kk >> 4)) * 8 + (kk & 7);
}
// First element of (page, kv head) in a layer's part of a pool.
template <int D>
static __device__ __forceinline__ size_t page_head(int page, int n_kv, int kvh) {
  return ((size_t)page * n_kv + kvh) * (GOOSE_PAGE * D);
}
