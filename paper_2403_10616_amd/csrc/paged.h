// The paged cache of keys and values, and the rows of new tokens that are read from and attend to it.
//
// cache: [n_pages][2][H_kv][page_size][dh], keys then values; position p of document b sits in page pages[b * pages_per_doc + p /
// page_size], slot p % page_size.  A head's share of a page is contiguous: page_size x dh elements, 2 KB for 16 positions of 64 bf16.
#pragma once
#include "visible.h"

namespace dipaco {

template <typename T> struct PagedArgs {
  const T* qkv;              // [T rows, (H + 2 H_kv) dh]
  const int* row_start;      // [B + 1]
  const int* cache_len;      // [B]
  const int* pages;          // [B, pages_per_doc]
  T* cache;
  T* o;                      // [T rows, H dh]
  float* lse;                // [T rows, H], or null
  int T_rows, B, max_new, H, H_kv, n_pages, page_shift, pages_per_doc;
  Window w;

  __device__ __forceinline__ int capacity() const { return pages_per_doc << page_shift; }
  __device__ __forceinline__ int cached(int b) const { return min(max(cache_len[b], 0), capacity()); }
  // the page of a position, or -1 where the table holds none
  __device__ __forceinline__ int page_of(int b, int pos) const {
    const int at = pos >> page_shift;
    if (at >= pages_per_doc) return -1;
    const int p = pages[(long)b * pages_per_doc + at];
    return (unsigned)p < (unsigned)n_pages ? p : -1;
  }
  template <int DH> __device__ __forceinline__ long key_offset(int page, int hk, int slot) const {
    return ((((long)page * 2 * H_kv + hk) << page_shift) + slot) * DH;
  }
  template <int DH> __device__ __forceinline__ long value_from_key() const { return ((long)H_kv << page_shift) * DH; }
};

}  // namespace dipaco
