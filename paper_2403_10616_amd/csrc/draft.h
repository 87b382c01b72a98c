// Drafted decoding: a document's new rows are a tree.  Row 0 is the last token that is certain; every other row is a drafted token whose parent is
// an earlier row of the document.
#pragma once
#include "visible.h"

namespace dipaco {

constexpr int DRAFT_MOST_ROWS = 1024;   // of a document
constexpr int draft_words(int max_new) { return (max_new + 63) / 64; }
// the parent of row i, or -1 for a root: what is no earlier row is none
__device__ __forceinline__ int draft_parent(int given, int i) { return given >= 0 && given < i ? given : -1; }

template <typename T> struct VerifyArgs {
  const T *target, *draft;   // [T rows, V] scores; draft: or null
  const int *tokens, *parent, *row_start;
  const float *u, *v;        // [T rows], [B]
  int *path, *kept, *next;   // [B, max_new], [B], [B]
  int T_rows, B, max_new, V;
  double rate, draft_rate;   // log2(e) / temperature; 0: all probability at the first maximum
  int distinct;
  double* rest;              // [B, V]: what a document's walk has left of the target's row; other parts of the workspace follow
};

constexpr int KEEP_MOST_LAYERS = 64;   // of a launch
struct KeepArgs {
  const int *path, *kept, *cache_len, *pages;
  int B, max_new, H_kv, n_pages, page_shift, pages_per_doc, row_vecs;   // row_vecs: 16-byte vectors of a head's row
  uint4* cache[KEEP_MOST_LAYERS];
};

}  // namespace dipaco
