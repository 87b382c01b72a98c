// The cache rows of a path through a tree of drafted tokens move behind the positions that were cached before: slot L + i takes the keys and values
// of slot L + path[i], in every layer and head.
//
// In place: path rises strictly, so a row's place lies in front of its source, and no place of an earlier row is the source of a later one.  A wave moves
// the rows of one layer, document and head in order, as many at a time as its lanes hold; those it has read before it writes may be the places of others.
#include <algorithm>

#include "draft.h"
#include "kernels.h"

namespace dipaco {

namespace {

__global__ void __launch_bounds__(256) cache_keep_rows(KeepArgs a, int first) {
  const int lane = threadIdx.x & 63, kh = blockIdx.y * 4 + (threadIdx.x >> 6), layer = blockIdx.z;
  const int b = first + blockIdx.x;
  if (kh >= 2 * a.H_kv) return;   // keys' heads, then values'
  const int* const path = a.path + (long)b * a.max_new;
  const int kept = min(max(a.kept[b], 0), a.max_new), cached = min(max(a.cache_len[b], 0), 0x7f000000);
  const int* const pages = a.pages + (long)b * a.pages_per_doc;
  uint4* const cache = a.cache[layer];
  auto row_of = [&](int pos) -> long {   // where the row of a position begins, -1 where the table has no page for it
    const int at = pos >> a.page_shift;
    const int page = at < a.pages_per_doc ? pages[at] : -1;
    if ((unsigned)page >= (unsigned)a.n_pages) return -1;
    return ((((long)page * 2 * a.H_kv + kh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) * a.row_vecs;
  };
  const int rows = 64 / a.row_vecs;   // at a time
  const int sub = lane / a.row_vecs, col = lane % a.row_vecs;
  int before = -1;                    // the path's last row so far
  for (int i0 = 0; i0 < kept; i0 += rows) {
    const int i = i0 + sub;
    const int from = i < kept && sub < rows ? path[i] : -1;
    int left = __shfl_up(from, a.row_vecs, WAVE);
    if (sub == 0) left = before;
    const bool rises = from > left && from < a.max_new;
    // rows from the first one on that does not rise are no path
    const unsigned long long bad = __builtin_amdgcn_ballot_w64(!rises && i < kept && sub < rows);
    const int good = bad ? __builtin_ctzll(bad) / a.row_vecs : rows;
    long to = -1, src = -1;
    if (sub < good && i < kept && from != i) {
      to = row_of(cached + i);
      src = row_of(cached + from);
    }
    if (to >= 0 && src >= 0) cache[to + col] = cache[src + col];   // the wave's reads come first: the store waits for them
    if (bad) break;
    before = __shfl(from, (rows - 1) * a.row_vecs, WAVE);
  }
}

}  // namespace

dipaco_status launch_cache_keep(KeepArgs a, void* const* caches, int n_layers, hipStream_t s) {
  for (int l0 = 0; l0 < n_layers; l0 += KEEP_MOST_LAYERS) {
    const int layers = std::min(n_layers - l0, KEEP_MOST_LAYERS);
    for (int l = 0; l < layers; ++l) a.cache[l] = static_cast<uint4*>(caches[l0 + l]);
    const int groups = (2 * a.H_kv + 3) / 4, most = (1 << 23) / (groups * layers);   // documents of a launch: H_kv < 2^15, so eight at least
    for (int b = 0; b < a.B; b += most) {
      cache_keep_rows<<<dim3(std::min(a.B - b, most), groups, layers), 256, 0, s>>>(a, b);
      DIPACO_LAUNCH_CHECK();
    }
  }
  return DIPACO_OK;
}

}  // namespace dipaco
