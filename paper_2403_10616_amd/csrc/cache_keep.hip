// The cache rows of a path through a tree of drafted tokens move behind the positions that were cached before: slot L + i takes the keys and values
// of slot L + path[i], in every layer and head.
//
// In place: path rises strictly, so a row's place lies in front of its source, and no place of an earlier row is the source of a later one.  A wave moves
// the rows of one layer, document and head in order, four loads of them ahead of their stores; those it has read before it writes may be the places of others.
//
// Bound by latency (kept, the path, pages, rows) and, with more waves than the chip holds, by how often that is paid: 12 layers of one document, 14 heads of 64, 6 rows,
// 3.5 us; 24 layers of 64 documents of up to 60 rows, 8 heads of 128, 57 MB read and written, 16 us (28 with one load at a time).
#include <algorithm>

#include "draft.h"
#include "kernels.h"

namespace dipaco {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));   // an array of HIP's own uint4 is kept in LDS

__global__ void __launch_bounds__(256) cache_keep_rows(KeepArgs a, int first) {
  const int lane = threadIdx.x & 63, kh = blockIdx.y * 4 + (threadIdx.x >> 6), layer = blockIdx.z;
  const int b = first + blockIdx.x;
  if (kh >= 2 * a.H_kv) return;   // keys' heads, then values'
  const int* const path = a.path + (long)b * a.max_new;
  const int kept = min(max(a.kept[b], 0), a.max_new), cached = min(max(a.cache_len[b], 0), 0x7f000000);
  const int* const pages = a.pages + (long)b * a.pages_per_doc;
  u32x4* const cache = reinterpret_cast<u32x4*>(a.cache[layer]);
  // Where the row of a position begins, -1 where the table has no page for it.  No load hangs on a branch: behind one the compiler waits for each by itself.
  auto page_of = [&](int pos) { return pages[min(pos >> a.page_shift, a.pages_per_doc - 1)]; };
  auto row_of = [&](int pos, int page) -> long {
    const long row = ((((long)page * 2 * a.H_kv + kh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) * a.row_vecs;
    return (unsigned)page < (unsigned)a.n_pages && pos >> a.page_shift < a.pages_per_doc ? row : -1;
  };
  constexpr int AHEAD = 4;
  const int rows = 64 / a.row_vecs, sub = lane / a.row_vecs, col = lane % a.row_vecs;   // rows a load or store
  int before = -1;                                                                    // the path's last row so far
  for (int i0 = 0; i0 < kept; i0 += 64) {
    // a row a lane: where it is and where it goes
    const int i = i0 + lane, from = i < kept ? path[i] : -1;
    int left = __shfl_up(from, 1, WAVE);
    if (lane == 0) left = before;
    const unsigned long long bad = __builtin_amdgcn_ballot_w64(i < kept && (from <= left || from >= a.max_new));
    const int n = min(bad ? __builtin_ctzll(bad) : 64, kept - i0);   // rows from the first one on that does not rise are no path
    const int to_page = page_of(cached + i), src_page = page_of(cached + max(from, 0));
    long to = row_of(cached + i, to_page), src = row_of(cached + max(from, 0), src_page);
    if (lane >= n || from == i || src < 0) to = -1;
    if (to < 0) src = 0;
    for (int r0 = 0; r0 < n; r0 += AHEAD * rows) {
      u32x4 v[AHEAD];
      long at[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int r = r0 + j * rows + sub;
        at[j] = __shfl(to, r & 63, WAVE);
        const long s = __shfl(src, r & 63, WAVE);   // 0 where nothing moves
        if (r >= n) at[j] = -1;
        v[j] = cache[s + col];
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (at[j] >= 0) cache[at[j] + col] = v[j];
    }
    if (bad) break;
    before = __shfl(from, 63, WAVE);
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
