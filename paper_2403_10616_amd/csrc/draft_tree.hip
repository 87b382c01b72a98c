// What rows of a tree of drafted tokens see: themselves and their ancestors, as bits, and how many ancestors that are.
//
// A thread holds a row; its bits and the row that they reach up to lie in LDS.  A round joins to a row's bits those of the row that they reach, which
// doubles their reach: ceil(log2(depth + 1)) rounds whatever the tree's shape, where following parents one by one takes a chain's length.
// Bound by latency: the rows' bounds, the parents, then rounds of an LDS read, two barriers and a write.  One document of 16 rows 1.8 us, 256 of up to 500, chains
// among them, 12 (13.8 with every word of every row and stores a row a lane).
#include "draft.h"
#include "kernels.h"

namespace dipaco {

namespace {

// An odd number of words from row to row: neighbours' words lie in other banks
template <int WORDS> constexpr int row_words() { return WORDS | 1; }

template <int WORDS>
__global__ void __launch_bounds__(DRAFT_MOST_ROWS) draft_tree_rows(const int* parent, const int* row_start, int* depth, uint64_t* seen, int T_rows, int max_new, int words,
                                                                   Divisor per_row, int b0) {
  constexpr int LD = row_words<WORDS>();
  extern __shared__ __attribute__((aligned(16))) uint64_t dt_smem[];   // [rows][LD] bits, then [rows] how far up they reach: the row, or -1
  const int i = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(i >> 6);   // rows of a wave see no row of a later one: words up to its own
  const RowRange r = ragged_rows(row_start, b0 + blockIdx.x, T_rows);
  const int n = min(r.count, max_new);
  int* const reach = reinterpret_cast<int*>(dt_smem + (size_t)max_new * LD);
  uint64_t mine[WORDS];
#pragma unroll
  for (int w = 0; w < WORDS; ++w) mine[w] = wave == w ? 1ull << (i & 63) : 0;
  int up = -1;
  if (i < n) {
    up = draft_parent(parent[r.first + i], i);
#pragma unroll
    for (int w = 0; w < WORDS; ++w)
      if (w <= wave) dt_smem[i * LD + w] = mine[w];
    reach[i] = up;
  }
  while (__syncthreads_or(up >= 0)) {
    int next = -1;
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < WORDS; ++w)   // the row's own wave is an earlier one, or this: it may hold fewer words
        if (w <= wave) mine[w] |= w <= up >> 6 ? dt_smem[up * LD + w] : 0;
      next = reach[up];
    }
    __syncthreads();
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < WORDS; ++w)
        if (w <= wave) dt_smem[i * LD + w] = mine[w];
      reach[i] = next;
    }
    up = next;
  }
  if (i < n) {
    int count = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) count += __builtin_popcountll(mine[w]);
    depth[r.first + i] = count - 1;
  }
  if (WORDS == 1) {
    if (i < n) seen[r.first + i] = mine[0];
    return;
  }
  // the rows' words lie one behind the other: from LDS, where a wave's rows hold words up to their own
  uint64_t* const out = seen + (long)r.first * words;
  for (int at = i; at < n * words; at += blockDim.x) {
    const int row = per_row(at), w = at - row * words;
    out[at] = w <= row >> 6 ? dt_smem[row * LD + w] : 0;
  }
}

}  // namespace

dipaco_status launch_draft_tree(const int* parent, const int* row_start, int* depth, uint64_t* seen, int T_rows, int B, int max_new, hipStream_t s) {
  const int words = draft_words(max_new);
  auto run = [&](auto Wc) -> dipaco_status {
    constexpr int WORDS = decltype(Wc)::value;
    static std::atomic<unsigned long long> lds_set{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(draft_tree_rows<WORDS>), DRAFT_MOST_ROWS * (8 * row_words<WORDS>() + 4), lds_set)) return st;
    launch_parts(B, [&](long long first, unsigned count) {
      draft_tree_rows<WORDS><<<count, (max_new + 63) / 64 * 64, (size_t)max_new * (8 * row_words<WORDS>() + 4), s>>>(parent, row_start, depth, seen, T_rows, max_new, words, Divisor(words), (int)first);
    });
    DIPACO_LAUNCH_CHECK();
    return DIPACO_OK;
  };
  using std::integral_constant;
  return words <= 1 ? run(integral_constant<int, 1>{}) : words <= 2 ? run(integral_constant<int, 2>{}) : words <= 4 ? run(integral_constant<int, 4>{})
       : words <= 8 ? run(integral_constant<int, 8>{}) : run(integral_constant<int, 16>{});
}

}  // namespace dipaco
