// The paged cache of keys and values, the rows of new tokens that attend to it, and how their work is cut.
//
// cache: [n_pages][2][H_kv][page_size][dh], keys then values; position p of document b sits in page pages[b * pages_per_doc + p /
// page_size], slot p % page_size.  A head's share of a page is contiguous: page_size x dh elements, 2 KB for 16 positions of 64 bf16.
//
// The query heads that read one key head, G of them, are rows of one product: row R of a document's n G packed rows is token R / G, head
// R % G of the group.  A workgroup takes a block of packed rows of a document and a key head, and a part ("split") of the keys that these see:
//   narrow: a document of up to 32 packed rows (fp32: 16) is one block; its workgroup's waves take the keys in turn.
//   wide:   128 packed rows, 32 a wave (fp32: 64, 16 a wave); the waves share the keys' tiles.
// Every eighth workgroup of a launch goes to the same eighth of the chip.  So workgroups that find nothing to do must not come at a fixed pace: wide
// blocks that a call does not have are its last workgroups (128 tokens over 16000 positions: 25 us, 32 with every other workgroup idle), and the narrow
// splits of a document, of which a short one leaves some idle, begin at another one of the eight each time.
// Rows of a tree (TreeArgs) are cut the same way; any of them may see any slot of the document's new rows, so that all blocks of a document have the same tiles,
// and in the tiles that hold such slots a row's bits are the mask (TreeView), two words a lane for 32 keys.
// A split's sums go to the workspace, and paged_join adds them; a block whose keys are one split's writes its rows itself.
#pragma once
#include "visible.h"

namespace dipaco {

// Tiles of 2^SHIFT keys that rows at positions lo .. hi see: those from `first` to that of position hi, then the sinks' in front of them.  The sinks last:
// every workgroup of a head asks for the same rows there, and a window's tile is in flight meanwhile.
template <int SHIFT> struct TileList {
  int near, first, count;   // `near` tiles from `first` on, `count` in all
  __device__ __forceinline__ TileList() : near(0), first(0), count(0) {}
  __device__ __forceinline__ TileList(const Window& w, int lo, int hi) {
    const int from = w.near_from(lo);
    first = min(from >> SHIFT, (hi >> SHIFT) + 1);   // hi, the table's last position, lies in front of the window where a document has outgrown it
    near = (hi >> SHIFT) + 1 - first;
    count = near + min((min(w.sinks, from) + (1 << SHIFT) - 1) >> SHIFT, first);
  }
  __device__ __forceinline__ int at(int t) const { return t < near ? first + t : t - near; }
};

// packed rows of a block, log2 of the keys of a tile, and the fewest keys of a split (in a narrow launch of few workgroups, of twice the waves, twice as many)
template <typename T> struct PagedCut { static constexpr int NARROW_ROWS = 32, NARROW_SHIFT = 5, WIDE_ROWS = 128, WIDE_SHIFT = 6, LEAST_KEYS = 512; };
template <> struct PagedCut<float> { static constexpr int NARROW_ROWS = 16, NARROW_SHIFT = 6, WIDE_ROWS = 64, WIDE_SHIFT = 5, LEAST_KEYS = 128; };
constexpr int PAGED_MOST_SPLITS = 64, PAGED_NARROW_GROUPS = 1024, PAGED_WIDE_GROUPS = 1024;   // splits, and the workgroups that they are to make

// n / d for n < 2^31: a multiplication by ceil(2^32 / d), whose result is at most one too high, and its correction.  As the compiler divides (40
// instructions, each waiting for the one before), the ten divisions in front of a one-token call's first load took a microsecond.
struct Divisor {
  uint32_t d, magic;
  __host__ __device__ Divisor() : d(1), magic(0) {}
  explicit Divisor(int v) : d(v), magic((uint32_t)(((1ull << 32) + v - 1) / v)) {}   // 0 for v = 1, whose quotient is n
  __device__ __forceinline__ int operator()(int n) const {
    if (d == 1) return n;
    const int q = (int)__umulhi((uint32_t)n, magic);
    return q - (q * (int)d > n ? 1 : 0);
  }
};

// The reference exponent of a row is -inf where it has seen nothing.  One that has seen scores, all of them -inf, has this instead once its keys are
// through: it loses against every finite reference, and if it stays the row is 0 / 0 as its definition is, not the 0 of a row that sees nothing.
constexpr float ALL_MINUS_INFINITY = -3.402823466e38f;

// What a row sees, key by key.  near: first position of its window
struct ChainView {
  int pos, near, sinks;   // up to position pos
  __device__ __forceinline__ bool sees(int key) const { return key <= pos && (key >= near || key < sinks); }
};
// A row of a tree: positions in front of `cached` by the window and the sinks, those behind by its bits, none behind `last`
struct TreeView {
  const uint32_t* bits;
  int words, cached, last, near, sinks;
  bool any;               // whether it has seen one of its bits' keys
  // the bits of the 32 positions from k0 on; set for positions in front of `cached`
  __device__ __forceinline__ uint32_t word(int k0) const {
    const int s = k0 - cached;
    uint32_t w = ~0u;
    if (s > -32) {
      const int i = s >> 5;
      const uint32_t a = i < 0 ? ~0u : i < words ? bits[i] : 0u, b = i + 1 < words ? bits[i + 1] : 0u;
      w = __builtin_amdgcn_alignbit(b, a, s & 31);
    }
    const int upto = last - k0;
    return upto >= 31 ? w : upto < 0 ? 0u : w & ((2u << upto) - 1);
  }
  // seen: as word, without keys that no page holds
  __device__ __forceinline__ void note(int k0, uint32_t seen) {
    any |= (k0 >= cached ? seen : cached - k0 >= 32 ? 0u : seen >> (cached - k0)) != 0;
  }
  __device__ __forceinline__ bool sees(int key) const { return (word(key) & 1) && (key >= cached || key >= near || key < sinks); }
};

template <typename T> struct PagedArgs {
  static constexpr bool TREE = false;   // a document's new rows see each other in order
  const T* qkv;              // [T rows, (H + 2 H_kv) dh]
  const int* row_start;      // [B + 1]
  const int* cache_len;      // [B]
  const int* pages;          // [B, pages_per_doc]
  T* cache;
  T* o;                      // [T rows, H dh]
  float* lse;                // [T rows, H], or null
  int T_rows, B, max_new, H, H_kv, n_pages, page_shift, pages_per_doc;
  Window w;
  Divisor group;             // H / H_kv
  Divisor narrow_splits, wide_splits;
  int narrow_keys;           // a narrow split has at least so many keys
  float* part;               // [splits][T rows][H][dh] sums
  float2* state;             // [splits][T rows][H] reference exponents and sums of exponentials; narrow and wide splits use the rows of their documents
  int narrow_turn;           // log2 of the (document, head)s behind which the order of their splits moves on by one
  // the split of the p-th workgroup of a document and head
  __device__ __forceinline__ int narrow_split(int p, int item) const {
    const int s = p + (item >> narrow_turn);
    return s - narrow_splits(s) * (int)narrow_splits.d;
  }
  __device__ __forceinline__ int capacity() const { return pages_per_doc << page_shift; }
  // A document may have outgrown its table: its rows keep their positions, and see of the table what the window and the sinks reach.  The bound is
  // arithmetic's: a row's position, at most 2^23 behind, stays below 2^31.
  __device__ __forceinline__ int cached(int b) const { return min(max(cache_len[b], 0), 0x7f000000); }
  // the page of a position, or -1 where the table holds none
  __device__ __forceinline__ int page_of(int b, int pos) const {
    const int at = pos >> page_shift;
    if (at >= pages_per_doc) return -1;
    const int p = pages[(long)b * pages_per_doc + at];
    return (unsigned)p < (unsigned)n_pages ? p : -1;
  }
  // whether a row at position pos, whose window begins at `near`, sees any of the n keys from k0 on, none behind `last`; k0 is a multiple of 16, and so are
  // pages' sizes: the keys of a run of 16 share one
  __device__ __forceinline__ bool sees_any(int b, int pos, int near, int last, int k0, int n) const {
    const int upto = min(min(pos, last), k0 + n - 1);
#pragma unroll 1
    for (int p = k0; p <= upto; p += 16)
      if ((min(p + 15, upto) >= near || p < w.sinks) && page_of(b, p) >= 0) return true;
    return false;
  }
  __device__ __forceinline__ bool sees_any(int b, const ChainView& x, int last, int k0, int n) const { return sees_any(b, x.pos, x.near, last, k0, n); }
  // a tree's row: its words have been looked at already
  __device__ __forceinline__ bool sees_any(int b, const TreeView& x, int last, int k0, int n) const { return x.any || sees_any(b, x.cached - 1, x.near, last, k0, n); }
  // of the row that is new token `token` of a document with `rows` of them from row0 on
  __device__ __forceinline__ ChainView view(int, int, int pos0, int last, int token) const { return {min(pos0 + token, last), w.near_from(pos0 + token), w.sinks}; }
  template <int DH> __device__ __forceinline__ long key_offset(int page, int hk, int slot) const {
    return ((((long)page * 2 * H_kv + hk) << page_shift) + slot) * DH;
  }
  template <int DH> __device__ __forceinline__ long value_from_key() const { return ((long)H_kv << page_shift) * DH; }
  template <int DH> __device__ __forceinline__ float* part_sums(int split, long row, int head) const { return part + (((long)split * T_rows + row) * H + head) * DH; }
  __device__ __forceinline__ float2* part_state(int split, long row, int head) const { return state + ((long)split * T_rows + row) * H + head; }
};

// The new rows are trees: a row's position is its depth behind the cached ones, and of the new rows it sees those of its bits
template <typename T> struct TreeArgs : PagedArgs<T> {
  static constexpr bool TREE = true;
  const int* depth;          // [T rows]
  const uint32_t* seen;      // [T rows, words]
  int words;
  int* plan;                 // null, or tiles a split, which the launch's first workgroup leaves for the join
  int most_items;            // with a plan: items of a key head that the launch has workgroups for
  __device__ __forceinline__ TreeView view(int row0, int rows, int pos0, int last, int token) const {
    token = min(token, rows - 1);
    const long row = row0 + token;
    const int pos = pos0 + min(max(depth[row], 0), token);
    return {seen + row * words, words, pos0, last, min(this->w.near_from(pos), pos0), this->w.sinks, false};
  }
};

template <typename T> __host__ __device__ __forceinline__ bool has_plan(const PagedArgs<T>&) { return false; }
template <typename T> __host__ __device__ __forceinline__ bool has_plan(const TreeArgs<T>& a) { return a.plan != nullptr; }
template <typename T> __device__ __forceinline__ int* plan_of(const PagedArgs<T>&) { return nullptr; }
template <typename T> __device__ __forceinline__ int* plan_of(const TreeArgs<T>& a) { return a.plan; }

// The item-th part of the wide blocks of trees (a block's tiles, cut into splits), for a key head.  Documents' lengths are known on the device alone, and a split of
// equal share of its document would take as long as the longest one: so here a split is so many tiles, the same for all documents, of which the workgroups at hand
// (`slots` are resident at once, one to TREE_ROUNDS rounds of them) end soonest; a workgroup's start and end take as long as TREE_START tiles.  Every wave reads the
// documents (64 at most), a lane each, and comes to the same end.
constexpr int TREE_DOCUMENTS = 64, TREE_ROUNDS = 3, TREE_START = 4;
__device__ __forceinline__ int lanes_upto(int v) {   // lane i: the sum of lanes 0 .. i
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast31 into rows 2 and 3
  return v;
}
struct TreeItem {
  int b, block, split, per, cached;   // b: -1 where there are fewer items
  RowRange rows;
  template <typename T> __device__ __forceinline__ TreeItem(const TreeArgs<T>& a, int item, int slots, int lane) : b(-1), block(0), split(0), per(0), cached(0), rows{0, 0} {
    using Cut = PagedCut<T>;
    int blocks = 0, tiles = 0, mine = 0;
    RowRange r{0, 0};
    if (lane < a.B) {
      r = ragged_rows(a.row_start, lane, a.T_rows);
      mine = a.cached(lane);
      const int n = min(r.count, a.max_new), packed = n * (int)a.group.d, last = min(mine + n, a.capacity()) - 1;
      if (packed > Cut::NARROW_ROWS) {
        blocks = (packed + Cut::WIDE_ROWS - 1) / Cut::WIDE_ROWS;
        tiles = last < 0 ? 1 : max(TileList<Cut::WIDE_SHIFT>(a.w, mine, last).count, 1);
      }
    }
    const int n_blocks = __builtin_amdgcn_readlane(lanes_upto(blocks), 63), longest = (int)wave_max((float)tiles) + 1;
    const float work = wave_sum((float)blocks * (float)tiles);
    const int least = max((longest + (int)a.wide_splits.d - 1) / (int)a.wide_splits.d, Cut::LEAST_KEYS >> Cut::WIDE_SHIFT);
    // splits of p tiles: at most work / p, and one a block for what is left over
    per = longest;
    float best = INFINITY;
#pragma unroll
    for (int k = 1; k <= TREE_ROUNDS; ++k) {
      const int room = k * slots / a.H_kv - n_blocks;
      const int p = max((int)(work * __builtin_amdgcn_rcpf((float)max(room, 1)) * 1.00001f) + 1, least);
      const float rounds = ceilf((work * __builtin_amdgcn_rcpf((float)p) + (float)n_blocks) * (float)a.H_kv / (float)slots), end = rounds * (float)(p + TREE_START);
      if (room >= 1 && end < best) {
        best = end;
        per = p;
      }
    }
    auto splits_of = [&](int p) {   // or one more, which finds nothing to do
      return (int)((float)(tiles + p - 1) * __builtin_amdgcn_rcpf((float)p) * 1.00001f);
    };
    int upto = lanes_upto(blocks * splits_of(per));
    if (__builtin_amdgcn_readlane(upto, 63) > a.most_items) {   // rounding may leave more than the launch holds
      per = longest;
      upto = lanes_upto(blocks);
    }
    if (item >= __builtin_amdgcn_readlane(upto, 63)) return;
    const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(upto <= item));
    b = at;
    const int i = item - (at ? __builtin_amdgcn_readlane(upto, at - 1) : 0), n = __builtin_amdgcn_readlane(blocks, at);
    split = i / n;
    block = i - split * n;
    cached = __builtin_amdgcn_readlane(mine, at);
    rows = {__builtin_amdgcn_readlane(r.first, at), __builtin_amdgcn_readlane(r.count, at)};
  }
};

// Workgroups of a launch of both kinds: n_wide of heads x splits x blocks, then those of splits x heads x documents
struct PagedOrder { Divisor heads, head_splits; int n_wide; };

// A block of packed rows of one document: which rows, the tiles that they see, and how many of these a split takes
template <int SHIFT> struct PagedBlock {
  int b, row0, rows, packed0, packed, pos0, last;   // rows row0 .. of the call, `rows` of them; packed rows packed0 .. of `packed`; position of row 0; last one
  int lo, hi;                                       // positions of the block's first and last row; TREE: of the document's new slots
  TileList<SHIFT> tiles;
  int per;                                          // tiles a split: split s has tiles s per ..
  template <typename A> __device__ __forceinline__ PagedBlock(const A& a, int b, int block, int block_rows, const Divisor& splits, int least_keys)
      : PagedBlock(a, b, ragged_rows(a.row_start, b, a.T_rows), a.cached(b), block, block_rows, splits, least_keys) {}
  template <typename A>
  __device__ __forceinline__ PagedBlock(const A& a, int b, const RowRange& r, int cached, int block, int block_rows, const Divisor& splits, int least_keys)
      : b(b) {
    const int G = a.group.d;
    pos0 = cached;
    row0 = r.first;
    rows = min(r.count, a.max_new);
    packed = rows * G;
    packed0 = block * block_rows;
    last = min(pos0 + rows, a.capacity()) - 1;
    per = lo = hi = 0;
    if (packed0 >= packed) return;
    if (A::TREE) {   // any row may see all of them
      lo = pos0;
      hi = pos0 + rows - 1;
    } else {
      lo = pos0 + a.group(packed0);
      hi = pos0 + a.group(min(packed, packed0 + block_rows) - 1);
    }
    if (last < 0) return;
    tiles = TileList<SHIFT>(a.w, lo, min(hi, last));
    if (tiles.count <= 0) { tiles.count = 0; return; }
    per = max(splits(tiles.count + (int)splits.d - 1), least_keys >> SHIFT);
  }
  // whether a split has tiles (the first one: whether or not it has), and whether it has them all
  __device__ __forceinline__ bool has(int split) const { return split == 0 || split * per < tiles.count; }
  __device__ __forceinline__ bool whole() const { return tiles.count <= per; }
};

// The i-th wide block of the call: its document (-1: there are fewer), which of the document's blocks, the document's rows and cached positions,
// which the whole wave has read anyway to find it.  Everything is wave-uniform.
struct WideBlock {
  int b, block, cached;
  RowRange rows;
  template <typename T> __device__ __forceinline__ WideBlock(const PagedArgs<T>& a, int i, int lane) : b(-1), block(0), cached(0), rows{0, 0} {
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      int n = 0, mine = 0;
      RowRange r{0, 0};
      if (b0 + lane < a.B) {
        r = ragged_rows(a.row_start, b0 + lane, a.T_rows);
        mine = a.cached(b0 + lane);
        const int packed = min(r.count, a.max_new) * (int)a.group.d;
        n = packed > PagedCut<T>::NARROW_ROWS ? (packed + PagedCut<T>::WIDE_ROWS - 1) / PagedCut<T>::WIDE_ROWS : 0;
      }
      int upto = n;   // blocks of documents b0 .. b0 + lane: a scan on the DPP lanes, of rows of 16, then across them
      upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
      upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
      upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
      upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
      upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, false);   // row_bcast15 into rows 1 and 3
      upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, false);   // row_bcast31 into rows 2 and 3
      const int all = __builtin_amdgcn_readlane(upto, 63);
      if (i < all) {
        const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(upto <= i));
        b = b0 + at;
        block = i - (at ? __builtin_amdgcn_readlane(upto, at - 1) : 0);
        cached = __builtin_amdgcn_readlane(mine, at);
        rows = {__builtin_amdgcn_readlane(r.first, at), __builtin_amdgcn_readlane(r.count, at)};
        return;
      }
      i -= all;
    }
  }
};

}  // namespace dipaco
