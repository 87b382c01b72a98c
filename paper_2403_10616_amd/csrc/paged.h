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
  template <int DH> __device__ __forceinline__ long key_offset(int page, int hk, int slot) const {
    return ((((long)page * 2 * H_kv + hk) << page_shift) + slot) * DH;
  }
  template <int DH> __device__ __forceinline__ long value_from_key() const { return ((long)H_kv << page_shift) * DH; }
  template <int DH> __device__ __forceinline__ float* part_sums(int split, long row, int head) const { return part + (((long)split * T_rows + row) * H + head) * DH; }
  __device__ __forceinline__ float2* part_state(int split, long row, int head) const { return state + ((long)split * T_rows + row) * H + head; }
};

// Workgroups of a launch of both kinds: n_wide of heads x splits x blocks, then those of splits x heads x documents
struct PagedOrder { Divisor heads, head_splits; int n_wide; };

// A block of packed rows of one document: which rows, the tiles that they see, and how many of these a split takes
template <int SHIFT> struct PagedBlock {
  int b, row0, rows, packed0, packed, pos0, last;   // rows row0 .. of the call, `rows` of them; packed rows packed0 .. of `packed`; position of row 0; last one
  int lo, hi;                                       // positions of the block's first and last row
  TileList<SHIFT> tiles;
  int per;                                          // tiles a split: split s has tiles s per ..
  template <typename T> __device__ __forceinline__ PagedBlock(const PagedArgs<T>& a, int b, int block, int block_rows, const Divisor& splits, int least_keys)
      : PagedBlock(a, b, ragged_rows(a.row_start, b, a.T_rows), a.cached(b), block, block_rows, splits, least_keys) {}
  template <typename T>
  __device__ __forceinline__ PagedBlock(const PagedArgs<T>& a, int b, const RowRange& r, int cached, int block, int block_rows, const Divisor& splits, int least_keys)
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
    lo = pos0 + a.group(packed0);
    hi = pos0 + a.group(min(packed, packed0 + block_rows) - 1);
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
