// Serving: keys and values of new tokens into a paged cache, and attention of these tokens over it (paged.h has the layout).
//
// append: a wave per row copies its k | v into the row's slot, 16 bytes a lane.  Bound by latency (a row's place takes three dependent
// loads: its document, the document's length, the page) and, for whole chunks, by the bytes: 35 tokens of 64 documents, 14 x 64, 3.0 us, 11984 tokens of 8, 8 x 128,
// 17 us (5.7 TB/s read and written).
//
// Attention: row r of document b is position cache_len[b] + r - row_start[b] and sees what a position sees under the window
// (visible.h), among the positions whose page the table holds.  paged.h says how a call is cut into workgroups; here are the plan and the launch
// that adds what was split.
#include <type_traits>

#include "kernels.h"
#include "paged.h"

namespace dipaco {

namespace {

template <typename T>
__global__ void __launch_bounds__(256) cache_append_rows(PagedArgs<T> a, int dh) {
  constexpr int VEC = Vec16<T>::N;
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.T_rows) return;
  const int b = find_document(a.row_start, a.B, row, lane);
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  if (row < r.first || row >= r.first + r.count) return;   // behind the last document
  const int pos = a.cached(b) + row - r.first, page = a.page_of(b, pos);
  if (page < 0) return;
  const int slot = pos & ((1 << a.page_shift) - 1), vecs = 2 * a.H_kv * dh / VEC, head = dh / VEC;
  const uint4* const from = reinterpret_cast<const uint4*>(a.qkv + (long)row * (a.H + 2 * a.H_kv) * dh + (long)a.H * dh);
  uint4* const to = reinterpret_cast<uint4*>(a.cache);
  for (int v = lane; v < vecs; v += 64) {
    const int kh = v / head;   // keys' heads, then values'
    to[((((long)page * 2 * a.H_kv + kh) << a.page_shift) + slot) * head + v % head] = from[v];
  }
}

// over the 16 lanes of a row, in every one of them: rotations of the row by 8, 4, 2, 1
template <int N> __device__ __forceinline__ float rotated16(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float group16_max(float v) {
  v = fmaxf(v, rotated16<8>(v));
  v = fmaxf(v, rotated16<4>(v));
  v = fmaxf(v, rotated16<2>(v));
  return fmaxf(v, rotated16<1>(v));
}
__device__ __forceinline__ float group16_sum(float v) {
  v += rotated16<8>(v);
  v += rotated16<4>(v);
  v += rotated16<2>(v);
  return v + rotated16<1>(v);
}

// The splits' sums of the blocks that were split, added in their order: HEADS heads of a row a wave, 64 / HEADS lanes each, which hold the splits' states
// (there are at most 64) and then columns of the head.  Bound by latency: its row's document, that document's rows and length, the states, the sums.  31 rows
// of 16 x 128, up to 4 splits, 4.8 us; 1253 rows of 14 x 64, 5 splits, 7 (one head a wave 10).
template <int DH, typename T, int HEADS>
__global__ void __launch_bounds__(256) paged_join(PagedArgs<T> a, Divisor waves) {   // of a row
  using Cut = PagedCut<T>;
  constexpr int LANES = 64 / HEADS, COLS = DH > LANES ? DH / LANES : 1, HELD = PAGED_MOST_SPLITS / LANES;
  const int lane = threadIdx.x & 63, sub = lane & (LANES - 1), item = blockIdx.x * 4 + (threadIdx.x >> 6), row = waves(item);
  if (row >= a.T_rows) return;   // whole waves leave
  const int head_of = HEADS * (item - row * (int)waves.d) + lane / LANES, head = min(head_of, a.H - 1);
  const int b = __builtin_amdgcn_readfirstlane(find_document(a.row_start, a.B, row, lane)), G = a.group.d;
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  const int rows = min(r.count, a.max_new);
  if (row < r.first || row >= r.first + rows) return;
  int tiles, per;
  if (rows * G <= Cut::NARROW_ROWS) {
    const PagedBlock<Cut::NARROW_SHIFT> blk(a, b, 0, Cut::NARROW_ROWS, a.narrow_splits, a.narrow_keys);
    tiles = blk.tiles.count;
    per = blk.per;
  } else {
    const PagedBlock<Cut::WIDE_SHIFT> blk(a, b, ((row - r.first) * G + head - a.group(head) * G) / Cut::WIDE_ROWS, Cut::WIDE_ROWS, a.wide_splits, Cut::LEAST_KEYS);
    tiles = blk.tiles.count;
    per = blk.per;
  }
  if (head_of >= a.H || tiles <= per) tiles = 0;   // a block of one split has been written by its workgroup
  if (!__any(tiles > 0)) return;
  float2 st[HELD];
  float m = -INFINITY, w[HELD], l = 0.f;
#pragma unroll
  for (int j = 0; j < HELD; ++j) {
    st[j] = make_float2(-INFINITY, 0.f);
    if ((LANES * j + sub) * per < tiles) st[j] = *a.part_state(LANES * j + sub, row, head);
    m = fmaxf(m, st[j].x);
  }
  m = HEADS == 1 ? wave_max(m) : group16_max(m);
#pragma unroll
  for (int j = 0; j < HELD; ++j) {
    w[j] = st[j].x == -INFINITY ? 0.f : exp2f(st[j].x - m);
    l = __builtin_fmaf(w[j], st[j].y, l);
  }
  l = HEADS == 1 ? wave_sum(l) : group16_sum(l);
  const float* const from = a.template part_sums<DH>(0, row, head) + COLS * (sub % (DH / COLS));
  const long step = (long)a.T_rows * a.H * DH;
  float v[COLS] = {};
#pragma unroll
  for (int j = 0; j < HELD; ++j) {
#pragma unroll
    for (int s0 = 0; s0 < LANES; s0 += 8) {   // eight splits at a time; one behind the last has no weight
      if (!__any((LANES * j + s0) * per < tiles)) break;
      float p[8][COLS];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int s = LANES * j + s0 + i;
        const float* const at = from + (s * per < tiles ? s : 0) * step;
        if constexpr (COLS == 1) {
          p[i][0] = *at;
        } else if constexpr (COLS == 2) {
          const float2 x = *reinterpret_cast<const float2*>(at);
          p[i][0] = x.x; p[i][1] = x.y;
        } else {
#pragma unroll
          for (int c = 0; c < COLS; c += 4) {
            const float4 x = *reinterpret_cast<const float4*>(at + c);
            p[i][c] = x.x; p[i][c + 1] = x.y; p[i][c + 2] = x.z; p[i][c + 3] = x.w;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool has = (LANES * j + s0 + i) * per < tiles;
        const float ws = __shfl(w[j], (lane - sub) + s0 + i, WAVE);
#pragma unroll
        for (int c = 0; c < COLS; ++c) v[c] = has ? __builtin_fmaf(ws, p[i][c], v[c]) : v[c];
      }
    }
  }
  if (tiles == 0 || COLS * sub >= DH) return;
  const float scale = m == -INFINITY ? 0.f : 1.f / l;
  T out[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) out[c] = from_f32<T>(v[c] * scale);
  T* const to = a.o + ((long)row * a.H + head) * DH + COLS * sub;
  constexpr int BYTES = COLS * (int)sizeof(T);
  if constexpr (COLS == 1) *to = out[0];
  else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(to) = __builtin_bit_cast(uint32_t, out);
  else if constexpr (BYTES == 8) *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, out);
  else {
#pragma unroll
    for (int c = 0; c < COLS; c += 16 / (int)sizeof(T)) {
      T part[16 / sizeof(T)];
#pragma unroll
      for (int e = 0; e < 16 / (int)sizeof(T); ++e) part[e] = out[c + e];
      *reinterpret_cast<uint4*>(to + c) = __builtin_bit_cast(uint4, part);
    }
  }
  if (a.lse && sub == 0) a.lse[(long)row * a.H + head] = (m + log2f(l)) * 0.6931471805599453f;
}

// How often a call's keys are cut: enough workgroups for the chip, none with less than LEAST_KEYS keys however long the documents are
struct PagedPlan { int narrow_splits, narrow_keys, wide_blocks, wide_splits; };
inline int most_splits(int64_t keys, int least) { return (int)std::min<int64_t>(PAGED_MOST_SPLITS, (keys + least - 1) / least); }
// Rows of partial sums that a workspace holds: `most` splits of every row, or as many as the workgroups that splits are made for have rows
constexpr size_t PAGED_GROUP_ROWS = std::max(PAGED_WIDE_GROUPS * PagedCut<bf16>::WIDE_ROWS, PAGED_NARROW_GROUPS * PagedCut<bf16>::NARROW_ROWS);
inline size_t partial_rows(int T_rows, int H, int64_t capacity) {
  return std::min((size_t)most_splits(capacity, PagedCut<float>::LEAST_KEYS) * T_rows, (size_t)T_rows + (PAGED_GROUP_ROWS + H - 1) / H);
}
template <typename T> PagedPlan plan(const PagedArgs<T>& a) {
  constexpr int NARROW_ROWS = PagedCut<T>::NARROW_ROWS, WIDE_ROWS = PagedCut<T>::WIDE_ROWS;
  const int G = a.H / a.H_kv, page_size = 1 << a.page_shift;
  const int64_t seen = std::min<int64_t>((int64_t)page_size * a.pages_per_doc, (int64_t)a.w.window + a.w.sinks + WIDE_ROWS);   // keys of a block, about
  const int most = most_splits(seen, PagedCut<T>::LEAST_KEYS);
  PagedPlan p;
  const int64_t packed = (int64_t)a.T_rows * G, longest = (int64_t)std::min(a.max_new, a.T_rows) * G;
  const int64_t heads = (int64_t)a.B * a.H_kv;
  p.narrow_splits = (int)std::min<int64_t>(most, (PAGED_NARROW_GROUPS + heads - 1) / heads);
  p.narrow_keys = PagedCut<T>::LEAST_KEYS;
  if (const int64_t half = (p.narrow_splits + 1) / 2; std::is_same<T, bf16>::value && heads * half <= 256 && longest <= NARROW_ROWS) {   // twice the waves a workgroup
    p.narrow_splits = (int)half;
    p.narrow_keys = 2 * PagedCut<T>::LEAST_KEYS;
  }
  p.wide_blocks = longest <= NARROW_ROWS ? 0 : (int)(packed / WIDE_ROWS + std::min<int64_t>(a.B, packed / (NARROW_ROWS + 1)));
  const int64_t wide = std::max<int64_t>(1, p.wide_blocks) * a.H_kv;
  p.wide_splits = (int)std::min<int64_t>(most, (PAGED_WIDE_GROUPS + wide - 1) / wide);
  // a call of narrow documents beside long chunks: the splits of the one have room for all rows of the other
  const int room = (int)std::min<size_t>(PAGED_MOST_SPLITS, partial_rows(a.T_rows, a.H, (int64_t)page_size * a.pages_per_doc) / a.T_rows);
  p.narrow_splits = std::min(p.narrow_splits, room);
  p.wide_splits = std::min(p.wide_splits, room);
  return p;
}

}  // namespace

template <typename T> dipaco_status launch_cache_append(const PagedArgs<T>& a, int dh, hipStream_t s) {
  cache_append_rows<T><<<(a.T_rows + 3) / 4, 256, 0, s>>>(a, dh);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
// Non-decreasing in every size but the heads'
size_t paged_workspace_bytes(int T_rows, int H, int dh, int page_size, int pages_per_doc) {
  return 256 + partial_rows(T_rows, H, (int64_t)page_size * pages_per_doc) * H * (dh + 2) * sizeof(float);
}
template <typename T> dipaco_status launch_attention_paged(PagedArgs<T> a, int dh, void* workspace, hipStream_t s) {
  const PagedPlan p = plan(a);
  a.narrow_splits = Divisor(p.narrow_splits);
  a.narrow_keys = p.narrow_keys;
  a.narrow_turn = 3 - std::min(3, __builtin_ctz(p.narrow_splits));   // n splits begin at 8 / gcd(8, n) places by themselves
  a.wide_splits = Divisor(p.wide_splits);
  a.state = static_cast<float2*>(workspace);
  const size_t states = (size_t)std::max(p.narrow_splits, p.wide_splits) * a.T_rows * a.H;
  a.part = static_cast<float*>(workspace) + (2 * states + 3) / 4 * 4;
  auto run = [&](auto DHc) -> dipaco_status {
    constexpr int DH = decltype(DHc)::value;
    if (dipaco_status st = p.wide_blocks ? launch_paged_both<DH>(a, p.wide_blocks, s) : launch_paged_narrow<DH>(a, s)) return st;
    if (p.narrow_splits > 1 || (p.wide_blocks && p.wide_splits > 1)) {
      // Four heads a wave where rows and heads are more than the chip holds waves.  A call's us at one a wave | four: 1 x 2000 tokens, 14 heads of 64, 36 |
      // 32; 1 x 512 over 8000, 16 of 128, 79 | 76; 1 x 128 over 16000, 14 of 64, 26 | 27; one over 30000, 32 of 128, 30.5 | 33.
      const bool four = (int64_t)a.T_rows * a.H >= 256 * 32;
      const int waves = four ? (a.H + 3) / 4 : a.H;   // of a row
      if (four) paged_join<DH, T, 4><<<(a.T_rows * waves + 3) / 4, 256, 0, s>>>(a, Divisor(waves));
      else paged_join<DH, T, 1><<<(a.T_rows * waves + 3) / 4, 256, 0, s>>>(a, Divisor(waves));
      DIPACO_LAUNCH_CHECK();
    }
    return DIPACO_OK;
  };
  return dh == 32 ? run(std::integral_constant<int, 32>{}) : dh == 64 ? run(std::integral_constant<int, 64>{}) : run(std::integral_constant<int, 128>{});
}
template dipaco_status launch_cache_append<float>(const PagedArgs<float>&, int, hipStream_t);
template dipaco_status launch_cache_append<bf16>(const PagedArgs<bf16>&, int, hipStream_t);
template dipaco_status launch_attention_paged<float>(PagedArgs<float>, int, void*, hipStream_t);
template dipaco_status launch_attention_paged<bf16>(PagedArgs<bf16>, int, void*, hipStream_t);

}  // namespace dipaco
