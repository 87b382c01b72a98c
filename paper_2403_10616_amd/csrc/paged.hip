// Serving: keys and values of new tokens into a paged cache, and attention of these tokens over it (paged.h has the layout).
//
// append: a wave per row copies its k | v into the row's slot, 16 bytes a lane.  Bound by latency (a row's place takes three dependent
// loads: its document, the document's length, the page) and, for whole chunks, by the bytes.
//
// Attention: row r of document b is position cache_len[b] + r - row_start[b] and sees what a position sees under the window
// (visible.h), among the positions whose page the table holds.  One wave per row and head, 64 keys at a time.
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
  const int pos = max(a.cache_len[b], 0) + row - r.first;
  const int page = pos < 0 ? -1 : a.page_of(b, pos);
  if (page < 0) return;
  const int slot = pos & ((1 << a.page_shift) - 1), vecs = 2 * a.H_kv * dh / VEC, head = dh / VEC;
  const uint4* const from = reinterpret_cast<const uint4*>(a.qkv + (long)row * (a.H + 2 * a.H_kv) * dh + (long)a.H * dh);
  uint4* const to = reinterpret_cast<uint4*>(a.cache);
  for (int v = lane; v < vecs; v += 64) {
    const int kh = v / head;   // keys' heads, then values'
    to[((((long)page * 2 * a.H_kv + kh) << a.page_shift) + slot) * head + v % head] = from[v];
  }
}

template <int DH> constexpr float head_scale() { return DH == 32 ? 0.17677669529663689f : DH == 64 ? 0.125f : 0.088388347648318447f; }

template <int DH, typename T> __device__ __forceinline__ float row_dot(const T* a, const T* b) {
  constexpr int VEC = Vec16<T>::N;
  float s = 0.f;
  for (int c = 0; c < DH; c += VEC) {
    float x[VEC], y[VEC];
    load_vec16(a + c, x);
    load_vec16(b + c, y);
#pragma unroll
    for (int e = 0; e < VEC; ++e) s = __builtin_fmaf(x[e], y[e], s);
  }
  return s;
}

template <int DH, typename T>
__global__ void __launch_bounds__(256) paged_rows(PagedArgs<T> a) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, hk = h / (a.H / a.H_kv);
  if (row >= a.T_rows) return;
  const int b = find_document(a.row_start, a.B, row, lane);
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  if (row < r.first || row >= r.first + min(r.count, a.max_new)) return;
  const int pos = a.cached(b) + row - r.first;
  const T* const q = a.qkv + (long)row * (a.H + 2 * a.H_kv) * DH + h * DH;
  float acc[2] = {0.f, 0.f}, m = -INFINITY, l = 0.f;
  const VisibleList vis(a.w, pos);
  for (int t0 = 0; t0 < vis.count; t0 += 64) {
    const int n = min(64, vis.count - t0), j = vis.at(t0 + lane);
    const int page = lane < n ? a.page_of(b, j) : -1;
    const long at = page < 0 ? 0 : a.template key_offset<DH>(page, hk, j & ((1 << a.page_shift) - 1));
    const float s = page < 0 ? -INFINITY : row_dot<DH>(q, a.cache + at) * head_scale<DH>();
    const float mn = fmaxf(m, wave_max(s));
    if (mn == -INFINITY) continue;   // nothing seen so far
    const float corr = expf(m - mn), p = expf(s - mn);
    m = mn;
    l = l * corr + wave_sum(p);
    acc[0] *= corr;
    acc[1] *= corr;
    for (int t = 0; t < n; ++t) {
      if (__builtin_amdgcn_readlane(page, t) < 0) continue;
      const float pt = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), t));
      const long from = __shfl(at, t, WAVE) + a.template value_from_key<DH>();
#pragma unroll
      for (int c = 0; c < (DH == 128 ? 2 : 1); ++c)
        if (DH >= 64 || lane < DH) acc[c] = __builtin_fmaf(pt, to_f32(a.cache[from + lane + 64 * c]), acc[c]);
    }
  }
  T* const out = a.o + ((long)row * a.H + h) * DH;
  const float scale = m == -INFINITY ? 0.f : 1.f / l;
#pragma unroll
  for (int c = 0; c < (DH == 128 ? 2 : 1); ++c)
    if (DH >= 64 || lane < DH) out[lane + 64 * c] = from_f32<T>(acc[c] * scale);
  if (a.lse && lane == 0) a.lse[(long)row * a.H + h] = m == -INFINITY ? -INFINITY : m + logf(l);
}

template <int DH, typename T> dipaco_status attend(const PagedArgs<T>& a, hipStream_t s) {
  paged_rows<DH, T><<<dim3((a.T_rows + 3) / 4, a.H), 256, 0, s>>>(a);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}

// The splits' sums of the blocks that were split, added in their order.  A workgroup per row, DH / 4 threads a head.
template <int DH, typename T>
__global__ void __launch_bounds__(256) paged_join(PagedArgs<T> a) {
  constexpr int PER = DH / 4;
  const int row = blockIdx.x, lane = threadIdx.x & 63, b = find_document(a.row_start, a.B, row, lane), G = a.group();
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  const int rows = min(r.count, a.max_new);
  if (row < r.first || row >= r.first + rows) return;
  const bool narrow = rows * G <= NARROW_ROWS;
  const int splits = narrow ? a.narrow_splits : a.wide_splits;
  for (int i = threadIdx.x; i < a.H * PER; i += 256) {
    const int head = i / PER, c = 4 * (i - head * PER), R = (row - r.first) * G + head % G;
    const int used = narrow ? PagedBlock<5>(a, b, 0, NARROW_ROWS, splits).used : PagedBlock<6>(a, b, R / WIDE_ROWS, WIDE_ROWS, splits).used;
    if (used <= 1) continue;   // its workgroup has written it
    float m = -INFINITY, l = 0.f;
    for (int s = 0; s < used; ++s) m = fmaxf(m, a.template part_state<DH>(splits, s, row, head)->x);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < used; ++s) {
      const float2 st = *a.template part_state<DH>(splits, s, row, head);
      if (st.x == -INFINITY) continue;
      const float w = exp2f(st.x - m);
      const float4 p = *reinterpret_cast<const float4*>(a.template part_sums<DH>(s, row, head) + c);
      l += w * st.y;
      v.x += w * p.x; v.y += w * p.y; v.z += w * p.z; v.w += w * p.w;
    }
    const float scale = m == -INFINITY ? 0.f : 1.f / l;
    T* const out = a.o + ((long)row * a.H + head) * DH + c;
    out[0] = from_f32<T>(v.x * scale);
    out[1] = from_f32<T>(v.y * scale);
    out[2] = from_f32<T>(v.z * scale);
    out[3] = from_f32<T>(v.w * scale);
    if (a.lse && c == 0) a.lse[(long)row * a.H + head] = (m + log2f(l)) * 0.6931471805599453f;
  }
}

// How often a call's keys are cut: enough workgroups for the chip, none with less than SPLIT_KEYS keys however long the documents are
struct PagedPlan { int narrow_splits, wide_blocks, wide_splits; };
inline int most_splits(int page_size, int pages_per_doc) {
  return (int)std::min<int64_t>(PAGED_MOST_SPLITS, ((int64_t)page_size * pages_per_doc + SPLIT_KEYS - 1) / SPLIT_KEYS);
}
template <typename T> PagedPlan plan(const PagedArgs<T>& a) {
  const int G = a.H / a.H_kv, page_size = 1 << a.page_shift;
  const int64_t seen = std::min<int64_t>((int64_t)page_size * a.pages_per_doc, (int64_t)a.w.window + a.w.sinks + WIDE_ROWS);   // keys of a block, about
  const int most = std::max(1, (int)std::min<int64_t>(most_splits(page_size, a.pages_per_doc), (seen + SPLIT_KEYS - 1) / SPLIT_KEYS));
  PagedPlan p;
  p.narrow_splits = (int)std::min<int64_t>(most, (PAGED_NARROW_GROUPS + (int64_t)a.B * a.H_kv - 1) / ((int64_t)a.B * a.H_kv));
  const int64_t packed = (int64_t)a.T_rows * G, longest = (int64_t)std::min(a.max_new, a.T_rows) * G;
  p.wide_blocks = longest <= NARROW_ROWS ? 0 : (int)(packed / WIDE_ROWS + std::min<int64_t>(a.B, packed / (NARROW_ROWS + 1)));
  const int64_t wide = std::max<int64_t>(1, p.wide_blocks) * a.H_kv;
  p.wide_splits = (int)std::min<int64_t>(most, (PAGED_WIDE_GROUPS + wide - 1) / wide);
  return p;
}

}  // namespace

template <typename T> dipaco_status launch_cache_append(const PagedArgs<T>& a, int dh, hipStream_t s) {
  cache_append_rows<T><<<(a.T_rows + 3) / 4, 256, 0, s>>>(a, dh);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
// Sums of at most `most` splits of T rows, and of no more packed rows than the plan's workgroups hold: a plan of n splits has at most
// GROUPS / n + 1 workgroups a split with up to 128 (32) packed rows each.  Non-decreasing in every size but the heads'.
size_t paged_workspace_bytes(int T_rows, int H, int dh, int page_size, int pages_per_doc) {
  const size_t most = most_splits(page_size, pages_per_doc);
  constexpr size_t GROUP_ROWS = std::max(PAGED_WIDE_GROUPS * WIDE_ROWS, PAGED_NARROW_GROUPS * NARROW_ROWS);
  const size_t rows = std::min(most * T_rows, (size_t)T_rows + (GROUP_ROWS + H - 1) / H);
  return 256 + rows * H * (dh + 2) * sizeof(float);
}
template <typename T> dipaco_status launch_attention_paged(PagedArgs<T> a, int dh, void* workspace, hipStream_t s) {
  if constexpr (std::is_same<T, bf16>::value) {
    const PagedPlan p = plan(a);
    a.narrow_splits = p.narrow_splits;
    a.wide_splits = p.wide_splits;
    a.part = static_cast<float*>(workspace);
    auto run = [&](auto DHc) -> dipaco_status {
      constexpr int DH = decltype(DHc)::value;
      if (p.wide_blocks)
        if (dipaco_status st = launch_paged_wide_mfma<DH>(a, p.wide_blocks, s)) return st;
      if (dipaco_status st = launch_paged_narrow_mfma<DH>(a, s)) return st;
      if (p.narrow_splits > 1 || (p.wide_blocks && p.wide_splits > 1)) {
        paged_join<DH, T><<<a.T_rows, 256, 0, s>>>(a);
        DIPACO_LAUNCH_CHECK();
      }
      return DIPACO_OK;
    };
    return dh == 32 ? run(std::integral_constant<int, 32>{}) : dh == 64 ? run(std::integral_constant<int, 64>{}) : run(std::integral_constant<int, 128>{});
  }
  return dh == 32 ? attend<32>(a, s) : dh == 64 ? attend<64>(a, s) : attend<128>(a, s);
}
template dipaco_status launch_cache_append<float>(const PagedArgs<float>&, int, hipStream_t);
template dipaco_status launch_cache_append<bf16>(const PagedArgs<bf16>&, int, hipStream_t);
template dipaco_status launch_attention_paged<float>(PagedArgs<float>, int, void*, hipStream_t);
template dipaco_status launch_attention_paged<bf16>(PagedArgs<bf16>, int, void*, hipStream_t);

}  // namespace dipaco
