// Serving: keys and values of new tokens into a paged cache, and attention of these tokens over it (paged.h has the layout).
//
// append: a wave per row copies its k | v into the row's slot, 16 bytes a lane.  Bound by latency (a row's place takes three dependent
// loads: its document, the document's length, the page) and, for whole chunks, by the bytes.
//
// Attention: row r of document b is position cache_len[b] + r - row_start[b] and sees what a position sees under the window
// (visible.h), among the positions whose page the table holds.  One wave per row and head, 64 keys at a time.
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

}  // namespace

template <typename T> dipaco_status launch_cache_append(const PagedArgs<T>& a, int dh, hipStream_t s) {
  cache_append_rows<T><<<(a.T_rows + 3) / 4, 256, 0, s>>>(a, dh);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
size_t paged_workspace_bytes(int T_rows, int B, int max_new, int H, int H_kv, int dh, int page_size, int pages_per_doc) {
  return 256;
}
template <typename T> dipaco_status launch_attention_paged(const PagedArgs<T>& a, int dh, void* workspace, hipStream_t s) {
  return dh == 32 ? attend<32>(a, s) : dh == 64 ? attend<64>(a, s) : attend<128>(a, s);
}
template dipaco_status launch_cache_append<float>(const PagedArgs<float>&, int, hipStream_t);
template dipaco_status launch_cache_append<bf16>(const PagedArgs<bf16>&, int, hipStream_t);
template dipaco_status launch_attention_paged<float>(const PagedArgs<float>&, int, void*, hipStream_t);
template dipaco_status launch_attention_paged<bf16>(const PagedArgs<bf16>&, int, void*, hipStream_t);

}  // namespace dipaco
