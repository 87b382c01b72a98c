// Attention of the rows of trees of drafted tokens over a paged cache: row i of a document, at position L + depth, sees the cached positions of its
// window and the sinks, and of the drafted rows (slots L ..) those of its bits.
//
// A wave per row and head; a lane takes a key of 64 at a time, then columns of the values.
#include "draft.h"
#include "kernels.h"
#include "paged.h"

namespace dipaco {

namespace {

template <int DH, typename T>
__global__ void __launch_bounds__(256) attention_tree_rows(PagedArgs<T> a, const int* depth, const uint64_t* seen, int words) {
  constexpr int VEC = Vec16<T>::N, COLS = DH > 64 ? DH / 64 : 1;
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y;
  if (row >= a.T_rows) return;
  const int b = find_document(a.row_start, a.B, row, lane);
  const RowRange r = ragged_rows(a.row_start, b, a.T_rows);
  const int n = min(r.count, a.max_new), i = row - r.first;
  if (i < 0 || i >= n) return;
  const int cached = a.cached(b), pos = cached + min(max(depth[row], 0), i), near = a.w.near_from(pos), hk = a.group(head);
  const int last = min(cached + n, a.capacity()) - 1;
  const T* const q = a.qkv + (long)row * (a.H + 2 * a.H_kv) * DH + head * DH;
  const float sc = 1.4426950408889634f / sqrtf((float)DH);
  float m = -INFINITY, l = 0.f, o[COLS] = {};
  bool any = false;
  const int from = min(near, cached);
  for (int part = 0; part < 2; ++part) {
    const int lo = part == 0 ? 0 : from, hi = part == 0 ? min(min(a.w.sinks, from), last + 1) : last + 1;
    for (int k0 = lo; k0 < hi; k0 += 64) {
      const int key = k0 + lane;
      bool sees = key < hi;
      if (sees && key >= cached) sees = (seen[(long)row * words + ((key - cached) >> 6)] >> ((key - cached) & 63)) & 1;
      const int page = sees ? a.page_of(b, key) : -1;
      sees = page >= 0;
      long at = 0;
      float s = -INFINITY;
      if (sees) {
        at = a.template key_offset<DH>(page, hk, key & ((1 << a.page_shift) - 1));
        float d = 0.f;
        for (int c = 0; c < DH; c += VEC) {
          float x[VEC], y[VEC];
          load_vec16(q + c, x);
          load_vec16(a.cache + at + c, y);
#pragma unroll
          for (int e = 0; e < VEC; ++e) d = __builtin_fmaf(x[e], y[e], d);
        }
        s = d * sc;
      }
      unsigned long long todo = __builtin_amdgcn_ballot_w64(sees);
      if (!todo) continue;
      any = true;
      const bool nan = __any(s != s);
      const float mn = fmaxf(m, wave_max(s));
      const float corr = m == mn ? 1.f : exp2f(m - mn);
      const float p = s == -INFINITY ? 0.f : exp2f(s - mn);
      l = l * corr + wave_sum(p);
      if (nan) l = NAN;
#pragma unroll
      for (int c = 0; c < COLS; ++c) o[c] *= corr;
      m = mn;
      while (todo) {
        const int k = __builtin_ctzll(todo);
        todo &= todo - 1;
        const float pk = __shfl(p, k, WAVE);
        const long v = __shfl(at, k, WAVE) + a.template value_from_key<DH>();
        if (DH >= 64 || lane < DH)
#pragma unroll
          for (int c = 0; c < COLS; ++c) o[c] = __builtin_fmaf(pk, to_f32(a.cache[v + lane + 64 * c]), o[c]);
      }
    }
  }
  const float scale = any ? 1.f / l : 0.f;
  T* const to = a.o + ((long)row * a.H + head) * DH;
  if (DH >= 64 || lane < DH)
#pragma unroll
    for (int c = 0; c < COLS; ++c) to[lane + 64 * c] = from_f32<T>(any ? o[c] * scale : 0.f);
  if (a.lse && lane == 0) a.lse[(long)row * a.H + head] = (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

template <typename T> dipaco_status launch_attention_tree(const PagedArgs<T>& a, const int* depth, const uint64_t* seen, int dh, void*, hipStream_t s) {
  const dim3 grid((a.T_rows + 3) / 4, a.H);
  const int words = draft_words(a.max_new);
  if (dh == 32) attention_tree_rows<32, T><<<grid, 256, 0, s>>>(a, depth, seen, words);
  else if (dh == 64) attention_tree_rows<64, T><<<grid, 256, 0, s>>>(a, depth, seen, words);
  else attention_tree_rows<128, T><<<grid, 256, 0, s>>>(a, depth, seen, words);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
template dipaco_status launch_attention_tree<float>(const PagedArgs<float>&, const int*, const uint64_t*, int, void*, hipStream_t);
template dipaco_status launch_attention_tree<bf16>(const PagedArgs<bf16>&, const int*, const uint64_t*, int, void*, hipStream_t);

}  // namespace dipaco
