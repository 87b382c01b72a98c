// fp32 attention under a sliding window with sinks on the matrix cores: what the kernels over a padded batch (attention_window_f32.hip) and over
// a paged cache (paged_f32.hip) share.  Layout and order of contraction are those of attention_f32.hip: 16 rows a wave, tiles of keys (queries)
// through registers into LDS in rows DH + 4 floats apart, two stages, the next tile's loads in flight during this one's products.
//
// Exponentials are base 2 on the hardware's instruction, log2(e) folded into the scale: its error (2^-22) is that of a product of a score of 8.
#pragma once
#include "attention_f32_tiles.h"
#include "attention_plain.h"
#include "paged.h"

namespace dipaco {

namespace {

constexpr int WF_WAVES = 4, WF_THREADS = 64 * WF_WAVES;
constexpr float WF_LOG2E = 1.4426950408889634f, WF_LN2 = 0.6931471805599453f;
template <int DH, int ROWS> constexpr int window_tile_floats() { return ROWS * row_stride<DH>(); }

// Two operands' tiles of ROWS rows: thread t moves float4 number t + 256 i of the first, then the same of the second
template <int DH, int ROWS> struct TileMover {
  static constexpr int VEC_ROW = DH / 4, N = ROWS * VEC_ROW / WF_THREADS;
  static_assert(N >= 1 && ROWS * VEC_ROW % WF_THREADS == 0, "");
  f32x4 v0[N], v1[N];
  // place(row, p0, p1): where row `row` of the tiles starts
  template <typename P> __device__ __forceinline__ void load(P place) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int n = threadIdx.x + WF_THREADS * i;
      const float *p0, *p1;
      place(n / VEC_ROW, p0, p1);
      v0[i] = *reinterpret_cast<const f32x4*>(p0 + 4 * (n % VEC_ROW));
      v1[i] = *reinterpret_cast<const f32x4*>(p1 + 4 * (n % VEC_ROW));
    }
  }
  __device__ __forceinline__ void store(float* stage) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int n = threadIdx.x + WF_THREADS * i;
      float* const at = stage + (n / VEC_ROW) * row_stride<DH>() + 4 * (n % VEC_ROW);
      *reinterpret_cast<f32x4*>(at) = v0[i];
      *reinterpret_cast<f32x4*>(at + window_tile_floats<DH, ROWS>()) = v1[i];
    }
  }
};

struct FRowSpan { int lo, hi; };   // a wave's rows: their first and last position (none: hi = -1)
enum FSeen { F_NONE = 0, F_SOME = 1, F_ALL = 2 };
// what rows of the span see of the 16 keys from k0 on (wave-uniform)
__device__ __forceinline__ int seen_16(const Window& w, const FRowSpan& r, int k0) {
  if (k0 > r.hi || (k0 + 15 < w.near_from(r.lo) && k0 >= w.sinks)) return F_NONE;
  return k0 + 15 <= r.lo && (k0 >= w.near_from(r.hi) || k0 + 15 < w.sinks) ? F_ALL : F_SOME;
}

// one query row for the four lanes that share l % 16
template <int DH> struct FSoftmaxRow {
  f32x4 o[DH / 16];
  float m, m_neg, l;   // reference exponent (base 2), its negative (0 while nothing has been seen), this lane's part of the sum
  __device__ __forceinline__ void clear() {
    zero_acc<DH>(o);
    m = -INFINITY;
    m_neg = 0.f;
    l = 0.f;
  }
};
// bit e: the lane's row sees key 4 g + e of the 16 from k0 on
__device__ __forceinline__ int seen_keys(const ChainView& x, int k0, int g) {
  int bits = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) bits |= x.sees(k0 + 4 * g + e) ? 1 << e : 0;
  return bits;
}
__device__ __forceinline__ int seen_keys(TreeView& x, int k0, int g) {
  const uint32_t word = x.word(k0) & 0xffffu;
  x.note(k0, word);
  int bits = word >> (4 * g);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int key = k0 + 4 * g + e;
    if (key < x.near && key >= x.sinks) bits &= ~(1 << e);
  }
  return bits;
}
// 16 keys, run t of the tile k_ (v_), from position k0 on
template <int DH, typename View>
__device__ __forceinline__ void attend_16(FSoftmaxRow<DH>& x, const RowFrag<DH>& qf, const float* k_, const float* v_, int t, int k0, bool masked, View& view,
                                          int m, int g) {
  const float sc = head_scale<DH>() * WF_LOG2E;
  f32x4 st = {0.f, 0.f, 0.f, 0.f};
  rows_product<DH>(st, k_, t, qf, m, g);
  float mx = -INFINITY;
  const int seen = masked ? seen_keys(view, k0, g) : 15;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (!(seen & (1 << e))) st[e] = -INFINITY;
    mx = fmaxf(mx, st[e]);
  }
  const float mn = fmaxf(x.m, max_groups(mx) * sc);
  if (__builtin_amdgcn_ballot_w64(mn > x.m + 8.0f) != 0) {   // wave-uniform; the reference may lag by 2^8
    const float corr = mn == x.m ? 1.f : __builtin_amdgcn_exp2f(x.m - mn);
    x.l *= corr;
#pragma unroll
    for (int d = 0; d < DH / 16; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) x.o[d][e] *= corr;
    x.m = mn;
    x.m_neg = mn == -INFINITY ? 0.f : -mn;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    st[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], sc, x.m_neg));
    x.l += st[e];
  }
  cols_product<DH>(x.o, v_, t, st, m, g);
}
// a tile of 32 keys: the runs that are seen
template <int DH, typename View>
__device__ __forceinline__ void attend_32(FSoftmaxRow<DH>& x, const RowFrag<DH>& qf, const float* k_, const float* v_, int k0, int holes, const Window& w,
                                          const FRowSpan& span, bool masked, View& view, int m, int g) {
  const int a = holes & 1 ? F_NONE : seen_16(w, span, k0), b = holes & 2 ? F_NONE : seen_16(w, span, k0 + 16);
  if (a != F_NONE) attend_16<DH>(x, qf, k_, v_, 0, k0, masked || a != F_ALL, view, m, g);
  if (b != F_NONE) attend_16<DH>(x, qf, k_, v_, 1, k0 + 16, masked || b != F_ALL, view, m, g);
}

}  // namespace

}  // namespace dipaco
