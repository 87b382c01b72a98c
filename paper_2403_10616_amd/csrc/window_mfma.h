// bf16 attention under a sliding window with sinks on the matrix cores: the pieces that the forward pass over a padded batch
// (attention_window_mfma.hip) and the one over a paged cache (paged_mfma.hip) share.
//
// Tiles, fragments and the order of contraction are those of attention_mfma.h: S^T = K.Q^T, so that a query's softmax state is a lane's and
// the probabilities are the next product's operand without leaving registers.  New here is which tiles are read: a workgroup walks
// the tiles of its rows' windows, then those of the sinks (TileList); a wave takes of each tile the halves of 32 keys that any of
// its 32 rows sees, and applies the mask only where some pair of the half is hidden.
//
// Bound: a half costs a wave DH / 8 matrix instructions of 32 cycles (head size 64: 256 cycles; with two numbers a probability, below, 3 DH / 16: head size 128
// 768) and about 80 vector instructions of four (16 of them exponentials, which take longer; 48 more to split probabilities), which a SIMD overlaps
// little, under a clock that the power limit sets (1.4 - 1.8 GHz).  Forward, us: 16 x 2048 positions, 14 heads of 64, window 512, 4 sinks 108 (490 TFLOP/s of
// visible pairs), window 2048 165; 2 x up to 32768, 16 heads of 128 on 4, window 4096 2340 (580); 8 x 2048, 8 heads, causal, of 128 111 (attention_mfma.h
// in the same run 119), of 64 50 (51).
//
// Probabilities enter the second product as in attention_mfma.h: as two bf16 numbers, 16 bits in all, for head sizes 32 and 128 (the output's own rounding hides
// the rest), rounded to bf16 for head size 64 (off by at most 2^-8 of each, as the output is).  Their sum is taken in fp32 before that, so
// that lse keeps fp32's digits.  Two numbers cost head size 128 a quarter to a third: 2 x up to 32768 positions, 16 heads on 4, window 4096, 1800 -> 2300 - 2450 us,
// the gradient on 4 x up to 8000, window 1000, 945 -> 1130 - 1190; what splits a pair of them by a dot product instruction saved 2 % and was left out.
#pragma once
#include "attention_mfma.h"
#include "paged.h"

namespace dipaco {

namespace {

// max of three, NaN ignored.  As an instruction of its own: fmaxf has the compiler quiet every operand first, one more instruction an element.
// The operands must not come straight from a matrix instruction: see max_of.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// The maximum of a score tile.  The first maximum is the compiler's (median with +inf), which waits for the matrix instructions that wrote the
// tile; the others depend on it.
__device__ __forceinline__ float max_of(const f32x16& st) {
  float mx = __builtin_amdgcn_fmed3f(st[0], st[15], INFINITY);
#pragma unroll
  for (int e = 1; e < 15; e += 2) mx = max3(mx, st[e], st[e + 1]);
  return mx;
}

// a wave's rows: their first and last position (none: hi = -1)
struct RowSpan { int lo, hi; };
// the larger of a lane's value and that of the lane 32 away, without a trip through LDS
__device__ __forceinline__ float max_over_halves(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
// What rows of the span see of the 32 keys from k0 on (wave-uniform): nothing, or SEEN and which bounds hide some pair: keys behind a row (UPPER), keys
// in front of a row's window (LOWER)
enum { SEEN = 1, UPPER = 2, LOWER = 4 };
__device__ __forceinline__ int seen_half(const Window& w, const RowSpan& r, int k0) {
  if (k0 > r.hi || (k0 + 31 < w.near_from(r.lo) && k0 >= w.sinks)) return 0;
  return SEEN | (k0 + 31 > r.lo ? UPPER : 0) | (k0 < w.near_from(r.hi) && k0 + 31 >= w.sinks ? LOWER : 0);
}
// v[e] = hidden where row pos does not see key k0 + acc_row(e).  A branch per bound, kept one by the empty statements: as selections the compiler would
// make of them they cost every tile 130 vector instructions (64 keys), more than its exponentials.
__device__ __forceinline__ void hide(f32x16& v, int seen, float hidden, int k0, int pos, int near, int sinks, int lane) {
  if (seen & UPPER) {
    asm volatile("");
    const int a = pos - k0 - 4 * (lane >> 5);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = 8 * (e >> 2) + (e & 3) > a ? hidden : v[e];
  }
  if (seen & LOWER) {
    asm volatile("");
    const int b = near - k0 - 4 * (lane >> 5), s = sinks - k0 - 4 * (lane >> 5);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = 8 * (e >> 2) + (e & 3) < b && 8 * (e >> 2) + (e & 3) >= s ? hidden : v[e];
  }
}

// One query row a lane pair: reference exponent, half row sum, O^T
template <int DH> struct SoftmaxRow {
  f32x16 o[DH / 32];
  float m, m_neg, l;   // m_neg = -m, 0 while nothing has been seen
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt) zero(o[dt]);
    m = -INFINITY;
    m_neg = 0.f;
    l = 0.f;
  }
};

// 32 keys from k0 on, of which the rows see `seen`.  k_, v_: their first row in LDS.  holes: bit per 16 keys that nobody sees.
// One path for all halves: with another one for two halves at a time the compiler kept two sets of accumulators and copied between them.
template <int DH>
__device__ __forceinline__ void attend_half(SoftmaxRow<DH>& x, const uint4 (&qf)[DH / 16], const char* k_, const char* v_, const FragOff& fo, const TrOff& to,
                                            int k0, int seen, int holes, int pos, int near, int sinks, int lane) {
  constexpr int KS = DH / 16, DT = DH / 32;
  f32x16 st;
  zero(st);
  // Keys are read in one go, and values while the scores are multiplied: left to the compiler the reads trickle in between the products, each
  // with a wait of its own.  16 x 2048 positions of 14 x 64, window 512: 96 us, 101 so.
  uint4 kf[KS], vf[DT][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kf[ks] = row_frag(k_, fo, ks, 0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) st = mfma16(kf[ks], qf[ks], st);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 2; ++i) vf[dt][i] = tr_read(v_, to, dt, i);
  __builtin_amdgcn_sched_barrier(0);
  hide(st, seen, -INFINITY, k0, pos, near, sinks, lane);
  if (holes) {   // wave-uniform
    asm volatile("");
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if ((holes >> (e >> 3)) & 1) st[e] = -INFINITY;
  }
  const float sc = score_scale<DH>() * LOG2E;
  const float mx = max_over_halves(max_of(st));
  // the reference may lag behind the running maximum by 2^8 (attention_mfma.h); rows that have seen nothing keep 0 for it
  const float mn = fmaxf(x.m, mx * sc);
  if (__builtin_amdgcn_ballot_w64(mn > x.m + 8.0f) != 0) {   // wave-uniform
    const float corr = mn == x.m ? 1.f : __builtin_amdgcn_exp2f(x.m - mn);
    x.l *= corr;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) x.o[dt][e] *= corr;
    x.m = mn;
    x.m_neg = mn == -INFINITY ? 0.f : -mn;
  }
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) st[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], sc, x.m_neg));
#pragma unroll
  for (int e = 0; e < 16; e += 2) { s0 += st[e]; s1 += st[e + 1]; }
  x.l += s0 + s1;
  const auto p0 = p_frag<split_p<DH>(), 0>(st), p1 = p_frag<split_p<DH>(), 8>(st);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    x.o[dt] = mfma_p(vf[dt][0], p0, x.o[dt]);
    x.o[dt] = mfma_p(vf[dt][1], p1, x.o[dt]);
  }
}
// a tile of 64 keys: the halves that are seen.  force: bounds to apply whatever the span says
template <int DH>
__device__ __forceinline__ void attend_tile(SoftmaxRow<DH>& x, const uint4 (&qf)[DH / 16], const char* k_, const char* v_, const FragOff& fo, const TrOff& to,
                                            int k0, int holes, const Window& w, const RowSpan& span, int force, int pos, int near, int lane) {
  const int a = (holes & 3) == 3 ? 0 : seen_half(w, span, k0), b = holes >> 2 == 3 ? 0 : seen_half(w, span, k0 + 32);
  if (a) attend_half<DH>(x, qf, k_, v_, fo, to, k0, a | force, holes & 3, pos, near, w.sinks, lane);
  if (b) attend_half<DH>(x, qf, k_ + 4096, v_ + 4096, fo, to, k0 + 32, b | force, holes >> 2, pos, near, w.sinks, lane);
}

// Two operands' rows of one document and head (keys and values; queries and output gradients), ld0 and ld1 elements apart
template <int DH, bool TWO_STRIDES = false> struct RowTiles {
  const bf16 *t0, *t1;
  int ld0, ld1, rows;
  uint32_t off[TWO_STRIDES ? 4 : 2];
  __device__ __forceinline__ uint32_t offset(int i, int row) const { return (uint32_t)(row * (i < 2 ? ld0 : ld1) * 2); }
  __device__ __forceinline__ RowTiles(const bf16* t0, const bf16* t1, int ld0, int ld1, int rows, int wave, int lane)
      : t0(t0), t1(t1), ld0(ld0), ld1(ld1), rows(rows) {
#pragma unroll
    for (int i = 0; i < (TWO_STRIDES ? 4 : 2); ++i) off[i] = offset(i, loader_row(i & 1, wave, lane)) + loader_column_bytes<DH>(i & 1, wave, lane);
  }
  // this wave's loads of a tile of 64 rows into a stage: rows behind the document's last one re-read it (callers give them no weight)
  __device__ __forceinline__ void issue(int tile, int wave, int lane, uint32_t stage_addr) const {
    constexpr int NP = panels<DH>();
    const int row0 = tile * 64;
    const bf16* const b0 = t0 + (long)row0 * ld0;
    const bf16* const b1 = t1 + (long)row0 * ld1;
    uint32_t at[4] = {off[0], off[1], off[TWO_STRIDES ? 2 : 0], off[TWO_STRIDES ? 3 : 1]};
    if (row0 + 64 > rows) {   // wave-uniform
#pragma unroll
      for (int i = 0; i < 4; ++i)
        at[i] = offset(i, min(loader_row(i & 1, wave, lane), rows - 1 - row0)) + loader_column_bytes<DH>(i & 1, wave, lane);
    }
#pragma unroll
    for (int i = 0; i < 4 * NP; ++i) {
      const int second = i / (2 * NP), panel = (i >> 1) % NP;   // compile-time
      load16_to_lds_at((second ? b1 : b0) + 64 * panel, at[2 * second + (i & 1)], stage_addr + (uint32_t)((wave + 4 * i) * 1024));
    }
  }
};

}  // namespace

}  // namespace dipaco
