// fp32 attention with a sliding window and sinks over packed rows of a padded batch, forward and backward (window_f32.h).
//
// A workgroup takes 64 queries (keys) of a head, 16 a wave.  Bound by the fp32 matrix cores on whole 16 x 16 tiles.  Us, forward | backward: 16 x 2048
// positions, 14 heads of 64, window 512, 4 sinks 525 | 1682 (101 | 79 TFLOP/s of what is needed; the backward pass multiplies 7 / 5 of it); 8 x 500, 8 heads of
// 64, window 100 21 | 51; 1 x 8192, 8 heads of 64 on 2, window 512, 4 sinks 96 | 322.  Rows that end with results that are not finite are taken again over the pairs that
// see each other alone (attention_plain.h).
#include "kernels.h"
#include "window_f32.h"

namespace dipaco {

namespace {

struct FWindowArgs {
  const float* qkv;
  const int* lengths;
  int B, S, H, H_kv;
  Window w;
};
constexpr int WF_ROWS = 16 * WF_WAVES, WF_TILE = 32;
template <int DH> constexpr int wf_stage() { return 2 * window_tile_floats<DH, WF_TILE>() + 2 * WF_TILE; }   // two operands, and two statistics a row

template <int DH>
__global__ void __launch_bounds__(WF_THREADS, 2) window_fwd_f32(FWindowArgs a, float* __restrict__ o, float* __restrict__ lse) {
  extern __shared__ __attribute__((aligned(16))) float wff_smem[];   // [stage][K | V]
  constexpr int STAGE = wf_stage<DH>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int n_bh = a.B * a.H, qb = (int)blockIdx.x / n_bh, bh = (int)blockIdx.x - qb * n_bh, b = bh / a.H, hd = bh - b * a.H, hk = hd / (a.H / a.H_kv);
  const int q0 = ((a.S + WF_ROWS - 1) / WF_ROWS - 1 - qb) * WF_ROWS, qw0 = q0 + 16 * wave, q = qw0 + m;
  const int rows = document_rows(a.lengths, b, a.S);
  const long ld = (long)(a.H + 2 * a.H_kv) * DH;
  const float* const base = a.qkv + (long)b * a.S * ld;
  const FRowSpan span{qw0, qw0 < rows ? min(qw0 + 15, rows - 1) : -1};
  const ChainView view{q, a.w.near_from(q), a.w.sinks};
  FSoftmaxRow<DH> x;
  x.clear();
  if (q0 < rows) {
    const float* const k = base + (a.H + hk) * DH;
    const RowFrag<DH> qf = load_row<DH>(base + q * ld + hd * DH, g, q < rows);
    const TileList<5> tiles(a.w, q0, min(q0 + WF_ROWS - 1, rows - 1));
    TileMover<DH, WF_TILE> next;
    auto load = [&](int t) {
      const int row0 = tiles.at(t) * 32;
      next.load([&](int r, const float*& p0, const float*& p1) {
        p0 = k + min(row0 + r, rows - 1) * ld;
        p1 = p0 + a.H_kv * DH;
      });
    };
    load(0);
    next.store(wff_smem);
    for (int t = 0; t < tiles.count; ++t) {
      const float* k_ = wff_smem + (t & 1) * STAGE;
      const bool more = t + 1 < tiles.count;
      if (more) load(t + 1);
      __syncthreads();   // tile t is in LDS, and everybody is done with the stage of tile t - 1
      attend_32<DH>(x, qf, k_, k_ + window_tile_floats<DH, WF_TILE>(), tiles.at(t) * 32, 0, a.w, span, false, view, m, g);
      if (more) next.store(wff_smem + ((t + 1) & 1) * STAGE);
    }
    x.l = sum_groups(x.l);
    if (__any(q < rows && plain::not_finite(x.o)) && q < rows) {
      plain::clear(x.o);
      const VisibleList vis(a.w, q);
#pragma unroll 1
      for (int t = 0; t < vis.count; ++t) {
        const float* kr = k + vis.at(t) * ld;
        plain::add_row(x.o, __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(base + q * ld + hd * DH, kr), head_scale<DH>() * WF_LOG2E, x.m_neg)),
                       kr + a.H_kv * DH, g);
      }
    }
  }
  if (q >= a.S) return;
  if (q >= rows) x.clear();
  store_row<DH>(o + (((long)b * a.S + q) * a.H + hd) * DH, x.o, g, q < rows ? 1.0f / x.l : 0.f);
  if (g == 0) lse[(long)bh * a.S + q] = q < rows ? (x.m + __builtin_amdgcn_logf(x.l)) * WF_LN2 : 0.f;   // v_log_f32 is log2
}

// D = rowsum(dO * O) and -lse log2(e) of every row, in rows padded to whole blocks of 128; 0 and -inf (probability 0) behind a document
template <int DH>
__global__ void __launch_bounds__(WF_THREADS) window_stats_f32(FWindowArgs a, const float* __restrict__ o, const float* __restrict__ d_o,
                                                               const float* __restrict__ lse, float* __restrict__ dsum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int n_bh = a.B * a.H, nb = (a.S + 127) / 128 * 2, bh = blockIdx.x / nb, b = bh / a.H, hd = bh - b * a.H;
  const int q = (blockIdx.x - bh * nb) * WF_ROWS + 16 * wave + m, rows = document_rows(a.lengths, b, a.S);
  const long at = (((long)b * a.S + q) * a.H + hd) * DH, Sp = nb * 64L;
  const float D = row_dot<DH>(load_row<DH>(d_o + at, g, q < rows), load_row<DH>(o + at, g, q < rows));
  if (g == 0) {
    dsum[bh * Sp + q] = D;
    dsum[(n_bh + bh) * Sp + q] = q < rows ? -lse[(long)bh * a.S + q] * WF_LOG2E : -INFINITY;
  }
}

template <int DH> __device__ __forceinline__ void window_dq_f32(const FWindowArgs& a, const float* __restrict__ d_o, const float* __restrict__ dsum,
                                                                float* __restrict__ dqkv, int bh, int qb, float* smem) {
  constexpr int STAGE = wf_stage<DH>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int b = bh / a.H, hd = bh - b * a.H, hk = hd / (a.H / a.H_kv), q0 = qb * WF_ROWS, qw0 = q0 + 16 * wave, q = qw0 + m;
  const int rows = document_rows(a.lengths, b, a.S);
  const long ld = (long)(a.H + 2 * a.H_kv) * DH, Sp = (a.S + 127) / 128 * 128L, grow = (((long)b * a.S + q) * a.H + hd) * DH;
  const float* const base = a.qkv + (long)b * a.S * ld;
  const float sc = head_scale<DH>() * WF_LOG2E;
  const FRowSpan span{qw0, qw0 < rows ? min(qw0 + 15, rows - 1) : -1};
  const int near = a.w.near_from(q);
  f32x4 dq[DH / 16];
  zero_acc<DH>(dq);
  if (q0 < rows) {
    const float* const k = base + (a.H + hk) * DH;
    const RowFrag<DH> qf = load_row<DH>(base + q * ld + hd * DH, g, q < rows), gf = load_row<DH>(d_o + grow, g, q < rows);
    const float D = dsum[bh * Sp + q], nlse2 = dsum[((long)a.B * a.H + bh) * Sp + q];
    const TileList<5> tiles(a.w, q0, min(q0 + WF_ROWS - 1, rows - 1));
    TileMover<DH, WF_TILE> next;
    auto load = [&](int t) {
      const int row0 = tiles.at(t) * 32;
      next.load([&](int r, const float*& p0, const float*& p1) {
        p0 = k + min(row0 + r, rows - 1) * ld;
        p1 = p0 + a.H_kv * DH;
      });
    };
    load(0);
    next.store(smem);
    for (int t = 0; t < tiles.count; ++t) {
      const float* k_ = smem + (t & 1) * STAGE;
      const float* v_ = k_ + window_tile_floats<DH, WF_TILE>();
      const bool more = t + 1 < tiles.count;
      if (more) load(t + 1);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k0 = tiles.at(t) * 32 + 16 * i, s = seen_16(a.w, span, k0);
        if (s == F_NONE) continue;   // wave-uniform
        f32x4 st = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
        rows_product<DH>(st, k_, i, qf, m, g);
        rows_product<DH>(dp, v_, i, gf, m, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // without the factor 1 / sqrt(d_head), which dQ gets when it is stored
          const int key = k0 + 4 * g + e;
          st[e] = s == F_ALL || (key <= q && (key >= near || key < a.w.sinks)) ? __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], sc, nlse2)) * (dp[e] - D) : 0.f;
        }
        cols_product<DH>(dq, k_, i, st, m, g);
      }
      if (more) next.store(smem + ((t + 1) & 1) * STAGE);
    }
    if (__any(q < rows && plain::not_finite(dq)) && q < rows) {
      plain::clear(dq);
      const VisibleList vis(a.w, q);
#pragma unroll 1
      for (int t = 0; t < vis.count; ++t) {
        const float* kr = k + vis.at(t) * ld;
        plain::add_row(dq, __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(base + q * ld + hd * DH, kr), sc, nlse2)) *
                               (plain::dot<DH>(d_o + grow, kr + a.H_kv * DH) - D), kr, g);
      }
    }
  }
  if (q >= a.S) return;
  if (q >= rows) zero_acc<DH>(dq);
  store_row<DH>(dqkv + ((long)b * a.S + q) * ld + hd * DH, dq, g, head_scale<DH>());
}

// A part's sums of 16 sinks, 32 DH floats (dK, then dV), in rows of their own of the q part of dqkv, H DH floats each
struct FSinkParts {
  int groups, parts, rows;   // of 16 sinks, parts a group, rows a part: ceil(32 / H)
  template <int DH> __device__ __forceinline__ float* at(float* dqkv, int b, int S, int H, long ld, int hk, int group, int part, int f) const {
    const int per_row = H * DH, row = ((hk * groups + group) * parts + part) * rows + f / per_row;
    return dqkv + ((long)b * S + row) * ld + f % per_row;
  }
};
enum { F_KEYS = 0, F_SINKS_WHOLE = 1, F_SINKS_PART = 2, F_KEYS_SHARED = 3 };

// where a wave's sums of its keys (four lanes each) are not finite: the pairs that see each other alone
template <int DH>
__device__ __forceinline__ void keys_if_not_finite(f32x4 (&dk)[DH / 16], f32x4 (&dv)[DH / 16], const FWindowArgs& a, const float* __restrict__ d_o,
                                                   const float* __restrict__ dsum, int b, int hk, int key, int key_last, int rows, int g) {
  if (!(__any(key < rows && (plain::not_finite(dk) || plain::not_finite(dv))) && key < rows)) return;
  const int G = a.H / a.H_kv;
  const long ld = (long)(a.H + 2 * a.H_kv) * DH, Sp = (a.S + 127) / 128 * 128L;
  const float* const base = a.qkv + (long)b * a.S * ld;
  const float* const krow = base + key * ld + (a.H + hk) * DH;
  plain::clear(dk);
  plain::clear(dv);
#pragma unroll 1
  for (int h = 0; h < G; ++h) {
    const float* const D = dsum + (long)(b * a.H + hk * G + h) * Sp;
    const float* const L = D + (long)a.B * a.H * Sp;
#pragma unroll 1
    for (int i = key; i <= key_last; ++i) {
      const float* qr = base + i * ld + (hk * G + h) * DH;
      const float* gr = d_o + (((long)b * a.S + i) * a.H + hk * G + h) * DH;
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(qr, krow), head_scale<DH>() * WF_LOG2E, L[i]));
      plain::add_row(dv, p, gr, g);
      plain::add_row(dk, p * (plain::dot<DH>(gr, krow + a.H_kv * DH) - D[i]), qr, g);
    }
  }
}
// a key's dK and dV; 0 behind the document
template <int DH>
__device__ __forceinline__ void store_keys(f32x4 (&dk)[DH / 16], f32x4 (&dv)[DH / 16], const FWindowArgs& a, float* __restrict__ dqkv, int b, int hk, int key, bool inside,
                                           int g) {
  if (!inside) { zero_acc<DH>(dk); zero_acc<DH>(dv); }
  float* const out = dqkv + ((long)b * a.S + key) * (a.H + 2 * a.H_kv) * DH + (a.H + hk) * DH;
  store_row<DH>(out, dk, g, head_scale<DH>());
  store_row<DH>(out + a.H_kv * DH, dv, g, 1.0f);
}

// dK and dV: 64 keys of a key head over the queries that see them under the window alone; or 16 sinks over all queries behind them, the
// waves two and two on the halves of a stage, for dV and for dK, whole or in parts (attention_window_mfma.hip).  A launch of few blocks of keys takes 16 keys a
// workgroup too: fewer than compute units (head size 128: than 160) where heads share keys, fewer than 64 where each has its own.  us whole | shared, head size 64,
// then 128: 1 x 2048, 16 heads on 4, window 256 (128 blocks) 144 | 104, 237 | 212; 24 on 6 (192) 158 | 147, 260 | 304; 64: 1 x 2000, 8 on 2, causal (64) 735 | 383;
// heads of their own: 1 x 300, 8 heads, window 64 (40) 18.2 | 16.1, 28.7 | 25.0; 1 x 512, 8, causal (64) 53.4 | 54.3, 91 | 95; 1 x 1024, 8, window 256 (128) 36 | 44,
// 61 | 102; 14, window 64 (224) 25 | 32.5, 42 | 62, causal 130 | 121, 234 | 303.
template <int DH, int KIND>
__device__ __forceinline__ void window_dkv_f32(const FWindowArgs& a, const float* __restrict__ d_o, const float* __restrict__ dsum, float* __restrict__ dqkv, int b,
                                               int hk, int k0, float* smem, const FSinkParts& sp, int part) {
  constexpr bool SINKS = KIND == F_SINKS_WHOLE || KIND == F_SINKS_PART, SHARED = KIND != F_KEYS;   // SHARED: the waves share 16 keys
  constexpr int BLOCK = SHARED ? 16 : WF_ROWS;
  constexpr int STAGE = wf_stage<DH>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int rows = document_rows(a.lengths, b, a.S), G = a.H / a.H_kv;
  const int sinks = rows <= a.w.window ? 0 : min(a.w.sinks, rows);   // a window that covers the document leaves the sinks nothing of their own
  if (SINKS && k0 >= sinks) return;
  const long ld = (long)(a.H + 2 * a.H_kv) * DH, Sp = (a.S + 127) / 128 * 128L;
  const int kw0 = k0 + (SHARED ? 0 : 16 * wave), key = kw0 + m, head0 = b * a.H + hk * G;
  const float* const base = a.qkv + (long)b * a.S * ld;
  const float* const krow = base + key * ld + (a.H + hk) * DH;
  const int last = SINKS ? rows - 1 : min(rows - 1, kw0 + 15 + a.w.window - 1), key_last = SINKS ? rows - 1 : min(rows - 1, key + a.w.window - 1);
  const bool idle = kw0 >= rows || (!SINKS && kw0 + 15 < sinks);
  const bool want_v = !SHARED || wave < 2, want_k = !SHARED || wave >= 2;
  const float sc = head_scale<DH>() * WF_LOG2E;
  f32x4 dk[DH / 16], dv[DH / 16];
  zero_acc<DH>(dk);
  zero_acc<DH>(dv);
  if (k0 < rows && (SINKS || k0 + BLOCK - 1 >= sinks)) {
    const RowFrag<DH> kf = load_row<DH>(krow, g, key < rows), vf = load_row<DH>(krow + a.H_kv * DH, g, key < rows);
    const int block_last = SINKS ? rows - 1 : min(rows - 1, k0 + BLOCK - 1 + a.w.window - 1);
    const int first = k0 >> 5, n_tiles = (block_last >> 5) + 1 - first;
    int steps = G * n_tiles, done = 0;   // steps of the parts in front of this one
    if constexpr (KIND == F_SINKS_PART) {
      const int per = (steps + sp.parts - 1) / sp.parts;
      done = min(part * per, steps);
      steps = min(per, steps - done);
    }
    TileMover<DH, WF_TILE> next;
    float next_stat = 0.f;
    int load_head = done / n_tiles, load_tile = first + done - load_head * n_tiles, qt = load_tile;
    auto load = [&]() {   // the heads of the group one after the other; threads 0 .. 31 move -lse log2(e), 32 .. 63 D
      const float* const q = base + (hk * G + load_head) * DH;
      const float* const go = d_o + ((long)b * a.S * a.H + hk * G + load_head) * DH;
      next.load([&](int r, const float*& p0, const float*& p1) {
        const long row = min(load_tile * 32 + r, rows - 1);
        p0 = q + row * ld;
        p1 = go + row * a.H * DH;
      });
      if (threadIdx.x < 2 * WF_TILE)
        next_stat = dsum[((threadIdx.x < WF_TILE ? (long)a.B * a.H : 0) + head0 + load_head) * Sp + load_tile * 32 + (threadIdx.x & (WF_TILE - 1))];
      if (++load_tile == first + n_tiles) { load_tile = first; ++load_head; }
    };
    auto store = [&](float* stage) {
      next.store(stage);
      if (threadIdx.x < 2 * WF_TILE) stage[2 * window_tile_floats<DH, WF_TILE>() + threadIdx.x] = next_stat;
    };
    if (steps > 0) {
      load();
      store(smem);
    }
    for (int n = 0; n < steps; ++n) {
      const float* q_ = smem + (n & 1) * STAGE;
      const float* g_ = q_ + window_tile_floats<DH, WF_TILE>();
      const float* Ls = g_ + window_tile_floats<DH, WF_TILE>();
      const bool more = n + 1 < steps;
      if (more) load();
      __syncthreads();
      const int q0 = qt * 32;
      if (++qt == first + n_tiles) qt = first;
#pragma unroll
      for (int i = 0; i < (SHARED ? 1 : 2); ++i) {
        const int t = SHARED ? wave & 1 : i, qh = q0 + 16 * t;
        if (idle || qh + 15 < kw0 || qh > last) continue;   // wave-uniform
        f32x4 st = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
        rows_product<DH>(st, q_, t, kf, m, g);
        if (want_k) rows_product<DH>(dp, g_, t, vf, m, g);
        const float4 Lq = *reinterpret_cast<const float4*>(Ls + 16 * t + 4 * g), Dq = *reinterpret_cast<const float4*>(Ls + WF_TILE + 16 * t + 4 * g);
        const float L[4] = {Lq.x, Lq.y, Lq.z, Lq.w}, D[4] = {Dq.x, Dq.y, Dq.z, Dq.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int q = qh + 4 * g + e;
          const float p = q < key || q > key_last ? 0.f : __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], sc, L[e]));
          st[e] = p;
          dp[e] = q < key || q > key_last ? 0.f : p * (dp[e] - D[e]);
        }
        if (want_v) cols_product<DH>(dv, g_, t, st, m, g);
        if (want_k) cols_product<DH>(dk, q_, t, dp, m, g);
      }
      if (more) store(smem + ((n + 1) & 1) * STAGE);
    }
    if constexpr (SHARED) {   // waves 1 and 3 hand their half of the queries over; then wave 2 its dK to wave 0
      constexpr int PER = DH / 16 * 4 * WAVE;
      static_assert(3 * PER <= 2 * STAGE, "the sums fit in the stages");
      auto put = [&](const f32x4 (&v)[DH / 16], float* at) {
#pragma unroll
        for (int d = 0; d < DH / 16; ++d) *reinterpret_cast<f32x4*>(at + (d * WAVE + lane) * 4) = v[d];
      };
      auto add = [&](f32x4 (&v)[DH / 16], const float* at) {
#pragma unroll
        for (int d = 0; d < DH / 16; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[d][e] += at[(d * WAVE + lane) * 4 + e];
      };
      __syncthreads();
      if (wave == 1) put(dv, smem);
      if (wave == 3) put(dk, smem + PER);
      __syncthreads();
      if (wave == 0) add(dv, smem);
      if (wave == 2) {
        add(dk, smem + PER);
        put(dk, smem + 2 * PER);
      }
      __syncthreads();
      if (wave != 0) return;
      add(dk, smem + 2 * PER);
    }
    if constexpr (KIND == F_SINKS_PART) {
#pragma unroll
      for (int d = 0; d < DH / 16; ++d) {
        *reinterpret_cast<f32x4*>(sp.at<DH>(dqkv, b, a.S, a.H, ld, hk, k0 >> 4, part, (d * WAVE + lane) * 4)) = dk[d];
        *reinterpret_cast<f32x4*>(sp.at<DH>(dqkv, b, a.S, a.H, ld, hk, k0 >> 4, part, ((DH / 16 + d) * WAVE + lane) * 4)) = dv[d];
      }
      return;
    }
    keys_if_not_finite<DH>(dk, dv, a, d_o, dsum, b, hk, key, key_last, rows, g);
  }
  if (SHARED && wave != 0) return;   // blocks behind the document
  if (key >= a.S || (SINKS ? key >= sinks : key < sinks)) return;
  store_keys<DH>(dk, dv, a, dqkv, b, hk, key, key < rows, g);
}
// The parts' sums of 16 sinks added in their order, a quarter of them a wave, and stored: a workgroup per document, key head, 16 sinks and 16 columns
template <int DH>
__global__ void __launch_bounds__(WF_THREADS) window_sinks_join_f32(FWindowArgs a, const float* __restrict__ d_o, const float* __restrict__ dsum,
                                                                    float* __restrict__ dqkv, FSinkParts sp) {
  constexpr int ND = DH / 16;
  __shared__ __attribute__((aligned(16))) f32x4 sums[3][WAVE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
  const int n_kv = a.B * a.H_kv, unit = blockIdx.x / (2 * ND), n = blockIdx.x - unit * 2 * ND, group = unit / n_kv, bk = unit - group * n_kv, b = bk / a.H_kv,
            hk = bk - b * a.H_kv;
  const int rows = document_rows(a.lengths, b, a.S), sinks = rows <= a.w.window ? 0 : min(a.w.sinks, rows);
  const long ld = (long)(a.H + 2 * a.H_kv) * DH;
  if (16 * group >= sinks) return;
  const int per = (sp.parts + 3) / 4, first = wave * per, end = min(first + per, sp.parts);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = first; p0 < end; p0 += 8) {   // eight parts at a time; those behind the last one count as zero
    f32x4 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const f32x4*>(sp.at<DH>(dqkv, b, a.S, a.H, ld, hk, group, min(p0 + i, end - 1), (n * WAVE + lane) * 4));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p0 + i < end) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[i][e];
      }
  }
  if (wave > 0) sums[wave - 1][lane] = v;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += sums[w][lane][e];
  const int key = 16 * group + (lane & 15);
  const f32x4 mine[1] = {v};
  if (__any(key < sinks && plain::not_finite(mine))) {
    f32x4 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) dk[d] = dv[d] = f32x4{INFINITY, 0.f, 0.f, 0.f};   // whatever it held: formed anew
    keys_if_not_finite<DH>(dk, dv, a, d_o, dsum, b, hk, key, rows - 1, rows, g);
#pragma unroll
    for (int d = 0; d < 2 * ND; ++d)
      if (d == n) v = d < ND ? dk[d < ND ? d : 0] : dv[d < ND ? 0 : d - ND];
  }
  if (key >= sinks) return;
  const float scale = n < ND ? head_scale<DH>() : 1.0f;
  *reinterpret_cast<float4*>(dqkv + ((long)b * a.S + key) * ld + (a.H + hk + (n < ND ? 0 : a.H_kv)) * DH + 16 * (n < ND ? n : n - ND) + 4 * g) =
      make_float4(v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale);
}
template <int DH>
__global__ void __launch_bounds__(WF_THREADS, 2) window_sink_parts_f32(FWindowArgs a, const float* __restrict__ d_o, const float* __restrict__ dsum,
                                                                       float* __restrict__ dqkv, FSinkParts sp) {
  extern __shared__ __attribute__((aligned(16))) float wpf_smem[];
  const int n_kv = a.B * a.H_kv, s = blockIdx.x / n_kv, bk = blockIdx.x - s * n_kv, b = bk / a.H_kv, group = s / sp.parts;
  window_dkv_f32<DH, F_SINKS_PART>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, 16 * group, wpf_smem, sp, s - group * sp.parts);
}

// One launch: the sinks' workgroups, which take longest, then those of dK / dV, then dQ's
template <int DH>
__global__ void __launch_bounds__(WF_THREADS, 2) window_bwd_f32(FWindowArgs a, const float* __restrict__ d_o, const float* __restrict__ dsum,
                                                                float* __restrict__ dqkv, int sink_blocks, bool shared) {
  extern __shared__ __attribute__((aligned(16))) float wbf_smem[];
  const int n_kv = a.B * a.H_kv, nb = (a.S + WF_ROWS - 1) / WF_ROWS;
  int i = blockIdx.x;
  if (i < sink_blocks * n_kv) {
    const int s = i / n_kv, bk = i - s * n_kv, b = bk / a.H_kv;
    window_dkv_f32<DH, F_SINKS_WHOLE>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, 16 * s, wbf_smem, FSinkParts{}, 0);
    return;
  }
  i -= sink_blocks * n_kv;
  const int key_blocks = shared ? 4 * nb : nb;
  if (i < n_kv * key_blocks) {
    const int kb = i / n_kv, bk = i - kb * n_kv, b = bk / a.H_kv;
    if (shared) window_dkv_f32<DH, F_KEYS_SHARED>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, 16 * kb, wbf_smem, FSinkParts{}, 0);
    else window_dkv_f32<DH, F_KEYS>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, WF_ROWS * kb, wbf_smem, FSinkParts{}, 0);
    return;
  }
  i -= n_kv * key_blocks;
  const int n_bh = a.B * a.H, qb = i / n_bh;
  window_dq_f32<DH>(a, d_o, dsum, dqkv, i - qb * n_bh, nb - 1 - qb, wbf_smem);
}

}  // namespace

template <int DH>
dipaco_status launch_window_fwd_f32(const float* qkv, const int* lengths, float* o, float* lse, int B, int S, int H, int H_kv, Window w, hipStream_t s) {
  constexpr int LDS = 2 * wf_stage<DH>() * (int)sizeof(float);
  static std::atomic<unsigned long long> lds_set{0};
  if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_fwd_f32<DH>), LDS, lds_set)) return st;
  window_fwd_f32<DH><<<B * H * ((S + WF_ROWS - 1) / WF_ROWS), WF_THREADS, LDS, s>>>(FWindowArgs{qkv, lengths, B, S, H, H_kv, w}, o, lse);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
template <int DH>
dipaco_status launch_window_bwd_f32(const float* qkv, const int* lengths, const float* o, const float* d_o, const float* lse, float* dqkv, float* dsum, int B,
                                    int S, int H, int H_kv, Window w, hipStream_t s) {
  constexpr int LDS = 2 * wf_stage<DH>() * (int)sizeof(float);
  static std::atomic<unsigned long long> lds_set{0};
  if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_bwd_f32<DH>), LDS, lds_set)) return st;
  const FWindowArgs a{qkv, lengths, B, S, H, H_kv, w};
  const int nb = (S + WF_ROWS - 1) / WF_ROWS, G = H / H_kv;
  int sink_blocks = w.window >= S ? 0 : (std::min(w.sinks, S) + 15) / 16;
  // As in attention_window_mfma.hip; stages of 32 queries, eight or more a part, 768 workgroups at a time.  us whole | cut (stages, those of the rest): 1 x 8192, 8
  // heads of 64 on 2, window 512 (1024, 50) 1400 | 320; 1 x 2048, 14 of 64, window 256 (64, 12) 130 | 104; 1 x 1000, 8, window 100 (32, 2) 51 | 46; 1 x 700, window
  // 64 (22, 1) 37 | 41; 1 x 16384, 14, window 1024 (512, 326) 1732 | 1721; 4 x 4000, 8 on 4, window 1000 (250, 178) 864 | 871; window 500, 8 heads (125, 94) 514 |
  // 529.  The first four with four stages a part 321, 99, 41, 33.5, with sixteen 328, 114, 56, 38.
  FSinkParts sp{sink_blocks, 1, (32 + H - 1) / H};
  const int64_t stages = (int64_t)G * ((S + 31) / 32), rest = (int64_t)2 * B * H * nb * ((w.window + 64) / 32 + 1) / 768;
  if (sink_blocks && stages > rest + 24 && 10 * stages > 18 * rest) sp.parts = (int)std::min<int64_t>(stages / 8, S / ((int64_t)H_kv * sink_blocks * sp.rows));
  window_stats_f32<DH><<<B * H * ((S + 127) / 128 * 2), WF_THREADS, 0, s>>>(a, o, d_o, lse, dsum);
  DIPACO_LAUNCH_CHECK();
  if (sink_blocks && sp.parts > 1) {
    static std::atomic<unsigned long long> parts_lds{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_sink_parts_f32<DH>), LDS, parts_lds)) return st;
    window_sink_parts_f32<DH><<<B * H_kv * sink_blocks * sp.parts, WF_THREADS, LDS, s>>>(a, d_o, dsum, dqkv, sp);
    DIPACO_LAUNCH_CHECK();
    window_sinks_join_f32<DH><<<B * H_kv * sink_blocks * (DH / 8), WF_THREADS, 0, s>>>(a, d_o, dsum, dqkv, sp);
    DIPACO_LAUNCH_CHECK();
    sink_blocks = 0;
  }
  const bool shared = (int64_t)B * H_kv * nb < (G == 1 ? 64 : DH == 128 ? 160 : 256);   // F_KEYS_SHARED, as measured at window_dkv_f32
  window_bwd_f32<DH><<<B * H_kv * (sink_blocks + (shared ? 4 : 1) * nb) + B * H * nb, WF_THREADS, LDS, s>>>(a, d_o, dsum, dqkv, sink_blocks, shared);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
#define DIPACO_WINDOW_F32(DH)                                                                                                                          \
  template dipaco_status launch_window_fwd_f32<DH>(const float*, const int*, float*, float*, int, int, int, int, Window, hipStream_t);                 \
  template dipaco_status launch_window_bwd_f32<DH>(const float*, const int*, const float*, const float*, const float*, float*, float*, int, int, int, \
                                                   int, Window, hipStream_t);
DIPACO_WINDOW_F32(32)
DIPACO_WINDOW_F32(64)
DIPACO_WINDOW_F32(128)

}  // namespace dipaco
