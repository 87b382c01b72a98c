// bf16 attention with a sliding window and sinks over packed rows of a padded batch (window_mfma.h has the forward pass's inner loops).
//
// Backward: dQ per block of 128 queries and dK / dV per block of 128 keys, each forming S and dO.V^T anew (seven products where one pass would need five), so
// that every output has one writer and a fixed order of sums.  Us: 16 x 2048, 14 heads of 64, window 512, 4 sinks 310 (the statistics 23 of them); 4 x 8000, 16
// heads of 128 on 4, window 1000 1335; 8 x 2048, 8 heads, causal, of 128 338 (attention_mfma.h in the same run 352), of 64 139 (154).
//
// Rows that a wave ends with results that are not finite are taken again over the pairs that see each other alone (attention_plain.h says
// why), so that such values reach exactly the rows that see them.
#include "kernels.h"
#include "window_mfma.h"

namespace dipaco {

namespace {

struct WindowArgs {
  const bf16* qkv;
  const int* lengths;
  int B, S, H, H_kv;
  Window w;
};

// ---- forward -----------------------------------------------------------------------------------------------------
// A workgroup per 128 queries of a head, the last ones first: under a window that covers the document these are the longest
// NG = 2: two groups of four waves take the block's tiles in turn, each in stages of its own, and their sums meet in LDS.
template <int DH, int NG>
__global__ void __launch_bounds__(AT_THREADS * NG, NG == 2 || DH == 128 ? 2 : 3) window_fwd_mfma(WindowArgs a, bf16* __restrict__ o, float* __restrict__ lse) {
  constexpr int KS = DH / 16, DT = DH / 32, TILE_BYTES = tile_bytes<DH>();
  extern __shared__ __attribute__((aligned(16))) char wf_rings[];   // [group][stage][K | V]
  const int lane = threadIdx.x & 63, wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  const int grp = NG == 1 ? 0 : wave_all >> 2, wave = wave_all & 3;
  char* const wf_smem = wf_rings + grp * 4 * TILE_BYTES;
  const int n_bh = a.B * a.H, qb = (int)blockIdx.x / n_bh, bh = (int)blockIdx.x - qb * n_bh, b = bh / a.H, hd = bh - b * a.H, hk = hd / (a.H / a.H_kv);
  const int q0 = ((a.S + 127) / 128 - 1 - qb) * 128, q = q0 + 32 * wave + r;
  const int rows = document_rows(a.lengths, b, a.S), ld = (a.H + 2 * a.H_kv) * DH;
  const bf16* const base = a.qkv + (long)b * a.S * ld;
  const bf16* const qrow = base + (long)q * ld + hd * DH;
  const RowSpan span{q0 + 32 * wave, q0 + 32 * wave < rows ? min(q0 + 32 * wave + 31, rows - 1) : -1};
  SoftmaxRow<DH> x;
  x.clear();
  const ChainView view{q, a.w.near_from(q), a.w.sinks};
  const float sc = score_scale<DH>() * LOG2E;
  if (q0 < rows) {
    uint4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = q < rows ? *reinterpret_cast<const uint4*>(qrow + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
    const FragOff fo = frag_offsets(lane);
    const TrOff to = tr_offsets(lane);
    const uint32_t smem_addr = (uint32_t)(uintptr_t)wf_smem;
    const bf16* const k = base + (a.H + hk) * DH;
    const RowTiles<DH> src(k, k + a.H_kv * DH, ld, ld, rows, wave, lane);
    const TileList<6> tiles(a.w, q0, min(q0 + 127, rows - 1));
    if (grp < tiles.count) src.issue(tiles.at(grp), wave, lane, smem_addr);
    auto tile = [&](auto CUR, int t) {
      constexpr int cur = decltype(CUR)::value;
      wait_vmcnt<0>();
      __syncthreads();   // tile t is in LDS, and nobody still reads the other stage
      if (t + NG < tiles.count) src.issue(tiles.at(t + NG), wave, lane, smem_addr + (1 - cur) * 2 * TILE_BYTES);
      if (NG == 2 && t >= tiles.count) return;
      const char* k_ = wf_smem + cur * 2 * TILE_BYTES;
      attend_tile<DH>(x, qf, k_, k_ + TILE_BYTES, fo, to, tiles.at(t) * 64, 0, a.w, span, 0, view, lane);
    };
    for (int t = 0; t < tiles.count; t += 2 * NG) {   // both groups walk as often as the first: the barriers are the workgroup's
      tile(std::integral_constant<int, 0>{}, t + grp);
      if (t + NG < tiles.count) tile(std::integral_constant<int, 1>{}, t + NG + grp);
    }
    if constexpr (NG == 2) {
      constexpr int PER = (16 * DT + 2) * WAVE;   // floats a wave hands over: O^T, the reference exponent, the half row sum
      static_assert(4 * PER * 4 <= NG * 4 * TILE_BYTES, "the sums fit in the rings");
      float* const at = reinterpret_cast<float*>(wf_rings) + wave * PER;
      __syncthreads();   // the rings have been read
      if (grp == 1) {
        hand_over(x.o, at, lane);
        at[16 * DT * WAVE + lane] = x.m;
        at[(16 * DT + 1) * WAVE + lane] = x.l;
      }
      __syncthreads();
      if (grp == 1) return;
      const float m1 = at[16 * DT * WAVE + lane], mn = fmaxf(x.m, m1);   // -inf: a group that has seen nothing
      const float c0 = x.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.m - mn), c1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - mn);
      x.l = x.l * c0 + at[(16 * DT + 1) * WAVE + lane] * c1;
      take_over(x.o, at, c0, c1, lane);
      x.m = mn;
      x.m_neg = -mn;
    }
    x.l += __shfl_xor(x.l, 32, WAVE);
    if (__any(q < rows && plain::not_finite(x.o)) && q < rows) {
      plain::clear(x.o);
      int q_again = q;
      asm volatile("" : "+v"(q_again));   // formed anew, not kept through the loop
      const VisibleList vis(a.w, q_again);
#pragma unroll 1
      for (int t = 0; t < vis.count; ++t) {
        const bf16* kr = src.t0 + (long)vis.at(t) * ld;
        plain::add_row(x.o, __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(base + (long)q_again * ld + hd * DH, kr), sc, x.m_neg)), kr + a.H_kv * DH, h);
      }
    }
  }
  if (grp == 1) return;   // blocks behind the document
  int q_out = q;          // addresses of the outputs are formed behind the loop
  asm volatile("" : "+v"(q_out));
  if (q_out < a.S) {
    bf16* const out = o + ((long)b * a.S + q_out) * a.H * DH + hd * DH;
    if (q_out >= rows) x.clear();
    store_transposed_out(out, x.o, h, q_out < rows ? 1.0f / x.l : 0.f);
    if (h == 0) lse[(long)bh * a.S + q_out] = q_out < rows ? (x.m + __builtin_amdgcn_logf(x.l)) * LN2 : 0.f;   // v_log_f32 is log2
  }
}

// ---- backward: -D = -rowsum(dO * O) and -lse log2(e) of every row, in rows padded to whole blocks of 128 -----------------------------
// -D is what the products dO.V^T start from: the subtraction costs nothing.  Behind a document D is 0 and -lse log2(e) is -inf (probability 0), so that the blocks below need no bounds check.
template <int DH>
__global__ void __launch_bounds__(AT_THREADS) window_stats_mfma(WindowArgs a, const bf16* __restrict__ o, const bf16* __restrict__ d_o,
                                                               const float* __restrict__ lse, float* __restrict__ dsum) {
  constexpr int LANES = DH / 8, ROWS = AT_THREADS / LANES;   // lanes of a row, rows of a workgroup at a time
  const int n_bh = a.B * a.H, nqb = (a.S + 127) / 128, bh = blockIdx.x / nqb, qb = blockIdx.x - bh * nqb, b = bh / a.H, hd = bh - b * a.H;
  const int c = 8 * (threadIdx.x % LANES), rows = document_rows(a.lengths, b, a.S);
  const long Sp = (long)nqb * 128;
#pragma unroll
  for (int i = 0; i < 128 / ROWS; ++i) {
    const int q = qb * 128 + ROWS * i + threadIdx.x / LANES;
    float D = 0.f;
    if (q < rows) {
      const size_t at = (((size_t)b * a.S + q) * a.H + hd) * DH + c;
      float x[8], y[8];
      load_vec16(o + at, x);
      load_vec16(d_o + at, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) D = __builtin_fmaf(x[e], y[e], D);
    }
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) D += __shfl_xor(D, m, WAVE);
    if (threadIdx.x % LANES == 0) {
      dsum[bh * Sp + q] = -D;
      dsum[(n_bh + bh) * Sp + q] = q < rows ? -lse[(long)bh * a.S + q] * LOG2E : -INFINITY;
    }
  }
}

// acc^T[dt] += (tile^T)[columns 32 dt .., the 32 rows from `tile` on] . src
template <int DT> __device__ __forceinline__ void mma_transposed_half(f32x16 (&acc)[DT], const char* tile, const TrOff& to, const f32x16& src) {
  if constexpr (split_p<32 * DT>()) {   // half a fragment at a time (attention_mfma.h: mma_transposed)
    const auto p0 = p_frag<true, 0>(src);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = mfma_p(tr_read(tile, to, dt, 0), p0, acc[dt]);
    const auto p1 = p_frag<true, 8>(src);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = mfma_p(tr_read(tile, to, dt, 1), p1, acc[dt]);
  } else {
    const uint4 p0 = pack8<0>(src), p1 = pack8<8>(src);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      acc[dt] = mfma16(tr_read(tile, to, dt, 0), p0, acc[dt]);
      acc[dt] = mfma16(tr_read(tile, to, dt, 1), p1, acc[dt]);
    }
  }
}

// ---- backward, dQ: 128 queries of a head ---------------------------------------------------------------------------
template <int DH> __device__ __forceinline__ void window_dq(const WindowArgs& a, const bf16* __restrict__ d_o, const float* __restrict__ dsum,
                                                            bf16* __restrict__ dqkv, int bh, int qb, char* smem) {
  constexpr int KS = DH / 16, DT = DH / 32, TILE_BYTES = tile_bytes<DH>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  const int b = bh / a.H, hd = bh - b * a.H, hk = hd / (a.H / a.H_kv), q0 = qb * 128, q = q0 + 32 * wave + r;
  const int rows = document_rows(a.lengths, b, a.S), ld = (a.H + 2 * a.H_kv) * DH;
  const long Sp = (a.S + 127) / 128 * 128L;
  const bf16* const base = a.qkv + (long)b * a.S * ld;
  const bf16* const qrow = base + (long)q * ld + hd * DH;
  const bf16* const grow = d_o + (((long)b * a.S + q) * a.H + hd) * DH;
  const RowSpan span{q0 + 32 * wave, q0 + 32 * wave < rows ? min(q0 + 32 * wave + 31, rows - 1) : -1};
  const int near = a.w.near_from(q);
  const float sc = score_scale<DH>() * LOG2E;
  f32x16 dq[DT];
  plain::clear(dq);
  if (q0 < rows) {
    uint4 qf[KS], gf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = q < rows ? *reinterpret_cast<const uint4*>(qrow + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
      gf[ks] = q < rows ? *reinterpret_cast<const uint4*>(grow + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
    }
    const float neg_d = dsum[bh * Sp + q], nlse2 = dsum[((long)a.B * a.H + bh) * Sp + q];
    const FragOff fo = frag_offsets(lane);
    const TrOff to = tr_offsets(lane);
    const uint32_t smem_addr = (uint32_t)(uintptr_t)smem;
    const bf16* const k = base + (a.H + hk) * DH;
    const RowTiles<DH> src(k, k + a.H_kv * DH, ld, ld, rows, wave, lane);
    const TileList<6> tiles(a.w, q0, min(q0 + 127, rows - 1));
    src.issue(tiles.at(0), wave, lane, smem_addr);
    f32x16 start;
#pragma unroll
    for (int e = 0; e < 16; ++e) start[e] = neg_d;
    for (int t = 0, cur = 0; t < tiles.count; ++t, cur ^= 1) {
      wait_vmcnt<0>();
      __syncthreads();   // tile t is in LDS, and nobody still reads the other stage
      if (t + 1 < tiles.count) src.issue(tiles.at(t + 1), wave, lane, smem_addr + (1 - cur) * 2 * TILE_BYTES);
      const int k0 = tiles.at(t) * 64;
      const char* k_ = smem + cur * 2 * TILE_BYTES;
      const char* v_ = k_ + TILE_BYTES;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int seen = seen_half(a.w, span, k0 + 32 * half);
        if (!seen) continue;   // wave-uniform
        f32x16 st, dp = start;
        zero(st);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          st = mfma16(row_frag(k_, fo, ks, half), qf[ks], st);
          dp = mfma16(row_frag(v_, fo, ks, half), gf[ks], dp);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)   // dS^T without the factor 1 / sqrt(d_head), which dQ gets when it is stored
          st[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], sc, nlse2)) * dp[e];
        hide(st, seen, 0.f, k0 + 32 * half, q, near, a.w.sinks, lane);
        mma_transposed_half(dq, k_ + 4096 * half, to, st);
      }
    }
    if (__any(q < rows && plain::not_finite(dq)) && q < rows) {
      plain::clear(dq);
      const VisibleList vis(a.w, q);
#pragma unroll 1
      for (int t = 0; t < vis.count; ++t) {
        const bf16* kr = k + (long)vis.at(t) * ld;
        plain::add_row(dq, __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(qrow, kr), sc, nlse2)) * (plain::dot<DH>(grow, kr + a.H_kv * DH) + neg_d), kr, h);
      }
    }
  }
  int q_out = q;
  asm volatile("" : "+v"(q_out));
  if (q_out < a.S) {
    if (q_out >= rows) plain::clear(dq);
    store_transposed_out(dqkv + ((long)b * a.S + q_out) * ld + hd * DH, dq, h, score_scale<DH>());
  }
}

// ---- backward, dK and dV ------------------------------------------------------------------------------------------
// Keys: 128 of a key head, 32 a wave, over the queries of every head of the group that see them under the window alone; the stages hold 64
// queries.  Sinks are seen by all queries behind them, a multiple of what the other keys take, so a workgroup takes only 32 of them (SINKS):
// its waves share the stage, two of them on each half of it, one for dV and one for dK, and the halves' sums meet at the end.
// A launch of few blocks of keys is made of such workgroups altogether (KEYS_SHARED): fewer than compute units where heads share keys (a block then takes the
// queries of a whole group and outlasts dQ's), fewer than 112 where each head has its own.  us whole | shared, head size 64, then 128: 1 x 8192, 8 heads on 1, window 512 (64 blocks)
// 146 | 80, 297 | 153; 1 x 4096, 16 on 4, window 256 (128) 57 | 42, 108 | 85; 2 x 4096, 12 on 3, window 1000 (192) 146 | 134, 305 | 299, window 256 60 | 56, 115 |
// 123; heads of their own: 1 x 512, 8 heads, causal (32) 22 | 17, 42 | 29; 1 x 2048, 6, window 256 (96) 20.3 | 19.2, 39 | 36.5; 8 heads (128) 18.9 | 20.1, 37 | 46,
// causal 59 | 56, 125 | 103; 10 heads, causal (160) 64 | 58.5, 131 | 127; 14 heads (224) 66.5 | 71.5, 139 | 144, window 256 25.6 | 32, 47 | 65.
// Where a workgroup for 32 sinks would still be the longest by far, the queries are cut among `parts` workgroups, whose sums lie in the rows of dqkv that dQ is
// written to afterwards (SinkParts), and window_sinks_join adds them.  1 x 32768 positions, 16 heads of 128 on 4, window 1024, 16 sinks: 3435 us
// uncut (without sinks 1378), 1449 cut; 8 heads of 64 on 1, 8192 positions, window 512, 4 sinks 772 | 106.
template <int DH> constexpr int window_dkv_stage() { return 2 * tile_bytes<DH>() + 2 * 64 * (int)sizeof(float); }   // Q | dO | -lse log2(e) | -D

// where a wave's sums of its keys (a lane pair each) are not finite: the pairs that see each other alone
template <int DH>
__device__ __forceinline__ void keys_if_not_finite(f32x16 (&dk)[DH / 32], f32x16 (&dv)[DH / 32], const WindowArgs& a, const bf16* __restrict__ d_o,
                                                   const float* __restrict__ dsum, int b, int hk, int key, int key_last, int rows, int h) {
  if (!(__any(key < rows && (plain::not_finite(dk) || plain::not_finite(dv))) && key < rows)) return;
  const int G = a.H / a.H_kv, ld = (a.H + 2 * a.H_kv) * DH;
  const long Sp = (a.S + 127) / 128 * 128L;
  const bf16* const base = a.qkv + (long)b * a.S * ld;
  const bf16* const krow = base + (long)key * ld + (a.H + hk) * DH;
  const float sc = score_scale<DH>() * LOG2E;
  plain::clear(dk);
  plain::clear(dv);
#pragma unroll 1
  for (int g = 0; g < G; ++g) {
    const float* const neg_d = dsum + (long)(b * a.H + hk * G + g) * Sp;
    const float* const L = neg_d + (long)a.B * a.H * Sp;
#pragma unroll 1
    for (int i = key; i <= key_last; ++i) {
      const bf16* qr = base + (long)i * ld + (hk * G + g) * DH;
      const bf16* gr = d_o + (((long)b * a.S + i) * a.H + hk * G + g) * DH;
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(qr, krow), sc, L[i]));
      plain::add_row(dv, p, gr, h);
      plain::add_row(dk, p * (plain::dot<DH>(gr, krow + a.H_kv * DH) + neg_d[i]), qr, h);
    }
  }
}
// a key's dK and dV; 0 behind the document
template <int DH>
__device__ __forceinline__ void store_keys(f32x16 (&dk)[DH / 32], f32x16 (&dv)[DH / 32], const WindowArgs& a, bf16* __restrict__ dqkv, int b, int hk, int key, bool inside,
                                           int h) {
  if (!inside) { plain::clear(dk); plain::clear(dv); }
  bf16* const out = dqkv + ((long)b * a.S + key) * (a.H + 2 * a.H_kv) * DH + (a.H + hk) * DH;
  store_transposed_out(out, dk, h, score_scale<DH>());
  store_transposed_out(out + a.H_kv * DH, dv, h, 1.0f);
}
// A part's sums of 32 sinks, 64 DH floats (dK, then dV, as hand_over leaves them), in rows of their own of the q part of dqkv, H DH / 2 floats each
struct SinkParts {
  int groups, parts, rows;   // of 32 sinks, parts a group, rows a part: ceil(128 / H)
  template <int DH> __device__ __forceinline__ float* at(bf16* dqkv, int b, int S, int H, int ld, int hk, int group, int part, int f) const {
    const int per_row = H * DH / 2, row = ((hk * groups + group) * parts + part) * rows + f / per_row;
    return reinterpret_cast<float*>(dqkv + ((long)b * S + row) * ld) + f % per_row;
  }
};
enum { KEYS = 0, SINKS_WHOLE = 1, SINKS_PART = 2, KEYS_SHARED = 3 };

template <int DH, int KIND>
__device__ __forceinline__ void window_dkv(const WindowArgs& a, const bf16* __restrict__ d_o, const float* __restrict__ dsum, bf16* __restrict__ dqkv, int b, int hk,
                                           int k0, char* smem, const SinkParts& sp, int part) {
  constexpr bool SINKS = KIND == SINKS_WHOLE || KIND == SINKS_PART, SHARED = KIND != KEYS;   // SHARED: the waves share 32 keys
  constexpr int BLOCK = SHARED ? 32 : 128;
  constexpr int KS = DH / 16, DT = DH / 32, TILE_BYTES = tile_bytes<DH>(), STAGE = window_dkv_stage<DH>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  const int rows = document_rows(a.lengths, b, a.S), ld = (a.H + 2 * a.H_kv) * DH, G = a.H / a.H_kv;
  const int sinks = rows <= a.w.window ? 0 : min(a.w.sinks, rows);   // a window that covers the document leaves the sinks nothing of their own
  if (SINKS && k0 >= sinks) return;
  const int kw0 = k0 + (SHARED ? 0 : 32 * wave), key = kw0 + r;
  const long Sp = (a.S + 127) / 128 * 128L;
  const bf16* const base = a.qkv + (long)b * a.S * ld;
  const bf16* const krow = base + (long)key * ld + (a.H + hk) * DH;
  // positions that see the wave's keys, and this lane's key
  const int last = SINKS ? rows - 1 : min(rows - 1, kw0 + 31 + a.w.window - 1);
  const int key_last = SINKS ? rows - 1 : min(rows - 1, key + a.w.window - 1);
  const bool idle = kw0 >= rows || (!SINKS && kw0 + 31 < sinks);
  const float sc = score_scale<DH>() * LOG2E;
  f32x16 dk[DT], dv[DT];
  plain::clear(dk);
  plain::clear(dv);
  if (k0 < rows && (SINKS || k0 + BLOCK - 1 >= sinks)) {
    uint4 kf[KS], vf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[ks] = key < rows ? *reinterpret_cast<const uint4*>(krow + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
      vf[ks] = key < rows ? *reinterpret_cast<const uint4*>(krow + a.H_kv * DH + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
    }
    FragOff fo = frag_offsets(lane);
    TrOff to = tr_offsets(lane);
    const uint32_t smem_addr = (uint32_t)(uintptr_t)smem;
    const int block_last = SINKS ? rows - 1 : min(rows - 1, k0 + BLOCK - 1 + a.w.window - 1);
    const int first = k0 >> 6, n_tiles = (block_last >> 6) + 1 - first;
    int steps = G * n_tiles, done = 0;   // steps of the parts in front of this one
    if constexpr (KIND == SINKS_PART) {
      const int per = (steps + sp.parts - 1) / sp.parts;
      done = min(part * per, steps);
      steps = min(per, steps - done);
    }
    const int head1 = done / n_tiles;    // the first step's head and tile
    const int head0 = b * a.H + hk * G;
    RowTiles<DH, true> src(base + hk * G * DH, d_o + ((long)b * a.S * a.H + hk * G) * DH, ld, a.H * DH, rows, wave, lane);
    // statistics of a tile's 64 queries: waves 0 and 2 fetch -lse log2(e), waves 1 and 3 fetch -D
    const float* stat = dsum + ((wave & 1 ? 0 : (long)a.B * a.H) + head0) * Sp + lane;
    const uint32_t stat_dst = 2 * TILE_BYTES + (wave & 1 ? 256 : 0);
    int next_tile = first + done - head1 * n_tiles;
    src.t0 += head1 * DH;
    src.t1 += head1 * DH;
    stat += head1 * Sp;
    auto issue = [&](int stage) {   // the next step's tile: the heads of the group one after the other
      src.issue(next_tile, wave, lane, smem_addr + stage * STAGE);
      load4_to_lds(stat + next_tile * 64, smem_addr + stage * STAGE + stat_dst);
      if (++next_tile == first + n_tiles) {
        next_tile = first;
        src.t0 += DH;
        src.t1 += DH;
        stat += Sp;
      }
    };
    int qt = next_tile;
    if (steps > 0) issue(0);
    for (int n = 0, cur = 0; n < steps; ++n, cur ^= 1) {
      wait_vmcnt<0>();
      __syncthreads();
      if (n + 1 < steps) issue(1 - cur);
      const int q0 = qt * 64;
      if (++qt == first + n_tiles) qt = first;
      const char* q_ = smem + cur * STAGE;
      const char* g_ = q_ + TILE_BYTES;
      const float* nlse2s = reinterpret_cast<const float*>(q_ + 2 * TILE_BYTES);
      const float* neg_ds = nlse2s + 64;
#pragma unroll
      for (int i = 0; i < (SHARED ? 1 : 2); ++i) {
        const int t = SHARED ? wave & 1 : i, qh = q0 + 32 * t;   // 32 queries
        if (idle || qh + 31 < kw0 || qh > last) continue;       // wave-uniform
        if constexpr (DH == 128) rederive_offsets(fo, to);
        const bool want_v = !SHARED || wave < 2, want_k = !SHARED || wave >= 2;
        // accumulator elements 4g .. 4g + 3 are queries 8g + 4h + (0..3) of the half: their statistics are 16 contiguous bytes
        f32x16 st, dp;
        zero(st);
        if (want_k) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float4 d = *reinterpret_cast<const float4*>(neg_ds + 32 * t + 8 * g + 4 * h);
            dp[4 * g] = d.x; dp[4 * g + 1] = d.y; dp[4 * g + 2] = d.z; dp[4 * g + 3] = d.w;
          }
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            st = mfma16(row_frag(q_ + 4096 * t, fo, ks, 0), kf[ks], st);
            dp = mfma16(row_frag(g_ + 4096 * t, fo, ks, 0), vf[ks], dp);
          }
        } else {
          zero(dp);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) st = mfma16(row_frag(q_ + 4096 * t, fo, ks, 0), kf[ks], st);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 Lq = *reinterpret_cast<const float4*>(nlse2s + 32 * t + 8 * g + 4 * h);
          const float Ls[4] = {Lq.x, Lq.y, Lq.z, Lq.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = 4 * g + j;
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], sc, Ls[j]));
            st[e] = p;
            dp[e] *= p;   // dS without 1 / sqrt(d_head), which dK gets when it is stored
          }
        }
        if (qh < kw0 + 31 || (!SINKS && qh + 31 > kw0 + a.w.window - 1)) {   // wave-uniform: some pair is hidden
          asm volatile("");   // a branch, not selections (window_mfma.h: hide)
          const int from = key - qh - 4 * h, upto = key_last - qh - 4 * h;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const bool hidden = 8 * (e >> 2) + (e & 3) < from || 8 * (e >> 2) + (e & 3) > upto;
            st[e] = hidden ? 0.f : st[e];
            dp[e] = hidden ? 0.f : dp[e];
          }
        }
        if (want_v) mma_transposed_half(dv, g_ + 4096 * t, to, st);
        if (want_k) mma_transposed_half(dk, q_ + 4096 * t, to, dp);
      }
    }
    if constexpr (SHARED) {   // the odd waves hand their half of the queries over; then wave 2 its dK to wave 0
      constexpr int PER = 16 * DT * WAVE;
      static_assert(3 * PER * 4 <= 2 * STAGE, "the sums fit in the stages");
      float* const at = reinterpret_cast<float*>(smem);
      __syncthreads();
      if (wave == 1) hand_over(dv, at, lane);
      if (wave == 3) hand_over(dk, at + PER, lane);
      __syncthreads();
      if (wave == 0) take_over(dv, at, 1.f, 1.f, lane);
      if (wave == 2) {
        take_over(dk, at + PER, 1.f, 1.f, lane);
        hand_over(dk, at + 2 * PER, lane);
      }
      __syncthreads();
      if (wave != 0) return;
      take_over(dk, at + 2 * PER, 0.f, 1.f, lane);
    }
    if constexpr (KIND == SINKS_PART) {
#pragma unroll
      for (int n = 0; n < 2 * DT; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16& v = n < DT ? dk[n < DT ? n : 0] : dv[n < DT ? 0 : n - DT];
          *reinterpret_cast<float4*>(sp.at<DH>(dqkv, b, a.S, a.H, ld, hk, k0 >> 5, part, ((n * 4 + g) * WAVE + lane) * 4)) =
              make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
        }
      return;
    }
    keys_if_not_finite<DH>(dk, dv, a, d_o, dsum, b, hk, key, key_last, rows, h);
  }
  if (SHARED && wave != 0) return;   // blocks behind the document
  int key_out = key;
  asm volatile("" : "+v"(key_out));
  if (key_out < a.S && (SINKS ? key_out < sinks : key_out >= sinks)) store_keys<DH>(dk, dv, a, dqkv, b, hk, key_out, key_out < rows, h);
}
// The parts' sums of 32 sinks added in their order, a quarter of them a wave, and stored: a workgroup per document, key head, 32 sinks and 32 columns
template <int DH>
__global__ void __launch_bounds__(AT_THREADS) window_sinks_join(WindowArgs a, const bf16* __restrict__ d_o, const float* __restrict__ dsum, bf16* __restrict__ dqkv,
                                                                SinkParts sp) {
  constexpr int DT = DH / 32;
  __shared__ __attribute__((aligned(16))) float sums[3][16 * WAVE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int n_kv = a.B * a.H_kv, unit = blockIdx.x / (2 * DT), n = blockIdx.x - unit * 2 * DT, group = unit / n_kv, bk = unit - group * n_kv, b = bk / a.H_kv,
            hk = bk - b * a.H_kv;
  const int rows = document_rows(a.lengths, b, a.S), ld = (a.H + 2 * a.H_kv) * DH, sinks = rows <= a.w.window ? 0 : min(a.w.sinks, rows);
  if (32 * group >= sinks) return;
  const int per = (sp.parts + 3) / 4, first = wave * per, end = min(first + per, sp.parts);
  f32x16 v[1];
  plain::clear(v);
  for (int p0 = first; p0 < end; p0 += 4) {   // four parts at a time; those behind the last one count as zero
    float4 w[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        w[i][g] = *reinterpret_cast<const float4*>(sp.at<DH>(dqkv, b, a.S, a.H, ld, hk, group, min(p0 + i, end - 1), ((n * 4 + g) * WAVE + lane) * 4));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p0 + i < end) {
#pragma unroll
        for (int g = 0; g < 4; ++g) { v[0][4 * g] += w[i][g].x; v[0][4 * g + 1] += w[i][g].y; v[0][4 * g + 2] += w[i][g].z; v[0][4 * g + 3] += w[i][g].w; }
      }
  }
  if (wave > 0) hand_over(v, sums[wave - 1], lane);
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) take_over(v, sums[w], 1.f, 1.f, lane);
  const int key = 32 * group + (lane & 31);
  if (__any(key < sinks && plain::not_finite(v))) {
    f32x16 dk[DT], dv[DT];
    plain::clear(dk);
    plain::clear(dv);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) { dk[dt][0] = INFINITY; dv[dt][0] = INFINITY; }   // whatever it held: formed anew
    keys_if_not_finite<DH>(dk, dv, a, d_o, dsum, b, hk, key, rows - 1, rows, h);
#pragma unroll
    for (int dt = 0; dt < 2 * DT; ++dt)
      if (dt == n) v[0] = dt < DT ? dk[dt < DT ? dt : 0] : dv[dt < DT ? 0 : dt - DT];
  }
  if (key >= sinks) return;
  bf16* const out = dqkv + ((long)b * a.S + key) * ld + (a.H + hk + (n < DT ? 0 : a.H_kv)) * DH + 32 * (n < DT ? n : n - DT);
#pragma unroll
  for (int g = 0; g < 4; ++g) store4(out + 8 * g + 4 * h, v[0], g, n < DT ? score_scale<DH>() : 1.0f);
}

// One launch: the sinks' workgroups, which take longest, then those of dK / dV, then dQ's.  A kernel for either kind of dK / dV: with both in one, head size 64
// has 169 registers, two waves a SIMD.
template <int DH, bool SHARED>
__global__ void __launch_bounds__(AT_THREADS, DH == 128 ? 2 : 3) window_bwd_mfma(WindowArgs a, const bf16* __restrict__ d_o, const float* __restrict__ dsum,
                                                                                 bf16* __restrict__ dqkv, int sink_blocks) {
  extern __shared__ __attribute__((aligned(16))) char wb_smem[];
  const int n_kv = a.B * a.H_kv, nb = (a.S + 127) / 128;
  int i = blockIdx.x;
  if (i < sink_blocks * n_kv) {
    const int s = i / n_kv, bk = i - s * n_kv, b = bk / a.H_kv;
    window_dkv<DH, SINKS_WHOLE>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, 32 * s, wb_smem, SinkParts{}, 0);
    return;
  }
  i -= sink_blocks * n_kv;
  const int key_blocks = SHARED ? 4 * nb : nb;
  if (i < n_kv * key_blocks) {
    const int kb = i / n_kv, bk = i - kb * n_kv, b = bk / a.H_kv;
    window_dkv<DH, SHARED ? KEYS_SHARED : KEYS>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, (SHARED ? 32 : 128) * kb, wb_smem, SinkParts{}, 0);
    return;
  }
  i -= n_kv * key_blocks;
  const int n_bh = a.B * a.H, qb = i / n_bh;
  window_dq<DH>(a, d_o, dsum, dqkv, i - qb * n_bh, nb - 1 - qb, wb_smem);
}

template <int DH>
__global__ void __launch_bounds__(AT_THREADS, 2) window_sink_parts(WindowArgs a, const bf16* __restrict__ d_o, const float* __restrict__ dsum, bf16* __restrict__ dqkv,
                                                                   SinkParts sp) {
  extern __shared__ __attribute__((aligned(16))) char wp_smem[];
  const int n_kv = a.B * a.H_kv, s = blockIdx.x / n_kv, bk = blockIdx.x - s * n_kv, b = bk / a.H_kv, group = s / sp.parts;
  window_dkv<DH, SINKS_PART>(a, d_o, dsum, dqkv, b, bk - b * a.H_kv, 32 * group, wp_smem, sp, s - group * sp.parts);
}

}  // namespace

template <int DH>
dipaco_status launch_window_fwd_mfma(const bf16* qkv, const int* lengths, bf16* o, float* lse, int B, int S, int H, int H_kv, Window w, hipStream_t s) {
  const int nqb = (S + 127) / 128, blocks = B * H * nqb;
  auto run = [&](auto NGc) -> dipaco_status {
    constexpr int NG = decltype(NGc)::value, LDS = NG * 4 * tile_bytes<DH>();
    static std::atomic<unsigned long long> lds_set{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_fwd_mfma<DH, NG>), LDS, lds_set)) return st;
    window_fwd_mfma<DH, NG><<<blocks, AT_THREADS * NG, LDS, s>>>(WindowArgs{qkv, lengths, B, S, H, H_kv, w}, o, lse);
    DIPACO_LAUNCH_CHECK();
    return DIPACO_OK;
  };
  // Two groups where the longest block's tiles, at least seven of them, are the launch's length: the blocks' tiles together are no more than 256 compute units
  // take in that time.  us one -> two (blocks, tiles), head size 64, then 128: 1 x 2048, 14 heads, window 512 (224, 11) 16.5 -> 14.3, 26.8 -> 25.3; 1 x 2000, 8
  // heads, causal (128, 32) 32.8 -> 24.7, 53 -> 44; 2 x 2048, 14 heads, causal (448, 32) 35.5 -> 30.6, 64 -> 59; 8 x 512, 8 heads, causal (256, 8) 11.2 -> 10.7,
  // 18.1 -> 18.7; beyond: 1 x 4096, 14 heads, window 512 (448, 11) 21.3 -> 24.5, 39 -> 46; 4 x 300, 8 heads, window 64 (96, 4) 7.0 -> 7.6; 1 x 300, 4 heads of
  // 128, causal (12, 6) 11.4 -> 12.2.
  const int tiles = std::min((w.window + w.sinks + 127) / 64 + 1, 2 * nqb), mean = std::min(tiles, nqb + 1);
  return tiles >= 7 && (int64_t)blocks * mean <= 256LL * tiles ? run(std::integral_constant<int, 2>{}) : run(std::integral_constant<int, 1>{});
}
template dipaco_status launch_window_fwd_mfma<32>(const bf16*, const int*, bf16*, float*, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_fwd_mfma<64>(const bf16*, const int*, bf16*, float*, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_fwd_mfma<128>(const bf16*, const int*, bf16*, float*, int, int, int, int, Window, hipStream_t);


template <int DH>
dipaco_status launch_window_bwd_mfma(const bf16* qkv, const int* lengths, const bf16* o, const bf16* d_o, const float* lse, bf16* dqkv, float* dsum, int B, int S,
                                     int H, int H_kv, Window w, hipStream_t s) {
  constexpr int LDS = 2 * window_dkv_stage<DH>();
  static_assert(LDS >= 4 * tile_bytes<DH>(), "dQ's stages fit");
  const WindowArgs a{qkv, lengths, B, S, H, H_kv, w};
  const int nb = (S + 127) / 128, G = H / H_kv;
  int sink_blocks = w.window >= S ? 0 : (std::min(w.sinks, S) + 31) / 32;
  // Parts of the sinks' queries, of 16 stages each or as many as the rows hold, where a workgroup that took them all would outlast the rest of the launch,
  // 512 workgroups at a time, by more than the two launches cost.  us whole | cut: the two of window_dkv; 4 x 8000 positions, 16 heads of 128 on 4, window
  // 1000, 16 sinks (1.7 times the rest) 1329 | 1340; 16384, 14 of 64, window 1024 (1.9 times) 287 | 277; 2048, 14 of 64, window 256 (26 stages more) 39.5 | 54.
  SinkParts sp{sink_blocks, 1, (128 + H - 1) / H};
  const int64_t stages = (int64_t)G * ((S + 63) / 64), rest = (int64_t)2 * B * H * nb * ((w.window + 128) / 64 + 1) / 512;
  if (sink_blocks && stages > rest + 40 && 10 * stages > 18 * rest)
    sp.parts = (int)std::min<int64_t>(stages / 16, S / ((int64_t)H_kv * sink_blocks * sp.rows));
  window_stats_mfma<DH><<<B * H * nb, AT_THREADS, 0, s>>>(a, o, d_o, lse, dsum);
  DIPACO_LAUNCH_CHECK();
  if (sink_blocks && sp.parts > 1) {
    static std::atomic<unsigned long long> parts_lds{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_sink_parts<DH>), LDS, parts_lds)) return st;
    window_sink_parts<DH><<<B * H_kv * sink_blocks * sp.parts, AT_THREADS, LDS, s>>>(a, d_o, dsum, dqkv, sp);
    DIPACO_LAUNCH_CHECK();
    window_sinks_join<DH><<<B * H_kv * sink_blocks * (DH / 16), AT_THREADS, 0, s>>>(a, d_o, dsum, dqkv, sp);
    DIPACO_LAUNCH_CHECK();
    sink_blocks = 0;
  }
  const bool shared = (int64_t)B * H_kv * nb < (G == 1 ? 112 : 256);   // KEYS_SHARED, as measured at window_dkv
  auto run = [&](auto SHAREDc) -> dipaco_status {
    constexpr bool SHARED = decltype(SHAREDc)::value;
    static std::atomic<unsigned long long> lds_set{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_bwd_mfma<DH, SHARED>), LDS, lds_set)) return st;
    window_bwd_mfma<DH, SHARED><<<B * H_kv * (sink_blocks + (SHARED ? 4 : 1) * nb) + B * H * nb, AT_THREADS, LDS, s>>>(a, d_o, dsum, dqkv, sink_blocks);
    DIPACO_LAUNCH_CHECK();
    return DIPACO_OK;
  };
  return shared ? run(std::true_type{}) : run(std::false_type{});
}
template dipaco_status launch_window_bwd_mfma<32>(const bf16*, const int*, const bf16*, const bf16*, const float*, bf16*, float*, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_bwd_mfma<64>(const bf16*, const int*, const bf16*, const bf16*, const float*, bf16*, float*, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_bwd_mfma<128>(const bf16*, const int*, const bf16*, const bf16*, const float*, bf16*, float*, int, int, int, int, Window,
                                                   hipStream_t);

}  // namespace dipaco
