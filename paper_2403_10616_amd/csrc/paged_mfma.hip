// bf16 attention of new tokens over a paged cache on the matrix cores (paged.h: how the work is cut; window_mfma.h: the arithmetic of a tile).
//
// Keys and values go from their pages straight into LDS, eight rows of one page a load.  The table's entries are fetched 64 at a time, a lane
// each: a load's page is then a wave-uniform value, and the loop waits for the table once in 16 tiles (wide) or 32 halves (narrow).
// What a load must not read (positions behind the document's last one, pages that the table does not name) is replaced by the last position's row,
// which nobody gives weight there.
//
// Bound, one token each: the bytes of the keys and values (64 documents of up to 16000, 31 of them with a token, 16 heads of 128 on 4: 110 us, 4.8 TB/s) or,
// for few keys, latency (one document of 1000, 14 heads of 64: 9 us, a microsecond each for the document's rows and length, the pages, the first keys, the
// join).  Chunks: as window_mfma.h, and a workgroup's start and end (6000 and 3500 cycles beside 2250 a tile of head size 64): 1 x 512 tokens over 8000, 16
// heads of 128 on 4, 76 us with the join (455 TFLOP/s); 4 x up to 512 (1253 in all) over up to 12000, 14 heads of 64, window 2048, 28 without it.  Trees: 1 x 16 rows
// over 1000, 14 heads of 64, 10; 32 x up to 64 over up to 16000, 16 heads of 128 on 4, 152 - 165 and the join's 13 (matrix cores 0.38 and vector ALU 0.35 of the cycles
// of the units at work; blocks of 128 rows are two thirds full); 2 x 400 over 12000, window 2048, 14 heads of 64, 35 and 6.
#include "kernels.h"
#include "window_mfma.h"

namespace dipaco {

namespace {

// v, the same in every lane, in scalar registers
__device__ __forceinline__ const char* uniform(const char* v) {
  const uint64_t a = (uint64_t)v;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ uint64_t lane_offset(uint64_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

using Cut = PagedCut<bf16>;

// where a document's keys of one head lie
template <int DH> struct PagePlace {
  const char* base;          // keys of this head in page 0
  long page_bytes, value_bytes;
  int b, shift, last;
  long safe;                 // the last position's key, from base
  __device__ __forceinline__ PagePlace(const PagedArgs<bf16>& a, int b, int hk, int last) : b(b), shift(a.page_shift), last(last) {
    base = reinterpret_cast<const char*>(a.cache + a.template key_offset<DH>(0, hk, 0));
    page_bytes = ((long)2 * a.H_kv << shift) * DH * 2;
    value_bytes = a.template value_from_key<DH>() * 2;
    const int page = a.page_of(b, last);
    safe = page < 0 ? 0 : page * page_bytes + (last & ((1 << shift) - 1)) * DH * 2;
  }
  __device__ __forceinline__ long at(int page, int pos) const { return page * page_bytes + (long)((pos & ((1 << shift) - 1)) * DH * 2); }
};

// A row of the block: which, and where its query lies
template <int DH> struct PagedRow {
  bool valid;
  long row;
  int head;
  const bf16* q;
  __device__ __forceinline__ PagedRow(const PagedArgs<bf16>& a, int R, int packed, int row0, int hk) {
    const int G = a.group.d, token = a.group(R);
    valid = R < packed;
    row = row0 + token;
    head = hk * G + R - token * G;
    q = a.qkv + row * (a.H + 2 * a.H_kv) * DH + head * DH;
  }
  __device__ __forceinline__ void load(uint4 (&qf)[DH / 16], int h) const {
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) qf[ks] = valid ? *reinterpret_cast<const uint4*>(q + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
  }
};
// o of a row over the keys k0 .. k0 + n - 1 that it sees, pair by pair: x.o += ...
template <int DH, typename View>
__device__ __forceinline__ void add_seen(SoftmaxRow<DH>& x, const PagedArgs<bf16>& a, const PagePlace<DH>& at, const PagedRow<DH>& row, const View& view, int k0, int n, int h) {
  const float sc = score_scale<DH>() * LOG2E;
#pragma unroll 1
  for (int key = k0; key < k0 + n; ++key) {
    const int page = key > at.last ? -1 : a.page_of(at.b, key);
    if (page < 0 || !view.sees(key)) continue;
    const char* const k = at.base + at.at(page, key);
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(row.q, reinterpret_cast<const bf16*>(k)), sc, x.m_neg));
    plain::add_row(x.o, p, reinterpret_cast<const bf16*>(k + at.value_bytes), h);
  }
}

// a row whose scores so far were all -inf has seen something if it sees any of the n keys from k0 on
template <int DH, typename View>
__device__ __forceinline__ void note_seen(SoftmaxRow<DH>& x, const PagedArgs<bf16>& a, const PagePlace<DH>& at, const PagedRow<DH>& row, const View& view, int k0, int n) {
  if (row.valid && x.m == -INFINITY && a.sees_any(at.b, view, at.last, k0, n)) x.m = ALL_MINUS_INFINITY;
}

// ---- wide ----------------------------------------------------------------------------------------------------------
// pw_smem: [stage][K | V]
template <int DH> constexpr int wide_slots() { return 256 * (DH == 32 ? 4 : DH == 64 ? 3 : 2); }   // workgroups that are resident at once: registers
// block: the wide block; a tree's launch with a plan (TreeItem): the item, whatever `split` is
template <int DH, typename A> __device__ __forceinline__ void wide_block(const A& a, int hk, int split, int block, char* pw_smem) {
  constexpr int KS = DH / 16, NP = panels<DH>(), TILE_BYTES = tile_bytes<DH>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  int b, cached, per = 0;
  RowRange of_document;
  bool found = false;
  if constexpr (A::TREE) {
    if (has_plan(a)) {
      const TreeItem item(a, block, wide_slots<DH>(), lane);
      b = item.b;
      cached = item.cached;
      of_document = item.rows;
      split = item.split;
      per = item.per;
      if (block == 0 && hk == 0 && threadIdx.x == 0) *plan_of(a) = per;
      block = item.block;
      found = true;
    }
  }
  if (!found) {
    const WideBlock at_block(a, block, lane);
    b = at_block.b;
    cached = at_block.cached;
    of_document = at_block.rows;
    block = at_block.block;
  }
  if (b < 0) return;
  PagedBlock<Cut::WIDE_SHIFT> blk(a, b, of_document, cached, block, Cut::WIDE_ROWS, a.wide_splits, Cut::LEAST_KEYS);
  if (A::TREE && per) blk.per = per;
  const int t0 = split * blk.per, n_tiles = min(blk.tiles.count - t0, blk.per);
  if (!blk.has(split)) return;
  const int r0 = blk.packed0 + 32 * wave;
  int R = r0 + r;
  auto view = a.view(blk.row0, blk.rows, blk.pos0, blk.last, a.group(R));
  // TREE: keys from pos0 on are seen by some rows and not by others
  const RowSpan span{A::TREE ? blk.pos0 - 1 : blk.pos0 + a.group(r0), r0 >= blk.packed ? -1 : A::TREE ? blk.hi : blk.pos0 + a.group(min(r0 + 31, blk.packed - 1))};
  SoftmaxRow<DH> x;
  x.clear();
  if (n_tiles > 0) {
    uint4 qf[KS];
    PagedRow<DH>(a, R, blk.packed, blk.row0, hk).load(qf, h);
    const FragOff fo = frag_offsets(lane);
    const TrOff to = tr_offsets(lane);
    const uint32_t smem_addr = (uint32_t)(uintptr_t)pw_smem;
    const PagePlace<DH> at(a, b, hk, blk.last);
    const uint32_t col = loader_column_bytes<DH>(0, wave, lane), off = (uint32_t)((lane >> 3) * DH * 2) + col;   // the same for both row groups of a wave
    int ids = 0;       // lane 4 (t % 16) + g: the page of rows 16 g .. of tile t
    uint64_t rows16 = 0;   // and where these rows' keys start, from at.base
    auto issue = [&](int t, int stage) -> int {
      const int tile = blk.tiles.at(t0 + t), row0 = tile * 64;
      if ((t & 15) == 0) {
        const int pos = blk.tiles.at(t0 + min(t + (lane >> 2), n_tiles - 1)) * 64 + 16 * (lane & 3);
        ids = a.page_of(b, min(pos, at.last));
        rows16 = (uint64_t)at.at(ids, pos);
      }
      const int l0 = 4 * (t & 15);
      const int holes = (int)((__builtin_amdgcn_ballot_w64(ids < 0) >> l0) & 15);
      const uint32_t dst = uniform(smem_addr + stage * 2 * TILE_BYTES + wave * 1024);
      if (holes == 0 && row0 + 63 <= at.last) {   // wave-uniform
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const char* const k = uniform(at.base + lane_offset(rows16, l0 + ((wave + 4 * i) >> 1)) + (wave & 1) * 8 * DH * 2);
          const char* const v = uniform(k + at.value_bytes);
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            load16_to_lds_at(k + 128 * p, off, dst + i * 4096 + p * PANEL_BYTES);
            load16_to_lds_at(v + 128 * p, off, dst + i * 4096 + TILE_BYTES + p * PANEL_BYTES);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int pos = row0 + 8 * (wave + 4 * i) + (lane >> 3);
          const int id = __shfl(ids, l0 + ((wave + 4 * i) >> 1), WAVE);
          const char* const k = at.base + (id < 0 || pos > at.last ? at.safe : at.at(id, pos)) + col;
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            load16_to_lds(k + 128 * p, dst + i * 4096 + p * PANEL_BYTES);
            load16_to_lds(k + at.value_bytes + 128 * p, dst + i * 4096 + TILE_BYTES + p * PANEL_BYTES);
          }
        }
      }
      return holes;
    };
    int holes = issue(0, 0);
    for (int t = 0; t < n_tiles; ++t) {
      wait_vmcnt<0>();
      __syncthreads();
      const int mine = holes;
      if (t + 1 < n_tiles) holes = issue(t + 1, (t + 1) & 1);
      const char* k_ = pw_smem + (t & 1) * 2 * TILE_BYTES;
      // a position behind the table's end holds no key: rows there see up to the last one that does
      attend_tile<DH>(x, qf, k_, k_ + TILE_BYTES, fo, to, blk.tiles.at(t0 + t) * 64, mine, a.w, span, blk.hi > at.last ? UPPER | LOWER : 0, view, lane);
    }
    x.l += __shfl_xor(x.l, 32, WAVE);
    asm volatile("" : "+v"(R));   // what follows is formed anew, not kept through the loop
    const PagedRow<DH> row(a, R, blk.packed, blk.row0, hk);
    if constexpr (!A::TREE) view = a.view(blk.row0, blk.rows, blk.pos0, blk.last, a.group(R));
    if (__any(row.valid && plain::not_finite(x.o)) && row.valid) {
      plain::clear(x.o);
      for (int t = 0; t < n_tiles; ++t) add_seen<DH>(x, a, at, row, view, blk.tiles.at(t0 + t) * 64, 64, h);
    }
    for (int t = 0; t < n_tiles && __any(row.valid && x.m == -INFINITY); ++t) note_seen<DH>(x, a, at, row, view, blk.tiles.at(t0 + t) * 64, 64);
  }
  asm volatile("" : "+v"(R));
  const PagedRow<DH> row(a, R, blk.packed, blk.row0, hk);
  if (!row.valid) return;
  if (blk.whole()) {
    store_transposed_out(a.o + (row.row * a.H + row.head) * DH, x.o, h, x.m == -INFINITY ? 0.f : 1.0f / x.l);
    if (a.lse && h == 0) a.lse[row.row * a.H + row.head] = (x.m + __builtin_amdgcn_logf(x.l)) * LN2;   // v_log_f32 is log2; -inf where nothing is seen
  } else {
    float* const sums = a.template part_sums<DH>(split, row.row, row.head);
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(sums + 32 * dt + 8 * g + 4 * h) = make_float4(x.o[dt][4 * g], x.o[dt][4 * g + 1], x.o[dt][4 * g + 2], x.o[dt][4 * g + 3]);
    if (h == 0) *a.part_state(split, row.row, row.head) = make_float2(x.m, x.l);
  }
}

// ---- narrow --------------------------------------------------------------------------------------------------------
// Waves of a workgroup and stages of a wave's ring.  Ordinary calls: four waves that wait for each half they read, and as many workgroups a unit as
// registers allow; launches of few workgroups: as many bytes in flight as a unit's LDS holds.
template <int DH> constexpr int narrow_stage() { return panels<DH>() * PANEL_BYTES; }   // 32 rows of K and V: a panel holds K's, then V's
// the rings, and in their place at the end what the waves add up: 16 accumulator elements a lane and 32 columns, reference exponent and sum
template <int DH, int NW, int NS> constexpr int narrow_lds() {
  constexpr int RINGS = NW * NS * narrow_stage<DH>(), SUMS = NW * WAVE * (16 * (DH / 32) + 2) * (int)sizeof(float);
  return RINGS > SUMS ? RINGS : SUMS;
}
// pn_smem: [wave][stage]
template <int DH, int NW, int NS, typename A> __device__ __forceinline__ void narrow_document(const A& a, int hk, int b, int split, char* pn_smem) {
  constexpr int KS = DH / 16, DT = DH / 32, NP = panels<DH>(), STAGE = narrow_stage<DH>(), LPW = 8 * NP;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  const PagedBlock<Cut::NARROW_SHIFT> blk(a, b, 0, Cut::NARROW_ROWS, a.narrow_splits, a.narrow_keys);
  if (blk.packed == 0 || blk.packed > Cut::NARROW_ROWS || !blk.has(split)) return;
  const int t0 = split * blk.per, end = min(t0 + blk.per, blk.tiles.count), n = (end - t0 - wave + NW - 1) / NW;   // this wave's halves: t0 + wave, + NW, ..
  const PagedRow<DH> row(a, r, blk.packed, blk.row0, hk);
  auto view = a.view(blk.row0, blk.rows, blk.pos0, blk.last, a.group(r));
  const RowSpan span{A::TREE ? blk.pos0 - 1 : blk.lo, blk.hi};
  SoftmaxRow<DH> x;
  x.clear();
  if (n > 0) {
    const FragOff fo = frag_offsets(lane);
    const TrOff to = tr_offsets(lane);
    char* const ring = pn_smem + wave * NS * STAGE;
    const uint32_t ring_addr = (uint32_t)(uintptr_t)ring;
    const PagePlace<DH> at(a, b, hk, blk.last);
    uint32_t col[2], off[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int c = (lane & 7) ^ swz64(8 * i + (lane >> 3));
      if (DH == 32) c &= 3;
      col[i] = (uint32_t)(c * 16);
      off[i] = (uint32_t)((lane >> 3) * DH * 2) + col[i];
    }
    int ids = 0;           // lane 2 (t % 32) + g: the page of rows 16 g .. of this wave's half t
    uint64_t rows16 = 0;   // and where these rows' keys start, from at.base
    auto half_at = [&](int t) { return blk.tiles.at(t0 + wave + NW * t) * 32; };
    auto holes_of = [&](unsigned long long none, int t) { return (int)((none >> (2 * (t & 31))) & 3); };
    unsigned long long none = 0;   // which of the lanes' pages are none; of the 32 halves before as well
    unsigned long long none_before = 0;
    auto issue = [&](int t) {
      const int row0 = half_at(t);
      if ((t & 31) == 0) {
        const int pos = half_at(min(t + (lane >> 1), n - 1)) + 16 * (lane & 1);
        ids = a.page_of(b, min(pos, at.last));
        rows16 = (uint64_t)at.at(ids, pos);
        none_before = none;
        none = __builtin_amdgcn_ballot_w64(ids < 0);
      }
      const int l0 = 2 * (t & 31);
      const uint32_t dst = uniform(ring_addr + (t % NS) * STAGE);
      if (holes_of(none, t) == 0 && row0 + 31 <= at.last) {   // wave-uniform
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const char* const k = uniform(at.base + lane_offset(rows16, l0 + (i >> 1)) + (i & 1) * 8 * DH * 2);
          const char* const v = uniform(k + at.value_bytes);
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            load16_to_lds_at(k + 128 * p, off[i & 1], dst + i * 1024 + p * PANEL_BYTES);
            load16_to_lds_at(v + 128 * p, off[i & 1], dst + i * 1024 + 4096 + p * PANEL_BYTES);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = row0 + 8 * i + (lane >> 3), id = __shfl(ids, l0 + (i >> 1), WAVE);
          const char* const k = at.base + (id < 0 || pos > at.last ? at.safe : at.at(id, pos)) + col[i & 1];
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            load16_to_lds(k + 128 * p, dst + i * 1024 + p * PANEL_BYTES);
            load16_to_lds(k + at.value_bytes + 128 * p, dst + i * 1024 + 4096 + p * PANEL_BYTES);
          }
        }
      }
    };
    // The rows' queries are asked for in front of the table, whose wait serves both.  A half's stage is filled again when its products have read it:
    // NS halves are in flight.
    uint4 qf[KS];
    row.load(qf, h);
    for (int t = 0; t < min(NS, n); ++t) issue(t);
    for (int t = 0; t < n; ++t) {
      wait_stages_but<LPW>(min(NS - 1, n - 1 - t));   // half t has landed: the loads behind it are those of the next halves
      asm volatile("" ::: "memory");
      const int k0 = half_at(t), holes = holes_of((t >> 5) == ((min(t + NS - 1, n - 1)) >> 5) ? none : none_before, t);
      const int s = holes == 3 ? 0 : seen_half(a.w, span, k0);
      const char* k_ = ring + (t % NS) * STAGE;
      if (s)
        attend_half<DH>(x, qf, k_, k_ + 4096, fo, to, k0, s | (blk.hi > at.last ? UPPER | LOWER : 0), holes, view, lane);
      asm volatile("" ::: "memory");
      if (t + NS < n) {
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));   // lgkmcnt(0): every read of the stage that is filled again has returned
        issue(t + NS);
      }
    }
    x.l += __shfl_xor(x.l, 32, WAVE);
    if (__any(row.valid && plain::not_finite(x.o)) && row.valid) {
      plain::clear(x.o);
      for (int t = 0; t < n; ++t) add_seen<DH>(x, a, at, row, view, half_at(t), 32, h);
    }
    for (int t = 0; t < n && __any(row.valid && x.m == -INFINITY); ++t) note_seen<DH>(x, a, at, row, view, half_at(t), 32);
  }
  // the waves' sums meet in LDS: wave w adds accumulator elements 4 g .. 4 g + 3 of every 32 columns for g = w, w + NW, ..
  constexpr int PER = 16 * DT * WAVE;
  float* const sums = reinterpret_cast<float*>(pn_smem);
  float2* const state = reinterpret_cast<float2*>(sums + NW * PER);
  __syncthreads();   // the rings have been read
  hand_over(x.o, sums + wave * PER, lane);
  state[wave * WAVE + lane] = make_float2(x.m, x.l);
  __syncthreads();
  if (!row.valid) return;
  float2 st[NW];
  float m = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    st[w] = state[w * WAVE + lane];
    m = fmaxf(m, st[w].x);
  }
  float c[NW], l = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    c[w] = st[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[w].x - m);
    l = __builtin_fmaf(st[w].y, c[w], l);
  }
  const bool whole = blk.whole();
  const float scale = !whole ? 1.f : m == -INFINITY ? 0.f : 1.0f / l;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g0 = 0; g0 < 4; g0 += NW) {
      const int g = g0 + wave;
      if (NW > 4 && g > 3) break;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float4 p = *reinterpret_cast<const float4*>(sums + w * PER + ((dt * 4 + g) * WAVE + lane) * 4);
        v.x = __builtin_fmaf(p.x, c[w], v.x); v.y = __builtin_fmaf(p.y, c[w], v.y); v.z = __builtin_fmaf(p.z, c[w], v.z); v.w = __builtin_fmaf(p.w, c[w], v.w);
      }
      const int at = 32 * dt + 8 * g + 4 * h;
      if (whole) {
        const bf16x4 out = {(bf16)(v.x * scale), (bf16)(v.y * scale), (bf16)(v.z * scale), (bf16)(v.w * scale)};
        *reinterpret_cast<bf16x4*>(a.o + (row.row * a.H + row.head) * DH + at) = out;
      } else {
        *reinterpret_cast<float4*>(a.template part_sums<DH>(split, row.row, row.head) + at) = v;
      }
    }
  if (wave == 0 && h == 0) {
    if (!whole) *a.part_state(split, row.row, row.head) = make_float2(m, l);
    else if (a.lse) a.lse[row.row * a.H + row.head] = (m + __builtin_amdgcn_logf(l)) * LN2;
  }
}

// Documents of a call that has only narrow ones
template <int DH, int NW, int NS, template <typename> class Args> __global__ void __launch_bounds__(WAVE * NW, 1) paged_narrow_mfma(Args<bf16> a, int b0) {
  extern __shared__ __attribute__((aligned(16))) char pn_smem[];
  const int hk = blockIdx.y, b = blockIdx.z + b0;
  narrow_document<DH, NW, NS>(a, hk, b, a.narrow_split(blockIdx.x, b * a.H_kv + hk), pn_smem);
}
// A call with wide blocks, and in the same launch behind them the narrow documents that it may have
template <int DH, template <typename> class Args> __global__ void __launch_bounds__(AT_THREADS, 2) paged_both_mfma(Args<bf16> a, PagedOrder order) {
  extern __shared__ __attribute__((aligned(16))) char pb_smem[];
  int i = blockIdx.x;
  if (i < order.n_wide) {
    if (Args<bf16>::TREE && has_plan(a)) {
      const int item = order.heads(i);
      wide_block<DH>(a, i - item * a.H_kv, 0, item, pb_smem);
      return;
    }
    const int block = order.head_splits(i), j = i - block * (int)order.head_splits.d, split = order.heads(j);
    wide_block<DH>(a, j - split * a.H_kv, split, block, pb_smem);
    return;
  }
  i -= order.n_wide;
  const int item = a.narrow_splits(i), b = order.heads(item);
  narrow_document<DH, 4, 1>(a, item - b * a.H_kv, b, a.narrow_split(i - item * (int)a.narrow_splits.d, item), pb_smem);
}

}  // namespace

template <int DH, template <typename> class Args> dipaco_status launch_paged_narrow(const Args<bf16>& a, hipStream_t s) {
  auto run = [&](auto NWc, auto NSc) -> dipaco_status {
    constexpr int NW = decltype(NWc)::value, NS = decltype(NSc)::value, LDS = narrow_lds<DH, NW, NS>();
    static std::atomic<unsigned long long> lds_set{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(paged_narrow_mfma<DH, NW, NS, Args>), LDS, lds_set)) return st;
    for (int b = 0; b < a.B; b += 65535) {   // documents are the grid's z
      paged_narrow_mfma<DH, NW, NS, Args><<<dim3(a.narrow_splits.d, a.H_kv, std::min(a.B - b, 65535)), WAVE * NW, LDS, s>>>(a, b);
      DIPACO_LAUNCH_CHECK();
    }
    return DIPACO_OK;
  };
  using std::integral_constant;
  // A launch of a workgroup a compute unit or less has a unit's LDS for each
  if (a.narrow_keys > PagedCut<bf16>::LEAST_KEYS) return run(integral_constant<int, DH == 128 ? 4 : 8>{}, integral_constant<int, 2>{});
  return run(integral_constant<int, DH == 128 ? 2 : 4>{}, integral_constant<int, DH == 128 ? 2 : 1>{});
}
template <int DH, template <typename> class Args> dipaco_status launch_paged_both(const Args<bf16>& a, int blocks, hipStream_t s) {
  constexpr int WIDE_LDS = 4 * tile_bytes<DH>(), NARROW_LDS = narrow_lds<DH, 4, 1>(), LDS = WIDE_LDS > NARROW_LDS ? WIDE_LDS : NARROW_LDS;
  static std::atomic<unsigned long long> lds_set{0};
  if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(paged_both_mfma<DH, Args>), LDS, lds_set)) return st;
  const int wide = a.H_kv * (int)a.wide_splits.d;
  auto launch = [&](const Args<bf16>& args, int n_wide) {
    const PagedOrder order{Divisor(a.H_kv), Divisor(wide), n_wide};
    paged_both_mfma<DH, Args><<<n_wide + a.B * a.H_kv * (int)a.narrow_splits.d, AT_THREADS, LDS, s>>>(args, order);
  };
  if constexpr (Args<bf16>::TREE) {
    Args<bf16> t = a;   // rounds of what is resident, and room for a split a block
    t.most_items = std::max(std::min(TREE_ROUNDS * wide_slots<DH>() / a.H_kv, a.most_items), blocks);
    launch(t, has_plan(a) ? t.most_items * a.H_kv : blocks * wide);
  } else {
    launch(a, blocks * wide);
  }
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
#define DIPACO_PAGED_MFMA(DH, ARGS)                                                      \
  template dipaco_status launch_paged_narrow<DH, ARGS>(const ARGS<bf16>&, hipStream_t); \
  template dipaco_status launch_paged_both<DH, ARGS>(const ARGS<bf16>&, int, hipStream_t);
DIPACO_PAGED_MFMA(32, PagedArgs) DIPACO_PAGED_MFMA(64, PagedArgs) DIPACO_PAGED_MFMA(128, PagedArgs)
DIPACO_PAGED_MFMA(32, TreeArgs) DIPACO_PAGED_MFMA(64, TreeArgs) DIPACO_PAGED_MFMA(128, TreeArgs)

}  // namespace dipaco
