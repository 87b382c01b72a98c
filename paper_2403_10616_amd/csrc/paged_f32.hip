// fp32 attention of new tokens over a paged cache on the matrix cores (paged.h: how the work is cut; window_f32.h: the arithmetic of a tile).
//
// The table's entries are fetched 64 at a time, a lane each (16 positions an entry); a thread takes the page of the row that it moves from the
// lane that holds it.  Rows that must not be read are replaced by the last position's, as in paged_mfma.hip.
// Us: 5 documents of up to 40 tokens over up to 700, 8 heads of 32 on 2 12.5 (of which the join 3.5); 1 x 500 over 1000, 8 heads of 64, 31; one token over
// 2000, 8 heads of 64, 9.8; trees of 5 documents of up to 25 rows over up to 700, 8 heads of 32 on 2, 12.7; 32 documents of up to 4000, 20 of them with a token, 8 heads of 64 on 2, 17.5 (2.2 TB/s).
#include "kernels.h"
#include "window_f32.h"

namespace dipaco {

namespace {

using Cut = PagedCut<float>;

// NARROW: 16 packed rows, which every wave holds; of a tile of 64 keys a wave takes 16.  Else 64 packed rows, 16 a wave, on tiles of 32 keys.
// b: the document, or the call's wide block; pf_smem: [stage][K | V]
template <int DH, bool NARROW, typename A> __device__ __forceinline__ void paged_part(const A& a, int hk, int split, int b, float* pf_smem) {
  constexpr int SHIFT = NARROW ? Cut::NARROW_SHIFT : Cut::WIDE_SHIFT, TILE = 1 << SHIFT, RUNS = TILE / 16, AHEAD = 64 / RUNS;
  constexpr int STAGE = 2 * window_tile_floats<DH, TILE>();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const Divisor& splits = NARROW ? a.narrow_splits : a.wide_splits;
  int block = 0, cached;
  RowRange rows;
  if constexpr (NARROW) {
    rows = ragged_rows(a.row_start, b, a.T_rows);
    cached = a.cached(b);
  } else {
    const WideBlock at(a, b, lane);
    b = at.b;
    if (b < 0) return;
    block = at.block;
    rows = at.rows;
    cached = at.cached;
  }
  const PagedBlock<SHIFT> blk(a, b, rows, cached, block, NARROW ? Cut::NARROW_ROWS : Cut::WIDE_ROWS, splits, NARROW ? a.narrow_keys : Cut::LEAST_KEYS);
  if (NARROW && (blk.packed == 0 || blk.packed > Cut::NARROW_ROWS)) return;
  if (!blk.has(split)) return;
  const int t0 = split * blk.per, n_tiles = min(blk.tiles.count - t0, blk.per);
  const int G = a.group.d, r0 = blk.packed0 + (NARROW ? 0 : 16 * wave), R = r0 + m, token = a.group(R), head = hk * G + R - token * G;
  const bool valid = R < blk.packed;
  auto view = a.view(blk.row0, blk.rows, blk.pos0, blk.last, token);
  const long row = blk.row0 + token;
  // TREE: keys from pos0 on are seen by some rows and not by others
  const FRowSpan span{A::TREE ? blk.pos0 - 1 : blk.pos0 + a.group(r0), r0 >= blk.packed ? -1 : A::TREE ? blk.hi : blk.pos0 + a.group(min(r0 + 15, blk.packed - 1))};
  const float* const q = a.qkv + row * (a.H + 2 * a.H_kv) * DH + head * DH;
  const float* const keys = a.cache + a.template key_offset<DH>(0, hk, 0);
  const long page_floats = ((long)2 * a.H_kv << a.page_shift) * DH, value = a.template value_from_key<DH>();
  const int in_page = (1 << a.page_shift) - 1;
  FSoftmaxRow<DH> x;
  x.clear();
  if (n_tiles > 0) {
    const RowFrag<DH> qf = load_row<DH>(q, g, valid);
    const int last_page = a.page_of(b, blk.last);
    const long safe = last_page < 0 ? 0 : last_page * page_floats + (long)(blk.last & in_page) * DH;
    TileMover<DH, TILE> next;
    int ids = 0;   // lane RUNS (t % AHEAD) + i: the page of run i of tile t
    auto load = [&](int t) -> int {
      const int k0 = blk.tiles.at(t0 + t) << SHIFT, l0 = RUNS * (t % AHEAD);
      if (t % AHEAD == 0) ids = a.page_of(b, min((blk.tiles.at(t0 + min(t + lane / RUNS, n_tiles - 1)) << SHIFT) + 16 * (lane % RUNS), blk.last));
      next.load([&](int r, const float*& p0, const float*& p1) {
        const int id = __shfl(ids, l0 + (r >> 4), WAVE), p = k0 + r;
        p0 = keys + (id < 0 || p > blk.last ? safe : id * page_floats + (long)(p & in_page) * DH);
        p1 = p0 + value;
      });
      return (int)((__builtin_amdgcn_ballot_w64(ids < 0) >> l0) & ((1 << RUNS) - 1));
    };
    int holes = load(0);
    next.store(pf_smem);
    for (int t = 0; t < n_tiles; ++t) {
      const float* k_ = pf_smem + (t & 1) * STAGE;
      const float* v_ = k_ + window_tile_floats<DH, TILE>();
      const int k0 = blk.tiles.at(t0 + t) << SHIFT, mine = holes;
      const bool more = t + 1 < n_tiles, beyond = blk.hi > blk.last;   // rows behind the table's end see up to the last position that it holds
      if (more) holes = load(t + 1);
      __syncthreads();
      if constexpr (NARROW) {
        const int s = (mine >> wave) & 1 ? F_NONE : seen_16(a.w, span, k0 + 16 * wave);
        if (s != F_NONE) attend_16<DH>(x, qf, k_, v_, wave, k0 + 16 * wave, beyond || s != F_ALL, view, m, g);
      } else {
        attend_32<DH>(x, qf, k_, v_, k0, mine, a.w, span, beyond, view, m, g);
      }
      if (more) next.store(pf_smem + ((t + 1) & 1) * STAGE);
    }
    x.l = sum_groups(x.l);
    if (__any(valid && plain::not_finite(x.o)) && valid) {
      plain::clear(x.o);
      for (int t = 0; t < n_tiles; ++t) {
        const int k0 = (blk.tiles.at(t0 + t) << SHIFT) + (NARROW ? 16 * wave : 0);
#pragma unroll 1
        for (int key = k0; key < k0 + (NARROW ? 16 : TILE); ++key) {
          const int page = key > blk.last ? -1 : a.page_of(b, key);
          if (page < 0 || !view.sees(key)) continue;
          const float* const k = keys + page * page_floats + (long)(key & in_page) * DH;
          plain::add_row(x.o, __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(q, k), head_scale<DH>() * WF_LOG2E, x.m_neg)), k + value, g);
        }
      }
    }
    for (int t = 0; t < n_tiles && __any(valid && x.m == -INFINITY); ++t)   // scores that were all -inf are not nothing (ALL_MINUS_INFINITY)
      if (valid && x.m == -INFINITY && a.sees_any(b, view, blk.last, (blk.tiles.at(t0 + t) << SHIFT) + (NARROW ? 16 * wave : 0), NARROW ? 16 : TILE)) x.m = ALL_MINUS_INFINITY;
  }
  if constexpr (NARROW) {   // the waves' sums meet in LDS: wave w adds columns 16 d + .. of every d with d % 4 = w
    constexpr int PER = DH / 16 * 4 * WAVE;
    static_assert(4 * PER + 8 * WAVE <= 2 * STAGE, "the sums fit in the stages");
    float2* const state = reinterpret_cast<float2*>(pf_smem + 4 * PER);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) *reinterpret_cast<f32x4*>(pf_smem + wave * PER + (d * WAVE + lane) * 4) = x.o[d];
    state[wave * WAVE + lane] = make_float2(x.m, x.l);
    __syncthreads();
    if (!valid) return;
    float mm = -INFINITY, c[4], l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, state[w * WAVE + lane].x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float2 s = state[w * WAVE + lane];
      c[w] = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - mm);
      l = __builtin_fmaf(s.y, c[w], l);
    }
    const float scale = !blk.whole() ? 1.f : mm == -INFINITY ? 0.f : 1.0f / l;
    float* const out = !blk.whole() ? a.template part_sums<DH>(split, row, head) : a.o + (row * a.H + head) * DH;
    for (int d = wave; d < DH / 16; d += 4) {
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const f32x4 p = *reinterpret_cast<const f32x4*>(pf_smem + w * PER + (d * WAVE + lane) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(p[e], c[w], v[e]);
      }
      *reinterpret_cast<float4*>(out + 16 * d + 4 * g) = make_float4(v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale);
    }
    if (wave == 0 && g == 0) {
      if (!blk.whole()) *a.part_state(split, row, head) = make_float2(mm, l);
      else if (a.lse) a.lse[row * a.H + head] = (mm + __builtin_amdgcn_logf(l)) * WF_LN2;
    }
  } else {
    if (!valid) return;
    if (!blk.whole()) {
      store_row<DH>(a.template part_sums<DH>(split, row, head), x.o, g, 1.f);
      if (g == 0) *a.part_state(split, row, head) = make_float2(x.m, x.l);
    } else {
      store_row<DH>(a.o + (row * a.H + head) * DH, x.o, g, x.m == -INFINITY ? 0.f : 1.0f / x.l);
      if (a.lse && g == 0) a.lse[row * a.H + head] = (x.m + __builtin_amdgcn_logf(x.l)) * WF_LN2;   // -inf where nothing is seen
    }
  }
}

template <int DH, bool NARROW, template <typename> class Args> __global__ void __launch_bounds__(WF_THREADS, NARROW && DH == 128 ? 1 : 2) paged_f32(Args<float> a, int first) {
  extern __shared__ __attribute__((aligned(16))) float pf_smem[];
  const int hk = NARROW ? blockIdx.y : blockIdx.x, b = blockIdx.z + first;
  paged_part<DH, NARROW>(a, hk, NARROW ? a.narrow_split(blockIdx.x, b * a.H_kv + hk) : blockIdx.y, b, pf_smem);
}
// Both kinds in a launch
template <int DH, template <typename> class Args> __global__ void __launch_bounds__(WF_THREADS, DH == 128 ? 1 : 2) paged_f32_both(Args<float> a, PagedOrder order) {
  extern __shared__ __attribute__((aligned(16))) float pfb_smem[];
  int i = blockIdx.x;
  if (i < order.n_wide) {
    const int block = order.head_splits(i), j = i - block * (int)order.head_splits.d, split = order.heads(j);
    paged_part<DH, false>(a, j - split * a.H_kv, split, block, pfb_smem);
    return;
  }
  i -= order.n_wide;
  const int item = a.narrow_splits(i), b = order.heads(item);
  paged_part<DH, true>(a, item - b * a.H_kv, a.narrow_split(i - item * (int)a.narrow_splits.d, item), b, pfb_smem);
}

template <int DH, bool NARROW> constexpr int paged_f32_lds() {
  return 2 * 2 * window_tile_floats<DH, 1 << (NARROW ? Cut::NARROW_SHIFT : Cut::WIDE_SHIFT)>() * (int)sizeof(float);
}

}  // namespace

template <int DH, template <typename> class Args> dipaco_status launch_paged_narrow(const Args<float>& a, hipStream_t s) {
  static std::atomic<unsigned long long> lds_set{0};
  if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(paged_f32<DH, true, Args>), paged_f32_lds<DH, true>(), lds_set)) return st;
  for (int b = 0; b < a.B; b += 65535) {   // documents are the grid's z
    paged_f32<DH, true, Args><<<dim3(a.narrow_splits.d, a.H_kv, std::min(a.B - b, 65535)), WF_THREADS, paged_f32_lds<DH, true>(), s>>>(a, b);
    DIPACO_LAUNCH_CHECK();
  }
  return DIPACO_OK;
}
template <int DH, template <typename> class Args> dipaco_status launch_paged_both(const Args<float>& a, int blocks, hipStream_t s) {
  static std::atomic<unsigned long long> lds_set{0};
  // One launch where the compute units hold all its workgroups at once: the narrow ones' LDS, twice the wide ones', then keeps nobody waiting.  Us, two launches
  // | one: 5 x up to 40 tokens over up to 700, 8 heads of 32 on 2, 13.6 | 12.5; 1 x 64 over 1000, 8 of 64, 16.7 | 15.7; 4 x up to 100 over up to 500, 8 of 128
  // on 2, level; and a launch less of the host's time, 15.7 | 12.4 a call of the first through the Python binding.
  constexpr int LDS = std::max(paged_f32_lds<DH, true>(), paged_f32_lds<DH, false>());
  const int64_t wide = (int64_t)a.H_kv * a.wide_splits.d, groups = wide * blocks + (int64_t)a.B * a.H_kv * a.narrow_splits.d;
  if (groups <= 256 * (163840 / LDS)) {
    static std::atomic<unsigned long long> both_set{0};
    if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(paged_f32_both<DH, Args>), LDS, both_set)) return st;
    const PagedOrder order{Divisor(a.H_kv), Divisor((int)wide), (int)wide * blocks};
    paged_f32_both<DH, Args><<<(int)groups, WF_THREADS, LDS, s>>>(a, order);
    DIPACO_LAUNCH_CHECK();
    return DIPACO_OK;
  }
  if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(paged_f32<DH, false, Args>), paged_f32_lds<DH, false>(), lds_set)) return st;
  for (int b = 0; b < blocks; b += 65535) {
    paged_f32<DH, false, Args><<<dim3(a.H_kv, a.wide_splits.d, std::min(blocks - b, 65535)), WF_THREADS, paged_f32_lds<DH, false>(), s>>>(a, b);
    DIPACO_LAUNCH_CHECK();
  }
  return launch_paged_narrow<DH>(a, s);
}
#define DIPACO_PAGED_F32(DH, ARGS)                                                        \
  template dipaco_status launch_paged_narrow<DH, ARGS>(const ARGS<float>&, hipStream_t); \
  template dipaco_status launch_paged_both<DH, ARGS>(const ARGS<float>&, int, hipStream_t);
DIPACO_PAGED_F32(32, PagedArgs) DIPACO_PAGED_F32(64, PagedArgs) DIPACO_PAGED_F32(128, PagedArgs)
DIPACO_PAGED_F32(32, TreeArgs) DIPACO_PAGED_F32(64, TreeArgs) DIPACO_PAGED_F32(128, TreeArgs)

}  // namespace dipaco
