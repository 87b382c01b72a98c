// bf16 attention with a sliding window and sinks over packed rows of a padded batch (window_mfma.h has the forward pass's inner loops).
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
template <int DH>
__global__ void __launch_bounds__(AT_THREADS, DH == 128 ? 2 : 3) window_fwd_mfma(WindowArgs a, bf16* __restrict__ o, float* __restrict__ lse) {
  constexpr int KS = DH / 16, TILE_BYTES = tile_bytes<DH>();
  extern __shared__ __attribute__((aligned(16))) char wf_smem[];   // [stage][K | V]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  const int n_bh = a.B * a.H, qb = (int)blockIdx.x / n_bh, bh = (int)blockIdx.x - qb * n_bh, b = bh / a.H, hd = bh - b * a.H, hk = hd / (a.H / a.H_kv);
  const int q0 = ((a.S + 127) / 128 - 1 - qb) * 128, q = q0 + 32 * wave + r;
  const int rows = document_rows(a.lengths, b, a.S), ld = (a.H + 2 * a.H_kv) * DH;
  const bf16* const base = a.qkv + (long)b * a.S * ld;
  const bf16* const qrow = base + (long)q * ld + hd * DH;
  const RowSpan span{q0 + 32 * wave, q0 + 32 * wave < rows ? min(q0 + 32 * wave + 31, rows - 1) : -1};
  SoftmaxRow<DH> x;
  x.clear();
  const int near = a.w.near_from(q);
  const float sc = score_scale<DH>() * LOG2E;
  if (q0 < rows) {
    uint4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = q < rows ? *reinterpret_cast<const uint4*>(qrow + 8 * (2 * ks + h)) : make_uint4(0, 0, 0, 0);
    const FragOff fo = frag_offsets(lane);
    const TrOff to = tr_offsets(lane);
    const uint32_t smem_addr = (uint32_t)(uintptr_t)wf_smem;
    const bf16* const k = base + (a.H + hk) * DH;
    const RowTiles<DH> src(k, k + a.H_kv * DH, ld, rows, wave, lane);
    const TileList tiles(a.w, q0, min(q0 + 127, rows - 1));
    src.issue(tiles.at(0), wave, lane, smem_addr);
    auto tile = [&](auto CUR, int t) {
      constexpr int cur = decltype(CUR)::value;
      wait_vmcnt<0>();
      __syncthreads();   // tile t is in LDS, and nobody still reads the other stage
      if (t + 1 < tiles.count) src.issue(tiles.at(t + 1), wave, lane, smem_addr + (1 - cur) * 2 * TILE_BYTES);
      const char* k_ = wf_smem + cur * 2 * TILE_BYTES;
      attend_tile<DH>(x, qf, k_, k_ + TILE_BYTES, fo, to, tiles.at(t) * 64, 0, a.w, span, q, near, lane);
    };
    for (int t = 0; t < tiles.count; t += 2) {
      tile(std::integral_constant<int, 0>{}, t);
      if (t + 1 < tiles.count) tile(std::integral_constant<int, 1>{}, t + 1);
    }
    x.l += __shfl_xor(x.l, 32, WAVE);
    if (__any(q < rows && plain::not_finite(x.o)) && q < rows) {
      plain::clear(x.o);
      const VisibleList vis(a.w, q);
#pragma unroll 1
      for (int t = 0; t < vis.count; ++t) {
        const bf16* kr = src.k + (long)vis.at(t) * ld;
        plain::add_row(x.o, __builtin_amdgcn_exp2f(__builtin_fmaf(plain::dot<DH>(qrow, kr), sc, x.m_neg)), kr + a.H_kv * DH, h);
      }
    }
  }
  int q_out = q;   // addresses of the outputs are formed behind the loop
  asm volatile("" : "+v"(q_out));
  if (q_out < a.S) {
    bf16* const out = o + ((long)b * a.S + q_out) * a.H * DH + hd * DH;
    if (q_out >= rows) x.clear();
    store_transposed_out(out, x.o, h, q_out < rows ? 1.0f / x.l : 0.f);
    if (h == 0) lse[(long)bh * a.S + q_out] = q_out < rows ? (x.m + __builtin_amdgcn_logf(x.l)) * LN2 : 0.f;   // v_log_f32 is log2
  }
}

}  // namespace

template <int DH>
dipaco_status launch_window_fwd_mfma(const bf16* qkv, const int* lengths, bf16* o, float* lse, int B, int S, int H, int H_kv, Window w, hipStream_t s) {
  constexpr int LDS = 2 * 2 * tile_bytes<DH>();
  static std::atomic<unsigned long long> lds_set{0};
  if (dipaco_status st = ensure_dynamic_lds(reinterpret_cast<const void*>(window_fwd_mfma<DH>), LDS, lds_set)) return st;
  window_fwd_mfma<DH><<<B * H * ((S + 127) / 128), AT_THREADS, LDS, s>>>(WindowArgs{qkv, lengths, B, S, H, H_kv, w}, o, lse);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
template dipaco_status launch_window_fwd_mfma<32>(const bf16*, const int*, bf16*, float*, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_fwd_mfma<64>(const bf16*, const int*, bf16*, float*, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_fwd_mfma<128>(const bf16*, const int*, bf16*, float*, int, int, int, int, Window, hipStream_t);

}  // namespace dipaco
