// Attention with a sliding window and sinks over the packed q | k | v rows of a padded batch, forward and backward.
//
//   vis(i) = { j <= i : j > i - window or j < sinks }      s_ij = q_i.k_j / sqrt(dh)      lse_i = log sum_{j in vis(i)} exp s_ij
//   o_i = sum_{vis(i)} exp(s_ij - lse_i) v_j
//   D_i = dO_i.o_i     dS_ij = P_ij (dO_i.v_j - D_i)     dq_i = sum_j dS_ij k_j / sqrt(dh)
//   dk_j = sum_{heads of the group} sum_{i sees j} dS_ij q_i / sqrt(dh)     dv_j = sum_{heads} sum_{i sees j} P_ij dO_i
//
// One wave per row and head.  The forward pass and dQ take 64 visible keys at a time: a lane forms one key's score, then the wave adds the
// values with the lanes on the head's columns.  dK / dV do the same over the rows that see a key.
#include <type_traits>

#include "kernels.h"
#include "visible.h"

namespace dipaco {

namespace {

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
__device__ __forceinline__ float lane_value(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
// columns of a head that a lane holds: lane and lane + 64
template <int DH> constexpr int cols() { return DH == 128 ? 2 : 1; }
template <int DH, typename T> __device__ __forceinline__ void add_row(float (&acc)[2], float w, const T* row, int lane) {
#pragma unroll
  for (int c = 0; c < cols<DH>(); ++c)
    if (DH >= 64 || lane < DH) acc[c] = __builtin_fmaf(w, to_f32(row[lane + 64 * c]), acc[c]);
}
template <int DH, typename T> __device__ __forceinline__ void store_cols(T* row, const float (&acc)[2], float scale, int lane) {
#pragma unroll
  for (int c = 0; c < cols<DH>(); ++c)
    if (DH >= 64 || lane < DH) row[lane + 64 * c] = from_f32<T>(acc[c] * scale);
}

template <int DH, typename T>
__global__ void __launch_bounds__(256) window_fwd_rows(const T* __restrict__ qkv, const int* __restrict__ lengths, T* __restrict__ o,
                                                       float* __restrict__ lse, int S, int H, int H_kv, Window w) {
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, b = blockIdx.z;
  if (i >= S) return;
  const long ld = (long)(H + 2 * H_kv) * DH;
  const T* const base = qkv + (long)b * S * ld;
  const T* const q = base + i * ld + h * DH;
  const T* const k = base + (H + h / (H / H_kv)) * DH;
  const T* const v = k + H_kv * DH;
  T* const out = o + (((long)b * S + i) * H + h) * DH;
  float acc[2] = {0.f, 0.f}, m = -INFINITY, l = 0.f;
  if (i >= document_rows(lengths, b, S)) {
    store_cols<DH>(out, acc, 0.f, lane);
    if (lane == 0) lse[((long)b * H + h) * S + i] = 0.f;
    return;
  }
  const VisibleList vis(w, i);
  for (int t0 = 0; t0 < vis.count; t0 += 64) {
    const int n = min(64, vis.count - t0);
    const float s = lane < n ? row_dot<DH>(q, k + vis.at(t0 + lane) * ld) * head_scale<DH>() : -INFINITY;
    const float mn = fmaxf(m, wave_max(s)), corr = expf(m - mn), p = expf(s - mn);
    m = mn;
    l = l * corr + wave_sum(p);
    acc[0] *= corr;
    acc[1] *= corr;
    for (int t = 0; t < n; ++t) add_row<DH>(acc, lane_value(p, t), v + vis.at(t0 + t) * ld, lane);
  }
  store_cols<DH>(out, acc, 1.f / l, lane);
  if (lane == 0) lse[((long)b * H + h) * S + i] = m + logf(l);
}

// D of every row, in rows padded to whole blocks of 128; 0 behind a document
template <int DH, typename T>
__global__ void __launch_bounds__(256) window_stats(const T* __restrict__ o, const T* __restrict__ d_o, const int* __restrict__ lengths,
                                                    float* __restrict__ dsum, int S, int S128, int H) {
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, b = blockIdx.z;
  if (i >= S128) return;
  float D = 0.f;
  if (i < document_rows(lengths, b, S)) {
    const long at = (((long)b * S + i) * H + h) * DH;
#pragma unroll
    for (int c = 0; c < cols<DH>(); ++c)
      if (DH >= 64 || lane < DH) D = __builtin_fmaf(to_f32(o[at + lane + 64 * c]), to_f32(d_o[at + lane + 64 * c]), D);
  }
  D = wave_sum(D);
  if (lane == 0) dsum[((long)b * H + h) * S128 + i] = D;
}

template <int DH, typename T>
__global__ void __launch_bounds__(256) window_dq_rows(const T* __restrict__ qkv, const int* __restrict__ lengths, const T* __restrict__ d_o,
                                                      const float* __restrict__ lse, const float* __restrict__ dsum, T* __restrict__ dqkv, int S,
                                                      int S128, int H, int H_kv, Window w) {
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, b = blockIdx.z;
  if (i >= S) return;
  const long ld = (long)(H + 2 * H_kv) * DH, row = (long)b * S + i;
  const T* const base = qkv + (long)b * S * ld;
  const T* const q = base + i * ld + h * DH;
  const T* const k = base + (H + h / (H / H_kv)) * DH;
  const T* const v = k + H_kv * DH;
  const T* const g = d_o + (row * H + h) * DH;
  float acc[2] = {0.f, 0.f};
  if (i < document_rows(lengths, b, S)) {
    const float L = lse[((long)b * H + h) * S + i], D = dsum[((long)b * H + h) * S128 + i];
    const VisibleList vis(w, i);
    for (int t0 = 0; t0 < vis.count; t0 += 64) {
      const int n = min(64, vis.count - t0);
      float ds = 0.f;
      if (lane < n) {
        const long j = vis.at(t0 + lane) * ld;
        ds = expf(row_dot<DH>(q, k + j) * head_scale<DH>() - L) * (row_dot<DH>(g, v + j) - D);
      }
      for (int t = 0; t < n; ++t) add_row<DH>(acc, lane_value(ds, t), k + vis.at(t0 + t) * ld, lane);
    }
  }
  store_cols<DH>(dqkv + row * ld + h * DH, acc, head_scale<DH>(), lane);
}

template <int DH, typename T>
__global__ void __launch_bounds__(256) window_dkv_rows(const T* __restrict__ qkv, const int* __restrict__ lengths, const T* __restrict__ d_o,
                                                       const float* __restrict__ lse, const float* __restrict__ dsum, T* __restrict__ dqkv, int S,
                                                       int S128, int H, int H_kv, Window w) {
  const int lane = threadIdx.x & 63, j = blockIdx.x * 4 + (threadIdx.x >> 6), hk = blockIdx.y, b = blockIdx.z, G = H / H_kv;
  if (j >= S) return;
  const long ld = (long)(H + 2 * H_kv) * DH;
  const T* const base = qkv + (long)b * S * ld;
  const T* const k = base + j * ld + (H + hk) * DH;
  const T* const v = k + H_kv * DH;
  const int rows = document_rows(lengths, b, S);
  float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
  if (j < rows) {
    const int last = w.last_seer(j, rows);
    for (int h = hk * G; h < (hk + 1) * G; ++h) {
      const float* const L = lse + ((long)b * H + h) * S;
      const float* const D = dsum + ((long)b * H + h) * S128;
      for (int i0 = j; i0 <= last; i0 += 64) {
        const int n = min(64, last + 1 - i0), i = i0 + lane;
        float p = 0.f, ds = 0.f;
        if (lane < n) {
          p = expf(row_dot<DH>(base + i * ld + h * DH, k) * head_scale<DH>() - L[i]);
          ds = p * (row_dot<DH>(d_o + (((long)b * S + i) * H + h) * DH, v) - D[i]);
        }
        for (int t = 0; t < n; ++t) {
          add_row<DH>(dv, lane_value(p, t), d_o + (((long)b * S + i0 + t) * H + h) * DH, lane);
          add_row<DH>(dk, lane_value(ds, t), base + (i0 + t) * ld + h * DH, lane);
        }
      }
    }
  }
  T* const out = dqkv + ((long)b * S + j) * ld + (H + hk) * DH;
  store_cols<DH>(out, dk, head_scale<DH>(), lane);
  store_cols<DH>(out + H_kv * DH, dv, 1.f, lane);
}

template <int DH, typename T>
dipaco_status fwd(const T* qkv, const int* lengths, T* o, float* lse, int B, int S, int H, int H_kv, Window w, hipStream_t s) {
  if constexpr (std::is_same<T, bf16>::value) return launch_window_fwd_mfma<DH>(qkv, lengths, o, lse, B, S, H, H_kv, w, s);
  window_fwd_rows<DH, T><<<dim3((S + 3) / 4, H, B), 256, 0, s>>>(qkv, lengths, o, lse, S, H, H_kv, w);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}
template <int DH, typename T>
dipaco_status bwd(const T* qkv, const int* lengths, const T* o, const T* d_o, const float* lse, T* dqkv, float* dsum, int B, int S, int H, int H_kv,
                  Window w, hipStream_t s) {
  if constexpr (std::is_same<T, bf16>::value) return launch_window_bwd_mfma<DH>(qkv, lengths, o, d_o, lse, dqkv, dsum, B, S, H, H_kv, w, s);
  const int S128 = (S + 127) / 128 * 128;
  window_stats<DH, T><<<dim3(S128 / 4, H, B), 256, 0, s>>>(o, d_o, lengths, dsum, S, S128, H);
  DIPACO_LAUNCH_CHECK();
  window_dq_rows<DH, T><<<dim3((S + 3) / 4, H, B), 256, 0, s>>>(qkv, lengths, d_o, lse, dsum, dqkv, S, S128, H, H_kv, w);
  DIPACO_LAUNCH_CHECK();
  window_dkv_rows<DH, T><<<dim3((S + 3) / 4, H_kv, B), 256, 0, s>>>(qkv, lengths, d_o, lse, dsum, dqkv, S, S128, H, H_kv, w);
  DIPACO_LAUNCH_CHECK();
  return DIPACO_OK;
}

}  // namespace

// documents per launch: rows x heads of a launch stay below what it may hold
static int documents_a_launch(int S, int H) { return std::max(1, std::min(32768, (1 << 23) / ((S + 3) / 4) / H)); }

template <typename T>
dipaco_status launch_window_fwd(const T* qkv, const int* lengths, T* o, float* lse, int B, int S, int H, int H_kv, int dh, Window w, hipStream_t s) {
  const int step = documents_a_launch(S, H);
  for (int b = 0; b < B; b += step) {
    const int n = std::min(step, B - b);
    const size_t row = (size_t)b * S;
    const T* const x = qkv + row * (H + 2 * H_kv) * dh;
    const int* const len = lengths ? lengths + b : nullptr;
    const dipaco_status st = dh == 32   ? fwd<32>(x, len, o + row * H * dh, lse + row * H, n, S, H, H_kv, w, s)
                             : dh == 64 ? fwd<64>(x, len, o + row * H * dh, lse + row * H, n, S, H, H_kv, w, s)
                                        : fwd<128>(x, len, o + row * H * dh, lse + row * H, n, S, H, H_kv, w, s);
    if (st != DIPACO_OK) return st;
  }
  return DIPACO_OK;
}
template <typename T>
dipaco_status launch_window_bwd(const T* qkv, const int* lengths, const T* o, const T* d_o, const float* lse, T* dqkv, float* dsum, int B, int S, int H,
                                int H_kv, int dh, Window w, hipStream_t s) {
  const int step = documents_a_launch(S, H);
  for (int b = 0; b < B; b += step) {
    const int n = std::min(step, B - b);
    const size_t row = (size_t)b * S, at = row * (H + 2 * H_kv) * dh, a = row * H * dh;
    const int* const len = lengths ? lengths + b : nullptr;
    const dipaco_status st = dh == 32   ? bwd<32>(qkv + at, len, o + a, d_o + a, lse + row * H, dqkv + at, dsum, n, S, H, H_kv, w, s)
                             : dh == 64 ? bwd<64>(qkv + at, len, o + a, d_o + a, lse + row * H, dqkv + at, dsum, n, S, H, H_kv, w, s)
                                        : bwd<128>(qkv + at, len, o + a, d_o + a, lse + row * H, dqkv + at, dsum, n, S, H, H_kv, w, s);
    if (st != DIPACO_OK) return st;
  }
  return DIPACO_OK;
}
template dipaco_status launch_window_fwd<float>(const float*, const int*, float*, float*, int, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_fwd<bf16>(const bf16*, const int*, bf16*, float*, int, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_bwd<float>(const float*, const int*, const float*, const float*, const float*, float*, float*, int, int, int, int, int,
                                                Window, hipStream_t);
template dipaco_status launch_window_bwd<bf16>(const bf16*, const int*, const bf16*, const bf16*, const float*, bf16*, float*, int, int, int, int, int,
                                               Window, hipStream_t);

}  // namespace dipaco
