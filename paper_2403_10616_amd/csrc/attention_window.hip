// Attention with a sliding window and sinks over the packed q | k | v rows of a padded batch: dispatch by element type and head size.
//
//   vis(i) = { j <= i : j > i - window or j < sinks }      s_ij = q_i.k_j / sqrt(dh)      lse_i = log sum_{j in vis(i)} exp s_ij
//   o_i = sum_{vis(i)} exp(s_ij - lse_i) v_j
//   D_i = dO_i.o_i     dS_ij = P_ij (dO_i.v_j - D_i)     dq_i = sum_j dS_ij k_j / sqrt(dh)
//   dk_j = sum_{heads of the group} sum_{i sees j} dS_ij q_i / sqrt(dh)     dv_j = sum_{heads} sum_{i sees j} P_ij dO_i
//
// bf16 runs in attention_window_mfma.hip, fp32 in attention_window_f32.hip, both on the matrix cores.
#include <type_traits>

#include "kernels.h"

namespace dipaco {

// run(DH, first document, documents, their first row): in as many launches as it takes to keep workgroups, of 64 rows or more each and three kinds
// in the backward pass, below 2^22
template <typename F> static dipaco_status in_parts(int B, int S, int H, int dh, F run) {
  const int step = std::max(1, std::min(B, (1 << 20) / ((S + 63) / 64) / H));
  for (int b = 0; b < B; b += step) {
    const int n = std::min(step, B - b);
    const size_t row = (size_t)b * S;
    const dipaco_status st = dh == 32   ? run(std::integral_constant<int, 32>{}, b, n, row)
                             : dh == 64 ? run(std::integral_constant<int, 64>{}, b, n, row)
                                        : run(std::integral_constant<int, 128>{}, b, n, row);
    if (st != DIPACO_OK) return st;
  }
  return DIPACO_OK;
}

template <typename T>
dipaco_status launch_window_fwd(const T* qkv, const int* lengths, T* o, float* lse, int B, int S, int H, int H_kv, int dh, Window w, hipStream_t s) {
  return in_parts(B, S, H, dh, [&](auto DHc, int b, int n, size_t row) {
    constexpr int DH = decltype(DHc)::value;
    const T* const x = qkv + row * (H + 2 * H_kv) * DH;
    const int* const len = lengths ? lengths + b : nullptr;
    if constexpr (std::is_same<T, bf16>::value) return launch_window_fwd_mfma<DH>(x, len, o + row * H * DH, lse + row * H, n, S, H, H_kv, w, s);
    else return launch_window_fwd_f32<DH>(x, len, o + row * H * DH, lse + row * H, n, S, H, H_kv, w, s);
  });
}
template <typename T>
dipaco_status launch_window_bwd(const T* qkv, const int* lengths, const T* o, const T* d_o, const float* lse, T* dqkv, float* dsum, int B, int S, int H,
                                int H_kv, int dh, Window w, hipStream_t s) {
  return in_parts(B, S, H, dh, [&](auto DHc, int b, int n, size_t row) {
    constexpr int DH = decltype(DHc)::value;
    const size_t at = row * (H + 2 * H_kv) * DH, a = row * H * DH;
    const int* const len = lengths ? lengths + b : nullptr;
    if constexpr (std::is_same<T, bf16>::value)
      return launch_window_bwd_mfma<DH>(qkv + at, len, o + a, d_o + a, lse + row * H, dqkv + at, dsum, n, S, H, H_kv, w, s);
    else return launch_window_bwd_f32<DH>(qkv + at, len, o + a, d_o + a, lse + row * H, dqkv + at, dsum, n, S, H, H_kv, w, s);
  });
}
template dipaco_status launch_window_fwd<float>(const float*, const int*, float*, float*, int, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_fwd<bf16>(const bf16*, const int*, bf16*, float*, int, int, int, int, int, Window, hipStream_t);
template dipaco_status launch_window_bwd<float>(const float*, const int*, const float*, const float*, const float*, float*, float*, int, int, int, int, int,
                                                Window, hipStream_t);
template dipaco_status launch_window_bwd<bf16>(const bf16*, const int*, const bf16*, const bf16*, const float*, bf16*, float*, int, int, int, int, int,
                                               Window, hipStream_t);

}  // namespace dipaco
