// fp32 attention on the matrix cores: the products of 16-row tiles that the kernels over whole sequences (attention_f32.hip) and those under a
// window and over a paged cache share.  attention_f32.hip describes the layout.
#pragma once
#include "common.h"

namespace dipaco {

namespace {

template <int DH> constexpr int row_stride() { return DH + 4; }

template <int DH> constexpr float head_scale() { return DH == 32 ? 0.17677669529663689f : DH == 64 ? 0.125f : 0.088388347648318447f; }

__device__ __forceinline__ f32x4 mfma4(float a, float b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float sum_groups(float v) {   // over the four lanes that share l % 16
  v += __shfl_xor(v, 16, WAVE);
  v += __shfl_xor(v, 32, WAVE);
  return v;
}
__device__ __forceinline__ float max_groups(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, WAVE));
  v = fmaxf(v, __shfl_xor(v, 32, WAVE));
  return v;
}

// a lane's share of one of its wave's 16 rows: columns 16 c + 4 (l / 16) .. + 3
template <int DH> struct RowFrag { float4 c[DH / 16]; };
template <int DH> __device__ __forceinline__ RowFrag<DH> load_row(const float* row, int g, bool valid) {
  RowFrag<DH> f;
#pragma unroll
  for (int c = 0; c < DH / 16; ++c)
    f.c[c] = valid ? *reinterpret_cast<const float4*>(row + 16 * c + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f);
  return f;
}
// acc (16 x 16) += rows 16 t .. + 15 of `tile`, contracted over the head with this wave's rows b
template <int DH>
__device__ __forceinline__ void rows_product(f32x4& acc, const float* tile, int t, const RowFrag<DH>& b, int m, int g) {
  const float* r = tile + (16 * t + m) * row_stride<DH>() + 4 * g;
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) {
    const float4 a = *reinterpret_cast<const float4*>(r + 16 * c);
    acc = mfma4(a.x, b.c[c].x, acc);
    acc = mfma4(a.y, b.c[c].y, acc);
    acc = mfma4(a.z, b.c[c].z, acc);
    acc = mfma4(a.w, b.c[c].w, acc);
  }
}
// acc^T[d] (16 head columns x this wave's 16 rows) += (rows 16 t .. + 15 of `tile`)^T . p
template <int DH>
__device__ __forceinline__ void cols_product(f32x4 (&acc)[DH / 16], const float* tile, int t, const f32x4& p, int m, int g) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float* r = tile + (16 * t + 4 * g + e) * row_stride<DH>() + m;
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) acc[d] = mfma4(r[16 * d], p[e], acc[d]);
  }
}
template <int DH> __device__ __forceinline__ void zero_acc(f32x4 (&acc)[DH / 16]) {
#pragma unroll
  for (int d = 0; d < DH / 16; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int DH> __device__ __forceinline__ void store_row(float* row, const f32x4 (&acc)[DH / 16], int g, float scale) {
#pragma unroll
  for (int d = 0; d < DH / 16; ++d)
    *reinterpret_cast<float4*>(row + 16 * d + 4 * g) =
        make_float4(acc[d][0] * scale, acc[d][1] * scale, acc[d][2] * scale, acc[d][3] * scale);
}
template <int DH> __device__ __forceinline__ float row_dot(const RowFrag<DH>& a, const RowFrag<DH>& b) {
  float d = 0.f;
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) d += (a.c[c].x * b.c[c].x + a.c[c].y * b.c[c].y) + (a.c[c].z * b.c[c].z + a.c[c].w * b.c[c].w);
  return sum_groups(d);
}

}  // namespace

}  // namespace dipaco
