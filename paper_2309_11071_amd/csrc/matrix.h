// What the products of rows share (linear.hip, gated.hip): fragments of the matrix instructions, pieces of rows, activations and their slopes.
#pragma once
#include "head.h"

namespace ink {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float F4 __attribute__((ext_vector_type(4)));

template <class T> struct Frag;              // 16 bytes of a row or of a column: what one lane gives a matrix instruction
template <> struct Frag<float> { typedef float V __attribute__((ext_vector_type(4))); };
template <> struct Frag<bf16> { typedef bf16 V __attribute__((ext_vector_type(8))); };
template <> struct Frag<f16> { typedef f16 V __attribute__((ext_vector_type(8))); };
template <class T> constexpr int kVec = 16 / (int)sizeof(T);      // elements of a fragment a lane
template <class T> constexpr int kStep = 2 * kVec<T>;             // depth of a fragment: lanes 0-31 hold its first half

__device__ __forceinline__ f32x16 mma(Frag<bf16>::V a, Frag<bf16>::V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(Frag<f16>::V a, Frag<f16>::V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(Frag<float>::V a, Frag<float>::V b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}
// Several products of one step: in 32 bits a step is four instructions, and those of one accumulator do not follow each other.
template <class T, int M, int N> __device__ __forceinline__ void mma_block(const typename Frag<T>::V (&a)[N], const typename Frag<T>::V (&b)[M], f32x16 (&c)[M][N]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int i = 0; i < M; i++)
#pragma unroll
        for (int n = 0; n < N; n++) c[i][n] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[n][j], b[i][j], c[i][n], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < M; i++)
#pragma unroll
      for (int n = 0; n < N; n++) c[i][n] = mma(a[n], b[i], c[i][n]);
  }
}
// Where a product's element stands in a lane: column (of the second operand) lane % 32, row 8 (e / 4) + 4 (lane / 32) + e % 4.

// Standard normal distribution function, with the density in `pdf`.  1 - Phi(|z|) = density * polynomial in 1 / (1 + p |z| / sqrt 2)
// (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26: error of erf at most 1.5e-7): one exponential serves both.
__device__ __forceinline__ float normal_cdf(float z, float &pdf) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118f, fabsf(z), 1.f));
  const float e = __builtin_amdgcn_exp2f(z * z * (-0.5f * 1.4426950408889634f));
  pdf = e * 0.3989422804014327f;
  const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  const float tail = 0.5f * poly * e;
  return z < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }

__device__ __forceinline__ float activate(float z, int act) {
  if (act == INK_ACT_RELU) return z < 0.f ? 0.f : z;             // NaN stays
  if (act == INK_ACT_GELU) { float pdf; return z * normal_cdf(z, pdf); }
  if (act == INK_ACT_SILU) return z * sigmoid(z);
  return z;
}
__device__ __forceinline__ float activate_grad(float z, int act) {
  if (act == INK_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
  if (act == INK_ACT_GELU) { float pdf; const float cdf = normal_cdf(z, pdf); return fmaf(z, pdf, cdf); }
  if (act == INK_ACT_SILU) { const float s = sigmoid(z); return s * fmaf(z, 1.f - s, 1.f); }
  return 1.f;
}

// the same of several elements, one decision for all of them
template <int N> __device__ __forceinline__ void activate_all(float v[N], int act) {
  if (act == INK_ACT_NONE) return;
  if (act == INK_ACT_RELU)
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = activate(v[e], INK_ACT_RELU);
  else if (act == INK_ACT_GELU)
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = activate(v[e], INK_ACT_GELU);
  else
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = activate(v[e], INK_ACT_SILU);
}
template <int N> __device__ __forceinline__ void scale_by_slope(float d[N], const float z[N], int act) {
  if (act == INK_ACT_RELU)
#pragma unroll
    for (int e = 0; e < N; e++) d[e] *= activate_grad(z[e], INK_ACT_RELU);
  else if (act == INK_ACT_GELU)
#pragma unroll
    for (int e = 0; e < N; e++) d[e] *= activate_grad(z[e], INK_ACT_GELU);
  else
#pragma unroll
    for (int e = 0; e < N; e++) d[e] *= activate_grad(z[e], INK_ACT_SILU);
}

// kVec elements k .. of one row of n elements as a fragment; past the row's end zeros, and nothing is read there.
template <class T> __device__ __forceinline__ typename Frag<T>::V row_frag(const T *row, int k, int n) {
  typedef typename Frag<T>::V V;
  typedef typename Pack<T, kVec<T>>::type P;
  if (k + kVec<T> <= n) { const P p = *reinterpret_cast<const P *>(row + k); return (V)p; }
  V v;
#pragma unroll
  for (int j = 0; j < kVec<T>; j++) v[j] = k + j < n ? row[k + j] : (T)0.f;
  return v;
}

// four neighbouring columns of a row
template <class T> __device__ __forceinline__ void load4(const T *p, int c, int n, float v[4]) {
  if (c + 4 <= n) return load_pack<T, 4>(p + c, v);
#pragma unroll
  for (int j = 0; j < 4; j++) v[j] = c + j < n ? (float)p[c + j] : 0.f;
}
template <class T> __device__ __forceinline__ void store4(T *p, int c, int n, const float v[4]) {
  if (c + 4 <= n) return store_pack<T, 4>(p + c, v);
#pragma unroll
  for (int j = 0; j < 4; j++)
    if (c + j < n) p[c + j] = (T)v[j];
}

// a piece of a row that starts `by` elements too early, moved down
template <class V> __device__ __forceinline__ V move_down(V v, int by, int size) {
  const unsigned __int128 u = __builtin_bit_cast(unsigned __int128, v) >> (8 * size * by);
  return __builtin_bit_cast(V, u);
}

// Bytes between rows in LDS: rows of 16 lanes' pieces fall on all banks, and in 32 bits two rows side by side nearly so.
template <class T, int TILES> constexpr int kGradPitch = TILES * 32 * (int)sizeof(T) + (sizeof(T) == 2 ? 16 : 144);

// Fragment of a step (2 kVec rows) of 32 columns of rows in LDS.  16 bits: of 16 lanes, lane 4 j + b gives the place of columns 4 b .. of
// row j, and lane i gets column i of the four rows.  Which rows of a step a lane holds is the same for both operands, and nothing else matters.
template <class T> __device__ __forceinline__ typename Frag<T>::V columns_frag(const char *rows, int pitch, int step, int tile) {
  const int l = lane_id(), half = l / 32;
  if constexpr (sizeof(T) == 2) {
    typedef short S4 __attribute__((ext_vector_type(4)));
    typedef S4 __attribute__((address_space(3))) *Lds;
    const char *at = rows + (step * 16 + half * 8 + l % 16 / 4) * pitch + (tile * 32 + l / 16 % 2 * 16 + l % 4 * 4) * 2;
    const S4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * pitch));
    typedef short S8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(typename Frag<T>::V, (S8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    typename Frag<T>::V v;
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = *reinterpret_cast<const float *>(rows + (step * 8 + 2 * j + half) * pitch + (tile * 32 + l % 32) * 4);
    return v;
  }
}

}  // namespace ink
