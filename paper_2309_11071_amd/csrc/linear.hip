// Matrix product of rows with its epilogue, y = act(x W + bias) + residual, and its gradient.
//
//   forward   z = x W + bias (kept if asked for),  y = act(z) + residual
//   gradient  dz = dy act'(z):  dx = dz W^T,  dweight = x^T dz,  dbias = sum over rows of dz
//
// W is [cols][out] as the layers' weights are.  The rows are many and both sides of W are short, so the product is bound by
// reading the rows and writing the results wherever 16-bit types are used, and by the matrix unit in 32 bits.  A wave takes 32 rows and
// all of a tile's columns: the rows go from memory straight into the registers that the matrix instructions read (lane = row,
// 16 bytes a load), W is laid out in LDS in the order in which the lanes read it, once per workgroup where it fits.  The product
// is formed transposed, W's columns as the instruction's rows, so that a lane ends up with four neighbouring columns of its row and stores
// them together.
//
// Products are exact (16-bit operands) or fused (32 bits), and summed in 32 bits; the epilogue is in 32 bits and y, z, dx, dweight and
// dbias are rounded once.  For 16-bit rows dz is rounded to the rows' type before the two products, which take 16-bit operands; dbias
// sums the unrounded values.  dweight is a sum over all rows: workgroups take slices of the rows and leave a
// partial matrix each, which k_weight_sum adds up in order (no atomics: the same call gives the same bits).
#include <algorithm>

#include "head.h"

namespace ink {

typedef float f32x16 __attribute__((ext_vector_type(16)));

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

struct LinearArgs {
  const void *in, *pre;                      // forward: rows of x; gradient: rows of dy, and z if there is an activation
  const void *weight, *bias, *res;
  void *out, *keep;                          // forward: y, z or NULL; gradient: dx
  int64_t rows, ld_in, ld_pre, ld_w, ld_res, ld_out, ld_keep;
  int depth, width, act, chunk;              // terms of a sum, columns of the result, elements of the depth in LDS at a time
};

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

// fragment of dz = dy act'(z), rounded to T
template <class T, class TI> __device__ __forceinline__ typename Frag<T>::V grad_frag(const TI *dy, const TI *pre, int k, int n, int act) {
  typename Frag<T>::V v;
  float d[kVec<T>], z[kVec<T>];
  if (k + kVec<T> <= n) {
    load_pack<TI, kVec<T>>(dy + k, d);
    if (act != INK_ACT_NONE) load_pack<TI, kVec<T>>(pre + k, z);
  } else {
#pragma unroll
    for (int j = 0; j < kVec<T>; j++) {
      d[j] = k + j < n ? (float)dy[k + j] : 0.f;
      z[j] = k + j < n && act != INK_ACT_NONE ? (float)pre[k + j] : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < kVec<T>; j++) v[j] = (T)(act != INK_ACT_NONE ? d[j] * activate_grad(z[j], act) : d[j]);
  return v;
}

// W to LDS, elements [k0, k0 + len) of the depth of columns [n0, n0 + 32 NT): fragment (step, tile) is 64 lanes of 16 bytes.
template <class T, int NT, bool TRANS>
__device__ __forceinline__ void stage_weights(const LinearArgs &a, typename Frag<T>::V *s_w, int k0, int len, int n0) {
  constexpr int VK = kVec<T>;
  const T *w = static_cast<const T *>(a.weight);
  const int kv = len / VK;
  if constexpr (TRANS) {                     // the depth runs along W's rows
    for (int i = threadIdx.x; i < kv * NT * 32; i += blockDim.x) {
      const int k = i % kv, n = i / kv;
      typename Frag<T>::V v{};
      if (n0 + n < a.width && k0 + k * VK < a.depth) v = row_frag<T>(w + (int64_t)(n0 + n) * a.ld_w, k0 + k * VK, a.depth);
      s_w[((k / 2) * NT + n / 32) * 64 + n % 32 + 32 * (k % 2)] = v;
    }
  } else {                                   // squares of VK x VK elements, transposed in registers
    constexpr int NB = NT * 32 / VK;
    for (int i = threadIdx.x; i < kv * NB; i += blockDim.x) {
      const int nb = i % NB, k = i / NB, n = nb * VK;
      typename Frag<T>::V rows[VK];
#pragma unroll
      for (int j = 0; j < VK; j++) {
        rows[j] = typename Frag<T>::V{};
        const int kk = k0 + k * VK + j;
        if (kk < a.depth && n0 + n < a.width) rows[j] = row_frag<T>(w + (int64_t)kk * a.ld_w, n0 + n, a.width);
      }
#pragma unroll
      for (int c = 0; c < VK; c++) {
        typename Frag<T>::V v;
#pragma unroll
        for (int j = 0; j < VK; j++) v[j] = rows[j][c];
        const int col = n + c;
        s_w[((k / 2) * NT + col / 32) * 64 + col % 32 + 32 * (k % 2)] = v;
      }
    }
  }
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

constexpr int kLinearThreads = 512;

// T: type of the operands, TI: of the rows read (GRAD: dy and z), TO: of the rows written.
template <class T, class TI, class TO, int NT, bool GRAD>
__global__ __launch_bounds__(kLinearThreads) void k_linear(LinearArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int VK = kVec<T>, KS = kStep<T>, U = 4;
  extern __shared__ __align__(16) char s_mem[];
  V *s_w = reinterpret_cast<V *>(s_mem);
  const int l = lane_id(), half = l / 32, waves = blockDim.x / kWave;
  const int n0 = blockIdx.y * (NT * 32);
  const bool resident = a.chunk >= a.depth;
  const int64_t tile = 32 * (int64_t)waves, tiles = (a.rows + tile - 1) / tile;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t mine = t * tile + (threadIdx.x / kWave) * 32 + l % 32;
    const int64_t r = mine < a.rows ? mine : a.rows - 1;
    const TI *in = static_cast<const TI *>(a.in) + r * a.ld_in;
    const TI *pre = static_cast<const TI *>(a.pre) + (a.pre ? r * a.ld_pre : 0);
    f32x16 acc[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) acc[i] = f32x16{};
    for (int k0 = 0; k0 < a.depth; k0 += a.chunk) {
      const int len = min(a.chunk, (a.depth - k0 + KS - 1) / KS * KS);
      if (!resident || t == blockIdx.x) {
        __syncthreads();
        stage_weights<T, NT, GRAD>(a, s_w, k0, len, n0);
        __syncthreads();
      }
      for (int s0 = 0; s0 < len / KS; s0 += U) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int k = k0 + (s0 + u) * KS + half * VK;
          if constexpr (GRAD) x[u] = grad_frag<T, TI>(in, pre, k, a.depth, a.act);
          else x[u] = row_frag<T>(in, k, a.depth);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
          if (s0 + u < len / KS)
#pragma unroll
            for (int i = 0; i < NT; i++) acc[i] = mma(s_w[((s0 + u) * NT + i) * 64 + l], x[u], acc[i]);
      }
    }
    if (mine >= a.rows) continue;
    TO *out = static_cast<TO *>(a.out) + r * a.ld_out;
#pragma unroll
    for (int i = 0; i < NT; i++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int c = n0 + i * 32 + 8 * e + 4 * half;
        if (c >= a.width) continue;
        float v[4] = {acc[i][4 * e], acc[i][4 * e + 1], acc[i][4 * e + 2], acc[i][4 * e + 3]};
        if constexpr (!GRAD) {
          if (a.bias) {
            float b[4];
            load4(static_cast<const T *>(a.bias), c, a.width, b);
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] += b[j];
          }
          if (a.keep) store4(static_cast<TO *>(a.keep) + r * a.ld_keep, c, a.width, v);
          if (a.act != INK_ACT_NONE)
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = activate(v[j], a.act);
          if (a.res) {
            float b[4];
            load4(static_cast<const TO *>(a.res) + r * a.ld_res, c, a.width, b);
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] += b[j];
          }
        }
        store4(out, c, a.width, v);
      }
  }
}

// ------------------------------------------------------------------------------------ a few rows
// One row and 32 columns a workgroup: lanes side by side take 16 bytes of a row of W, the rest of the workgroup splits the depth.
template <class T, class TO>
__global__ __launch_bounds__(kHeadThreads) void k_linear_few(LinearArgs a) {
  constexpr int VK = kVec<T>, CL = 32 / VK, SL = kHeadThreads / CL, W = kHeadThreads / kWave;
  __shared__ float s_sum[W][32];
  const int cl = threadIdx.x % CL, sl = threadIdx.x / CL, n0 = blockIdx.x * 32, n = n0 + cl * VK;
  const int64_t r = blockIdx.y;
  const T *x = static_cast<const T *>(a.in) + r * a.ld_in, *w = static_cast<const T *>(a.weight);
  float acc[VK];
#pragma unroll
  for (int j = 0; j < VK; j++) acc[j] = 0.f;
  if (n < a.width)
    for (int k = sl; k < a.depth; k += SL) {
      const float xv = (float)x[k];
      const typename Frag<T>::V v = row_frag<T>(w + (int64_t)k * a.ld_w, n, a.width);
#pragma unroll
      for (int j = 0; j < VK; j++) acc[j] = fmaf(xv, (float)v[j], acc[j]);
    }
#pragma unroll
  for (int j = 0; j < VK; j++) {
#pragma unroll
    for (int o = CL; o < kWave; o <<= 1) acc[j] += __shfl_xor(acc[j], o, kWave);
    if (lane_id() < CL) s_sum[threadIdx.x / kWave][cl * VK + j] = acc[j];
  }
  __syncthreads();
  const int c = n0 + threadIdx.x;
  if (threadIdx.x >= 32 || c >= a.width) return;
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < W; i++) v += s_sum[i][threadIdx.x];
  if (a.bias) v += (float)static_cast<const T *>(a.bias)[c];
  if (a.keep) static_cast<TO *>(a.keep)[r * a.ld_keep + c] = (TO)v;
  v = activate(v, a.act);
  if (a.res) v += (float)static_cast<const TO *>(a.res)[r * a.ld_res + c];
  static_cast<TO *>(a.out)[r * a.ld_out + c] = (TO)v;
}

// ------------------------------------------------------------------------------------ gradient of the weights
struct WeightGradArgs {
  const void *x, *dy, *pre;
  float *part, *part_bias;                   // [slices][cols][out], [slices][out]
  int64_t rows, ld_x, ld_dy, ld_pre, slice;  // rows of a slice
  int cols, out, act;
};

constexpr int kGradRows = 64;                // rows in LDS at a time

// Squares of VK rows x VK columns, transposed in registers: fragment (step, tile) holds 32 columns of 2 VK rows, a lane VK rows of a column.
// `get(row, column)` gives VK elements of a row.
template <class T, int NT, class Get> __device__ __forceinline__ void stage_rows(typename Frag<T>::V *s, Get get) {
  constexpr int VK = kVec<T>, NB = NT * 32 / VK, RB = kGradRows / VK;
  for (int i = threadIdx.x; i < NB * RB; i += kLinearThreads) {
    const int nb = i % NB, rb = i / NB;
    typename Frag<T>::V rows[VK];
#pragma unroll
    for (int j = 0; j < VK; j++) rows[j] = get(rb * VK + j, nb * VK);
#pragma unroll
    for (int c = 0; c < VK; c++) {
      typename Frag<T>::V v;
#pragma unroll
      for (int j = 0; j < VK; j++) v[j] = rows[j][c];
      const int col = nb * VK + c;
      s[((rb / 2) * NT + col / 32) * 64 + col % 32 + 32 * (rb % 2)] = v;
    }
  }
}

// Tile of 32 KT columns of x by 32 NT columns of dz over a slice of the rows.  Eight waves: wave w has x tiles w % KW ..
template <class T, class TI, int KT, int NT>
__global__ __launch_bounds__(kLinearThreads) void k_weight_grad(WeightGradArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int W = kLinearThreads / kWave, KW = KT < W ? KT : W, NW = W / KW, KP = KT / KW, NP = (NT + NW - 1) / NW;
  constexpr int STEPS = kGradRows / kStep<T>;
  __shared__ V s_x[STEPS * KT * 64], s_z[STEPS * NT * 64];
  const int w = threadIdx.x / kWave, l = lane_id();
  const int kt0 = (w % KW) * KP, nt0 = (w / KW) * NP;
  const int k0 = blockIdx.x * (KT * 32), n0 = blockIdx.y * (NT * 32);
  const int64_t r_begin = blockIdx.z * a.slice, r_end = min(r_begin + a.slice, a.rows);
  f32x16 acc[KP][NP];
#pragma unroll
  for (int i = 0; i < KP; i++)
#pragma unroll
    for (int j = 0; j < NP; j++) acc[i][j] = f32x16{};
  for (int64_t r0 = r_begin; r0 < r_end; r0 += kGradRows) {
    __syncthreads();
    stage_rows<T, KT>(s_x, [&](int r, int c) {
      V v{};
      if (r0 + r < r_end && k0 + c < a.cols) v = row_frag<T>(static_cast<const T *>(a.x) + (r0 + r) * a.ld_x, k0 + c, a.cols);
      return v;
    });
    stage_rows<T, NT>(s_z, [&](int r, int c) {
      V v{};
      if (r0 + r < r_end && n0 + c < a.out)
        v = grad_frag<T, TI>(static_cast<const TI *>(a.dy) + (r0 + r) * a.ld_dy,
                             static_cast<const TI *>(a.pre) + (a.pre ? (r0 + r) * a.ld_pre : 0), n0 + c, a.out, a.act);
      return v;
    });
    __syncthreads();
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      V z[NP];
#pragma unroll
      for (int j = 0; j < NP; j++) z[j] = s_z[(s * NT + min(nt0 + j, NT - 1)) * 64 + l];
#pragma unroll
      for (int i = 0; i < KP; i++) {
        const V x = s_x[(s * KT + kt0 + i) * 64 + l];
#pragma unroll
        for (int j = 0; j < NP; j++) acc[i][j] = mma(z[j], x, acc[i][j]);
      }
    }
  }
  float *part = a.part + (int64_t)blockIdx.z * a.cols * a.out;
#pragma unroll
  for (int i = 0; i < KP; i++)
#pragma unroll
    for (int j = 0; j < NP; j++) {
      const int k = k0 + (kt0 + i) * 32 + l % 32;
      if (k >= a.cols || nt0 + j >= NT) continue;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int c = n0 + (nt0 + j) * 32 + 8 * e + 4 * (l / 32);
        const float v[4] = {acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        if (c < a.out) store4(part + (int64_t)k * a.out, c, a.out, v);
      }
    }
}

// column sums of dz over a slice of the rows: 64 columns a workgroup, a wave takes every fourth row
template <class TI> __global__ __launch_bounds__(kHeadThreads) void k_bias_grad(WeightGradArgs a) {
  constexpr int W = kHeadThreads / kWave;
  __shared__ float s_sum[W][kWave];
  const int w = threadIdx.x / kWave, c = blockIdx.x * kWave + lane_id();
  const int64_t r_begin = blockIdx.y * a.slice, r_end = min(r_begin + a.slice, a.rows);
  float t = 0.f;
  if (c < a.out)
    for (int64_t r = r_begin + w; r < r_end; r += W) {
      const float d = (float)static_cast<const TI *>(a.dy)[r * a.ld_dy + c];
      t += a.act != INK_ACT_NONE ? d * activate_grad((float)static_cast<const TI *>(a.pre)[r * a.ld_pre + c], a.act) : d;
    }
  s_sum[w][lane_id()] = t;
  __syncthreads();
  if (w || c >= a.out) return;
  t = 0.f;
#pragma unroll
  for (int i = 0; i < W; i++) t += s_sum[i][lane_id()];
  a.part_bias[(int64_t)blockIdx.y * a.out + c] = t;
}

// partial sums of n elements from `slices` slices to their sum
__global__ __launch_bounds__(kHeadThreads) void k_weight_sum(const float *part, int64_t n, int slices, int type, int out, void *to, int64_t ld_to) {
  const int64_t i = (int64_t)blockIdx.x * kHeadThreads + threadIdx.x;
  if (i >= n) return;
  float t = 0.f;
  for (int s = 0; s < slices; s++) t += part[s * n + i];
  store_any(to, i / out * ld_to + i % out, type, t);
}

// ------------------------------------------------------------------------------------ host side
constexpr int64_t kFewRows = 16;
constexpr int kWeightLds = 64 << 10;

// tiles of 32 columns a workgroup takes: all columns up to eight tiles, fewer where that leaves the card empty
static int linear_tiles(int64_t rows, int width) {
  const int all = (width + 31) / 32;
  int nt = all >= 8 ? 8 : all > 6 ? 8 : all > 4 ? 6 : all > 2 ? 4 : 2;
  while (nt > 2 && (rows + 255) / 256 * ((all + nt - 1) / nt) < 256) nt = nt == 6 ? 4 : nt / 2;
  return nt;
}

template <class T, class TI, class TO, int NT, bool GRAD> static void linear_launch(LinearArgs a, Launches &run) {
  constexpr int KS = kStep<T>;
  const int padded = (a.depth + KS - 1) / KS * KS, most = kWeightLds / (NT * 32 * (int)sizeof(T)) / KS * KS;
  a.chunk = std::min(padded, most);
  const int lds = a.chunk * NT * 32 * (int)sizeof(T);
  const int threads = a.rows <= 128 * 256 ? 256 : kLinearThreads;
  const int64_t tile = threads / 2;
  const unsigned gy = (unsigned)((a.width + NT * 32 - 1) / (NT * 32));
  const int64_t tiles = (a.rows + tile - 1) / tile;
  const int64_t most_x = a.chunk >= a.depth ? std::max<int64_t>(1, 1024 / gy) : tiles;
  run.lds = lds;
  run(k_linear<T, TI, TO, NT, GRAD>, dim3((unsigned)std::min(tiles, most_x), gy), dim3(threads), a);
  run.lds = 0;
}
template <class T, class TI, class TO, bool GRAD> static void linear_run(const LinearArgs &a, Launches &run) {
  if constexpr (!GRAD)
    if (a.rows <= kFewRows) return run(k_linear_few<T, TO>, dim3((a.width + 31) / 32, (unsigned)a.rows), dim3(kHeadThreads), a);
  switch (linear_tiles(a.rows, a.width)) {
    case 2: return linear_launch<T, TI, TO, 2, GRAD>(a, run);
    case 4: return linear_launch<T, TI, TO, 4, GRAD>(a, run);
    case 6: return linear_launch<T, TI, TO, 6, GRAD>(a, run);
    default: return linear_launch<T, TI, TO, 8, GRAD>(a, run);
  }
}

struct GradPlan { int kt, nt, slices; int64_t slice; };
static GradPlan grad_plan(int64_t rows, int cols, int out) {
  GradPlan p;
  p.kt = cols > 64 ? 4 : 2;
  p.nt = out > 64 ? 4 : 2;
  const int64_t tiles = (int64_t)((cols + p.kt * 32 - 1) / (p.kt * 32)) * ((out + p.nt * 32 - 1) / (p.nt * 32));
  const int64_t blocks = (rows + kGradRows - 1) / kGradRows;
  const int64_t slices = std::max<int64_t>(1, std::min<int64_t>(blocks, 512 / tiles));
  p.slice = (blocks + slices - 1) / slices * kGradRows;
  p.slices = (int)((rows + p.slice - 1) / p.slice);
  return p;
}

template <class T, class TI> static void weight_grad_run(const WeightGradArgs &a, const GradPlan &p, Launches &run) {
  const dim3 grid((a.cols + p.kt * 32 - 1) / (p.kt * 32), (a.out + p.nt * 32 - 1) / (p.nt * 32), p.slices), block(kLinearThreads);
  if (a.part) {
    if (p.kt == 2) run(p.nt == 2 ? k_weight_grad<T, TI, 2, 2> : k_weight_grad<T, TI, 2, 4>, grid, block, a);
    else run(p.nt == 2 ? k_weight_grad<T, TI, 4, 2> : k_weight_grad<T, TI, 4, 4>, grid, block, a);
  }
  if (a.part_bias) run(k_bias_grad<TI>, dim3((a.out + kWave - 1) / kWave, p.slices), dim3(kHeadThreads), a);
}

static const char *linear_check(int64_t rows, int32_t cols, int32_t out, int32_t type, int32_t io_type, int32_t act) {
  if (!known_type(type)) return "unknown type";
  if (io_type != type && io_type != INK_F32) return "the results' type must be the rows' type or INK_F32";
  if (act < INK_ACT_NONE || act > INK_ACT_SILU) return "unknown activation";
  if (rows < 0 || rows > kMaxHeadRows) return "rows out of range";
  if (cols < 1 || cols > INK_MAX_IN_DIM || out < 1 || out > INK_MAX_IN_DIM) return "cols and out must be 1 .. INK_MAX_IN_DIM";
  return nullptr;
}

}  // namespace ink

using namespace ink;

extern "C" ink_status ink_linear(const void *x, int64_t ld_x, const void *weight, int64_t ld_w, const void *bias, const void *residual,
                                 int64_t ld_res, int64_t rows, int32_t cols, int32_t out, int32_t type, int32_t out_type, int32_t act,
                                 void *y, int64_t ld_y, void *pre, int64_t ld_pre, void *hip_stream) {
  const char *who = "ink_linear";
  if (const char *why = linear_check(rows, cols, out, type, out_type, act)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (!good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "%s: x is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(weight, cols, out, ld_w, type, false)) return fail_call(INK_E_ARG, "%s: weight is NULL, not aligned to its type or has rows that overlap", who);
  if (!aligned_to(bias, type_size(type))) return fail_call(INK_E_ARG, "%s: bias is not aligned to its type", who);
  if (residual && !good_matrix(residual, rows, out, ld_res, out_type, false)) return fail_call(INK_E_ARG, "%s: residual is not aligned to its type or has rows that overlap", who);
  if (!good_matrix(y, rows, out, ld_y, out_type, true)) return fail_call(INK_E_ARG, "%s: y is NULL, not aligned to its type or has rows that overlap", who);
  if (pre && !good_matrix(pre, rows, out, ld_pre, out_type, true)) return fail_call(INK_E_ARG, "%s: pre is not aligned to its type or has rows that overlap", who);
  if (rows == 0) return INK_OK;
  LinearArgs a{};
  a.in = x; a.weight = weight; a.bias = bias; a.res = residual; a.out = y; a.keep = pre;
  a.rows = rows; a.ld_in = ld_x; a.ld_w = ld_w; a.ld_res = ld_res; a.ld_out = ld_y; a.ld_keep = ld_pre;
  a.depth = cols; a.width = out; a.act = act;
  Launches run(hip_stream);
  if (type == INK_F32) linear_run<float, float, float, false>(a, run);
  else if (type == INK_BF16) out_type == INK_F32 ? linear_run<bf16, bf16, float, false>(a, run) : linear_run<bf16, bf16, bf16, false>(a, run);
  else out_type == INK_F32 ? linear_run<f16, f16, float, false>(a, run) : linear_run<f16, f16, f16, false>(a, run);
  return run.done(who);
}

extern "C" size_t ink_linear_backward_work(int64_t rows, int32_t cols, int32_t out) {
  if (rows < 1 || rows > kMaxHeadRows || cols < 1 || cols > INK_MAX_IN_DIM || out < 1 || out > INK_MAX_IN_DIM) return 0;
  return (size_t)grad_plan(rows, cols, out).slices * ((size_t)cols + 1) * (size_t)out * sizeof(float);
}

extern "C" ink_status ink_linear_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const void *weight, int64_t ld_w,
                                          const void *pre, int64_t ld_pre, int64_t rows, int32_t cols, int32_t out, int32_t type,
                                          int32_t dy_type, int32_t act, void *dx, int64_t ld_dx, void *dweight, int64_t ld_dw,
                                          void *dbias, void *work, size_t work_bytes, void *hip_stream) {
  const char *who = "ink_linear_backward";
  if (const char *why = linear_check(rows, cols, out, type, dy_type, act)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (type == INK_F16 && dy_type == INK_F32)
    return fail_call(INK_E_ARG, "%s: 16-bit floats of INK_F16 do not hold the range of a 32-bit gradient: pass dy as INK_F16, scaled", who);
  if (!good_matrix(dy, rows, out, ld_dy, dy_type, false)) return fail_call(INK_E_ARG, "%s: dy is NULL, not aligned to its type or has rows that overlap", who);
  if (act != INK_ACT_NONE && !good_matrix(pre, rows, out, ld_pre, dy_type, false))
    return fail_call(INK_E_ARG, "%s: pre is NULL, not aligned to its type or has rows that overlap", who);
  if (dx && !good_matrix(weight, cols, out, ld_w, type, false)) return fail_call(INK_E_ARG, "%s: weight is NULL, not aligned to its type or has rows that overlap", who);
  if (dx && !good_matrix(dx, rows, cols, ld_dx, type, true)) return fail_call(INK_E_ARG, "%s: dx is not aligned to its type or has rows that overlap", who);
  if (dweight && !good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "%s: x is NULL, not aligned to its type or has rows that overlap", who);
  if (dweight && !good_matrix(dweight, cols, out, ld_dw, type, true)) return fail_call(INK_E_ARG, "%s: dweight is not aligned to its type or has rows that overlap", who);
  if (!aligned_to(dbias, type_size(type))) return fail_call(INK_E_ARG, "%s: dbias is not aligned to its type", who);
  if (rows > 0 && (dweight || dbias) && (!work || !aligned_to(work, 16) || work_bytes < ink_linear_backward_work(rows, cols, out)))
    return fail_call(INK_E_ARG, "%s: work holds less than ink_linear_backward_work bytes or is not aligned to 16", who);
  Launches run(hip_stream);
  if (dx && rows > 0) {
    LinearArgs a{};
    a.in = dy; a.pre = act == INK_ACT_NONE ? nullptr : pre; a.weight = weight; a.out = dx;
    a.rows = rows; a.ld_in = ld_dy; a.ld_pre = ld_pre; a.ld_w = ld_w; a.ld_out = ld_dx;
    a.depth = out; a.width = cols; a.act = act;
    if (type == INK_F32) linear_run<float, float, float, true>(a, run);
    else if (type == INK_F16) linear_run<f16, f16, f16, true>(a, run);
    else dy_type == INK_F32 ? linear_run<bf16, float, bf16, true>(a, run) : linear_run<bf16, bf16, bf16, true>(a, run);
  }
  if (dweight || dbias) {
    GradPlan p{};
    WeightGradArgs a{};
    if (rows > 0) {
      p = grad_plan(rows, cols, out);
      a.x = x; a.dy = dy; a.pre = act == INK_ACT_NONE ? nullptr : pre;
      a.part = static_cast<float *>(work);
      a.part_bias = dbias ? a.part + (int64_t)p.slices * cols * out : nullptr;
      if (!dweight) a.part = nullptr;
      a.rows = rows; a.ld_x = ld_x; a.ld_dy = ld_dy; a.ld_pre = ld_pre; a.slice = p.slice;
      a.cols = cols; a.out = out; a.act = act;
      if (type == INK_F32) weight_grad_run<float, float>(a, p, run);
      else if (type == INK_F16) weight_grad_run<f16, f16>(a, p, run);
      else dy_type == INK_F32 ? weight_grad_run<bf16, float>(a, p, run) : weight_grad_run<bf16, bf16>(a, p, run);
    }
    const int64_t n = (int64_t)cols * out;  // no rows: zeros
    if (dweight) run(k_weight_sum, dim3((unsigned)((n + kHeadThreads - 1) / kHeadThreads)), dim3(kHeadThreads), a.part, n, p.slices, type, out, dweight, ld_dw);
    if (dbias) run(k_weight_sum, dim3((out + kHeadThreads - 1) / kHeadThreads), dim3(kHeadThreads), a.part_bias, (int64_t)out, p.slices, type, out, dbias, (int64_t)out);
  }
  return run.done(who);
}
