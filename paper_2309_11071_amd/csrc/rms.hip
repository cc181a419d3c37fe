// Root-mean-square norm of rows, with the addition of a residual before it and an output in 8 bits, and its gradient.
//
//   forward   t = x + residual, rounded to the rows' type (the residual stream that goes on),  r = 1 / sqrt(sum t^2 / n + eps),
//             y = t r weight;  in 8 bits: scale = max |y| / 448, codes = y / scale to the nearest e4m3 number
//   gradient  h = t r,  g = dy weight:   dx = r (g - h mean(g h)) + d_total,  dweight = sum over rows of dy h
//
// Bound by memory, at the rate of a copy (5.09 TB/s) where a wave holds a row: 2.45M x 256 bf16 with a residual 974 us (5.03 GB), gradient of 2.45M x 128
// bf16 478 us (2.52 GB, 5 of them for the partial rows' sum), 1M x 602 bf16 to 8 bits 912 us (4.22 GB, 4.6 TB/s: rows of 602 codes start anywhere, and a lane
// stores 8 bytes of them).  A row of 128 by itself 3.3 us.
//
// The statistics and y are those of the sum as it is stored, so that the gradient, which reads the stored sum, is that of the same
// function.  Laid out as the layer norm is (norm.hip): L lanes hold a row, V elements a load, at most 4 loads a
// lane; a row is read once; the last load of a row ends at the row's end.  Rows that a wave does not hold have a workgroup of 256 threads, and one of
// 1024 where those do not hold them.  Sums and statistics are in 32 bits, outputs are rounded once; the 8-bit codes are rounded from the 32-bit
// y.  dweight is a sum over all rows: partial rows by workgroup, added in their order (no atomics: the same call gives the same bits).
#include <algorithm>

#include "rowgroup.h"

namespace ink {

struct RmsArgs {
  const void *x, *res, *weight;            // gradient: x is the stored sum, res the gradient that arrives there (or NULL)
  const void *dy;
  void *y, *total;                         // gradient: y is dx (or NULL)
  float *rstd, *scale;                     // forward: rstd written where not NULL; gradient: read
  float *part;                             // gradient: [workgroups][cols], or NULL
  int64_t rows, ld_x, ld_res, ld_dy, ld_y, ld_total;
  int cols, param_type;
  float eps;
};

constexpr int kMidThreads = 256;

template <int L> __device__ __forceinline__ float row_max(float x, float *s) {
  x = group_all<(L > kWave ? kWave : L)>(x, [](float a, float b) { return fmaxf(a, b); });
  if constexpr (L > kWave) {
    if (lane_id() == 0) s[threadIdx.x / kWave] = x;
    __syncthreads();
    x = s[0];
#pragma unroll
    for (int i = 1; i < L / kWave; i++) x = fmaxf(x, s[i]);
    __syncthreads();
  }
  return x;
}

// V codes (a multiple of 4, or 1) of numbers within the range of e4m3; NaN stays NaN
template <int V> __device__ __forceinline__ void store_codes(uint8_t *p, const float v[V]) {
  if constexpr (V == 1) *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[0], 0, false);
  else {
    typedef uint32_t W __attribute__((ext_vector_type(V / 4), aligned(1)));
    W w;
#pragma unroll
    for (int j = 0; j < V / 4; j++) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * j], v[4 * j + 1], 0, false);
      w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * j + 2], v[4 * j + 3], lo, true);
    }
    *reinterpret_cast<W *>(p) = w;
  }
}

template <class T, int L, int NV, int V, bool FULL, bool CODES>
__global__ __launch_bounds__(norm_threads<L>()) void k_rms_norm(RmsArgs a) {
  constexpr int G = norm_threads<L>() / L;
  __shared__ float s_sum[L > kWave ? L / kWave : 1];
  const NormPlace<L, V, FULL> p(a.cols);
  float w[NV][V];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int j = 0; j < V; j++) w[i][j] = a.weight ? load_any(a.weight, p.at(i) + j, a.param_type) : 1.f;
  const float n = (float)a.cols;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += (int64_t)gridDim.x * G) {
    const int64_t mine = r0 + threadIdx.x / L;
    const bool on = mine < a.rows;
    const int64_t r = on ? mine : a.rows - 1;                 // a group without a row repeats the last one and stores nothing
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x;
    float v[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) load_pack<T, V>(x + p.at(i), v[i]);
    if (a.res) {
      const T *q = static_cast<const T *>(a.res) + r * a.ld_res;
      float e[NV][V];
#pragma unroll
      for (int i = 0; i < NV; i++) load_pack<T, V>(q + p.at(i), e[i]);
      T *t = static_cast<T *>(a.total) + r * a.ld_total;
#pragma unroll
      for (int i = 0; i < NV; i++) {
#pragma unroll
        for (int j = 0; j < V; j++) v[i][j] = (float)(T)(v[i][j] + e[i][j]);
        if (on && p.any(i)) store_pack<T, V>(t + p.at(i), v[i]);
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) sum += p.live(i, j) ? v[i][j] * v[i][j] : 0.f;
    const float rstd = 1.f / sqrtf(row_sum<L>(sum, s_sum) / n + a.eps);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) {
        v[i][j] = v[i][j] * rstd * w[i][j];
        if constexpr (CODES) top = fmaxf(top, fabsf(v[i][j]) <= 3.4028235e38f ? fabsf(v[i][j]) : INFINITY);       // NaN counts as infinite
      }
    float scale = 1.f;
    if constexpr (CODES) {
      top = row_max<L>(top, s_sum);
      // below the smallest normal scale the row counts as zeros; with a number that is none, the row is none
      scale = top == INFINITY ? NAN : top < 448.f * 1.17549435e-38f ? 0.f : top / 448.f;
      const float by = scale == 0.f ? 0.f : 1.f / scale;
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) v[i][j] *= by;
    }
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      if (!p.any(i)) continue;
      if constexpr (CODES) store_codes<V>(static_cast<uint8_t *>(a.y) + r * a.ld_y + p.at(i), v[i]);
      else store_pack<T, V>(static_cast<T *>(a.y) + r * a.ld_y + p.at(i), v[i]);
    }
    if (p.q == 0) {
      if (a.rstd) a.rstd[r] = rstd;
      if constexpr (CODES) a.scale[r] = scale;
    }
  }
}

template <class T, int L, int NV, int V, bool FULL>
__global__ __launch_bounds__(norm_threads<L>()) void k_rms_norm_grad(RmsArgs a) {
  constexpr int G = norm_threads<L>() / L;
  __shared__ float s_sum[L > kWave ? L / kWave : 1];
  const NormPlace<L, V, FULL> p(a.cols);
  float w[NV][V], dw[NV][V];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int j = 0; j < V; j++) {
      w[i][j] = a.weight ? load_any(a.weight, p.at(i) + j, a.param_type) : 1.f;
      dw[i][j] = 0.f;
    }
  const float n = (float)a.cols;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += (int64_t)gridDim.x * G) {
    const int64_t mine = r0 + threadIdx.x / L;
    const bool on = mine < a.rows;
    const int64_t r = on ? mine : a.rows - 1;
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x, *dy = static_cast<const T *>(a.dy) + r * a.ld_dy;
    float h[NV][V], g[NV][V], e[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) { load_pack<T, V>(x + p.at(i), h[i]); load_pack<T, V>(dy + p.at(i), g[i]); }
    if (a.res) {
      const T *q = static_cast<const T *>(a.res) + r * a.ld_res;
#pragma unroll
      for (int i = 0; i < NV; i++) load_pack<T, V>(q + p.at(i), e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) e[i][j] = 0.f;
    }
    const float rstd = a.rstd[r];
    float along = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) {
        h[i][j] *= rstd;
        dw[i][j] += on ? g[i][j] * h[i][j] : 0.f;             // a repeated element's sums are dropped at the end
        g[i][j] *= w[i][j];
        along += p.live(i, j) ? g[i][j] * h[i][j] : 0.f;
      }
    if (!a.y) continue;
    along = row_sum<L>(along, s_sum) / n;
    if (!on) continue;
    T *dx = static_cast<T *>(a.y) + r * a.ld_y;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; j++) o[j] = rstd * (g[i][j] - h[i][j] * along) + e[i][j];
      if (p.any(i)) store_pack<T, V>(dx + p.at(i), o);
    }
  }
  if (!a.part) return;
  // one partial row a workgroup: first over the groups of a wave, then over the waves
  float *out = a.part + (int64_t)blockIdx.x * a.cols;
  if constexpr (L > kWave) {
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++)
        if (p.any(i) && p.live(i, j)) out[p.at(i) + j] = dw[i][j];
  } else {
    constexpr int W = kHeadThreads / kWave, N = NV * V * L;    // columns that a group's lanes stand for
    __shared__ float s_part[W][N];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) {
        float t = dw[i][j];
#pragma unroll
        for (int o = L; o < kWave; o <<= 1) t += __shfl_xor(t, o, kWave);
        if (lane_id() < L && p.any(i) && p.live(i, j)) s_part[threadIdx.x / kWave][p.at(i) + j] = t;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += kHeadThreads) {
      float t = 0.f;
#pragma unroll
      for (int v = 0; v < W; v++) t += s_part[v][c];
      out[c] = t;
    }
  }
}

__global__ __launch_bounds__(1024) void k_rms_params(const float *part, int n_part, int cols, int param_type, void *dweight) {
  sum_partial_rows(part, n_part, cols, cols, param_type, dweight);
}

// Threads of a row of n_vec vectors: the smallest group that holds it with at most 4 vectors each.
static int rms_lanes(int n_vec) {
  int l = 4;
  while (l < kWave && n_vec > 4 * l) l *= 2;
  return n_vec <= 4 * l ? l : n_vec <= 4 * kMidThreads ? kMidThreads : kWideThreads;
}

// workgroups: enough rows to fill the card, and in the gradient so few that a partial row stands for several rows
static int64_t rms_blocks(int64_t rows, int lanes, bool grad) {
  const int64_t per = lanes > kWave ? 1 : kHeadThreads / lanes;
  const int64_t want = (rows + per - 1) / per;
  const int64_t most = lanes == kWideThreads ? 512 : grad ? 1024 : 2048;
  return std::max<int64_t>(1, std::min(want, most));
}

template <class T, int L, int NV, int V, bool FULL> static void rms_launch(const RmsArgs &a, bool grad, Launches &run) {
  const dim3 grid((unsigned)rms_blocks(a.rows, L, grad)), block(norm_threads<L>());
  if (grad) run(k_rms_norm_grad<T, L, NV, V, FULL>, grid, block, a);
  else run(a.scale ? k_rms_norm<T, L, NV, V, FULL, true> : k_rms_norm<T, L, NV, V, FULL, false>, grid, block, a);
}

template <class T, int L, int V> static void rms_vectors(const RmsArgs &a, int nv, bool grad, Launches &run) {
  if constexpr (L <= kWave)
    if (nv == 4 && a.cols == L * 4 * V) return rms_launch<T, L, 4, V, true>(a, grad, run);
  if constexpr (L == 4)
    if (nv == 1) return rms_launch<T, L, 1, V, false>(a, grad, run);
  if constexpr (L == 4 || L > kWave)
    if (nv <= 2) return rms_launch<T, L, 2, V, false>(a, grad, run);
  if constexpr (L != kWideThreads || INK_MAX_IN_DIM > 2 * V * L) {         // (16-bit rows of 1024 threads have two vectors each at most)
    if (nv <= 3) return rms_launch<T, L, 3, V, false>(a, grad, run);
    rms_launch<T, L, 4, V, false>(a, grad, run);
  }
}

template <class T> static void rms_dispatch(const RmsArgs &a, bool grad, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  if (a.cols < V) return rms_launch<T, 8, 1, 1, false>(a, grad, run);
  const int n_vec = (a.cols + V - 1) / V, l = rms_lanes(n_vec), nv = (n_vec + l - 1) / l;
  switch (l) {
    case 4: return rms_vectors<T, 4, V>(a, nv, grad, run);
    case 8: return rms_vectors<T, 8, V>(a, nv, grad, run);
    case 16: return rms_vectors<T, 16, V>(a, nv, grad, run);
    case 32: return rms_vectors<T, 32, V>(a, nv, grad, run);
    case 64: return rms_vectors<T, 64, V>(a, nv, grad, run);
    case kMidThreads: return rms_vectors<T, kMidThreads, V>(a, nv, grad, run);
    default: return rms_vectors<T, kWideThreads, V>(a, nv, grad, run);
  }
}

static int64_t rms_grad_blocks(int64_t rows, int cols, int type) {
  const int V = 16 / type_size(type);
  return rms_blocks(rows, cols < V ? 8 : rms_lanes((cols + V - 1) / V), true);
}

static void rms_run(const RmsArgs &a, int type, bool grad, Launches &run) {
  if (type == INK_F32) rms_dispatch<float>(a, grad, run);
  else if (type == INK_BF16) rms_dispatch<bf16>(a, grad, run);
  else rms_dispatch<f16>(a, grad, run);
}

// what both calls check alike
static const char *rms_check(int64_t rows, int32_t cols, int32_t type, int32_t param_type, const void *weight, const void *other) {
  if (!known_type(type)) return "unknown type";
  if (param_type != type && param_type != INK_F32) return "param_type must be the rows' type or INK_F32";
  if (rows < 0 || rows > kMaxHeadRows) return "rows out of range";
  if (cols < 1 || cols > INK_MAX_IN_DIM) return "cols must be 1 .. INK_MAX_IN_DIM";
  if (!aligned_to(weight, type_size(param_type)) || !aligned_to(other, type_size(param_type))) return "a parameter is not aligned to its type";
  return nullptr;
}

}  // namespace ink

using namespace ink;

extern "C" ink_status ink_rms_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_res, const void *weight, int64_t rows,
                                   int32_t cols, int32_t type, int32_t param_type, float eps, int32_t out_type, void *y, int64_t ld_y,
                                   float *scale, void *total, int64_t ld_total, float *rstd, void *hip_stream) {
  const char *who = "ink_rms_norm";
  if (const char *why = rms_check(rows, cols, type, param_type, weight, nullptr)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (!(eps > 0.f) || eps > 3e38f) return fail_call(INK_E_ARG, "%s: eps must be positive and finite", who);
  if (out_type != type && out_type != INK_E4M3) return fail_call(INK_E_ARG, "%s: out_type must be the rows' type or INK_E4M3", who);
  if (!good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "%s: x is NULL, not aligned to its type or has rows that overlap", who);
  if (residual && !good_matrix(residual, rows, cols, ld_res, type, false)) return fail_call(INK_E_ARG, "%s: residual is not aligned to its type or has rows that overlap", who);
  if (residual && !good_matrix(total, rows, cols, ld_total, type, true)) return fail_call(INK_E_ARG, "%s: total is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(y, rows, cols, ld_y, out_type, true)) return fail_call(INK_E_ARG, "%s: y is NULL, not aligned to its type or has rows that overlap", who);
  if (!aligned_to(rstd, 4)) return fail_call(INK_E_ARG, "%s: rstd is not aligned", who);
  if (out_type == INK_E4M3 && rows > 0 && (!scale || !aligned_to(scale, 4))) return fail_call(INK_E_ARG, "%s: scale is NULL or not aligned", who);
  if (rows == 0) return INK_OK;
  RmsArgs a{};
  a.x = x; a.res = residual; a.weight = weight; a.y = y; a.total = total; a.rstd = rstd; a.scale = out_type == INK_E4M3 ? scale : nullptr;
  a.rows = rows; a.cols = cols; a.ld_x = ld_x; a.ld_res = ld_res; a.ld_y = ld_y; a.ld_total = ld_total; a.param_type = param_type; a.eps = eps;
  Launches run(hip_stream);
  rms_run(a, type, false, run);
  return run.done(who);
}

extern "C" size_t ink_rms_norm_backward_work(int64_t rows, int32_t cols, int32_t type) {
  if (!known_type(type) || rows < 1 || rows > kMaxHeadRows || cols < 1 || cols > INK_MAX_IN_DIM) return 0;
  return (size_t)rms_grad_blocks(rows, cols, type) * (size_t)cols * sizeof(float);
}

extern "C" ink_status ink_rms_norm_backward(const void *dy, int64_t ld_dy, const void *total, int64_t ld_total, const float *rstd,
                                            const void *weight, const void *d_total, int64_t ld_dt, int64_t rows, int32_t cols, int32_t type,
                                            int32_t param_type, void *dx, int64_t ld_dx, void *dweight, void *work, size_t work_bytes,
                                            void *hip_stream) {
  const char *who = "ink_rms_norm_backward";
  if (const char *why = rms_check(rows, cols, type, param_type, weight, dweight)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (!good_matrix(dy, rows, cols, ld_dy, type, false)) return fail_call(INK_E_ARG, "%s: dy is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(total, rows, cols, ld_total, type, false)) return fail_call(INK_E_ARG, "%s: total is NULL, not aligned to its type or has rows that overlap", who);
  if (d_total && !good_matrix(d_total, rows, cols, ld_dt, type, false)) return fail_call(INK_E_ARG, "%s: d_total is not aligned to its type or has rows that overlap", who);
  if (rows > 0 && (!rstd || !aligned_to(rstd, 4))) return fail_call(INK_E_ARG, "%s: rstd is NULL or not aligned", who);
  if (dx && !good_matrix(dx, rows, cols, ld_dx, type, true)) return fail_call(INK_E_ARG, "%s: dx is not aligned to its type or has rows that overlap", who);
  if (rows > 0 && dweight && (!work || !aligned_to(work, 16) || work_bytes < ink_rms_norm_backward_work(rows, cols, type)))
    return fail_call(INK_E_ARG, "%s: work holds less than ink_rms_norm_backward_work bytes or is not aligned to 16", who);
  Launches run(hip_stream);
  RmsArgs a{};
  a.x = total; a.res = d_total; a.dy = dy; a.weight = weight; a.y = dx; a.rstd = const_cast<float *>(rstd);
  a.part = dweight ? static_cast<float *>(work) : nullptr;
  a.rows = rows; a.cols = cols; a.ld_x = ld_total; a.ld_res = ld_dt; a.ld_dy = ld_dy; a.ld_y = ld_dx; a.param_type = param_type;
  if (rows > 0 && (dx || dweight)) rms_run(a, type, true, run);
  if (dweight)                             // no rows: zeros
    run(k_rms_params, dim3((cols + 31) / 32), dim3(1024), a.part, rows > 0 ? rms_grad_blocks(rows, cols, type) : 0, cols, param_type, dweight);
  return run.done(who);
}
