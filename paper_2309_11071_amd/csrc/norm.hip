// Layer norm of rows and its gradient.
//
//   forward   mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps),  y = (x - mean) rstd weight + bias
//   gradient  h = (x - mean) rstd,  g = dy weight:   dx = rstd (g - mean(g) - h mean(g h)),
//             dweight = sum over rows of dy h,  dbias = sum over rows of dy
//
// Both are bound by memory, eight to eleven operations an element against 4 to 12 bytes, and run at the rate of a copy (5.0 TB/s)
// where a wave holds a row: 2.45M x 256 bf16 forward 504 us, 233k x 602 f32 gradient 332 us, 5 of them for the partial rows' sum.  So a row is read once: L lanes hold it
// in registers, V elements (16 bytes) a load and NV loads a lane, and the variance is taken of the differences from the mean
// without a second read.  L is the smallest group that holds a row with NV <= 4: the fewer lanes a row has, the fewer steps
// its sums take and the more rows a wave has under way.  The last load of a row that is no multiple of V elements starts V
// elements before the row's end, so that no lane loads element by element; what it repeats is left out of the sums and
// written twice with the same value.  Sums and statistics are in 32 bits; y, dx, dweight and dbias are rounded once, at the store.
//
// The weights' gradient is a sum over all rows: a lane keeps those of its columns in registers over all rows that its workgroup
// takes, the workgroup adds up its groups in LDS and leaves one partial row, and k_norm_params adds the partial
// rows in their order.  No atomics: the same call gives the same bits.
//
// Rows that a wave does not hold (f32 from 1025 columns on, 16 bits from 2049) have a workgroup of 1024 threads each, which little more than that
// leaves idle: f32 200k x 1100 takes 2.4 times a copy's time forward and 2.8 in the gradient, 100k x 2048 1.3 and 1.7, 50k x 4096 0.9 and 1.1, 20k x 8192
// 0.9 and 0.9; bf16 100k x 2100 3.0 and 2.7, 50k x 4096 1.6 and 1.5, 20k x 16384 1.0 and 1.0.
#include <algorithm>

#include "rowgroup.h"

namespace ink {

struct NormArgs {
  const void *x, *dy, *weight, *bias;
  void *y;                                 // forward: y, gradient: dx (or NULL)
  float *mean, *rstd;                      // forward: written where not NULL; gradient: read
  float *part;                             // gradient: [workgroups][2][cols], or NULL
  int64_t rows, ld_x, ld_dy, ld_y;
  int cols, param_type;
  float eps;
};

template <class T, int L, int NV, int V, bool FULL>
__global__ __launch_bounds__(norm_threads<L>()) void k_layer_norm(NormArgs a) {
  constexpr int G = norm_threads<L>() / L;
  __shared__ float s_sum[L > kWave ? L / kWave : 1];
  const NormPlace<L, V, FULL> p(a.cols);
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int j = 0; j < V; j++) {
      w[i][j] = a.weight ? load_any(a.weight, p.at(i) + j, a.param_type) : 1.f;
      b[i][j] = a.bias ? load_any(a.bias, p.at(i) + j, a.param_type) : 0.f;
    }
  const float n = (float)a.cols;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += (int64_t)gridDim.x * G) {
    const int64_t mine = r0 + threadIdx.x / L;
    const int64_t r = mine < a.rows ? mine : a.rows - 1;      // a group without a row repeats the last one and stores nothing
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x;
    float v[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) load_pack<T, V>(x + p.at(i), v[i]);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) sum += p.live(i, j) ? v[i][j] : 0.f;
    const float mean = row_sum<L>(sum, s_sum) / n;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) {
        v[i][j] -= mean;
        sum += p.live(i, j) ? v[i][j] * v[i][j] : 0.f;
      }
    const float rstd = 1.f / sqrtf(row_sum<L>(sum, s_sum) / n + a.eps);
    if (mine >= a.rows) continue;
    T *y = static_cast<T *>(a.y) + r * a.ld_y;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; j++) o[j] = v[i][j] * rstd * w[i][j] + b[i][j];
      if (p.any(i)) store_pack<T, V>(y + p.at(i), o);
    }
    if (p.q == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

template <class T, int L, int NV, int V, bool FULL>
__global__ __launch_bounds__(norm_threads<L>()) void k_layer_norm_grad(NormArgs a) {
  constexpr int G = norm_threads<L>() / L;
  __shared__ float s_sum[L > kWave ? L / kWave : 1];
  const NormPlace<L, V, FULL> p(a.cols);
  float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int j = 0; j < V; j++) {
      w[i][j] = a.weight ? load_any(a.weight, p.at(i) + j, a.param_type) : 1.f;
      dw[i][j] = db[i][j] = 0.f;
    }
  const float n = (float)a.cols;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += (int64_t)gridDim.x * G) {
    const int64_t mine = r0 + threadIdx.x / L;
    const bool on = mine < a.rows;
    const int64_t r = on ? mine : a.rows - 1;
    const T *x = static_cast<const T *>(a.x) + r * a.ld_x, *dy = static_cast<const T *>(a.dy) + r * a.ld_dy;
    float h[NV][V], g[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) { load_pack<T, V>(x + p.at(i), h[i]); load_pack<T, V>(dy + p.at(i), g[i]); }
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sg = 0.f, sgh = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) {
        h[i][j] = (h[i][j] - mean) * rstd;
        dw[i][j] += on ? g[i][j] * h[i][j] : 0.f;             // a repeated element's sums are dropped at the end
        db[i][j] += on ? g[i][j] : 0.f;
        g[i][j] *= w[i][j];
        sg += p.live(i, j) ? g[i][j] : 0.f;
        sgh += p.live(i, j) ? g[i][j] * h[i][j] : 0.f;
      }
    if (!a.y) continue;
    sg = row_sum<L>(sg, s_sum) / n;
    sgh = row_sum<L>(sgh, s_sum) / n;
    if (!on) continue;
    T *dx = static_cast<T *>(a.y) + r * a.ld_y;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      float o[V];
#pragma unroll
      for (int j = 0; j < V; j++) o[j] = rstd * (g[i][j] - sg - h[i][j] * sgh);
      if (p.any(i)) store_pack<T, V>(dx + p.at(i), o);
    }
  }
  if (!a.part) return;
  // one partial row a workgroup: first over the groups of a wave, then over the waves
  float *out = a.part + (int64_t)blockIdx.x * 2 * a.cols;
  if constexpr (L > kWave) {
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++)
        if (p.any(i) && p.live(i, j)) { out[p.at(i) + j] = dw[i][j]; out[a.cols + p.at(i) + j] = db[i][j]; }
  } else {
    constexpr int W = kHeadThreads / kWave, N = NV * V * L;    // columns that a group's lanes stand for
    __shared__ float s_part[W][N];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) {
          float t = k ? db[i][j] : dw[i][j];
#pragma unroll
          for (int o = L; o < kWave; o <<= 1) t += __shfl_xor(t, o, kWave);
          if (lane_id() < L && p.any(i) && p.live(i, j)) s_part[threadIdx.x / kWave][p.at(i) + j] = t;
        }
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += kHeadThreads) {
        float t = 0.f;
#pragma unroll
        for (int v = 0; v < W; v++) t += s_part[v][c];
        out[k * a.cols + c] = t;
      }
    }
  }
}

// Partial rows to the gradients of weight and bias: 32 columns a workgroup, 32 threads a column.
__global__ __launch_bounds__(1024) void k_norm_params(const float *part, int n_part, int cols, int param_type, void *dweight, void *dbias) {
  void *out = blockIdx.y ? dbias : dweight;
  if (out) sum_partial_rows(part + blockIdx.y * cols, n_part, 2 * (int64_t)cols, cols, param_type, out);
}

// Lanes and loads of a row of n_vec vectors: the smallest group that holds it with at most 4 vectors a lane.
static int norm_lanes(int n_vec) {
  int l = 4;
  while (l < kWave && n_vec > 4 * l) l *= 2;
  return n_vec > 4 * l ? kWideThreads : l;
}

// workgroups: enough rows to fill the card, and in the gradient so few that a partial row stands for several rows
static int64_t norm_blocks(int64_t rows, int lanes, bool grad) {
  const int64_t per = lanes > kWave ? 1 : kHeadThreads / lanes;
  const int64_t want = (rows + per - 1) / per;
  const int64_t most = lanes > kWave ? 512 : grad ? 1024 : 2048;
  return std::max<int64_t>(1, std::min(want, most));
}

template <class T, int L, int NV, int V, bool FULL> static void norm_launch(const NormArgs &a, bool grad, Launches &run) {
  const dim3 grid((unsigned)norm_blocks(a.rows, L, grad)), block(norm_threads<L>());
  run(grad ? k_layer_norm_grad<T, L, NV, V, FULL> : k_layer_norm<T, L, NV, V, FULL>, grid, block, a);
}

template <class T, int L, int V> static void norm_vectors(const NormArgs &a, int nv, bool grad, Launches &run) {
  if constexpr (L != kWideThreads)
    if (nv == 4 && a.cols == L * 4 * V) return norm_launch<T, L, 4, V, true>(a, grad, run);
  if constexpr (L == 4 || L == kWideThreads) {
    if (nv == 1) return norm_launch<T, L, 1, V, false>(a, grad, run);
    if (nv == 2) return norm_launch<T, L, 2, V, false>(a, grad, run);
  }
  if constexpr (L != kWideThreads || INK_MAX_IN_DIM > 2 * V * L) {         // (16-bit rows of a workgroup have two vectors a thread at most)
    if (nv <= 3) return norm_launch<T, L, 3, V, false>(a, grad, run);
    norm_launch<T, L, 4, V, false>(a, grad, run);
  }
}

template <class T> static void norm_dispatch(const NormArgs &a, bool grad, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  if (a.cols < V) return norm_launch<T, 8, 1, 1, false>(a, grad, run);
  const int n_vec = (a.cols + V - 1) / V, l = norm_lanes(n_vec), nv = (n_vec + l - 1) / l;
  switch (l) {
    case 4: return norm_vectors<T, 4, V>(a, nv, grad, run);
    case 8: return norm_vectors<T, 8, V>(a, nv, grad, run);
    case 16: return norm_vectors<T, 16, V>(a, nv, grad, run);
    case 32: return norm_vectors<T, 32, V>(a, nv, grad, run);
    case 64: return norm_vectors<T, 64, V>(a, nv, grad, run);
    default: return norm_vectors<T, kWideThreads, V>(a, nv, grad, run);
  }
}

static int64_t norm_grad_blocks(int64_t rows, int cols, int type) {
  const int V = 16 / type_size(type);
  return norm_blocks(rows, cols < V ? 8 : norm_lanes((cols + V - 1) / V), true);
}

static void norm_run(const NormArgs &a, int type, bool grad, Launches &run) {
  if (type == INK_F32) norm_dispatch<float>(a, grad, run);
  else if (type == INK_BF16) norm_dispatch<bf16>(a, grad, run);
  else norm_dispatch<f16>(a, grad, run);
}

// what both calls check alike
static const char *norm_check(int64_t rows, int32_t cols, int32_t type, int32_t param_type, const void *weight, const void *other) {
  if (!known_type(type)) return "unknown type";
  if (param_type != type && param_type != INK_F32) return "param_type must be the rows' type or INK_F32";
  if (rows < 0 || rows > kMaxHeadRows) return "rows out of range";
  if (cols < 1 || cols > INK_MAX_IN_DIM) return "cols must be 1 .. INK_MAX_IN_DIM";
  if (!aligned_to(weight, type_size(param_type)) || !aligned_to(other, type_size(param_type))) return "a parameter is not aligned to its type";
  return nullptr;
}

}  // namespace ink

using namespace ink;

extern "C" ink_status ink_layer_norm(const void *x, int64_t ld_x, const void *weight, const void *bias, int64_t rows, int32_t cols,
                                     int32_t type, int32_t param_type, float eps, void *y, int64_t ld_y, float *mean, float *rstd,
                                     void *hip_stream) {
  if (const char *why = norm_check(rows, cols, type, param_type, weight, bias)) return fail_call(INK_E_ARG, "ink_layer_norm: %s", why);
  if (!(eps > 0.f) || eps > 3e38f) return fail_call(INK_E_ARG, "ink_layer_norm: eps must be positive and finite");
  if (!good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "ink_layer_norm: x is NULL, not aligned to its type or has rows that overlap");
  if (!good_matrix(y, rows, cols, ld_y, type, true)) return fail_call(INK_E_ARG, "ink_layer_norm: y is NULL, not aligned to its type or has rows that overlap");
  if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return fail_call(INK_E_ARG, "ink_layer_norm: mean or rstd is not aligned");
  if (rows == 0) return INK_OK;
  NormArgs a{};
  a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd;
  a.rows = rows; a.cols = cols; a.ld_x = ld_x; a.ld_y = ld_y; a.param_type = param_type; a.eps = eps;
  Launches run(hip_stream);
  norm_run(a, type, false, run);
  return run.done("ink_layer_norm");
}

extern "C" size_t ink_layer_norm_backward_work(int64_t rows, int32_t cols, int32_t type) {
  if (!known_type(type) || rows < 1 || rows > kMaxHeadRows || cols < 1 || cols > INK_MAX_IN_DIM) return 0;
  return (size_t)norm_grad_blocks(rows, cols, type) * 2 * (size_t)cols * sizeof(float);
}

extern "C" ink_status ink_layer_norm_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const float *mean,
                                              const float *rstd, const void *weight, int64_t rows, int32_t cols, int32_t type,
                                              int32_t param_type, void *dx, int64_t ld_dx, void *dweight, void *dbias, void *work,
                                              size_t work_bytes, void *hip_stream) {
  const char *who = "ink_layer_norm_backward";
  if (const char *why = norm_check(rows, cols, type, param_type, weight, dweight)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (!aligned_to(dbias, type_size(param_type))) return fail_call(INK_E_ARG, "%s: dbias is not aligned to its type", who);
  if (!good_matrix(dy, rows, cols, ld_dy, type, false)) return fail_call(INK_E_ARG, "%s: dy is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "%s: x is NULL, not aligned to its type or has rows that overlap", who);
  if (rows > 0 && (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4))) return fail_call(INK_E_ARG, "%s: mean or rstd is NULL or not aligned", who);
  if (dx && !good_matrix(dx, rows, cols, ld_dx, type, true)) return fail_call(INK_E_ARG, "%s: dx is not aligned to its type or has rows that overlap", who);
  const bool params = dweight || dbias;
  if (rows > 0 && params && (!work || !aligned_to(work, 4) || work_bytes < ink_layer_norm_backward_work(rows, cols, type)))
    return fail_call(INK_E_ARG, "%s: work holds less than ink_layer_norm_backward_work bytes", who);
  Launches run(hip_stream);
  NormArgs a{};
  a.x = x; a.dy = dy; a.weight = weight; a.y = dx; a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
  a.part = params ? static_cast<float *>(work) : nullptr;
  a.rows = rows; a.cols = cols; a.ld_x = ld_x; a.ld_dy = ld_dy; a.ld_y = ld_dx; a.param_type = param_type;
  if (rows > 0 && (dx || params)) norm_run(a, type, true, run);
  if (params)                              // no rows: zeros
    run(k_norm_params, dim3((cols + 31) / 32, 2), dim3(1024), a.part, rows > 0 ? norm_grad_blocks(rows, cols, type) : 0, cols,
        param_type, dweight, dbias);
  return run.done(who);
}
