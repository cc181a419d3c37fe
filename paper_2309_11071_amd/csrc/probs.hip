// Log probabilities of given classes, entropy and the best alternatives of rows of logits, and the gradient.
//
//   z = scale * logit,  m = max z,  S = sum e^(z - m),  U = sum (z - m) e^(z - m)
//   lse = m + log S,  log p_t = z_t - lse,  entropy = -sum p log p = log S - U / S
//   gradient of g log p_t + h entropy:  scale (g ([c = t] - p_c) - h p_c (log p_c + entropy))
//
// The alternatives are the classes of the largest logits, compared as they stand in memory: equal ones by the lower class, NaN
// before everything, -0 equal to +0.  A class at -inf is masked (p = 0); a row of masked classes has lse = log p = -inf, entropy
// and gradient 0.  Sums and statistics are in 32 bits.
//
// Bound by memory: a row is read once.  Short rows (k_probs_rows): L lanes hold a row in registers, in at most 4 loads a lane; the
// maximum comes first and the sums after it, from the registers.  Long rows (k_probs_long): a workgroup, or several for parts
// of a row where there are few rows, runs over the row with a running maximum that the sums follow; k_probs_join
// puts the parts together.  The alternatives are kept as a sorted list a lane: an element goes through the list by
// one comparison a place, and at the end the group takes the best head of all lists, once per alternative.
#include <algorithm>

#include "head.h"

namespace ink {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ProbsArgs {
  const void *logits;
  const void *targets;                      // int32 or int64, or NULL
  float *logp, *entropy, *lse, *top_logp;   // each may be NULL
  int32_t *top_ids;
  float *part_stats;                        // long rows in parts: [rows][parts][3]: m, S, U
  uint32_t *part_ord;                       // [rows][parts][top]
  int32_t *part_id;
  int64_t rows, ld, classes, part_len;
  int parts, top, wide_targets;
  float scale;
};

__device__ __forceinline__ int64_t target_of(const void *targets, int wide, int64_t r) {
  if (!targets) return -1;
  return wide ? static_cast<const int64_t *>(targets)[r] : (int64_t)static_cast<const int32_t *>(targets)[r];
}

// Order of logits as unsigned numbers: larger logits have larger ones, all NaN the largest, -0 that of +0; 0 stands for nothing.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);              // -0 + 0 = +0
  const uint32_t o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return v != v ? 0xffffffffu : o;
}
__device__ __forceinline__ float of_order(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);      // all ones: a NaN
}

// A list of the K best elements of a lane, best first.
//   f32            order and class apart
//   bf16 and f16   one number: the 16 bits of the order above 65535 - index, the index being the class (short rows) or the place
//                  among the lane's elements (long rows), so that a place of the list costs two instructions instead of five
template <class T, int K> struct Best {
  uint32_t o[K > 0 ? K : 1];
  int32_t id[K > 0 ? K : 1];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < K; k++) { o[k] = 0; id[k] = 0x7fffffff; }
  }
  __device__ __forceinline__ void put(uint32_t x, int32_t i) {         // classes come in ascending order
    bool up = false;                       // from its place on everything moves down: equal ones keep their order
#pragma unroll
    for (int k = 0; k < K; k++) {
      up |= x > o[k];
      const uint32_t a = up ? x : o[k]; const int32_t b = up ? i : id[k];
      x = up ? o[k] : x; i = up ? id[k] : i;
      o[k] = a; id[k] = b;
    }
  }
  __device__ __forceinline__ void pop(bool mine) {
#pragma unroll
    for (int k = 0; k + 1 < K; k++) { o[k] = mine ? o[k + 1] : o[k]; id[k] = mine ? id[k + 1] : id[k]; }
    o[K - 1] = mine ? 0 : o[K - 1]; id[K - 1] = mine ? 0x7fffffff : id[K - 1];
  }
};

// The 16 bits of a bf16 or f16 in the same order.
template <class T> __device__ __forceinline__ uint32_t order16(T v) {
  const uint32_t u = __builtin_bit_cast(uint16_t, v);
  constexpr uint32_t inf = __is_same(T, bf16) ? 0x7f80u : 0x7c00u;
  uint32_t o = u & 0x8000u ? u ^ 0xffffu : u | 0x8000u;
  o = u == 0x8000u ? 0x8000u : o;
  return (u & 0x7fffu) > inf ? 0xffffu : o;
}
template <class T> __device__ __forceinline__ float of_order16(uint32_t o) {
  const uint16_t u = (uint16_t)(o & 0x8000u ? o ^ 0x8000u : o ^ 0xffffu);
  return (float)__builtin_bit_cast(T, u);
}

// Best of a group's heads, taken off its list: every lane gets it.
template <int L, int K> __device__ __forceinline__ void take_best(Best<float, K> &b, uint32_t &o, int32_t &id) {
  o = group_all<L>(b.o[0], [](uint32_t x, uint32_t y) { return x > y ? x : y; });
  const int32_t c = b.o[0] == o ? b.id[0] : 0x7fffffff;
  id = group_all<L>(c, [](int32_t x, int32_t y) { return x < y ? x : y; });
  b.pop(c == id && b.o[0] == o);
}

struct RowStats { float m, s, u; };
__device__ __forceinline__ float safe_max(float m) { return m == -__builtin_inff() ? 0.f : m; }

// e^(z - m) and its product with z - m; a masked class (z = -inf) adds nothing to either
__device__ __forceinline__ void add_term(float z, float m, float &s, float &u) {
  const float t = z - m, e = __builtin_amdgcn_exp2f(t * kLog2e);
  s += e;
  u = fmaf(fmaxf(t, -1e30f), e, u);
}
// sums over `from` relative to the maximum `to`
__device__ __forceinline__ void rescale(RowStats &a, float to) {
  const float d = safe_max(a.m) - to, f = a.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(d * kLog2e);
  a.u = f == 0.f ? 0.f : (a.u + a.s * d) * f;
  a.s *= f;
  a.m = to;
}

// what a row's statistics say, written by one lane
__device__ __forceinline__ float finish_row(const ProbsArgs &a, int64_t r, float m, float s, float u, float z_target, bool has) {
  const bool none = s == 0.f;
  const float ls = logf(s), lse = none ? -__builtin_inff() : m + ls;
  if (a.lse) a.lse[r] = lse;
  if (a.entropy) a.entropy[r] = none ? 0.f : ls - u / s;
  if (a.logp) a.logp[r] = !has ? 0.f : none ? -__builtin_inff() : z_target - lse;
  return lse;
}
__device__ __forceinline__ void write_top(const ProbsArgs &a, int64_t r, int j, float v, int32_t id, float lse) {
  const float z = v * a.scale;
  if (a.top_ids) a.top_ids[r * a.top + j] = id;
  if (a.top_logp) a.top_logp[r * a.top + j] = lse == -__builtin_inff() ? lse : z - lse;
}

// ------------------------------------------------------------------------------------ short rows
template <class T, int L, int NV, int V, int K>
__global__ __launch_bounds__(kHeadThreads) void k_probs_rows(ProbsArgs a) {
  constexpr int G = kHeadThreads / L;
  constexpr bool PACKED = sizeof(T) == 2;
  const int q = threadIdx.x % L, C = (int)a.classes;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += (int64_t)gridDim.x * G) {
    const int64_t mine = r0 + threadIdx.x / L;
    const int64_t r = mine < a.rows ? mine : a.rows - 1;
    const T *x = static_cast<const T *>(a.logits) + r * a.ld;
    typename Pack<T, V>::type raw[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) raw[i] = *reinterpret_cast<const typename Pack<T, V>::type *>(x + min((i * L + q) * V, C - V));
    const int64_t t = target_of(a.targets, a.wide_targets, r);
    const bool has = t >= 0 && t < C;
    const float zt = has ? (float)x[t] * a.scale : 0.f;
    float z[NV][V];
    float m = -__builtin_inff();
    Best<T, PACKED ? 0 : K> best;                          // f32
    uint32_t packed[PACKED && K > 0 ? K : 1];
    best.clear();
    if constexpr (PACKED)
#pragma unroll
      for (int k = 0; k < K; k++) packed[k] = 0;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int first = (i * L + q) * V, at = min(first, C - V);
#pragma unroll
      for (int j = 0; j < V; j++) {
        T e;
        if constexpr (V == 1) e = raw[i]; else e = raw[i][j];
        const bool live = at + j >= first;                 // the rest is a repetition of the vector before
        z[i][j] = live ? (float)e * a.scale : -__builtin_inff();
        m = fmaxf(m, z[i][j]);
        if constexpr (K > 0) {
          if constexpr (PACKED) {
            uint32_t key = live ? order16<T>(e) << 16 | (uint32_t)(0xffff - (at + j)) : 0u;
#pragma unroll
            for (int k = 0; k < K; k++) { const uint32_t hi = max(packed[k], key); key = min(packed[k], key); packed[k] = hi; }
          } else best.put(live ? order_of((float)e) : 0u, at + j);
        }
      }
    }
    m = group_all<L>(m, [](float p, float p2) { return fmaxf(p, p2); });
    const float ms = safe_max(m);
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) add_term(z[i][j], ms, s, u);
    s = group_sum<L>(s);
    u = group_sum<L>(u);
    const bool on = mine < a.rows;
    float lse = 0.f;
    if (on && q == 0) lse = finish_row(a, r, ms, s, u, zt, has);
    else lse = s == 0.f ? -__builtin_inff() : ms + logf(s);
    if constexpr (K > 0) {
#pragma unroll
      for (int k = 0; k < K; k++) {
        uint32_t o; int32_t id; float v;
        if constexpr (PACKED) {
          o = group_all<L>(packed[0], [](uint32_t p, uint32_t p2) { return p > p2 ? p : p2; });
          const bool me = packed[0] == o;
#pragma unroll
          for (int i = 0; i + 1 < K; i++) packed[i] = me ? packed[i + 1] : packed[i];
          packed[K - 1] = me ? 0 : packed[K - 1];
          id = 0xffff - (int32_t)(o & 0xffffu);
          v = of_order16<T>(o >> 16);
        } else {
          take_best<L, K>(best, o, id);
          v = of_order(o);
        }
        if (on && q == k % L && k < a.top) write_top(a, r, k, v, id, lse);
      }
    }
  }
}

// ------------------------------------------------------------------------------------ long rows
// the K best of a workgroup's lists to s_o / s_id, best first; all threads call it
template <int K> __device__ __forceinline__ void block_best(Best<float, K> &b, uint32_t *s_o, int32_t *s_id) {
  constexpr int W = kHeadThreads / kWave;
  const int w = threadIdx.x / kWave, l = lane_id();
#pragma unroll
  for (int k = 0; k < K; k++) {
    uint32_t o; int32_t id;
    take_best<kWave, K>(b, o, id);
    if (l == 0) { s_o[w * K + k] = o; s_id[w * K + k] = id; }
  }
  __syncthreads();
  if (w == 0) {
    Best<float, K> c;
    c.clear();
    if (l < W)
#pragma unroll
      for (int k = 0; k < K; k++) { c.o[k] = s_o[l * K + k]; c.id[k] = s_id[l * K + k]; }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < K; k++) {
      uint32_t o; int32_t id;
      take_best<kWave, K>(c, o, id);
      if (l == 0) { s_o[W * K + k] = o; s_id[W * K + k] = id; }
    }
  }
  __syncthreads();
}

template <class T, int V, int K>
__global__ __launch_bounds__(kHeadThreads) void k_probs_long(ProbsArgs a) {
  constexpr int W = kHeadThreads / kWave, KS = K > 0 ? K : 1;
  constexpr bool PACKED = sizeof(T) == 2;
  __shared__ float s_m[W], s_s[W], s_u[W];
  __shared__ uint32_t s_o[(W + 1) * KS];
  __shared__ int32_t s_id[(W + 1) * KS];
  const int64_t r = blockIdx.x / (unsigned)a.parts;
  const int part = (int)(blockIdx.x % (unsigned)a.parts);
  const int64_t c0 = part * a.part_len, c1 = min(c0 + a.part_len, a.classes);    // part_len is a multiple of V
  const T *x = static_cast<const T *>(a.logits) + r * a.ld;
  RowStats st = {-__builtin_inff(), 0.f, 0.f};
  Best<float, K> best;
  best.clear();
  uint32_t packed[KS];
#pragma unroll
  for (int k = 0; k < KS; k++) packed[k] = 0;
  uint32_t floor_o = 0;                    // K elements of the wave are at least this large
  int64_t refresh = 1;
  int step = 0;
  const int64_t n_vec = (c1 - c0 + V - 1) / V;
  for (int64_t i0 = 0; i0 < n_vec; i0 += kHeadThreads, step++) {
    const int64_t i = i0 + threadIdx.x;
    const int64_t first = c0 + i * V;
    const int64_t at = min(first, a.classes - V);
    const typename Pack<T, V>::type raw = *reinterpret_cast<const typename Pack<T, V>::type *>(x + at);
    float z[V];
    uint32_t o[V];
    float vm = -__builtin_inff();
    uint32_t vo = 0;
#pragma unroll
    for (int j = 0; j < V; j++) {
      const bool live = at + j >= first && first < c1;
      z[j] = live ? (float)raw[j] * a.scale : -__builtin_inff();
      vm = fmaxf(vm, z[j]);
      if constexpr (K > 0) {
        if constexpr (PACKED) o[j] = live ? order16<T>(raw[j]) : 0u;
        else o[j] = live ? order_of((float)raw[j]) : 0u;
        vo = max(vo, o[j]);
      }
    }
    if (vm > st.m) rescale(st, vm);
    const float ms = safe_max(st.m);
#pragma unroll
    for (int j = 0; j < V; j++) add_term(z[j], ms, st.s, st.u);
    if constexpr (K > 0) {
      const uint32_t last = PACKED ? packed[KS - 1] >> 16 : best.o[KS - 1];
      if (__any(vo > last && vo >= floor_o)) {
#pragma unroll
        for (int j = 0; j < V; j++) {
          if (!__any(o[j] > (PACKED ? packed[KS - 1] >> 16 : best.o[KS - 1]) && o[j] >= floor_o)) continue;
          if constexpr (PACKED) {
            uint32_t key = o[j] ? o[j] << 16 | (uint32_t)(0xffff - (step * V + j)) : 0u;
#pragma unroll
            for (int k = 0; k < K; k++) { const uint32_t hi = max(packed[k], key); key = min(packed[k], key); packed[k] = hi; }
          } else best.put(o[j], (int32_t)(at + j));
        }
      }
      if (step + 1 == refresh) {           // at steps 1, 2, 4, ...: the K-th best of the lanes' best
        refresh *= 2;
        uint32_t head = PACKED ? packed[0] >> 16 : best.o[0];
#pragma unroll
        for (int k = 0; k < K; k++) {
          floor_o = group_all<kWave>(head, [](uint32_t p, uint32_t p2) { return p > p2 ? p : p2; });
          const uint64_t who = __ballot(head == floor_o);
          head = lane_id() == __ffsll((unsigned long long)who) - 1 ? 0u : head;
        }
      }
    }
  }
  // the workgroup's sums
  const float m = group_all<kWave>(st.m, [](float p, float p2) { return fmaxf(p, p2); });
  if (lane_id() == 0) s_m[threadIdx.x / kWave] = m;
  __syncthreads();
  float bm = s_m[0];
#pragma unroll
  for (int w = 1; w < W; w++) bm = fmaxf(bm, s_m[w]);
  rescale(st, safe_max(bm));
  st.s = group_sum<kWave>(st.s);
  st.u = group_sum<kWave>(st.u);
  if (lane_id() == 0) { s_s[threadIdx.x / kWave] = st.s; s_u[threadIdx.x / kWave] = st.u; }
  if constexpr (K > 0) {
    if constexpr (PACKED)                  // from places among the lane's elements to classes
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int e = 0xffff - (int)(packed[k] & 0xffffu);
        const int64_t first = c0 + ((int64_t)(e / V) * kHeadThreads + threadIdx.x) * V;
        best.o[k] = packed[k] ? order_of(of_order16<T>(packed[k] >> 16)) : 0u;
        best.id[k] = packed[k] ? (int32_t)(min(first, a.classes - V) + e % V) : 0x7fffffff;
      }
    block_best<K>(best, s_o, s_id);
  } else __syncthreads();
  float s = 0.f, u = 0.f;
#pragma unroll
  for (int w = 0; w < W; w++) { s += s_s[w]; u += s_u[w]; }
  if (a.parts > 1) {
    const int64_t p = r * a.parts + part;
    if (threadIdx.x == 0) { a.part_stats[3 * p] = bm; a.part_stats[3 * p + 1] = s; a.part_stats[3 * p + 2] = u; }
    if (K > 0 && (int)threadIdx.x < a.top) {
      a.part_ord[p * a.top + threadIdx.x] = s_o[W * KS + threadIdx.x];
      a.part_id[p * a.top + threadIdx.x] = s_id[W * KS + threadIdx.x];
    }
    return;
  }
  const float ms = safe_max(bm);
  const float lse = s == 0.f ? -__builtin_inff() : ms + logf(s);
  if (threadIdx.x == 0) {
    const int64_t t = target_of(a.targets, a.wide_targets, r);
    const bool has = t >= 0 && t < a.classes;
    finish_row(a, r, ms, s, u, has ? (float)x[t] * a.scale : 0.f, has);
  }
  if (K > 0 && (int)threadIdx.x < a.top) write_top(a, r, threadIdx.x, of_order(s_o[W * KS + threadIdx.x]), s_id[W * KS + threadIdx.x], lse);
}

// Parts of a row, at most 64, to the row: one wave a row, a part a lane.
template <class T, int K>
__global__ __launch_bounds__(kWave) void k_probs_join(ProbsArgs a) {
  const int64_t r = blockIdx.x;
  const int l = lane_id();
  const int64_t p = r * a.parts + min(l, a.parts - 1);
  RowStats st = {a.part_stats[3 * p], a.part_stats[3 * p + 1], a.part_stats[3 * p + 2]};
  if (l >= a.parts) st = {-__builtin_inff(), 0.f, 0.f};
  const float m = safe_max(group_all<kWave>(st.m, [](float x, float y) { return fmaxf(x, y); }));
  rescale(st, m);
  const float s = group_sum<kWave>(st.s), u = group_sum<kWave>(st.u);
  const float lse = s == 0.f ? -__builtin_inff() : m + logf(s);
  if (l == 0) {
    const T *x = static_cast<const T *>(a.logits) + r * a.ld;
    const int64_t t = target_of(a.targets, a.wide_targets, r);
    const bool has = t >= 0 && t < a.classes;
    finish_row(a, r, m, s, u, has ? (float)x[t] * a.scale : 0.f, has);
  }
  if constexpr (K > 0) {
    Best<float, K> b;
    b.clear();
    if (l < a.parts)
#pragma unroll
      for (int k = 0; k < K; k++)
        if (k < a.top) { b.o[k] = a.part_ord[p * a.top + k]; b.id[k] = a.part_id[p * a.top + k]; }
    uint32_t my_o = 0; int32_t my_id = 0;
#pragma unroll
    for (int k = 0; k < K; k++) {
      uint32_t o; int32_t id;
      take_best<kWave, K>(b, o, id);
      if (l == k) { my_o = o; my_id = id; }
    }
    if (l < a.top) write_top(a, r, l, of_order(my_o), my_id, lse);
  }
}

// ------------------------------------------------------------------------------------ gradient
struct ProbsGradArgs {
  const void *logits, *targets;
  const float *lse, *entropy, *g_logp, *g_entropy;
  void *out;
  int64_t rows, ld, ld_out, classes, chunks;     // chunks: pieces of a row, one a group of lanes
  int wide_targets;
  float scale;
};

template <class T, int L, int NV, int V>
__global__ __launch_bounds__(kHeadThreads) void k_probs_grad(ProbsGradArgs a) {
  constexpr int G = kHeadThreads / L;
  const int q = threadIdx.x % L;
  const int64_t n = a.rows * a.chunks;
  for (int64_t i0 = (int64_t)blockIdx.x * G + threadIdx.x / L; i0 < n; i0 += (int64_t)gridDim.x * G) {
    int64_t r = i0, c0 = 0;
    if (a.chunks > 1) { r = i0 / a.chunks; c0 = (i0 - r * a.chunks) * (L * NV * V); }
    const T *x = static_cast<const T *>(a.logits) + r * a.ld;
    T *out = static_cast<T *>(a.out) + r * a.ld_out;
    float z[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) load_pack<T, V>(x + min(c0 + (i * L + q) * V, a.classes - V), z[i]);
    const int64_t t = target_of(a.targets, a.wide_targets, r);
    float lse = a.lse[r];
    const bool none = lse == -__builtin_inff();            // every class masked: no gradient
    lse = none ? 0.f : lse;
    const float g = a.g_logp && t >= 0 && t < a.classes && !none ? a.g_logp[r] : 0.f;
    const float h = a.g_entropy && !none ? a.g_entropy[r] : 0.f, ent = a.g_entropy ? a.entropy[r] : 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t first = c0 + (i * L + q) * V, at = min(first, a.classes - V);
      float o[V];
#pragma unroll
      for (int j = 0; j < V; j++) {
        const float lp = z[i][j] * a.scale - lse, p = __builtin_amdgcn_exp2f(lp * kLog2e);
        const float d = p * (-g - h * (fmaxf(lp, -1e30f) + ent)) + (at + j == t ? g : 0.f);
        o[j] = d * a.scale;
      }
      if (first < a.classes) store_pack<T, V>(out + at, o);
    }
  }
}

// ------------------------------------------------------------------------------------ host side
constexpr int kProbsVectors = 4;            // loads a lane, at most, of a short row
static int probs_lanes(int64_t n_vec) {
  int l = 2;
  while (l < kWave && n_vec > kProbsVectors * l) l *= 2;
  return l;
}
static bool probs_long(int64_t classes, int type) {
  const int V = 16 / type_size(type);
  return (classes + V - 1) / V > kProbsVectors * kWave;
}
// Parts of a long row: so many that the launch has about 1024 workgroups, none shorter than four loads a thread.
static int probs_parts(int64_t rows, int64_t classes, int type, int64_t *len) {
  const int64_t V = 16 / type_size(type), n_vec = (classes + V - 1) / V;
  int64_t parts = std::min<int64_t>({kWave, std::max<int64_t>(1, 1024 / rows), (n_vec + 4 * kHeadThreads - 1) / (4 * kHeadThreads)});
  const int64_t most = (int64_t)65536 / V * kHeadThreads;  // places that 16 bits number (see Best)
  const int64_t per = std::min((n_vec + parts - 1) / parts, most);
  parts = (n_vec + per - 1) / per;
  *len = per * V;
  return (int)parts;
}

template <class T, int L, int K> static void probs_rows(const ProbsArgs &a, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  const int64_t n_vec = (a.classes + V - 1) / V, per = kHeadThreads / L;
  const dim3 grid((unsigned)std::min<int64_t>((a.rows + per - 1) / per, 16384));
  if (a.classes < V) { if constexpr (L == 8) run(k_probs_rows<T, 8, 1, 1, K>, grid, dim3(kHeadThreads), a); return; }
  run(n_vec <= 3 * L ? k_probs_rows<T, L, 3, V, K> : k_probs_rows<T, L, 4, V, K>, grid, dim3(kHeadThreads), a);
}

template <class T, int K> static void probs_top(const ProbsArgs &a, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  if (probs_long(a.classes, sizeof(T) == 4 ? INK_F32 : INK_BF16)) {
    run(k_probs_long<T, V, K>, dim3((unsigned)(a.rows * a.parts)), dim3(kHeadThreads), a);
    if (a.parts > 1) run(k_probs_join<T, K>, dim3((unsigned)a.rows), dim3(kWave), a);
    return;
  }
  const int64_t n_vec = (a.classes + V - 1) / V;
  switch (a.classes < V ? 8 : probs_lanes(n_vec)) {
    case 2: return probs_rows<T, 2, K>(a, run);
    case 4: return probs_rows<T, 4, K>(a, run);
    case 8: return probs_rows<T, 8, K>(a, run);
    case 16: return probs_rows<T, 16, K>(a, run);
    case 32: return probs_rows<T, 32, K>(a, run);
    default: return probs_rows<T, 64, K>(a, run);
  }
}

// lists of 1, 3, 5, 8 and 16 places: what is asked for most, and little more than what is asked for
template <class T> static void probs_dispatch(const ProbsArgs &a, Launches &run) {
  if (a.top == 0) return probs_top<T, 0>(a, run);
  if (a.top == 1) return probs_top<T, 1>(a, run);
  if (a.top <= 3) return probs_top<T, 3>(a, run);
  if (a.top <= 5) return probs_top<T, 5>(a, run);
  if (a.top <= 8) return probs_top<T, 8>(a, run);
  probs_top<T, 16>(a, run);
}

template <class T, int L> static void grad_launch(const ProbsGradArgs &a, int nv, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  const int64_t per = kHeadThreads / L, n = a.rows * a.chunks;
  const dim3 grid((unsigned)std::min<int64_t>((n + per - 1) / per, 1 << 20)), block(kHeadThreads);
  if (nv == 1) run(k_probs_grad<T, L, 1, V>, grid, block, a);
  else if (nv == 2) run(k_probs_grad<T, L, 2, V>, grid, block, a);
  else if (nv == 3) run(k_probs_grad<T, L, 3, V>, grid, block, a);
  else run(k_probs_grad<T, L, 4, V>, grid, block, a);
}

template <class T> static void grad_dispatch(ProbsGradArgs a, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  if (a.classes < V) {
    const int64_t per = kHeadThreads / 8;
    return run(k_probs_grad<T, 8, 1, 1>, dim3((unsigned)std::min<int64_t>((a.rows + per - 1) / per, 1 << 20)), dim3(kHeadThreads), a);
  }
  const int64_t n_vec = (a.classes + V - 1) / V;
  int l = 4;
  while (l < kWave && n_vec > 4 * l) l *= 2;
  const int nv = (int)std::min<int64_t>(4, (n_vec + l - 1) / l);
  a.chunks = (n_vec + l * nv - 1) / (l * nv);
  switch (l) {
    case 4: return grad_launch<T, 4>(a, nv, run);
    case 8: return grad_launch<T, 8>(a, nv, run);
    case 16: return grad_launch<T, 16>(a, nv, run);
    case 32: return grad_launch<T, 32>(a, nv, run);
    default: return grad_launch<T, 64>(a, nv, run);
  }
}

static const char *probs_check(const void *targets, int32_t target_bytes, int64_t rows, int64_t classes, int32_t type, float scale) {
  if (!known_type(type)) return "unknown type";
  if (rows < 0 || rows > kMaxHeadRows) return "rows out of range";
  if (classes < 1 || classes > INK_MAX_CLASSES) return "classes must be 1 .. INK_MAX_CLASSES";
  if (!(scale > 0.f) || scale > 3e38f) return "scale must be positive and finite";
  if (targets && target_bytes != 4 && target_bytes != 8) return "target_bytes must be 4 or 8";
  if (targets && !aligned_to(targets, target_bytes)) return "targets are not aligned";
  return nullptr;
}

}  // namespace ink

using namespace ink;

extern "C" size_t ink_log_probs_work(int64_t rows, int64_t classes, int32_t type, int32_t top) {
  if (!known_type(type) || rows < 1 || rows > kMaxHeadRows || classes < 1 || classes > INK_MAX_CLASSES || top < 0 || top > INK_MAX_TOP) return 0;
  if (!probs_long(classes, type)) return 0;
  int64_t len;
  const int parts = probs_parts(rows, classes, type, &len);
  return parts == 1 ? 0 : (size_t)rows * parts * (3 + 2 * (size_t)top) * 4;
}

extern "C" ink_status ink_log_probs(const void *logits, int64_t ld, const void *targets, int32_t target_bytes, int64_t rows,
                                    int64_t classes, int32_t type, float scale, int32_t top, float *logp, float *entropy, float *lse,
                                    int32_t *top_ids, float *top_logp, void *work, size_t work_bytes, void *hip_stream) {
  const char *who = "ink_log_probs";
  if (const char *why = probs_check(targets, target_bytes, rows, classes, type, scale)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (top < 0 || top > INK_MAX_TOP || top > classes) return fail_call(INK_E_ARG, "%s: top must be 0 .. min(classes, INK_MAX_TOP)", who);
  if (!good_matrix(logits, rows, classes, ld, type, false)) return fail_call(INK_E_ARG, "%s: logits is NULL, not aligned to its type or has rows that overlap", who);
  for (const void *p : {(const void *)logp, (const void *)entropy, (const void *)lse, (const void *)top_ids, (const void *)top_logp})
    if (!aligned_to(p, 4)) return fail_call(INK_E_ARG, "%s: an output is not aligned", who);
  if (rows == 0) return INK_OK;
  const size_t need = ink_log_probs_work(rows, classes, type, top);
  if (need && (!work || !aligned_to(work, 4) || work_bytes < need)) return fail_call(INK_E_ARG, "%s: work holds less than ink_log_probs_work bytes", who);
  ProbsArgs a{};
  a.logits = logits; a.targets = targets; a.wide_targets = target_bytes == 8;
  a.logp = logp; a.entropy = entropy; a.lse = lse; a.top_ids = top_ids; a.top_logp = top_logp;
  a.rows = rows; a.ld = ld; a.classes = classes; a.top = top; a.scale = scale; a.parts = 1;
  if (probs_long(classes, type)) {
    a.parts = probs_parts(rows, classes, type, &a.part_len);
    if (rows * a.parts > kMaxHeadRows) return fail_call(INK_E_RANGE, "%s: too many rows of so many classes", who);
    a.part_stats = static_cast<float *>(work);
    a.part_ord = reinterpret_cast<uint32_t *>(a.part_stats + 3 * rows * a.parts);
    a.part_id = reinterpret_cast<int32_t *>(a.part_ord + rows * a.parts * top);
  }
  Launches run(hip_stream);
  if (type == INK_F32) probs_dispatch<float>(a, run);
  else if (type == INK_BF16) probs_dispatch<bf16>(a, run);
  else probs_dispatch<f16>(a, run);
  return run.done(who);
}

extern "C" ink_status ink_log_probs_backward(const void *logits, int64_t ld, const void *targets, int32_t target_bytes,
                                             const float *lse, const float *entropy, const float *g_logp, const float *g_entropy,
                                             int64_t rows, int64_t classes, int32_t type, float scale, void *dlogits, int64_t ld_out,
                                             void *hip_stream) {
  const char *who = "ink_log_probs_backward";
  if (const char *why = probs_check(targets, target_bytes, rows, classes, type, scale)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (!good_matrix(logits, rows, classes, ld, type, false)) return fail_call(INK_E_ARG, "%s: logits is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(dlogits, rows, classes, ld_out, type, true)) return fail_call(INK_E_ARG, "%s: dlogits is NULL, not aligned to its type or has rows that overlap", who);
  if (rows > 0 && !lse) return fail_call(INK_E_ARG, "%s: lse is NULL", who);
  if (g_entropy && !entropy) return fail_call(INK_E_ARG, "%s: g_entropy without entropy", who);
  if (!g_logp && !g_entropy && rows > 0) return fail_call(INK_E_ARG, "%s: neither g_logp nor g_entropy", who);
  for (const void *p : {(const void *)lse, (const void *)entropy, (const void *)g_logp, (const void *)g_entropy})
    if (!aligned_to(p, 4)) return fail_call(INK_E_ARG, "%s: a statistic or a gradient is not aligned", who);
  if (rows == 0) return INK_OK;
  ProbsGradArgs a{};
  a.logits = logits; a.targets = targets; a.wide_targets = target_bytes == 8; a.lse = lse; a.entropy = entropy;
  a.g_logp = g_logp; a.g_entropy = g_entropy; a.out = dlogits;
  a.rows = rows; a.ld = ld; a.ld_out = ld_out; a.classes = classes; a.chunks = 1; a.scale = scale;
  Launches run(hip_stream);
  if (type == INK_F32) grad_dispatch<float>(a, run);
  else if (type == INK_BF16) grad_dispatch<bf16>(a, run);
  else grad_dispatch<f16>(a, run);
  return run.done(who);
}
