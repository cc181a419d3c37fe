// Log probabilities of given classes, entropy and the best alternatives of rows of logits, and the gradient.
//
//   z = scale * logit,  m = max z,  S = sum e^(z - m),  U = sum (z - m) e^(z - m)
//   lse = m + log S,  log p_t = (z_t - m) - log S,  entropy = -sum p log p = log S - U / S
//   gradient of g log p_t + h entropy:  scale (g ([c = t] - p_c) - h p_c (log p_c + entropy))
//
// log p is a difference of logits and log S: formed of those it has the same digits wherever a row lies, which z - lse has near zero only
// (47 logits near 20000: 1.0e-6 off, and 9.8e-4).  S, not lse, says whether a row has a class left.
//
// The alternatives are the classes of the largest logits, compared as they stand in memory: equal ones by the lower class, NaN
// before everything, -0 equal to +0.  A class at -inf is masked (p = 0); a row of masked classes has lse = log p = -inf, entropy
// and gradient 0.  Sums and statistics are in 32 bits.
//
// Bound by memory: a row is read once.  Short rows (k_probs_rows): L lanes hold a row in registers, in at most 4 loads a lane; the
// maximum comes first and the sums after it, from the registers.  Long rows (k_probs_long): a workgroup, or several for parts
// of a row where there are few rows, runs over the row with a running maximum that the sums follow; k_probs_join
// puts the parts together.
//
// The alternatives are what costs instructions.  They are kept as a sorted list a lane, and at the end the group takes the best head
// of all lists, once per alternative.  An element is one number, its order above its class, so that a place of the list costs one
// instruction (the median of the place, the one above and the element).  16-bit logits and their classes fit into 32 bits; of 32-bit logits
// the lowest bits give way to the class, and where that leaves the order open (equal upper bits at the list's end or within it), or a row
// has NaN, its wave's rows are done again by full comparisons.  In long rows a wave skips what is below K values it has seen.
// Equal upper bits are rare among continuous 32-bit logits, not among rounded ones: 1M x 172 f32 with 5 alternatives takes 214 us, of logits that were
// bf16 342, f16 236, of relu's zeros where few classes are above them 399 (2.45M x 47 148, 261, 182, 272).
//
// 2.45M x 47 bf16: without alternatives 56 us (4.9 TB/s), with 5 99 (vector instructions, some 700 for 32 rows); 512 x 100003 f16 29 and, with 8,
// 46; the gradient of 1M x 172 f32 235 (6.0 TB/s), 340 where every row is far from zero.
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
  int parts, top, wide_targets, id_bits;    // id_bits: of a number in a list that stand for the class (32-bit logits)
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

// A list of the K best elements of a lane, best first, order and class apart: five instructions a place.
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

// the place of x in a sorted list of numbers, best first: the median of three neighbours, from the end on
__device__ __forceinline__ uint32_t median(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("v_med3_u32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int K> __device__ __forceinline__ void put_number(uint32_t (&list)[K], uint32_t x) {
#pragma unroll
  for (int k = K - 1; k > 0; k--) list[k] = median(list[k - 1], list[k], x);
  list[0] = max(list[0], x);
}
// order_of without the care for NaN
__device__ __forceinline__ uint32_t order_of_number(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
// bits of a number that stand for the class: what the order of a type leaves
template <class T> constexpr int kIdBits = __is_same(T, bf16) ? 16 : 13;

// Best of a group's heads, taken off its list: every lane gets it.
template <int L, int K> __device__ __forceinline__ void take_best(Best<float, K> &b, uint32_t &o, int32_t &id) {
  o = group_all<L>(b.o[0], [](uint32_t x, uint32_t y) { return x > y ? x : y; });
  const int32_t c = b.o[0] == o ? b.id[0] : 0x7fffffff;
  id = group_all<L>(c, [](int32_t x, int32_t y) { return x < y ? x : y; });
  b.pop(c == id && b.o[0] == o);
}

// maximum of the logits, sum of e^(z - z_max) and of its products with (z - z_max) log2 e
struct RowStats { float m, s, u; };
__device__ __forceinline__ float safe_max(float m) { return m == -__builtin_inff() ? 0.f : m; }

// adds a logit; scale2 = scale log2 e.  A masked class (-inf) adds nothing to either sum.
__device__ __forceinline__ void add_term(float f, float m, float scale2, float &s, float &u) {
  const float t = (f - m) * scale2, e = __builtin_amdgcn_exp2f(t);
  s += e;
  u = fmaf(fmaxf(t, -1e30f), e, u);
}
// the sums relative to another maximum
__device__ __forceinline__ void rescale(RowStats &a, float to, float scale2) {
  const float d = (safe_max(a.m) - to) * scale2, f = a.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(d);
  a.u = f == 0.f ? 0.f : (a.u + a.s * d) * f;
  a.s *= f;
  a.m = to;
}

// log p of a logit of a row with maximum m (safe_max's) and log_s = log S, which is -inf where every class is masked
__device__ __forceinline__ float log_p(float logit, float m, float log_s, float scale) {
  return log_s == -__builtin_inff() ? log_s : (logit - m) * scale - log_s;
}
// what a row's statistics say, written by one lane
__device__ __forceinline__ void finish_row(const ProbsArgs &a, int64_t r, float m, float s, float u, float log_s, float target, bool has) {
  const bool none = s == 0.f;
  if (a.lse) {                               // one of finite logits is finite: the largest number where it passes the range
    const float lse = m * a.scale + log_s;
    a.lse[r] = none || lse != lse ? lse : __builtin_amdgcn_fmed3f(lse, -__FLT_MAX__, __FLT_MAX__);
  }
  if (a.entropy) a.entropy[r] = none ? 0.f : log_s - u * kLn2 / s;
  if (a.logp) a.logp[r] = has ? log_p(target, m, log_s, a.scale) : 0.f;
}
__device__ __forceinline__ void write_top(const ProbsArgs &a, int64_t r, int j, float v, int32_t id, float m, float log_s) {
  if (a.top_ids) a.top_ids[r * a.top + j] = id;
  if (a.top_logp) a.top_logp[r * a.top + j] = log_p(v, m, log_s, a.scale);
}

// ------------------------------------------------------------------------------------ short rows
template <class T, int L, int NV, int V, int K>
__global__ __launch_bounds__(kHeadThreads) void k_probs_rows(ProbsArgs a) {
  constexpr int G = kHeadThreads / L;
  constexpr bool EXACT = sizeof(T) == 2;     // a number holds order and class
  constexpr int KL = EXACT ? K : K + 1;      // ... or one more place says whether the last one is certain
  const int q = threadIdx.x % L, C = (int)a.classes;
  const float scale2 = a.scale * kLog2e;
  const uint32_t low = (1u << (EXACT ? kIdBits<T> : a.id_bits)) - 1;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += (int64_t)gridDim.x * G) {
    const int64_t mine = r0 + threadIdx.x / L;
    const int64_t r = mine < a.rows ? mine : a.rows - 1;
    const T *x = static_cast<const T *>(a.logits) + r * a.ld;
    float f[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++) load_pack<T, V>(x + min((i * L + q) * V, C - V), f[i]);
    const int64_t t = target_of(a.targets, a.wide_targets, r);
    const bool has = t >= 0 && t < C;
    const float target = has ? (float)x[t] : 0.f;
    uint32_t list[KL > 0 ? KL : 1];
#pragma unroll
    for (int k = 0; k < KL; k++) list[k] = 0;
    // all vectors but the last are whole (NV is the least that holds the row); of that one the rest repeats the vector before
    const int last = ((NV - 1) * L + q) * V, last_at = min(last, C - V);
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int at = i + 1 < NV ? (i * L + q) * V : last_at;
#pragma unroll
      for (int j = 0; j < V; j++) {
        uint32_t number = 0;
        if constexpr (K > 0) number = (order_of_number(f[i][j]) & ~low) | (low - (uint32_t)(at + j));
        if (i + 1 == NV) {
          const bool live = at + j >= last;
          f[i][j] = live ? f[i][j] : -__builtin_inff();
          number = live ? number : 0u;
        }
        m = fmaxf(m, f[i][j]);
        if constexpr (K > 0) put_number<KL>(list, number);
      }
    }
    m = safe_max(group_all<L>(m, [](float p, float p2) { return fmaxf(p, p2); }));
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
      for (int j = 0; j < V; j++) add_term(f[i][j], m, scale2, s, u);
    s = group_sum<L>(s);
    u = group_sum<L>(u);
    const bool on = mine < a.rows;
    const float log_s = logf(s);
    if (on && q == 0) finish_row(a, r, m, s, u, log_s, target, has);
    if constexpr (K > 0) {
      uint32_t o[KL];
      bool open = s != s;                    // a NaN (or +inf) in the row
#pragma unroll
      for (int k = 0; k < KL; k++) {
        o[k] = group_all<L>(list[0], [](uint32_t p, uint32_t p2) { return p > p2 ? p : p2; });
        const bool me = list[0] == o[k];
#pragma unroll
        for (int i = 0; i + 1 < KL; i++) list[i] = me ? list[i + 1] : list[i];
        list[KL - 1] = me ? 0 : list[KL - 1];
        if constexpr (!EXACT)
          if (k > 0) open |= k <= a.top && o[k] != 0 && ((o[k] ^ o[k - 1]) & ~low) == 0;
      }
      int32_t id[K > L ? (K + L - 1) / L : 1];               // this lane's alternatives: q, q + L, ...
      float v[K > L ? (K + L - 1) / L : 1];
      if (!__any(open)) {
#pragma unroll
        for (int i = 0; i * L < K; i++) {
          uint32_t mine_o = o[i * L];
#pragma unroll
          for (int k = 1; k < L; k++)
            if (i * L + k < K) mine_o = q == k ? o[i * L + k] : mine_o;
          id[i] = (int32_t)(low - (mine_o & low));
          if constexpr (EXACT) v[i] = of_order(mine_o & 0x80000000u ? mine_o & ~low : mine_o | low);
          else v[i] = on && i * L + q < a.top ? (float)x[id[i]] : 0.f;
        }
      } else {                               // once more from memory: rare, and not to cost the usual case registers
        Best<float, K> best;
        best.clear();
#pragma unroll 1
        for (int c = q; c < C; c += L) best.put(order_of((float)x[c]), c);
#pragma unroll
        for (int k = 0; k < K; k++) {
          uint32_t oo; int32_t ii;
          take_best<L, K>(best, oo, ii);
          if (q == k % L) { id[k / L] = ii; v[k / L] = of_order(oo); }
        }
      }
#pragma unroll
      for (int i = 0; i * L < K; i++)
        if (on && i * L + q < a.top) write_top(a, r, i * L + q, v[i], id[i], m, log_s);
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

// TW: threads of a row (or part): a workgroup, or one wave where there are rows for all of them, which then needs no LDS at the end.
template <class T, int V, int K, int TW>
__global__ __launch_bounds__(kHeadThreads) void k_probs_long(ProbsArgs a) {
  constexpr int W = kHeadThreads / kWave, G = kHeadThreads / TW, KS = K > 0 ? K : 1;
  // 16-bit logits: a number is the order above the place among the lane's elements, of which probs_parts leaves few enough
  constexpr bool EXACT = sizeof(T) == 2;
  constexpr uint32_t low = (1u << kIdBits<T>) - 1;
  __shared__ float s_m[W], s_s[W], s_u[W];
  __shared__ uint32_t s_o[(W + 1) * KS];
  __shared__ int32_t s_id[(W + 1) * KS];
  const int tid = threadIdx.x % TW;
  const float scale2 = a.scale * kLog2e;
  for (int64_t item = (int64_t)blockIdx.x * G + threadIdx.x / TW; item < a.rows * a.parts; item += (int64_t)gridDim.x * G) {
    auto order_of_list = [](uint32_t number) { return number == 0 ? 0u : number & 0x80000000u ? number & ~low : number | low; };
    const int64_t r = item / a.parts;
    const int part = (int)(item - r * a.parts);
    const int64_t c0 = part * a.part_len, c1 = min(c0 + a.part_len, a.classes);    // part_len is a multiple of V
    const T *x = static_cast<const T *>(a.logits) + r * a.ld;
    RowStats st = {-__builtin_inff(), 0.f, 0.f};
    Best<float, K> best;
    best.clear();
    uint32_t list[KS];
#pragma unroll
    for (int k = 0; k < KS; k++) list[k] = 0;
    float floor_f = -__builtin_inff();       // K elements of the wave are at least this large
    int64_t refresh = 1, step = 0;
    const int64_t n_vec = (c1 - c0 + V - 1) / V;
    for (int64_t i0 = 0; i0 < n_vec; i0 += TW, step++) {
      const int64_t first = c0 + (i0 + tid) * V, at = min(first, a.classes - V);
      float f[V];
      load_pack<T, V>(x + at, f);
      const bool whole = i0 + TW < n_vec;    // of the last vectors some repeat elements or are past the part
      if (!whole)
#pragma unroll
        for (int j = 0; j < V; j++) f[j] = at + j >= first && first < c1 ? f[j] : -__builtin_inff();
      float vm = f[0];
#pragma unroll
      for (int j = 1; j < V; j++) vm = fmaxf(vm, f[j]);
      if (vm > st.m) rescale(st, vm, scale2);
      const float ms = safe_max(st.m);
#pragma unroll
      for (int j = 0; j < V; j++) add_term(f[j], ms, scale2, st.s, st.u);
      if constexpr (K > 0) {
        if (__any(vm >= floor_f)) {
#pragma unroll
          for (int j = 0; j < V; j++) {
            if (!__any(f[j] >= floor_f)) continue;
            const uint32_t o = f[j] >= floor_f && (whole || (at + j >= first && first < c1)) ? order_of_number(f[j]) : 0u;
            if constexpr (EXACT) put_number<KS>(list, o ? (o & ~low) | (low - (uint32_t)(step * V + j)) : 0u);
            else if (__any(o > best.o[KS - 1])) best.put(o, (int32_t)(at + j));
          }
        }
        if (step + 1 == refresh) {           // at steps 1, 2, 4, ...: what K of the lanes' best reach
          refresh *= 2;
          const uint32_t head = EXACT ? list[0] : best.o[0];
          uint32_t o = 0;                    // the largest number of 16 bits (then zeros) that K heads reach, bit by bit
#pragma unroll
          for (int bit = 31; bit >= 16; bit--)
            if (__popcll(__ballot(head >= (o | 1u << bit))) >= K) o |= 1u << bit;
          if (o > 0x007fffffu) floor_f = of_order(o);        // (above -inf)
        }
      }
    }
    // the row's sums
    float bm = group_all<kWave>(st.m, [](float p, float p2) { return fmaxf(p, p2); });
    if constexpr (TW > kWave) {
      if (lane_id() == 0) s_m[threadIdx.x / kWave] = bm;
      __syncthreads();
      bm = s_m[0];
#pragma unroll
      for (int w = 1; w < W; w++) bm = fmaxf(bm, s_m[w]);
    }
    rescale(st, safe_max(bm), scale2);
    float s = group_sum<kWave>(st.s), u = group_sum<kWave>(st.u);
    if constexpr (TW > kWave) {
      if (lane_id() == 0) { s_s[threadIdx.x / kWave] = s; s_u[threadIdx.x / kWave] = u; }
      __syncthreads();
      s = u = 0.f;
#pragma unroll
      for (int w = 0; w < W; w++) { s += s_s[w]; u += s_u[w]; }
    }
    if constexpr (K > 0) {
      if constexpr (EXACT)                   // from places to classes
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int64_t e = low - (list[k] & low), first = c0 + (e / V * TW + tid) * V;
          best.o[k] = list[k] ? order_of_list(list[k]) : 0u;
          best.id[k] = list[k] ? (int32_t)(min(first, a.classes - V) + e % V) : 0x7fffffff;
        }
      if (s != s) {                          // a NaN (or +inf) in the part: comparisons skipped it
        best.clear();
        for (int64_t i = tid; i < n_vec; i += TW) {
          const int64_t first = c0 + i * V, at = min(first, a.classes - V);
          float f[V];
          load_pack<T, V>(x + at, f);
#pragma unroll
          for (int j = 0; j < V; j++) best.put(at + j >= first ? order_of(f[j]) : 0u, (int32_t)(at + j));
        }
      }
      if constexpr (TW > kWave) block_best<K>(best, s_o, s_id);
    }
    const int64_t p = r * a.parts + part;
    if (a.parts > 1) {
      if (threadIdx.x == 0) { a.part_stats[3 * p] = bm; a.part_stats[3 * p + 1] = s; a.part_stats[3 * p + 2] = u; }
      if (K > 0 && (int)threadIdx.x < a.top) {
        a.part_ord[p * a.top + threadIdx.x] = s_o[W * KS + threadIdx.x];
        a.part_id[p * a.top + threadIdx.x] = s_id[W * KS + threadIdx.x];
      }
    } else {
      const float m = safe_max(bm), log_s = logf(s);
      if (tid == 0) {
        const int64_t t = target_of(a.targets, a.wide_targets, r);
        const bool has = t >= 0 && t < a.classes;
        finish_row(a, r, m, s, u, log_s, has ? (float)x[t] : 0.f, has);
      }
      if constexpr (K > 0) {
        uint32_t o = 0;
        int32_t id = 0;
        if constexpr (TW > kWave) {
          if (tid < K) { o = s_o[W * KS + tid]; id = s_id[W * KS + tid]; }
        } else {
#pragma unroll
          for (int k = 0; k < K; k++) {
            uint32_t oo; int32_t ii;
            take_best<kWave, K>(best, oo, ii);
            if (tid == k) { o = oo; id = ii; }
          }
        }
        if (tid < a.top) write_top(a, r, tid, of_order(o), id, m, log_s);
      }
    }
    if constexpr (TW > kWave) __syncthreads();               // LDS is the next row's
  }
}

// Parts of a row, at most 64, to the row: one wave a row, a part a lane.
template <class T, int K>
__global__ __launch_bounds__(kWave) void k_probs_join(ProbsArgs a) {
  const int l = lane_id();
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int64_t p = r * a.parts + min(l, a.parts - 1);
    RowStats st = {a.part_stats[3 * p], a.part_stats[3 * p + 1], a.part_stats[3 * p + 2]};
    if (l >= a.parts) st = {-__builtin_inff(), 0.f, 0.f};
    const float m = safe_max(group_all<kWave>(st.m, [](float x, float y) { return fmaxf(x, y); }));
    rescale(st, m, a.scale * kLog2e);
    const float s = group_sum<kWave>(st.s), u = group_sum<kWave>(st.u);
    const float log_s = logf(s);
    if (l == 0) {
      const T *x = static_cast<const T *>(a.logits) + r * a.ld;
      const int64_t t = target_of(a.targets, a.wide_targets, r);
      const bool has = t >= 0 && t < a.classes;
      finish_row(a, r, m, s, u, log_s, has ? (float)x[t] : 0.f, has);
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
      if (l < a.top) write_top(a, r, l, of_order(my_o), my_id, m, log_s);
    }
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

// Beyond this lse of 32 bits is off by more than 1.5e-5, and so would be every p that is formed with it; at a type's lowest values
// it holds nothing of log S at all.
constexpr float kFarLse = 256.f;

// The gradient by one logit, from its class's log probability.  p comes in two factors: the hardware's exponential knows no subnormal
// results, which 32-bit and bf16 gradients have.  Below log p = -200 both factors are zero, and what they multiply has to be finite.
struct GradTerm {
  float g, h, ent, scale;                    // gradients of log p_t and entropy, 0 where there are none
  __device__ __forceinline__ float operator()(float lp, bool target) const {
    const float root = __builtin_amdgcn_exp2f(lp * (0.5f * kLog2e));
    return (root * (-g - h * (fmaxf(lp, -200.f) + ent)) * root + (target ? g : 0.f)) * scale;
  }
};

// A row far from zero, by one group of lanes: maximum and sum anew, then its gradient.  Three reads instead of one.
template <class T, int L, int V> __device__ __forceinline__ void far_row(const ProbsGradArgs &a, const T *x, T *out, int64_t t, GradTerm term) {
  const int q = threadIdx.x % L;
  const float scale2 = a.scale * kLog2e;
  float m = -__builtin_inff(), s = 0.f;
#pragma unroll 1
  for (int64_t first = q * V; first < a.classes; first += L * V) {
    float f[V];
    load_pack<T, V>(x + min(first, a.classes - V), f);
#pragma unroll
    for (int j = 0; j < V; j++) m = fmaxf(m, f[j]);
  }
  m = safe_max(group_all<L>(m, [](float p, float p2) { return fmaxf(p, p2); }));
#pragma unroll 1
  for (int64_t first = q * V; first < a.classes; first += L * V) {
    const int64_t at = min(first, a.classes - V);
    float f[V];
    load_pack<T, V>(x + at, f);
#pragma unroll
    for (int j = 0; j < V; j++) s += at + j >= first ? __builtin_amdgcn_exp2f((f[j] - m) * scale2) : 0.f;
  }
  const float log_s = logf(group_sum<L>(s));
#pragma unroll 1
  for (int64_t first = q * V; first < a.classes; first += L * V) {
    const int64_t at = min(first, a.classes - V);
    float f[V];
    load_pack<T, V>(x + at, f);
#pragma unroll
    for (int j = 0; j < V; j++) f[j] = term(log_p(f[j], m, log_s, a.scale), at + j == t);
    store_pack<T, V>(out + at, f);
  }
}

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
    float lse = a.lse[r], g = a.g_logp ? a.g_logp[r] : 0.f, h = 0.f, ent = 0.f;
    if (a.g_entropy) { h = a.g_entropy[r]; ent = a.entropy[r]; }
    const bool none = lse == -__builtin_inff();            // every class masked: no gradient
    lse = none ? 0.f : lse;
    h = none ? 0.f : h;
    g = none || t < 0 || t >= a.classes ? 0.f : g;
    const GradTerm term = {g, h, ent, a.scale};
    const bool far = fabsf(lse) > kFarLse;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t first = c0 + (i * L + q) * V, at = min(first, a.classes - V);
      float o[V];
#pragma unroll
      for (int j = 0; j < V; j++) o[j] = term(z[i][j] * a.scale - lse, at + j == t);
      if (first < a.classes && !far) store_pack<T, V>(out + at, o);
    }
    // rare; a group's lanes agree, and of a row in pieces the first one's group does all
    if (far && c0 == 0) far_row<T, L, V>(a, x, out, t, term);
  }
}

// ------------------------------------------------------------------------------------ host side
constexpr int64_t kWaveRows = 4096;         // long rows of which a wave takes one: 16 waves a CU
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
  const int64_t most = (int64_t)8192 * kHeadThreads;       // elements of a part: a lane's places have 13 bits
  static_assert(INK_MAX_CLASSES <= kWave * 8192ll * kHeadThreads, "64 parts are enough");
  parts = std::max(parts, (n_vec * V + most - 1) / most);
  const int64_t per = (n_vec + parts - 1) / parts;
  parts = (n_vec + per - 1) / per;
  *len = per * V;
  return (int)parts;
}

template <class T, int L, int K> static void probs_rows(const ProbsArgs &a, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  const int64_t n_vec = (a.classes + V - 1) / V, per = kHeadThreads / L;
  const dim3 grid((unsigned)std::min<int64_t>((a.rows + per - 1) / per, 16384));
  if (a.classes < V) { if constexpr (L == 8) run(k_probs_rows<T, 8, 1, 1, K>, grid, dim3(kHeadThreads), a); return; }
  if constexpr (L == 2) {                    // (wider groups hold more than two vectors a lane)
    if (n_vec <= L) return run(k_probs_rows<T, L, 1, V, K>, grid, dim3(kHeadThreads), a);
    if (n_vec <= 2 * L) return run(k_probs_rows<T, L, 2, V, K>, grid, dim3(kHeadThreads), a);
  }
  run(n_vec <= 3 * L ? k_probs_rows<T, L, 3, V, K> : k_probs_rows<T, L, 4, V, K>, grid, dim3(kHeadThreads), a);
}

template <class T, int K> static void probs_top(const ProbsArgs &a, Launches &run) {
  constexpr int V = 16 / sizeof(T);
  if (probs_long(a.classes, sizeof(T) == 4 ? INK_F32 : INK_BF16)) {
    if (a.parts == 1 && a.rows >= kWaveRows && a.classes <= 8192 * kWave)
      return run(k_probs_long<T, V, K, kWave>, dim3((unsigned)std::min<int64_t>((a.rows + 3) / 4, 1 << 20)), dim3(kHeadThreads), a);
    run(k_probs_long<T, V, K, kHeadThreads>, dim3((unsigned)std::min<int64_t>(a.rows * a.parts, 1 << 20)), dim3(kHeadThreads), a);
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
  if constexpr (L == 4) {                    // (wider groups hold more than two vectors a lane)
    if (nv == 1) return run(k_probs_grad<T, L, 1, V>, grid, block, a);
    if (nv == 2) return run(k_probs_grad<T, L, 2, V>, grid, block, a);
  }
  run(nv <= 3 ? k_probs_grad<T, L, 3, V> : k_probs_grad<T, L, 4, V>, grid, block, a);
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
  if (!(scale > 0.f) || scale > 2.3e38f) return "scale must be positive and at most 2.3e38";       // scale log2 e is a number
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
  while (a.id_bits < 16 && (1 << a.id_bits) < classes) a.id_bits++;
  if (probs_long(classes, type)) {
    a.parts = probs_parts(rows, classes, type, &a.part_len);
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
