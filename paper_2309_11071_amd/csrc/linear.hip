// Matrix product of rows with its epilogue, y = act(x W + bias) + residual, and its gradient.
//
//   forward   z = x W + bias (kept if asked for),  y = act(z) + residual
//   gradient  dz = dy act'(z):  dx = dz W^T,  dweight = x^T dz,  dbias = sum over rows of dz
//
// W is [cols][out] as the layers' weights are.  The rows are many and both sides of W are short, so 16-bit products are bound by
// reading the rows and writing the results, 32-bit ones by the matrix unit.  Every product is formed transposed, W's columns as
// the instruction's rows, so that a lane ends up with four neighbouring columns of its row.  Which kernel:
//
//   up to 64 rows, 64k results  k_linear_few     a row and 32 columns a workgroup; W is what is read: 1 x 602 x 256 bf16 5 us
//   from 32768 rows on          k_linear_stream  W in registers, rows in a stream; up to 640 terms (16 bits) or 256 (32 bits)
//   enough rows for 256 tiles   k_linear_tile    128 rows by 64 or 128 columns
//   else                        k_linear_small   32 by 32, eight waves share the depth: 100 x 602 x 256 f32 37 us in tiles, 11 (the call) so
//
// The stream against the tiles, in one run: 50k x 128 x 47 bf16 11 and 14 us, 200k x 128 x 128 26 and 40, 200k x 256 x 256 59 and 91; f32 of 128 x 64,
// which the matrix unit holds up, 50k rows 19 and 19, 200k 49 and 54.
//
// Products are exact (16-bit operands) or fused (32 bits), and summed in 32 bits; the epilogue is in 32 bits and y, z, dx, dweight and
// dbias are rounded once.  For 16-bit rows dz is rounded to the rows' type before the two products, as a program that keeps dz in memory
// has it: an error of the size of the results' own rounding (612k x 128 x 172 bf16 with gelu 0.0024 from 64 bits, 0.0017 rounded once).  dz in two
// 16-bit parts gives results rounded once; the second part's conversions, its room in LDS and its matrix instructions cost 612k x 128 x 172 242 us instead of
// 194, 128 x 47 113 instead of 110, 256 x 256, whose registers it does not fit, 1016 instead of 556.  dbias sums the unrounded values.  dweight is
// a sum over all rows: workgroups take slices of the rows and leave a partial matrix each, which k_grad_sum adds up in order (no
// atomics: the same call gives the same bits).
#include <algorithm>
#include <type_traits>

#include "matrix.h"

namespace ink {

struct LinearArgs {
  const void *in, *pre;                      // forward: rows of x; gradient: rows of dy, and z if there is an activation
  const void *weight, *bias, *res;
  void *out, *keep;                          // forward: y, z or NULL; gradient: dx
  int64_t rows, ld_in, ld_pre, ld_w, ld_res, ld_out, ld_keep;
  int depth, width, act;                     // terms of a sum, columns of the result
};

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

// Four neighbouring columns of a row of results, from the registers of the products: bias, z, activation, residual, y.
template <class T, class TO, bool GRAD> __device__ __forceinline__ void finish4(const LinearArgs &a, int64_t r, int c, float v[4]) {
  if constexpr (!GRAD) {
    float q[4];
    if (a.bias) {
      load4(static_cast<const T *>(a.bias), c, a.width, q);
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] += q[j];
    }
    if (a.keep) store4(static_cast<TO *>(a.keep) + r * a.ld_keep, c, a.width, v);
    activate_all<4>(v, a.act);
    if (a.res) {
      load4(static_cast<const TO *>(a.res) + r * a.ld_res, c, a.width, q);
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] += q[j];
    }
  }
  store4(static_cast<TO *>(a.out) + r * a.ld_out, c, a.width, v);
}

// a fragment of a row of rows read: x, or dz of dy and z
template <class T, class TI, bool GRAD> __device__ __forceinline__ typename Frag<T>::V in_frag(const LinearArgs &a, int64_t r, int k) {
  const TI *x = static_cast<const TI *>(a.in) + r * a.ld_in;
  if constexpr (GRAD) return grad_frag<T, TI>(x, static_cast<const TI *>(a.pre) + (a.pre ? r * a.ld_pre : 0), k, a.depth, a.act);
  else return row_frag<T>(x, k, a.depth);
}

// ------------------------------------------------------------------------------------ tiles
// T: type of the operands, TI: of the rows read (GRAD: dy and z), TO: of the rows written.
// 128 rows by 64 NTW columns a workgroup, 64 by 32 NTW a wave, 128 bytes of the depth in LDS at a time: while one piece is
// multiplied the next is on its way in registers.  For 32-bit rows, which the matrix unit bounds, and depths whose W the registers of a
// workgroup do not hold.  233k x 602 x 256 f32 takes 674 us (106 TFLOP/s).  One buffer and three workgroups a CU against two buffers (one barrier a
// piece) and two workgroups, both before products of different accumulators took turns: 782 and 815 us; tiles of 64 rows and four workgroups 789.
template <class T, class TI, class TO, int NTW, bool GRAD>
__global__ __launch_bounds__(256, 3) void k_linear_tile(LinearArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int VK = kVec<T>, KC = 8 * VK, BM = 128, BN = 64 * NTW, NT = 2 * NTW, P = 9;      // P: 16-byte pieces between rows of x
  constexpr int NX = BM * 8 / 256;
  constexpr int NW = GRAD ? BN * 8 / 256 : VK, SQ = BN / VK * 8;           // W in pieces of its rows, or in squares (forward)
  __shared__ V s_x[BM * P], s_w[BN * 8];
  const int tid = threadIdx.x, l = lane_id(), half = l / 32, wm = tid / kWave / 2, wn = tid / kWave % 2;
  // workgroups go to the eight chiplets in turn: the column tiles of the same rows are eight apart, so that one L2 serves them
  const int gy = (a.width + BN - 1) / BN, id = blockIdx.x / 8;
  const int64_t m0 = ((int64_t)(id / gy) * 8 + blockIdx.x % 8) * BM;
  const int n0 = id % gy * BN;
  if (m0 >= a.rows) return;
  const T *w = static_cast<const T *>(a.weight);
  V x[NX], wv[NW];
  const int kp = tid % 8 * VK;               // this thread's place in 128 bytes of the depth
  const TI *xp[NX], *zp[NX];
#pragma unroll
  for (int j = 0; j < NX; j++) {
    const int64_t r = min(m0 + tid / 8 + 32 * j, a.rows - 1);
    xp[j] = static_cast<const TI *>(a.in) + r * a.ld_in;
    zp[j] = GRAD && a.pre ? static_cast<const TI *>(a.pre) + r * a.ld_pre : nullptr;
  }
  const int wn_at = GRAD ? tid / 8 : tid % (BN / VK) * VK, wk_at = GRAD ? kp : tid / (BN / VK) * VK;      // first column, first k
  const bool inside = n0 + BN <= a.width;
  auto fetch = [&](int k0) {
    const bool whole = k0 + KC <= a.depth;   // no piece is cut by the end of the depth
#pragma unroll
    for (int j = 0; j < NX; j++) {
      if constexpr (GRAD) x[j] = grad_frag<T, TI>(xp[j], zp[j], k0 + kp, whole ? 0x7fffffff : a.depth, a.act);
      else x[j] = row_frag<T>(xp[j], k0 + kp, whole ? 0x7fffffff : a.depth);
    }
    if (whole && inside) {
      if (GRAD || tid < SQ)
#pragma unroll
        for (int j = 0; j < NW; j++) {
          const T *at = w + (GRAD ? (int64_t)(n0 + wn_at + 32 * j) * a.ld_w + k0 + wk_at : (int64_t)(k0 + wk_at + j) * a.ld_w + n0 + wn_at);
          wv[j] = (V)*reinterpret_cast<const typename Pack<T, VK>::type *>(at);
        }
      return;
    }
#pragma unroll
    for (int j = 0; j < NW; j++) {
      wv[j] = V{};
      const int n = n0 + wn_at + (GRAD ? 32 * j : 0), k = k0 + wk_at + (GRAD ? 0 : j);
      if ((!GRAD && tid >= SQ) || k >= a.depth || n >= a.width) continue;
      if constexpr (GRAD) wv[j] = row_frag<T>(w + (int64_t)n * a.ld_w, k, a.depth);
      else wv[j] = row_frag<T>(w + (int64_t)k * a.ld_w, n, a.width);
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int j = 0; j < NX; j++) s_x[(tid / 8 + 32 * j) * P + tid % 8] = x[j];
    if constexpr (GRAD) {
#pragma unroll
      for (int j = 0; j < NW; j++) {
        const int n = tid / 8 + 32 * j, p = tid % 8;
        s_w[((p / 2) * NT + n / 32) * 64 + n % 32 + 32 * (p % 2)] = wv[j];
      }
    } else if (tid < SQ) {
      const int p = tid / (BN / VK);
#pragma unroll
      for (int c = 0; c < VK; c++) {
        V v;
#pragma unroll
        for (int j = 0; j < VK; j++) v[j] = wv[j][c];
        const int n = tid % (BN / VK) * VK + c;
        s_w[((p / 2) * NT + n / 32) * 64 + n % 32 + 32 * (p % 2)] = v;
      }
    }
  };
  f32x16 acc[2][NTW];
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int n = 0; n < NTW; n++) acc[i][n] = f32x16{};
  fetch(0);
  put();
  __syncthreads();
  for (int k0 = 0; k0 < a.depth; k0 += KC) {
    const bool more = k0 + KC < a.depth;
    if (more) fetch(k0 + KC);
#pragma unroll
    for (int s = 0; s < 4; s++) {
      V xs[2], ws[NTW];
#pragma unroll
      for (int i = 0; i < 2; i++) xs[i] = s_x[(wm * 64 + i * 32 + l % 32) * P + 2 * s + half];
#pragma unroll
      for (int n = 0; n < NTW; n++) ws[n] = s_w[(s * NT + wn * NTW + n) * 64 + l];
      mma_block<T>(ws, xs, acc);
    }
    __syncthreads();
    if (more) put();
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int64_t r = m0 + wm * 64 + i * 32 + l % 32;
    if (r >= a.rows) continue;
#pragma unroll
    for (int n = 0; n < NTW; n++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int c = n0 + (wn * NTW + n) * 32 + 8 * e + 4 * half;
        float v[4] = {acc[i][n][4 * e], acc[i][n][4 * e + 1], acc[i][n][4 * e + 2], acc[i][n][4 * e + 3]};
        if (c < a.width) finish4<T, TO, GRAD>(a, r, c, v);
      }
  }
}

// ------------------------------------------------------------------------------------ not many rows
// 32 rows by 32 columns a workgroup, whose eight waves share the depth: where tiles of 128 rows would leave most of the card without work.
// The fragments come straight from memory (W's columns, forward, element by element: 32 lanes side by side).
constexpr int kSmallWaves = 8;
template <class T, class TI, class TO, bool GRAD>
__global__ __launch_bounds__(kWave * kSmallWaves) void k_linear_small(LinearArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int VK = kVec<T>, KS = kStep<T>;
  __shared__ float s_acc[kSmallWaves][32][36];
  const int wave = threadIdx.x / kWave, l = lane_id(), half = l / 32;
  const int64_t r0 = (int64_t)blockIdx.x * 32, r = min(r0 + l % 32, a.rows - 1);
  const int n0 = blockIdx.y * 32, n = n0 + l % 32;
  const T *w = static_cast<const T *>(a.weight);
  f32x16 acc = f32x16{};
#pragma unroll 2
  for (int k0 = wave * KS; k0 < a.depth; k0 += kSmallWaves * KS) {
    const int k = k0 + half * VK;
    const V x = in_frag<T, TI, GRAD>(a, r, k);
    V wv{};
    if constexpr (GRAD) {
      if (n < a.width) wv = row_frag<T>(w + (int64_t)n * a.ld_w, k, a.depth);
    } else {
#pragma unroll
      for (int j = 0; j < VK; j++)
        if (n < a.width && k + j < a.depth) wv[j] = w[(int64_t)(k + j) * a.ld_w + n];
    }
    acc = mma(wv, x, acc);
  }
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const F4 v = {acc[4 * e], acc[4 * e + 1], acc[4 * e + 2], acc[4 * e + 3]};
    *reinterpret_cast<F4 *>(&s_acc[wave][l % 32][8 * e + 4 * half]) = v;
  }
  __syncthreads();
  if (threadIdx.x >= 256) return;
  const int row = threadIdx.x / 8, c = threadIdx.x % 8 * 4;
  F4 t = F4{};
#pragma unroll
  for (int i = 0; i < kSmallWaves; i++) t += *reinterpret_cast<const F4 *>(&s_acc[i][row][c]);
  float v[4] = {t[0], t[1], t[2], t[3]};
  if (r0 + row < a.rows && n0 + c < a.width) finish4<T, TO, GRAD>(a, r0 + row, n0 + c, v);
}

// ------------------------------------------------------------------------------------ many rows
// Rows in a stream.  A workgroup of WM x WN waves holds W in registers for good: a wave has the fragments of its 32 NTW columns over
// the whole depth (KS steps).  It takes 32 WM rows at a time: all threads load them side by side (16 bytes a lane, whole lines), a tile
// ahead, and put them into LDS, from where every wave reads the fragments of its 32 rows; the product goes through
// LDS in 32 bits once more, so that residual, z and y are read and written in whole lines too.  Bound by memory in 16 bits: 2.45M x 256 x
// 256 with residual and z 1.0 ms (5.02 GB, 4.9 TB/s), without 0.59 (4.2), 2.45M x 128 x 64 167 us (5.6); the matrix unit is busy 15 % of the time.  In
// 32 bits the matrix unit and memory take turns: 2.45M x 128 x 64 460 us, 87 TFLOP/s.  The group sizes are the fastest of those
// measured: 612k x 602 x 256 bf16 with all 40 steps of 32 columns a wave 473 us, with 20-step halves and 64 columns a wave 672, with halves over sixteen
// waves 622; 612k x 602 x 47 split four ways 174, unsplit 639.  Not all fit the registers (256 with two waves a SIMD, 128 with four): the
// forms of 40 steps spill 37 to 94, those of 8 steps a wave at four waves a SIMD 6 to 12 in the gradient, 93 there with 32-bit rows.
struct StreamArgs {
  LinearArgs a;
  int chunks, pitch, flat;                   // 16-byte pieces of a row's depth; floats between rows of results in LDS; see emit
};

template <class T, class TI, class TO, int KS, int NTW, int WN, int WM, int WK, int PER, bool GRAD>
__global__ __launch_bounds__(kWave * WN * WM * WK, PER) void k_linear_stream(StreamArgs sa) {
  const LinearArgs &a = sa.a;
  typedef typename Frag<T>::V V;
  typedef typename Pack<TI, kVec<T>>::type In;
  constexpr int VK = kVec<T>, THREADS = kWave * WN * WM * WK, MR = 32 * WM, NT = NTW * WN, BN = 32 * NT, STEPS = KS * WK;
  constexpr int P = STEPS * 32 + 16;         // bytes between rows in LDS: 16 lanes' pieces fall on all banks
  constexpr int NL = (MR * 2 * STEPS + THREADS - 1) / THREADS;
  constexpr int OE = 16 / sizeof(TO), NO = (MR * BN / OE + THREADS - 1) / THREADS, PART = MR * (BN + 4);
  constexpr int ROOM = MR * P + WK * PART * 4, STEP_BYTES = BN * 32;       // W goes through the same LDS, in as few pieces as it takes
  constexpr int PS = STEPS * STEP_BYTES <= ROOM ? STEPS : STEPS / 2 * STEP_BYTES <= ROOM ? STEPS / 2 : 4;
  static_assert(STEPS % PS == 0 && PS * STEP_BYTES <= ROOM, "whole pieces");
  extern __shared__ __align__(16) char s_mem[];
  char *s_x = s_mem;
  float *s_o = reinterpret_cast<float *>(s_mem + MR * P), *s_b = s_o + WK * PART;
  const int tid = threadIdx.x, l = lane_id(), half = l / 32, wave = tid / kWave, wn = wave % WN, wm = wave / WN % WM, wk = wave / (WN * WM);
  const int n0 = blockIdx.y * BN, width = min(BN, a.width - n0);
  const int64_t tiles = (a.rows + MR - 1) / MR;
  const bool narrow = a.depth < VK;
  // This thread's pieces of a tile of rows: place in LDS, and offsets from the tile's first row, the same for every tile.
  In in[NL], pre[GRAD ? NL : 1];
  int lds_at[NL];
  uint32_t in_at[NL], pre_at[GRAD ? NL : 1];               // bytes
  uint32_t tails = 0;                        // pieces that the end of the depth cuts
#pragma unroll
  for (int j = 0; j < NL; j++) {
    const int i = min(tid + j * THREADS, MR * sa.chunks - 1);       // a thread without a piece repeats the last
    const int row = i / sa.chunks, c = i - row * sa.chunks, at = narrow ? 0 : min(c * VK, a.depth - VK);
    lds_at[j] = row * P + c * 16;
    in_at[j] = (__umul24(row, (uint32_t)a.ld_in) + at) * (uint32_t)sizeof(TI);
    if constexpr (GRAD) pre_at[j] = (__umul24(row, (uint32_t)a.ld_pre) + at) * (uint32_t)sizeof(TI);
    if (c * VK + VK > a.depth) tails |= 1u << j;
  }
  auto load = [&](const TI *base, uint32_t at) -> In {     // a uniform base and 32 bits a lane: one register of address
    const TI *x = reinterpret_cast<const TI *>(reinterpret_cast<const char *>(base) + at);
    if (!narrow) return *reinterpret_cast<const In *>(x);
    In v;
#pragma unroll
    for (int e = 0; e < VK; e++) v[e] = e < a.depth ? x[e] : (TI)0.f;
    return v;
  };
  auto fetch = [&](int64_t t) {
    const TI *x = static_cast<const TI *>(a.in) + t * MR * a.ld_in;
    const TI *z = GRAD && a.pre ? static_cast<const TI *>(a.pre) + t * MR * a.ld_pre : nullptr;
    const int64_t left = a.rows - t * MR;
    if (left >= MR) {
#pragma unroll
      for (int j = 0; j < NL; j++) {
        in[j] = load(x, in_at[j]);
        if constexpr (GRAD) if (z) pre[j] = load(z, pre_at[j]);
      }
    } else {                                 // the last rows once more in place of those past the end
#pragma unroll
      for (int j = 0; j < NL; j++) {
        const int row = lds_at[j] / P;
        const uint32_t over = max(0, row - (int)left + 1) * (uint32_t)sizeof(TI);
        in[j] = load(x, in_at[j] - over * (uint32_t)a.ld_in);
        if constexpr (GRAD) if (z) pre[j] = load(z, pre_at[j] - over * (uint32_t)a.ld_pre);
      }
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int j = 0; j < NL; j++) {
      V v;
      if constexpr (GRAD) {
        float d[VK];
#pragma unroll
        for (int e = 0; e < VK; e++) d[e] = (float)in[j][e];
        if (a.act != INK_ACT_NONE) {
          float z[VK];
#pragma unroll
          for (int e = 0; e < VK; e++) z[e] = (float)pre[j][e];
          scale_by_slope<VK>(d, z, a.act);
        }
#pragma unroll
        for (int e = 0; e < VK; e++) v[e] = (T)d[e];
      } else v = (V)in[j];
      if (!narrow && (tails >> j & 1)) v = move_down(v, VK - a.depth % VK, sizeof(T));
      *reinterpret_cast<V *>(s_x + lds_at[j]) = v;
    }
  };
  // This thread's pieces of the results: 16 bytes of a row, or (flat: rows of an odd length that stand one behind the other) of the
  // whole tile, which is then one row here.
  typedef typename Pack<TO, OE>::type Out;
  uint32_t out_row[NO];
  int out_col[NO];
  const int pieces = (width + OE - 1) / OE;
#pragma unroll
  for (int j = 0; j < NO; j++) {
    const int i = tid + j * THREADS;
    out_row[j] = sa.flat ? 0 : i / pieces;
    out_col[j] = (sa.flat ? i : i - (int)out_row[j] * pieces) * OE;
  }
  auto place = [&](auto *base, int64_t ld, int j) {
    typedef std::conditional_t<std::is_const_v<std::remove_pointer_t<decltype(base)>>, const char, char> Byte;
    return reinterpret_cast<decltype(base)>(reinterpret_cast<Byte *>(base) + (__umul24(out_row[j], (uint32_t)ld) + out_col[j]) * (uint32_t)sizeof(TO));
  };
  int64_t t = blockIdx.x;
  if (t < tiles) fetch(t);                   // on its way while W is laid out
  V w[KS][NTW];
#pragma unroll
  for (int k0 = 0; k0 < STEPS; k0 += PS) {
    __syncthreads();
    stage_weights<T, NT, GRAD>(a, reinterpret_cast<V *>(s_mem), k0 * kStep<T>, PS * kStep<T>, n0);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < PS; s++)
      if (WK == 1 || wk == (k0 + s) / KS)
#pragma unroll
        for (int i = 0; i < NTW; i++) w[(k0 + s) % KS][i] = reinterpret_cast<V *>(s_mem)[(s * NT + wn * NTW + i) * 64 + l];
  }
  __syncthreads();
  for (int i = tid; i < MR * P / 16; i += THREADS) reinterpret_cast<V *>(s_x)[i] = V{};      // past the depth it stays zero
  for (int i = tid; i < BN; i += THREADS) s_b[i] = !GRAD && a.bias && i < width ? (float)static_cast<const T *>(a.bias)[n0 + i] : 0.f;
  __syncthreads();                           // the zeros are there
  for (; t < tiles; t += gridDim.x) {
    put();
    __syncthreads();
    if (t + gridDim.x < tiles) fetch(t + gridDim.x);
    const int rows = (int)min((int64_t)MR, a.rows - t * MR);
    const int row_n = sa.flat ? 1 : rows, col_n = sa.flat ? rows * width : width;
    Out res[GRAD ? 1 : NO];
    if constexpr (!GRAD)
      if (a.res) {
        const TO *q = static_cast<const TO *>(a.res) + t * MR * a.ld_res + n0;
#pragma unroll
        for (int j = 0; j < NO; j++)
          if ((int)out_row[j] < row_n && out_col[j] + OE <= col_n) res[j] = *reinterpret_cast<const Out *>(place(q, a.ld_res, j));
      }
    f32x16 acc[NTW];
#pragma unroll
    for (int i = 0; i < NTW; i++) acc[i] = f32x16{};
    const char *xs = s_x + (wm * 32 + l % 32) * P + wk * (KS * 32) + half * 16;
#pragma unroll
    for (int k = 0; k < KS; k++) {
      const V x = *reinterpret_cast<const V *>(xs + k * 32);
#pragma unroll
      for (int i = 0; i < NTW; i++) acc[i] = mma(w[k][i], x, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < NTW; i++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int c = (wn * NTW + i) * 32 + 8 * e + 4 * half;
        F4 v = {acc[i][4 * e], acc[i][4 * e + 1], acc[i][4 * e + 2], acc[i][4 * e + 3]};
        if constexpr (!GRAD)
          if (wk == 0) v += *reinterpret_cast<const F4 *>(s_b + c);
        float *o = s_o + wk * PART + (wm * 32 + l % 32) * sa.pitch + c;
        if (!sa.flat) *reinterpret_cast<F4 *>(o) = v;
        else
#pragma unroll
          for (int j = 0; j < 4; j++)
            if (c + j < width) o[j] = v[j];
      }
    __syncthreads();
    TO *to = static_cast<TO *>(a.out) + t * MR * a.ld_out + n0;
    TO *keep = !GRAD && a.keep ? static_cast<TO *>(a.keep) + t * MR * a.ld_keep + n0 : nullptr;
#pragma unroll
    for (int j = 0; j < NO; j++) {
      if ((int)out_row[j] >= row_n || out_col[j] >= col_n) continue;
      const F4 *o = reinterpret_cast<const F4 *>(s_o + ((int)__umul24(out_row[j], (uint32_t)sa.pitch) + out_col[j]));
      float v[OE];
#pragma unroll
      for (int e = 0; e < OE; e++) v[e] = o[e / 4][e % 4];
#pragma unroll
      for (int q = 1; q < WK; q++)           // the parts of the depth, in order
#pragma unroll
        for (int e = 0; e < OE; e++) v[e] += o[q * (PART / 4) + e / 4][e % 4];
      const bool whole = out_col[j] + OE <= col_n;
      if constexpr (!GRAD) {
        if (keep && whole) store_pack<TO, OE>(place(keep, a.ld_keep, j), v);
        if (keep && !whole)
#pragma unroll
          for (int e = 0; e < OE; e++)
            if (out_col[j] + e < col_n) place(keep, a.ld_keep, j)[e] = (TO)v[e];
        activate_all<OE>(v, a.act);
        if (a.res) {
          if (whole)
#pragma unroll
            for (int e = 0; e < OE; e++) v[e] += (float)res[j][e];
          else {
            const TO *q = place(static_cast<const TO *>(a.res) + t * MR * a.ld_res + n0, a.ld_res, j);
#pragma unroll
            for (int e = 0; e < OE; e++)
              if (out_col[j] + e < col_n) v[e] += (float)q[e];
          }
        }
      }
      if (whole) store_pack<TO, OE>(place(to, a.ld_out, j), v);
      else
#pragma unroll
        for (int e = 0; e < OE; e++)
          if (out_col[j] + e < col_n) place(to, a.ld_out, j)[e] = (TO)v[e];
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

// ------------------------------------------------------------------------------------ gradient
// dweight = x^T dz and dbias over a slice of the rows, and (DX) dx = dz W^T of its rows on the way, so that dy, z and x are read once.
// A workgroup has the sums of 32 KT columns of x by 32 NT of dz in registers, (KT / 2) (NT / 2) tiles a wave, and takes 32 rows at a time
// (64 with eight waves, which larger tiles take), one piece ahead in registers.  All threads load x, dy and z side by side, 16 bytes a lane, form dz once and put both into LDS row by row.  The
// sums run over the rows, so their fragments are columns: 16-bit ones come from the transposing LDS read, 32-bit ones element by
// element.  The partial sums are left in the fragments' order and k_grad_sum puts them where they belong.  dbias without dweight takes the
// same kernel, whose products are then of zeros.
// 612k x 128 x 172 bf16: without an activation 142 us (3.7 TB/s of the bytes it cannot do without), with gelu 198: the slope is formed once an
// element, and its 25 instructions are what bounds that.
struct GradArgs {
  const void *x, *dy, *pre, *weight;
  void *dx;
  float *part, *part_bias;                   // fragments of [slices][tiles][KT][NT], or NULL; [slices][32 NT tiles], or NULL
  int64_t rows, ld_x, ld_dy, ld_pre, ld_w, ld_dx, slice;
  int cols, out, act;
};

template <class T, class TI, int KT, int NT, int WAVES, bool DX>
__global__ __launch_bounds__(kWave * WAVES, 2) void k_linear_grad(GradArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int ROWS = 8 * WAVES, THREADS = kWave * WAVES, WN = WAVES / 2;     // waves: two by the columns of x, WN by those of dz
  constexpr int VK = kVec<T>, STEPS = ROWS / kStep<T>, CX = KT * 32 / VK, CZ = NT * 32 / VK;      // pieces of a row
  constexpr int NX = ROWS * CX / THREADS, NZ = ROWS * CZ / THREADS;
  constexpr int KP = KT / 2, NP = NT / WN, DP = (KT + WAVES - 1) / WAVES, DS = CZ / 2;      // tiles a wave; column tiles of dx a wave, steps of its depth
  constexpr int PX = kGradPitch<T, KT>, PZ = kGradPitch<T, NT>, PD = KT * 32 + 4, PB = NT * 32 + 4;
  constexpr int kLds = ROWS * (PX + PZ + (DX ? PD * 4 : 0)), kLdsBias = ROWS * PB * 4;
  static_assert(KT % 2 == 0 && NT % WN == 0 && (!DX || WAVES == 4), "every wave has its tiles; dx is formed of 32 rows");
  __shared__ __align__(16) char s_mem[kLds > kLdsBias ? kLds : kLdsBias];
  __shared__ __align__(16) float s_db[NZ * VK > 16 ? ROWS * PB : 1];
  char *s_x = s_mem, *s_z = s_mem + ROWS * PX;
  float *s_dx = reinterpret_cast<float *>(s_z + ROWS * PZ);
  const int tid = threadIdx.x, l = lane_id(), half = l / 32, wave = tid / kWave;
  const int k0 = blockIdx.x * (KT * 32), n0 = blockIdx.y * (NT * 32);
  const int64_t r_begin = blockIdx.z * a.slice, r_end = min(r_begin + a.slice, a.rows);
  const int x_cols = a.x ? a.cols : 0;
  V w[DX ? DP : 1][DX ? DS : 1];
  if constexpr (DX)
#pragma unroll
    for (int i = 0; i < DP; i++)
#pragma unroll
      for (int s = 0; s < DS; s++) {
        const int k = (wave + WAVES * i) * 32 + l % 32, n = s * kStep<T> + half * VK;
        w[i][s] = V{};
        if (k < a.cols && n < a.out) w[i][s] = row_frag<T>(static_cast<const T *>(a.weight) + (int64_t)k * a.ld_w, n, a.out);
      }
  f32x16 acc[KP][NP];
#pragma unroll
  for (int i = 0; i < KP; i++)
#pragma unroll
    for (int j = 0; j < NP; j++) acc[i][j] = f32x16{};
  // Eight threads share a row: pieces tid % 8, + 8, ... of row tid / 8.  A piece that the matrix's end cuts starts earlier and is moved
  // down; one past it, or of a row past the slice, is not loaded and put down as zero.
  typedef typename Pack<T, VK>::type PT;
  typedef typename Pack<TI, VK>::type PI;
  const int my_row = tid / 8, my_piece = tid % 8;
  const T *xp = static_cast<const T *>(a.x) + (a.x ? (r_begin + my_row) * a.ld_x : 0);
  const TI *yp = static_cast<const TI *>(a.dy) + (r_begin + my_row) * a.ld_dy, *zp = static_cast<const TI *>(a.pre) + (a.pre ? (r_begin + my_row) * a.ld_pre : 0);
  PT x[NX];
  PI dy[NZ], pre[NZ];
  // Column sums of dz: in registers, or, where those are wanted elsewhere, in LDS, each place this thread's own.
  constexpr bool DB_LDS = NZ * VK > 16;
  float db[DB_LDS ? 1 : NZ][VK];
#pragma unroll
  for (int j = 0; j < NZ; j++)
#pragma unroll
    for (int e = 0; e < VK; e++) {
      if constexpr (DB_LDS) s_db[my_row * PB + (my_piece + 8 * j) * VK + e] = 0.f;
      else db[j][e] = 0.f;
    }
  auto load = [&](auto *row, int c, int n) {
    typedef std::remove_const_t<std::remove_pointer_t<decltype(row)>> E;
    typedef typename Pack<E, VK>::type P;
    if (n >= VK) return *reinterpret_cast<const P *>(row + min(c, n - VK));
    P v;
#pragma unroll
    for (int e = 0; e < VK; e++) v[e] = e < n ? row[e] : (E)0.f;
    return v;
  };
  auto fetch = [&](int64_t left) {           // rows left in the slice
    if (my_row < left) {
#pragma unroll
      for (int j = 0; j < NX; j++) {
        const int c = k0 + (my_piece + 8 * j) * VK;
        if (c < x_cols) x[j] = load(xp, c, x_cols);
      }
#pragma unroll
      for (int j = 0; j < NZ; j++) {
        const int c = n0 + (my_piece + 8 * j) * VK;
        if (c < a.out) {
          dy[j] = load(yp, c, a.out);
          if (a.act != INK_ACT_NONE) pre[j] = load(zp, c, a.out);
        }
      }
    }
    xp += ROWS * a.ld_x;
    yp += ROWS * a.ld_dy;
    zp += ROWS * a.ld_pre;
  };
  auto put = [&](int64_t left) {
#pragma unroll
    for (int j = 0; j < NX; j++) {
      const int c = k0 + (my_piece + 8 * j) * VK;
      V v{};
      if (my_row < left && c < x_cols) {
        v = (V)x[j];
        if (c + VK > x_cols && x_cols >= VK) v = move_down(v, c + VK - x_cols, sizeof(T));
      }
      *reinterpret_cast<V *>(s_x + my_row * PX + (my_piece + 8 * j) * 16) = v;
    }
#pragma unroll
    for (int j = 0; j < NZ; j++) {
      const int c = n0 + (my_piece + 8 * j) * VK;
      V v{};
      if (my_row < left && c < a.out) {
        float d[VK];
#pragma unroll
        for (int e = 0; e < VK; e++) d[e] = (float)dy[j][e];
        if (a.act != INK_ACT_NONE) {
          float z[VK];
#pragma unroll
          for (int e = 0; e < VK; e++) z[e] = (float)pre[j][e];
          scale_by_slope<VK>(d, z, a.act);
        }
#pragma unroll
        for (int e = 0; e < VK; e++) {
          if constexpr (DB_LDS) s_db[my_row * PB + (my_piece + 8 * j) * VK + e] += d[e];
          else db[j][e] += d[e];
          v[e] = (T)d[e];
        }
        if (c + VK > a.out && a.out >= VK) v = move_down(v, c + VK - a.out, sizeof(T));
      }
      *reinterpret_cast<V *>(s_z + my_row * PZ + (my_piece + 8 * j) * 16) = v;
    }
  };
  if (r_begin < r_end) fetch(r_end - r_begin);
  for (int64_t r0 = r_begin; r0 < r_end; r0 += ROWS) {
    put(r_end - r0);
    __syncthreads();
    if (r0 + ROWS < r_end) fetch(r_end - r0 - ROWS);
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      V zs[NP], xs[KP];
#pragma unroll
      for (int j = 0; j < NP; j++) zs[j] = columns_frag<T>(s_z, PZ, s, wave / 2 * NP + j);
#pragma unroll
      for (int i = 0; i < KP; i++) xs[i] = columns_frag<T>(s_x, PX, s, wave % 2 * KP + i);
      mma_block<T>(zs, xs, acc);
    }
    if constexpr (DX) {
#pragma unroll
      for (int i = 0; i < DP; i++) {
        if (wave + WAVES * i >= KT) continue;
        f32x16 d = f32x16{};
#pragma unroll
        for (int s = 0; s < DS; s++) d = mma(w[i][s], *reinterpret_cast<const V *>(s_z + l % 32 * PZ + (2 * s + half) * 16), d);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const F4 v = {d[4 * e], d[4 * e + 1], d[4 * e + 2], d[4 * e + 3]};
          *reinterpret_cast<F4 *>(s_dx + (l % 32) * PD + (wave + WAVES * i) * 32 + 8 * e + 4 * half) = v;
        }
      }
    }
    __syncthreads();
    if constexpr (DX) {
      const int rows = (int)min((int64_t)ROWS, r_end - r0);
#pragma unroll
      for (int j = 0; j < NX; j++) {
        const int c = (my_piece + 8 * j) * VK;
        if (my_row >= rows || c >= a.cols) continue;
        const F4 *o = reinterpret_cast<const F4 *>(s_dx + my_row * PD + c);
        T *to = static_cast<T *>(a.dx) + (r0 + my_row) * a.ld_dx + c;
        float v[VK];
#pragma unroll
        for (int e = 0; e < VK; e++) v[e] = o[e / 4][e % 4];
        if (c + VK <= a.cols) store_pack<T, VK>(to, v);
        else
#pragma unroll
          for (int e = 0; e < VK; e++)
            if (c + e < a.cols) to[e] = (T)v[e];
      }
    }
  }
  const int64_t tile = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * gridDim.y + blockIdx.y;
  if (a.part) {
    float *part = a.part + tile * (KT * NT * 1024);
#pragma unroll
    for (int i = 0; i < KP; i++)
#pragma unroll
      for (int j = 0; j < NP; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const F4 v = {acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
          reinterpret_cast<F4 *>(part)[(((wave % 2 * KP + i) * NT + wave / 2 * NP + j) * 4 + e) * 64 + l] = v;
        }
  }
  if (!a.part_bias || blockIdx.x) return;
  // column sums of dz: each thread's of its row's pieces, over the ROWS rows.  A moved piece's first columns belong to the one before.
  float *s_sum = DB_LDS ? s_db : reinterpret_cast<float *>(s_mem);           // [ROWS][PB]
  float own[NZ][VK];
#pragma unroll
  for (int j = 0; j < NZ; j++)
#pragma unroll
    for (int e = 0; e < VK; e++) {
      if constexpr (DB_LDS) own[j][e] = s_db[my_row * PB + (my_piece + 8 * j) * VK + e];
      else own[j][e] = db[j][e];
    }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < NZ; j++) {
    const int cb = my_piece + 8 * j, c = n0 + cb * VK, over = c + VK > a.out && a.out >= VK ? c + VK - a.out : 0;
#pragma unroll
    for (int e = 0; e < VK; e++)
      if (c < a.out && e >= over && c - over + e < a.out) s_sum[my_row * PB + cb * VK + e - over] = own[j][e];
  }
  __syncthreads();
  for (int c = tid; c < NT * 32; c += THREADS) {
    if (n0 + c >= a.out) continue;
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; r++) t += s_sum[r * PB + c];
    a.part_bias[((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * (NT * 32) + c] = t;
  }
}

// Partial sums of all slices: 64 elements, four by four, a workgroup; 16 threads share a sum.  The last workgroups do the bias.
struct GradSumArgs {
  const float *part, *part_bias;
  void *dweight, *dbias;
  int64_t ld_dw;
  int slices, type, cols, out, kt, nt, tiles_k, tiles_n, weight_groups;
};
__global__ __launch_bounds__(256) void k_grad_sum(GradSumArgs a) {
  __shared__ F4 s[16][17];
  const int x = threadIdx.x % 16, y = threadIdx.x / 16;
  const bool bias = (int)blockIdx.x >= a.weight_groups;
  const int64_t n = bias ? (int64_t)a.tiles_n * a.nt * 32 : (int64_t)a.tiles_k * a.tiles_n * a.kt * a.nt * 1024;
  const float *part = bias ? a.part_bias : a.part;
  const int64_t i = ((int64_t)(bias ? blockIdx.x - a.weight_groups : blockIdx.x) * 16 + x) * 4;
  F4 t = F4{};
  if (i < n)
#pragma unroll 8
    for (int p = y; p < a.slices; p += 16) t += *reinterpret_cast<const F4 *>(part + p * n + i);
  s[y][x] = t;
  __syncthreads();
  if (y || i >= n) return;
  t = F4{};
#pragma unroll
  for (int p = 0; p < 16; p++) t += s[p][x];
  if (bias) {
    for (int e = 0; e < 4; e++)
      if (i + e < a.out) store_any(a.dbias, i + e, a.type, t[e]);
    return;
  }
  const int per = a.kt * a.nt * 1024, tile = (int)(i / per), f = (int)(i - (int64_t)tile * per), frag = f / 1024, e = f / 256 % 4, lane = f / 4 % 64;
  const int tk = tile / a.tiles_n, tn = tile - tk * a.tiles_n, fk = frag / a.nt, fn = frag - fk * a.nt;
  const int k = (tk * a.kt + fk) * 32 + lane % 32, c = (tn * a.nt + fn) * 32 + 8 * e + 4 * (lane / 32);
  if (k >= a.cols) return;
  for (int j = 0; j < 4; j++)
    if (c + j < a.out) store_any(a.dweight, (int64_t)k * a.ld_dw + c + j, a.type, t[j]);
}

// ------------------------------------------------------------------------------------ host side
// Rows that workgroups take one by one (k_linear_few), each asking for all of W.  Both kernels' time goes with the depth; what is asked for again comes on
// top, so the limit is on rows times columns.  us a call, k_linear_few and k_linear_small: bf16 4096 x 4096 16 rows (at the limit) 35 and 76, 32 rows 83
// and 77; 16384 x 16384 4 rows 391 and 492, 8 rows 913 and 491, 64 rows 9720 and 536; 256 x 16384 4 rows 8.7 and 8.6, 64 rows 54 and 10; 16384 x 256
// 64 rows 91 and 331; f32 4096 x 4096 16 rows 42 and 46, 32 rows 86 and 50; 16384 x 16384 4 rows 296 and 316, 8 rows 719 and 318.
constexpr int64_t kFewRows = 64, kFewResults = 64 * 1024;
constexpr int64_t kStreamRows = 32 * 1024;   // rows from which on a workgroup that lays out W for itself takes several tiles
template <class T, class TI, class TO, int KS, int NTW, int WN, int WM, int WK, int PER, bool GRAD>
static void stream_launch(const LinearArgs &a, Launches &run) {
  constexpr int MR = 32 * WM, BN = 32 * NTW * WN, OE = 16 / (int)sizeof(TO), WAVES = WN * WM * WK;
  StreamArgs s{a, (a.depth + kVec<T> - 1) / kVec<T>, BN + 4, 0};
  s.flat = a.width <= BN && a.width % OE != 0 && a.ld_out == a.width && (!a.keep || a.ld_keep == a.width) && (!a.res || a.ld_res == a.width);
  if (s.flat) s.pitch = a.width;
  const unsigned gy = (unsigned)((a.width + BN - 1) / BN);
  const int64_t tiles = (a.rows + MR - 1) / MR;
  constexpr int lds = MR * (KS * WK * 32 + 16) + WK * MR * (BN + 4) * 4 + BN * 4;
  static_assert(lds <= 160 << 10 && lds >= 4 * BN * 32, "LDS holds the tiles, and W's pieces on their way to the registers");
  constexpr int per_cu = std::max(1, std::min((160 << 10) / lds, 4 * PER / WAVES));
  run.lds = lds;
  run(k_linear_stream<T, TI, TO, KS, NTW, WN, WM, WK, PER, GRAD>, dim3((unsigned)std::min<int64_t>(tiles, std::max(1u, 256 * per_cu / gy)), gy),
      dim3(kWave * WAVES), s);
  run.lds = 0;
}
// whether the rows are so many that a workgroup takes several tiles, and W fits the registers
template <class T, class TI, class TO, bool GRAD> static bool stream_run(const LinearArgs &a, Launches &run) {
  if (a.rows < kStreamRows) return false;
  for (const int64_t ld : {a.ld_in, a.ld_pre, a.ld_res, a.ld_out, a.ld_keep})
    if (ld >= 1 << 22) return false;         // offsets within a tile are 32-bit
  const int steps = (a.depth + kStep<T> - 1) / kStep<T>;
  if constexpr (sizeof(T) == 2) {
    if (steps <= 8) {
      if (a.width <= 64) stream_launch<T, TI, TO, 8, 1, 2, 2, 1, 2, GRAD>(a, run);
      else if (a.width <= 128) stream_launch<T, TI, TO, 8, 2, 2, 2, 1, 2, GRAD>(a, run);
      else stream_launch<T, TI, TO, 8, 2, 4, 1, 1, 2, GRAD>(a, run);
    } else if (steps <= 16) {
      if (a.width <= 64) stream_launch<T, TI, TO, 8, 1, 2, 1, 2, 4, GRAD>(a, run);
      else if (a.width <= 128) stream_launch<T, TI, TO, 16, 1, 4, 1, 1, 2, GRAD>(a, run);
      else stream_launch<T, TI, TO, 16, 1, 8, 1, 1, 2, GRAD>(a, run);
    } else if (steps <= 40) {
      if (a.width <= 64) stream_launch<T, TI, TO, 10, 1, 2, 1, 4, 2, GRAD>(a, run);
      else if (a.width <= 128) stream_launch<T, TI, TO, 20, 1, 4, 1, 2, 2, GRAD>(a, run);
      else stream_launch<T, TI, TO, 40, 1, 8, 1, 1, 2, GRAD>(a, run);
    } else return false;
  } else {
    if (steps <= 16) {
      if (a.width <= 64) stream_launch<T, TI, TO, 8, 1, 2, 1, 2, 4, GRAD>(a, run);
      else if (a.width <= 128) stream_launch<T, TI, TO, 16, 1, 4, 1, 1, 2, GRAD>(a, run);
      else stream_launch<T, TI, TO, 16, 1, 8, 1, 1, 2, GRAD>(a, run);
    } else if (steps <= 32) {
      if (a.width <= 64) stream_launch<T, TI, TO, 16, 1, 2, 1, 2, 2, GRAD>(a, run);
      else if (a.width <= 128) stream_launch<T, TI, TO, 16, 1, 4, 1, 2, 2, GRAD>(a, run);
      else stream_launch<T, TI, TO, 32, 1, 8, 1, 1, 2, GRAD>(a, run);
    } else return false;
  }
  return true;
}

template <class T, class TI, class TO, bool GRAD> static void linear_run(const LinearArgs &a, Launches &run) {
  if constexpr (!GRAD)
    if (a.rows <= kFewRows && a.rows * a.width <= kFewResults) return run(k_linear_few<T, TO>, dim3((a.width + 31) / 32, (unsigned)a.rows), dim3(kHeadThreads), a);
  if (stream_run<T, TI, TO, GRAD>(a, run)) return;
  const int64_t tiles = (a.rows + 127) / 128;
  const int ntw = a.width <= 64 ? 1 : 2, gy = (a.width + 64 * ntw - 1) / (64 * ntw);
  if (tiles * gy < 256) {
    const dim3 grid((unsigned)((a.rows + 31) / 32), (a.width + 31) / 32);
    return run(k_linear_small<T, TI, TO, GRAD>, grid, dim3(kWave * kSmallWaves), a);
  }
  const dim3 grid((unsigned)((tiles + 7) / 8 * 8 * gy));
  run(ntw == 1 ? k_linear_tile<T, TI, TO, 1, GRAD> : k_linear_tile<T, TI, TO, 2, GRAD>, grid, dim3(256), a);
}

// How the gradient's sums are cut: tiles of 32 kt columns by 32 nt of dz, and slices of the rows, two workgroups of four waves a CU or one
// of eight.  `wide`: 16-bit rows, whose registers leave room for tiles of 256 columns of x; dy and z, read again for every such tile, are
// then read half as often.  bf16, four waves and eight: 612k x 256 x 256 with gelu 695 and 604 us, 612k x 256 x 100 330 and 297, 100k x 1000 x 500
// 820 and 764, but 128 x 256 (one tile of x either way) 402 and 408, and 10000 rows 39 and 46.
struct GradPlan { int kt, nt, waves, tiles_k, tiles_n, slices; int64_t slice, part, part_bias; bool whole; };
static GradPlan grad_plan(int64_t rows, int cols, int out, bool wide) {
  GradPlan p{};
  const int k = (cols + 31) / 32, n = (out + 31) / 32;
  p.waves = 4;
  p.kt = k <= 2 ? 2 : k <= 4 || n > 2 ? 4 : 8;
  p.nt = p.kt == 8 || n <= 2 ? 2 : n <= 4 ? 4 : n <= 6 ? 6 : 4;
  if (wide && rows >= kStreamRows && k > 4 && n > 2) {
    p.waves = 8;
    p.kt = 8;
    p.nt = n > 4 ? 8 : 4;
  }
  p.tiles_k = (k + p.kt - 1) / p.kt;
  p.tiles_n = (n + p.nt - 1) / p.nt;
  p.whole = p.tiles_k == 1 && p.tiles_n == 1;
  const int per = 8 * p.waves;               // rows at a time
  const int64_t blocks = (rows + per - 1) / per, tiles = (int64_t)p.tiles_k * p.tiles_n;
  const int64_t slices = std::max<int64_t>(1, std::min<int64_t>((blocks + 1) / 2, 2048 / p.waves / tiles));
  p.slice = (blocks + slices - 1) / slices * per;
  p.slices = (int)((rows + p.slice - 1) / p.slice);
  p.part = p.slices * tiles * p.kt * p.nt * 1024;
  p.part_bias = (int64_t)p.slices * p.tiles_n * p.nt * 32;
  return p;
}

template <class T, class TI, int KT, int NT> static void grad_launch(const GradArgs &a, const GradPlan &p, Launches &run) {
  const dim3 grid(p.tiles_k, p.tiles_n, p.slices);
  if constexpr (sizeof(T) == sizeof(TI) && (sizeof(T) == 2 || NT <= 4))
    if (a.dx) return run(k_linear_grad<T, TI, KT, NT, 4, true>, grid, dim3(kWave * 4), a);
  run(k_linear_grad<T, TI, KT, NT, 4, false>, grid, dim3(kWave * 4), a);
}
template <class T, class TI> static void grad_run(const GradArgs &a, const GradPlan &p, Launches &run) {
  if constexpr (sizeof(T) == 2 && sizeof(TI) == 2)
    if (p.waves == 8) {
      const dim3 grid(p.tiles_k, p.tiles_n, p.slices), block(kWave * 8);
      return run(p.nt == 8 ? k_linear_grad<T, TI, 8, 8, 8, false> : k_linear_grad<T, TI, 8, 4, 8, false>, grid, block, a);
    }
  if (p.kt == 8) return grad_launch<T, TI, 8, 2>(a, p, run);
  if (p.kt == 2) {
    if (p.nt == 2) return grad_launch<T, TI, 2, 2>(a, p, run);
    if (p.nt == 4) return grad_launch<T, TI, 2, 4>(a, p, run);
    return grad_launch<T, TI, 2, 6>(a, p, run);
  }
  if (p.nt == 2) return grad_launch<T, TI, 4, 2>(a, p, run);
  if (p.nt == 4) return grad_launch<T, TI, 4, 4>(a, p, run);
  grad_launch<T, TI, 4, 6>(a, p, run);
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
  const GradPlan p = grad_plan(rows, cols, out, false), q = grad_plan(rows, cols, out, true);     // enough for every type
  return (size_t)std::max(p.part + p.part_bias, q.part + q.part_bias) * sizeof(float);
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
  GradPlan p{};
  if (rows > 0) p = grad_plan(rows, cols, out, type != INK_F32 && type == dy_type);
  // dx in the same pass where one workgroup has all columns of both matrices and, in 32 bits, the registers for it
  const bool sums = dweight || dbias, together = dx && sums && rows > 0 && p.whole && p.waves == 4 && type == dy_type && (type != INK_F32 || p.nt <= 4);
  if (act == INK_ACT_NONE) pre = nullptr;
  if (dx && rows > 0 && !together) {
    LinearArgs a{};
    a.in = dy; a.pre = pre; a.weight = weight; a.out = dx;
    a.rows = rows; a.ld_in = ld_dy; a.ld_pre = ld_pre; a.ld_w = ld_w; a.ld_out = ld_dx;
    a.depth = out; a.width = cols; a.act = act;
    if (type == INK_F32) linear_run<float, float, float, true>(a, run);
    else if (type == INK_F16) linear_run<f16, f16, f16, true>(a, run);
    else dy_type == INK_F32 ? linear_run<bf16, float, bf16, true>(a, run) : linear_run<bf16, bf16, bf16, true>(a, run);
  }
  if (sums) {
    GradSumArgs s{};
    s.type = type; s.cols = cols; s.out = out; s.dweight = dweight; s.dbias = dbias; s.ld_dw = ld_dw;
    s.kt = s.nt = 2; s.tiles_k = (cols + 63) / 64; s.tiles_n = (out + 63) / 64;        // no rows: zeros
    if (rows > 0) {
      GradArgs a{};
      a.x = x; a.dy = dy; a.pre = pre; a.weight = weight; a.dx = together ? dx : nullptr;
      a.part = dweight ? static_cast<float *>(work) : nullptr;
      a.part_bias = dbias ? static_cast<float *>(work) + p.part : nullptr;
      a.rows = rows; a.ld_x = ld_x; a.ld_dy = ld_dy; a.ld_pre = ld_pre; a.ld_w = ld_w; a.ld_dx = ld_dx; a.slice = p.slice;
      a.cols = cols; a.out = out; a.act = act;
      if (!dweight) a.x = nullptr;           // not read
      if (type == INK_F32) grad_run<float, float>(a, p, run);
      else if (type == INK_F16) grad_run<f16, f16>(a, p, run);
      else dy_type == INK_F32 ? grad_run<bf16, float>(a, p, run) : grad_run<bf16, bf16>(a, p, run);
      s.part = a.part; s.part_bias = a.part_bias; s.slices = p.slices;
      s.kt = p.kt; s.nt = p.nt; s.tiles_k = p.tiles_k; s.tiles_n = p.tiles_n;
    }
    s.weight_groups = dweight ? s.tiles_k * s.tiles_n * s.kt * s.nt * 16 : 0;
    const int bias_groups = dbias ? (s.tiles_n * s.nt + 1) / 2 : 0;
    run(k_grad_sum, dim3(s.weight_groups + bias_groups), dim3(256), s);
  }
  return run.done(who);
}
