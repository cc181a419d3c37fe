// The gated pair of projections, h = act(x Wg) * (x Wu), and its gradient.
//
//   forward   g = x Wg, u = x Wu (8-bit rows and weights: times the row's and the column's scale),  h = act(g) u
//   gradient  g and u formed anew from x;  dg = dh u act'(g), du = dh act(g);
//             dx = dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du
//
// As in linear.hip every product is formed transposed, the weights' columns as the instruction's rows, so that a lane ends up with four
// neighbouring columns of its row, here of g and of u: act(g) u needs nothing of another lane.  Which kernel, forward:
//
//   up to 16 rows, 64k results   k_gated_few     a row and 32 columns a workgroup; the weights are what is read: 1 x 256 x 683 bf16 6 us; not of 8-bit rows
//   from 16384 or 32768 rows on  k_gated_stream  the weights in registers, rows in a stream; depths of up to 256 (16 bits), 128 (32 bits) or 512 (8 bits, with
//                                                16-bit results)
//   else                         k_gated_tile    128 rows by 64 columns, both operands through LDS; 32-bit results of 8-bit rows at any size
//
// What bounds the stream: reading rows and writing h (16 bits, 128 columns), the vector instructions of the activation (8 bits, whose products take a
// quarter of the time), the matrix unit (32 bits).  Figures at each kernel.
//
// The gradient does not keep g and u: forming them again costs 4 rows cols hidden operations, keeping them 8 bytes an element of h written and
// read (1M x 128 x 344 bf16: 0.16 ms of the matrix unit against 0.55 ms of memory).  dg and du are left in work memory once, in the rows' type, for the two
// products that read them: an error of the size of the results' own rounding (233k x 256 x 683 bf16 0.0024 from 64 bits where rounding the results alone
// gives 0.0017).  float16 rows keep their range besides (GatedRange).  A few rows are kept in 32 bits.  The weights' gradients are sums over all
// rows: workgroups take slices of the rows and leave a partial matrix each, added up in order (no atomics: the same call gives the same bits).
#include <algorithm>
#include <type_traits>

#include "matrix.h"

namespace ink {

// 8-bit operands.  The matrix instructions of 8-bit floats add the products of eight neighbouring places (k = 8 i .. 8 i + 7) in units of 2^-13 of the
// largest 2^(e_x + e_w) of the eight, e being a number's exponent and -6 for numbers below 2^-6, and drop what lies below; the eights, and what was summed before,
// are added in 32 bits.  Measured: beside 448 * 448 and its negative a product of 8 counts, one of 7.5 does not, and in another eight it does.  So each of seven
// products loses less than 2^-13 of the largest max(|x|, 2^-6) max(|w|, 2^-6), typically 1.4e-5 of a sum of 64 to 1024 products: beside what rounding rows and weights to
// 8 bits has cost (2^-4 of each number) little, a hundredth of a bfloat16 result's rounding and a tenth of a float16 one's; but of a sum whose large products cancel it may
// be all that is left.  That is taken for 16-bit results, and said in the header; 32-bit results are formed in bfloat16, which holds every e4m3 number and
// whose products and sums are exact and in 32 bits, at 2.5 times the time (612.5k x 256 x 1024: 620 us to float16, 1581 to 32 bits).
typedef uint8_t e4m3;                        // held as its bits
template <> struct Frag<e4m3> { typedef int V __attribute__((ext_vector_type(8))); };      // 32 elements a lane
__device__ __forceinline__ f32x16 mma(Frag<e4m3>::V a, Frag<e4m3>::V b, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);       // both e4m3, no block scales
}

typedef int Piece __attribute__((ext_vector_type(4)));                // 16 bytes
typedef int PieceAny __attribute__((ext_vector_type(4), aligned(1)));

// Elements k .. of a row of n elements of TL, as many as a piece of T holds (8-bit numbers may become 16-bit ones on the way); past the row's end
// zeros, and nothing is read there.  In two steps, so that nothing waits for the load where it is asked for: a piece that the row's
// end cuts is the row's last bytes, which piece_of moves down.  SHORT: rows that hold no whole piece, element by element.
template <class TL, class T> struct RawOf { typedef Piece V; };
template <> struct RawOf<e4m3, bf16> { typedef uint64_t V; };
template <class TL, class T, bool SHORT> __device__ __forceinline__ typename RawOf<TL, T>::V raw_piece(const TL *row, int k, int n) {
  typedef typename RawOf<TL, T>::V V;
  constexpr int N = sizeof(V) / sizeof(TL);
  if constexpr (SHORT) {
    typedef std::conditional_t<sizeof(TL) == 1, uint8_t, std::conditional_t<sizeof(TL) == 2, uint16_t, uint32_t>> Bits;
    unsigned __int128 v = 0;
#pragma unroll
    for (int j = 0; j < N; j++)
      if (k + j < n) v |= (unsigned __int128)reinterpret_cast<const Bits *>(row)[k + j] << (8 * sizeof(TL) * j);
    if constexpr (sizeof(V) == 8) return (uint64_t)v;
    else return __builtin_bit_cast(Piece, v);
  } else if constexpr (sizeof(V) == 8) {
    typedef uint64_t W __attribute__((aligned(1)));
    return *reinterpret_cast<const W *>(row + min(k, n - N));
  } else return (Piece)*reinterpret_cast<const PieceAny *>(row + min(k, n - N));
}
template <class TL, class T, bool SHORT> __device__ __forceinline__ Piece piece_of(typename RawOf<TL, T>::V v, int k, int n) {
  typedef typename RawOf<TL, T>::V V;
  constexpr int N = sizeof(V) / sizeof(TL);
  if constexpr (!SHORT)
    if (k + N > n) {
      if constexpr (sizeof(V) == 8) v = k < n ? v >> 8 * (k + N - n) : 0;
      else v = k < n ? move_down(v, k + N - n, sizeof(TL)) : Piece{};
    }
  if constexpr (sizeof(V) == 8) {
    typedef T R __attribute__((ext_vector_type(8)));
    R r;
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int w = (int)(uint32_t)(v >> 32 * j);
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
      r[4 * j] = (T)lo[0]; r[4 * j + 1] = (T)lo[1]; r[4 * j + 2] = (T)hi[0]; r[4 * j + 3] = (T)hi[1];
    }
    return __builtin_bit_cast(Piece, r);
  } else return v;
}

// The range of dg and du of float16 rows: both may pass 65504, or lie below 2^-24 where many of them or a large weight make a result of them.
// So 32 rows by 32 columns of them, a block, are held in units of 2^K.  K is 0 while the block's largest number lies between 2^-4 and 65504, and every number is
// then what its rounding gives; else a multiple of 4 or 16, so that neighbouring blocks mostly agree.  A row of the block whose largest number would fall below 2^-12 there, and any
// row of up to 65504 in a block beyond it, has units 2^-d times as large, so that a row beside one of quite another size keeps its own numbers: dx is formed
// row by row.  For the sums over rows all are brought to the block's units.  The sums of products change their units, by a power of two, where the next block has others.
// What it costs: 233k x 256 x 683 906 -> 944 us, 1M x 128 x 344 1297 -> 1412 us, most of it in the forming of dg and du; with sizes that differ from row to row by up to
// 2^23 1230 and 1814 us.
struct GatedRange {
  int32_t *unit;                             // [row blocks][across]: 2 K, and 1 more where a row has units of its own
  uint8_t *finer;                            // [row blocks][across][32]: d of the block's rows, written where that is so
  int across;                                // blocks side by side: dg's, then du's
};
template <class T> constexpr bool kRanged = std::is_same_v<T, f16>;

__device__ __forceinline__ int exponent_of(float a) { return (int)(__float_as_uint(a) >> 23) - 127; }            // of a >= 0
__device__ __forceinline__ int unit_for(float top) {
  const int e = exponent_of(top);
  return top > 65504.f ? (e - 10) / 4 * 4 : top > 0.f && e < -4 ? -((11 - e) / 16 * 16) : 0;
}
// Brings 16 numbers a lane, lanes l and l ^ 32 a row's 32, a wave a block's, to their units, and writes these down.  Infinities and NaN stay and do not count.
__device__ __forceinline__ void to_units(float v[16], const GatedRange &range, int64_t row_block, int column_block) {
  const int64_t block = row_block * range.across + column_block;
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 16; j++) top = fmaxf(top, fabsf(v[j]));                   // the larger of a NaN and a number is the number
  // Units of 1 for all, as a rule: seen by comparisons alone (with the reductions below for every block 233k x 256 x 683 973 us instead of 944)
  int code = 0;
  const bool ordinary = __builtin_amdgcn_ballot_w64(top >= 0.000244140625f || top == 0.f) == ~0ull;
  if (!ordinary || __builtin_amdgcn_ballot_w64(top > 65504.f) || !__builtin_amdgcn_ballot_w64(top >= 0.0625f)) {
    if (__builtin_amdgcn_ballot_w64(top == INFINITY)) {
      top = 0.f;
#pragma unroll
      for (int j = 0; j < 16; j++) top = fmaxf(top, fabsf(v[j]) <= 3.4028235e38f ? fabsf(v[j]) : 0.f);
    }
    const auto larger = [](float a, float b) { return fmaxf(a, b); };
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const int unit = __builtin_amdgcn_readfirstlane(unit_for(group_all<32>(top, larger)));
    const int calm = min(unit, 0), finer = unit - (top > 65504.f || (top > 0.f && exponent_of(top) - calm < -12) ? unit_for(top) : calm);
    const bool uneven = __builtin_amdgcn_ballot_w64(finer != 0) != 0;
#pragma unroll
    for (int j = 0; j < 16; j++) v[j] = __builtin_amdgcn_ldexpf(v[j], finer - unit);
    if (uneven) range.finer[block * 32 + lane_id() % 32] = (uint8_t)finer;
    code = 2 * unit + uneven;
  }
  range.unit[block] = code;                  // by all lanes: a store under a condition would make the next wait for rows one for all stores
}
// A product's sums so far from units of 2^was to those of 2^unit
template <int N> __device__ __forceinline__ void change_units(f32x16 (&acc)[N], int was, int unit) {
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int e = 0; e < 16; e++) acc[n][e] = __builtin_amdgcn_ldexpf(acc[n][e], was - unit);
}

struct GatedArgs {
  const void *x, *gate, *up, *dh;
  const float *x_scale, *gate_scale, *up_scale;
  void *out;                                 // forward: h; gradient: [rows][2 pad] of dg and du
  int64_t rows, ld_x, ld_gate, ld_up, ld_dh, ld_out;
  int cols, hidden, act, pad;                // pad: hidden rounded up to 32
  GatedRange range;                          // gradient, float16
};

constexpr int kChunk = 128, kChunkPitch = kChunk + 16;     // bytes of the depth in LDS at a time, and between rows there
constexpr int kTileHidden = 64;                            // columns of Wg and of Wu a tile takes

template <class T> constexpr int kTypeStep = sizeof(T) == 1 ? 64 : 32 / (int)sizeof(T);    // depth of a matrix instruction's fragments
template <class T> constexpr int kChunkK = kChunk / (int)sizeof(T);

// Fragment of step s of 32 rows of an operand whose depth runs along its rows in LDS.
template <class T> __device__ __forceinline__ typename Frag<T>::V rows_frag(const char *rows, int pitch, int s) {
  const int l = lane_id(), half = l / 32;
  const char *at = rows + (l % 32) * pitch;
  if constexpr (sizeof(T) == 1) {
    const Piece a = *reinterpret_cast<const Piece *>(at + s * 64 + half * 32), b = *reinterpret_cast<const Piece *>(at + s * 64 + half * 32 + 16);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else return *reinterpret_cast<const typename Frag<T>::V *>(at + s * 32 + half * 16);
}
// The same of 32 columns of an operand whose depth runs down its columns, with the depth in the order that rows_frag has it.
template <class T> __device__ __forceinline__ typename Frag<T>::V deep_frag(const char *rows, int pitch, int s, int tile) {
  if constexpr (sizeof(T) == 2) return columns_frag<T>(rows, pitch, s, tile);
  else {
    const int l = lane_id(), half = l / 32;
    typename Frag<T>::V v;
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = *reinterpret_cast<const float *>(rows + (s * 8 + half * 4 + j) * pitch + (tile * 32 + l % 32) * 4);
    return v;
  }
}

// What the lanes of a wave have put into LDS is there for its other lanes: a wave's accesses are in order, so this holds the compiler alone.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// z Phi(z) = max(z, 0) - |z| (1 - Phi(|z|)), with 1 - Phi as normal_cdf has it (half of the polynomial's factors taken in): three instructions fewer
// than a choice by z's sign, which has cost no less time (612.5k x 256 x 1024 of 8 bits 633 us, with the choice 627; 2.45M x 128 x 344 bf16 817 and 815).  The
// clamp keeps infinity times 0 away.
__device__ __forceinline__ float gelu(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118f, fabsf(z), 1.f));
  const float e = __builtin_amdgcn_exp2f(z * z * (-0.5f * 1.4426950408889634f));
  const float tail = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f) * e;
  return fmaf(-fminf(fabsf(z), 3.4028235e38f), tail, fmaxf(z, 0.f));
}

// h of a lane's elements in place of g: one decision for all of them, whose exponentials are then under way side by side
template <int N> __device__ __forceinline__ void gate_all(float g[N], const float u[N], int act) {
  if (act == INK_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; j++) g[j] = gelu(g[j]);
  } else activate_all<N>(g, act);
#pragma unroll
  for (int j = 0; j < N; j++) g[j] *= u[j];
}
// value and slope of an activation, which share their exponential
__device__ __forceinline__ float activate_both(float z, float &slope, int act) {
  if (act == INK_ACT_RELU) { slope = z > 0.f ? 1.f : z <= 0.f ? 0.f : z; return z < 0.f ? 0.f : z; }
  if (act == INK_ACT_GELU) { float pdf; const float cdf = normal_cdf(z, pdf); slope = fmaf(z, pdf, cdf); return z * cdf; }
  if (act == INK_ACT_SILU) { const float s = sigmoid(z); slope = s * fmaf(z, 1.f - s, 1.f); return z * s; }
  slope = 1.f;
  return z;
}
// dg and du in place of g and u
template <int N, int ACT> __device__ __forceinline__ void gate_grad_of(float g[N], float u[N], const float dh[N]) {
#pragma unroll
  for (int j = 0; j < N; j++) {
    float slope;
    const float a = activate_both(g[j], slope, ACT);
    g[j] = dh[j] * u[j] * slope;
    u[j] = dh[j] * a;
  }
}
template <int N> __device__ __forceinline__ void gate_grad_all(float g[N], float u[N], const float dh[N], int act) {
  if (act == INK_ACT_SILU) gate_grad_of<N, INK_ACT_SILU>(g, u, dh);
  else if (act == INK_ACT_GELU) gate_grad_of<N, INK_ACT_GELU>(g, u, dh);
  else if (act == INK_ACT_RELU) gate_grad_of<N, INK_ACT_RELU>(g, u, dh);
  else gate_grad_of<N, INK_ACT_NONE>(g, u, dh);
}

// ------------------------------------------------------------------------------------ tiles
// 128 rows by 64 columns of h a workgroup, 64 by 32 a wave (a tile of Wg and one of Wu, so that g and u of an element meet in a lane), 128 bytes
// of the depth at a time: while one piece is multiplied the next is on its way in registers.  16-bit weights lie in LDS as they do in memory, and the
// transposing read makes fragments of their columns.  100k x 602 x 1605 bf16 700 us (550 TFLOP/s), which LDS bounds: a wave reads 4 KB of it for four
// products of 32 cycles.
// TL: type of the operands in memory, T: in the products, TO: of h.  GRAD: dg and du go to `out` in place of h.
template <class TL, class T, class TO, bool GRAD, bool SHORT>
__global__ __launch_bounds__(256, 2) void k_gated_tile(GatedArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int RB = 2, BM = 64 * RB, KC = kChunkK<T>, PE = 16 / sizeof(T), STEPS = KC / kTypeStep<T>;
  constexpr bool DEEP = sizeof(TL) != 1;     // the depth runs down the weights' columns
  constexpr int PW = DEEP ? 2 * kTileHidden * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 16) : kChunkPitch;
  constexpr int NX = BM * 8 / 256, NW = 4;
  constexpr int PO = kTileHidden * (int)sizeof(TO) + 16;
  constexpr int kLoop = BM * kChunkPitch + (DEEP ? KC : 2 * kTileHidden) * PW, kEnd = BM * PO * (GRAD ? 2 : 1);
  __shared__ __align__(16) char s_mem[kLoop > kEnd ? kLoop : kEnd];
  char *s_x = s_mem, *s_w = s_mem + BM * kChunkPitch;
  const int tid = threadIdx.x, l = lane_id(), half = l / 32, wm = tid / kWave / 2, wn = tid / kWave % 2;
  // workgroups go to the eight chiplets in turn: the column tiles of the same rows are eight apart, so that one L2 serves them
  const int gy = (a.hidden + kTileHidden - 1) / kTileHidden, id = blockIdx.x / 8;
  const int64_t m0 = ((int64_t)(id / gy) * 8 + blockIdx.x % 8) * BM;
  const int n0 = id % gy * kTileHidden;
  if (m0 >= a.rows) return;
  typename RawOf<TL, T>::V x[NX], w[NW];
  const TL *xp[NX];
#pragma unroll
  for (int j = 0; j < NX; j++) xp[j] = static_cast<const TL *>(a.x) + min(m0 + tid / 8 + 32 * j, a.rows - 1) * a.ld_x;
  // This thread's pieces of the weights: a place in rows of Wg and Wu, some rows apart (rows of the weights, or of what is multiplied with one column).
  constexpr int C = DEEP ? kTileHidden / PE : 8, WR = DEEP ? 256 / (2 * C) : 32;       // pieces of a row of Wg; rows apart
  const int wc = DEEP ? tid % (2 * C) : tid % 8;
  const bool up = DEEP && wc >= C;
  const int wn_at = n0 + wc % C * PE;        // DEEP: first column
  auto fetch = [&](int k0) {
#pragma unroll
    for (int j = 0; j < NX; j++) x[j] = raw_piece<TL, T, SHORT>(xp[j], k0 + tid % 8 * PE, a.cols);
#pragma unroll
    for (int j = 0; j < NW; j++) {
      if constexpr (DEEP) {
        const int k = min(k0 + tid / (2 * C) + WR * j, a.cols - 1);
        w[j] = raw_piece<TL, T, SHORT>(static_cast<const TL *>(up ? a.up : a.gate) + (int64_t)k * (up ? a.ld_up : a.ld_gate), wn_at, a.hidden);
      } else {
        const int n = min(n0 + (tid / 8 + 32 * j) % kTileHidden, a.hidden - 1);
        w[j] = raw_piece<TL, T, SHORT>(static_cast<const TL *>(j >= 2 ? a.up : a.gate) + (int64_t)n * (j >= 2 ? a.ld_up : a.ld_gate), k0 + wc * PE, a.cols);
      }
    }
  };
  auto put = [&](int k0) {
#pragma unroll
    for (int j = 0; j < NX; j++)
      *reinterpret_cast<Piece *>(s_x + (tid / 8 + 32 * j) * kChunkPitch + tid % 8 * 16) = piece_of<TL, T, SHORT>(x[j], k0 + tid % 8 * PE, a.cols);
#pragma unroll
    for (int j = 0; j < NW; j++) {
      if constexpr (DEEP) {                    // rows past the depth are zeros, as x is there
        const int k = tid / (2 * C) + WR * j;
        *reinterpret_cast<Piece *>(s_w + k * PW + wc * 16) = k0 + k < a.cols ? piece_of<TL, T, SHORT>(w[j], wn_at, a.hidden) : Piece{};
      } else *reinterpret_cast<Piece *>(s_w + (tid / 8 + 32 * j) * PW + wc * 16) = piece_of<TL, T, SHORT>(w[j], k0 + wc * PE, a.cols);
    }
  };
  f32x16 g[RB], u[RB];
#pragma unroll
  for (int i = 0; i < RB; i++) g[i] = u[i] = f32x16{};
  fetch(0);
  put(0);
  __syncthreads();
  for (int k0 = 0; k0 < a.cols; k0 += KC) {
    const bool more = k0 + KC < a.cols;
    if (more) fetch(k0 + KC);
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      V ws[2], xs[RB];
      if constexpr (DEEP) {
        ws[0] = deep_frag<T>(s_w, PW, s, wn);
        ws[1] = deep_frag<T>(s_w, PW, s, 2 + wn);
      } else {
        ws[0] = rows_frag<T>(s_w + wn * 32 * PW, PW, s);
        ws[1] = rows_frag<T>(s_w + (kTileHidden + wn * 32) * PW, PW, s);
      }
#pragma unroll
      for (int i = 0; i < RB; i++) xs[i] = rows_frag<T>(s_x + (wm * RB + i) * 32 * kChunkPitch, kChunkPitch, s);
      if constexpr (sizeof(T) == 4) {          // the four instructions of a step take turns among the accumulators
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int i = 0; i < RB; i++) {
            g[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(ws[0][j], xs[i][j], g[i], 0, 0, 0);
            u[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(ws[1][j], xs[i][j], u[i], 0, 0, 0);
          }
      } else
#pragma unroll
        for (int i = 0; i < RB; i++) {
          g[i] = mma(ws[0], xs[i], g[i]);
          u[i] = mma(ws[1], xs[i], u[i]);
        }
    }
    __syncthreads();
    if (more) put(k0 + KC);
    __syncthreads();
  }
  // Through LDS, so that dh is read and h, dg and du are written in whole lines.
  constexpr int OE = 16 / sizeof(TO), OP = kTileHidden / OE, NO = BM * OP / 256;      // elements of a piece, pieces of a row, pieces a thread
  if constexpr (GRAD) {
#pragma unroll
    for (int j = 0; j < NO; j++) {
      const int i = tid + 256 * j, row = i / OP, c = i % OP;
      const int64_t r = min(m0 + row, a.rows - 1);
      const Piece v = raw_piece<TO, TO, SHORT>(static_cast<const TO *>(a.dh) + r * a.ld_dh, n0 + c * OE, a.hidden);
      *reinterpret_cast<Piece *>(s_mem + row * PO + c * 16) = piece_of<TO, TO, SHORT>(v, n0 + c * OE, a.hidden);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < RB; i++) {
    const int row = (wm * RB + i) * 32 + l % 32;
    float scale = 1.f;
    if constexpr (!DEEP) scale = a.x_scale[min(m0 + row, a.rows - 1)];
    float gv[16], uv[16];
    TO *at = reinterpret_cast<TO *>(s_mem + row * PO) + wn * 32 + 4 * half;      // four neighbouring columns, four times 8 apart
#pragma unroll
    for (int e = 0; e < 16; e++) {
      gv[e] = g[i][e];
      uv[e] = u[i][e];
      if constexpr (!DEEP) {
        const int n = min(n0 + wn * 32 + 8 * (e / 4) + 4 * half + e % 4, a.hidden - 1);
        gv[e] *= scale * a.gate_scale[n];
        uv[e] *= scale * a.up_scale[n];
      }
    }
    if constexpr (GRAD) {
      float dh[16];
#pragma unroll
      for (int e = 0; e < 4; e++) load_pack<TO, 4>(at + 8 * e, dh + 4 * e);
      gate_grad_all<16>(gv, uv, dh, a.act);
      if (n0 + kTileHidden > a.hidden)         // behind the last column the products that follow find zeros, whatever x holds
#pragma unroll
        for (int e = 0; e < 16; e++)
          if (n0 + wn * 32 + 8 * (e / 4) + 4 * half + e % 4 >= a.hidden) gv[e] = uv[e] = 0.f;
      if constexpr (kRanged<TO>)
        if (n0 + wn * 32 < a.pad) {
          to_units(gv, a.range, m0 / 32 + wm * RB + i, n0 / 32 + wn);
          to_units(uv, a.range, m0 / 32 + wm * RB + i, (a.pad + n0) / 32 + wn);
        }
#pragma unroll
      for (int e = 0; e < 4; e++) store_pack<TO, 4>(at + BM * PO / (int)sizeof(TO) + 8 * e, uv + 4 * e);
    } else gate_all<16>(gv, uv, a.act);
#pragma unroll
    for (int e = 0; e < 4; e++) store_pack<TO, 4>(at + 8 * e, gv + 4 * e);
  }
  __syncthreads();
  if constexpr (GRAD) {
#pragma unroll
    for (int j = 0; j < 2 * NO; j++) {
      const int i = tid + 256 * j, row = i / OP, c = i % OP, part = row / BM;
      const int64_t r = m0 + row % BM;
      if (r < a.rows && n0 + c * OE < a.pad)
        *reinterpret_cast<Piece *>(static_cast<TO *>(a.out) + r * a.ld_out + part * a.pad + n0 + c * OE) = *reinterpret_cast<const Piece *>(s_mem + row * PO + c * 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NO; j++) {
      const int i = tid + 256 * j, row = i / OP, c = i % OP, n = n0 + c * OE;
      const int64_t r = m0 + row;
      if (r >= a.rows || n >= a.hidden) continue;
      const Piece v = *reinterpret_cast<const Piece *>(s_mem + row * PO + c * 16);
      TO *to = static_cast<TO *>(a.out) + r * a.ld_out + n;
      if (n + OE <= a.hidden) *reinterpret_cast<PieceAny *>(to) = v;
      else {
        const TO *from = reinterpret_cast<const TO *>(s_mem + row * PO) + c * OE;
        for (int e = 0; n + e < a.hidden; e++) to[e] = from[e];
      }
    }
  }
}

// ------------------------------------------------------------------------------------ many rows
// Rows in a stream past weights in registers: a wave has the fragments of 32 columns of Wg and of Wu over the whole depth (KS steps) for good, a
// workgroup WN waves side by side and WM below each other.  It takes 32 WM rows at a time; all threads load them side by side, a
// tile ahead, into one of two buffers in LDS, from where every wave reads the fragments of its rows: one barrier a tile.  The results
// turn in LDS that is the wave's own, from four columns a lane to 64 bytes of a row side by side, so no wave waits for another's activations.  The
// next tile's rows go into LDS before this tile's results are stored: memory answers in order, so a wait for rows asked for is one for all
// stores before them, and those of the tile before have had the products' time (2.45M x 128 x 344 bf16: 812 us with the stores first).
struct StreamPlan { int groups, row_groups; };               // workgroups side by side, and below each other
template <class T, class TO, int KS, int WN, int WM, int PER, bool GRAD>
__global__ __launch_bounds__(kWave * WN * WM, PER) void k_gated_stream(GatedArgs a, StreamPlan plan) {
  typedef typename Frag<T>::V V;
  constexpr bool DEEP = sizeof(T) != 1;
  constexpr int THREADS = kWave * WN * WM, MR = 32 * WM;
  constexpr int KB = KS * kTypeStep<T> * (int)sizeof(T), P = KB + 16;        // bytes of a row, and between rows in LDS
  constexpr int PE = 16 / sizeof(T), ROWS = THREADS / (KB / 16), NL = (MR + ROWS - 1) / ROWS;     // a thread's piece has one place in rows ROWS apart
  constexpr int OE = 16 / sizeof(TO), OP = 32 / OE, OROWS = kWave / OP, NO = 32 / OROWS;          // a wave stores OROWS rows of 32 columns at once
  constexpr int PO = 32 * (int)sizeof(TO) + 16, OWN = 32 * PO * (GRAD ? 2 : 1);                 // a wave's 32 rows of 32 results
  constexpr int PWT = 32 * (int)sizeof(T) + 16;              // a step of W on its way to the registers
  static_assert(THREADS % (KB / 16) == 0, "whole rows of pieces");
  static_assert(!DEEP || 2 * kTypeStep<T> * PWT <= OWN, "a step of W fits a wave's own memory");
  extern __shared__ __align__(16) char s_mem[];
  char *s_x = s_mem;
  const int tid = threadIdx.x, l = lane_id(), half = l / 32, wave = __builtin_amdgcn_readfirstlane(tid / kWave), wn = wave % WN, wm = wave / WN;
  char *s_own = s_mem + 2 * MR * P + wave * OWN;
  // workgroups go to the eight chiplets in turn: those that read the same rows are eight apart
  const int id = blockIdx.x / 8, group = id % plan.groups;
  const int64_t first = (int64_t)(id / plan.groups) * 8 + blockIdx.x % 8, tiles = (a.rows + MR - 1) / MR;
  // A wave that the last column cuts takes the last 32 columns instead, some of which the wave before it has too: the same numbers.  (dg and du
  // are stored up to whole tiles, with zeros.)
  const int n_first = (group * WN + wn) * 32, n0 = GRAD || n_first >= a.hidden ? n_first : max(0, min(n_first, a.hidden - 32));
  // Addresses are a uniform base and 32 bits a lane.  A piece that the row's end cuts is loaded from its last 16 bytes and moved down, one
  // past it is zero; of the last tile the last row stands in for those past the end.
  const int row = tid / (KB / 16), col = tid % (KB / 16) * PE;
  const uint32_t x_at = (__umul24(row, (uint32_t)a.ld_x) + min(col, a.cols - PE)) * (uint32_t)sizeof(T);
  Piece x[NL];
  auto fetch = [&](int64_t t) {
    const char *base = reinterpret_cast<const char *>(static_cast<const T *>(a.x) + t * MR * a.ld_x);
    const int left = (int)min(a.rows - t * MR, (int64_t)MR);
#pragma unroll
    for (int j = 0; j < NL; j++) {
      if (MR % ROWS && j == NL - 1 && row + j * ROWS >= MR) continue;
      uint32_t at = x_at;
      if (left < MR) at -= max(0, row + j * ROWS - left + 1) * (uint32_t)a.ld_x * (uint32_t)sizeof(T);
      x[j] = (Piece)*reinterpret_cast<const PieceAny *>(base + (int64_t)j * ROWS * a.ld_x * (int)sizeof(T) + (int64_t)(int32_t)at);
    }
  };
  auto put = [&](int buffer) {
#pragma unroll
    for (int j = 0; j < NL; j++) {
      if (MR % ROWS && j == NL - 1 && row + j * ROWS >= MR) continue;
      if (col + PE > a.cols) x[j] = col < a.cols ? move_down(x[j], col + PE - a.cols, sizeof(T)) : Piece{};
      *reinterpret_cast<Piece *>(s_x + (buffer * MR + j * ROWS + row) * P + tid % (KB / 16) * 16) = x[j];
    }
  };
  int64_t t = first;
  if (t < tiles) fetch(t);
  V w[2][KS];
  if constexpr (DEEP) {
    constexpr int PR = 32 / PE;              // pieces of a step's row: 64 lanes take a whole step
    const int k = l / PR, n = n0 + l % PR * PE;
    Piece q[2][KS];
#pragma unroll
    for (int s = 0; s < KS; s++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int kk = s * kTypeStep<T> + k;
        const T *from = static_cast<const T *>(h ? a.up : a.gate) + (int64_t)min(kk, a.cols - 1) * (h ? a.ld_up : a.ld_gate);
        q[h][s] = (Piece)*reinterpret_cast<const PieceAny *>(from + min(n, a.hidden - PE));
        if (kk >= a.cols || n >= a.hidden) q[h][s] = Piece{};
        else if (n + PE > a.hidden) q[h][s] = move_down(q[h][s], n + PE - a.hidden, sizeof(T));
      }
#pragma unroll
    for (int s = 0; s < KS; s++) {
#pragma unroll
      for (int h = 0; h < 2; h++) *reinterpret_cast<Piece *>(s_own + h * kTypeStep<T> * PWT + k * PWT + l % PR * 16) = q[h][s];
      wave_order();
#pragma unroll
      for (int h = 0; h < 2; h++) w[h][s] = deep_frag<T>(s_own + h * kTypeStep<T> * PWT, PWT, 0, 0);
      wave_order();
    }
  } else {
    const int n = n0 + l % 32;
#pragma unroll
    for (int s = 0; s < KS; s++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        Piece q[2];
#pragma unroll
        for (int j = 0; j < 2; j++) {
          const int k = s * kTypeStep<T> + half * 32 + 16 * j;
          const T *from = static_cast<const T *>(h ? a.up : a.gate) + (int64_t)min(n, a.hidden - 1) * (h ? a.ld_up : a.ld_gate);
          q[j] = (Piece)*reinterpret_cast<const PieceAny *>(from + min(k, a.cols - PE));
          if (k >= a.cols || n >= a.hidden) q[j] = Piece{};
          else if (k + PE > a.cols) q[j] = move_down(q[j], k + PE - a.cols, sizeof(T));
        }
        w[h][s] = __builtin_shufflevector(q[0], q[1], 0, 1, 2, 3, 4, 5, 6, 7);
      }
  }
  F4 *s_scale = reinterpret_cast<F4 *>(s_mem + 2 * MR * P + WN * WM * OWN) + wave * 16;      // 8-bit weights: scales of this wave's columns
  if constexpr (!DEEP) {
    reinterpret_cast<float *>(s_scale)[l] = (l < 32 ? a.gate_scale : a.up_scale)[min(n0 + l % 32, a.hidden - 1)];
    wave_order();
  }
  const bool whole = n0 + 32 <= a.hidden;
  const int orow = l / OP, ocol = l % OP * OE;               // this lane's piece of the results: rows OROWS apart
  const uint32_t o_at = (__umul24(orow, (uint32_t)a.ld_out) + ocol) * (uint32_t)sizeof(TO);
  const uint32_t d_at = GRAD ? (__umul24(orow, (uint32_t)a.ld_dh) + max(0, min(n0 + ocol, a.hidden - OE))) * (uint32_t)sizeof(TO) : 0;
  if (t >= tiles) return;                    // the whole workgroup
  const int64_t last = t + (tiles - 1 - t) / plan.row_groups * plan.row_groups;
  // What else a tile reads, a tile ahead: dh of the wave's rows (64 bytes or more side by side), scales of its 8-bit rows.
  constexpr int ND = 32 / OROWS;
  Piece dhp[GRAD ? ND : 1];
  float scale = 1.f;
  auto fetch_more = [&](int64_t t, auto plain) {
    const int64_t my_row = t * MR + wm * 32;
    if constexpr (!DEEP) scale = a.x_scale[min(my_row + l % 32, a.rows - 1)];
    if constexpr (GRAD)
#pragma unroll
      for (int j = 0; j < ND; j++) {
        if constexpr (plain()) {
          const char *base = reinterpret_cast<const char *>(static_cast<const TO *>(a.dh) + (my_row + j * OROWS) * a.ld_dh);
          dhp[j] = (Piece)*reinterpret_cast<const PieceAny *>(base + d_at);
        } else {
          const int64_t r = min(my_row + j * OROWS + orow, a.rows - 1);
          dhp[j] = (Piece)*reinterpret_cast<const PieceAny *>(static_cast<const TO *>(a.dh) + r * a.ld_dh + min(n0 + ocol, a.hidden - OE));
        }
      }
  };
  // One tile.  PLAIN: not this workgroup's last one, and all 32 columns there: the stores are then under no condition, and the wait for the next
  // tile's rows is not one for them (one wave of a launch with a condition on its stores: 2.45M x 128 x 344 bf16 940 us).
  auto tile = [&](int64_t t, int buffer, auto plain) {
    constexpr bool PLAIN = plain();
    __syncthreads();
    const int64_t my_row = t * MR + wm * 32;
    f32x16 g = f32x16{}, u = f32x16{};
    const char *xs = s_x + (buffer * MR + wm * 32) * P;
    // fragments are asked for AHEAD steps before their products: left alone, the compiler asks for one at a time and waits for it
    constexpr int AHEAD = sizeof(T) == 2 ? 4 : 2;
    V f[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; s++) f[s] = rows_frag<T>(xs, P, s);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < KS; s++) {
      const V xf = f[s % AHEAD];
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
          g = __builtin_amdgcn_mfma_f32_32x32x2f32(w[0][s][j], xf[j], g, 0, 0, 0);
          u = __builtin_amdgcn_mfma_f32_32x32x2f32(w[1][s][j], xf[j], u, 0, 0, 0);
        }
      } else {
        g = mma(w[0][s], xf, g);
        u = mma(w[1][s], xf, u);
      }
      if (s + AHEAD < KS) f[s % AHEAD] = rows_frag<T>(xs, P, s + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (GRAD) {
#pragma unroll
      for (int j = 0; j < ND; j++) {
        Piece &d = dhp[j];
        if (!whole && n0 + ocol + OE > a.hidden) d = n0 + ocol < a.hidden ? move_down(d, n0 + ocol + OE - a.hidden, sizeof(TO)) : Piece{};
        *reinterpret_cast<Piece *>(s_own + (orow + j * OROWS) * PO + l % OP * 16) = d;
      }
      wave_order();
    }
    constexpr int N = GRAD || !DEEP ? 8 : 16;      // elements at a time: registers
    constexpr bool WHOLE = GRAD && kRanged<TO>;    // stored when all are there: a block's units follow from all of it
    float all_g[WHOLE ? 16 : N], all_u[WHOLE ? 16 : N];
#pragma unroll
    for (int q = 0; q < 16 / N; q++) {
      float *gv = all_g + (WHOLE ? N * q : 0), *uv = all_u + (WHOLE ? N * q : 0);
      TO *at = reinterpret_cast<TO *>(s_own + (l % 32) * PO) + 16 * q + 4 * half;          // four neighbouring columns at a time, 8 apart
#pragma unroll
      for (int e = 0; e < N; e++) {
        gv[e] = g[8 * q + e];
        uv[e] = u[8 * q + e];
        if constexpr (!DEEP) {
          gv[e] *= scale * s_scale[4 * q + 2 * (e / 4) + half][e % 4];
          uv[e] *= scale * s_scale[8 + 4 * q + 2 * (e / 4) + half][e % 4];
        }
      }
      if constexpr (GRAD) {
        float dh[8];
#pragma unroll
        for (int e = 0; e < 2; e++) load_pack<TO, 4>(at + 8 * e, dh + 4 * e);
        gate_grad_all<8>(gv, uv, dh, a.act);
        if (!whole)                          // behind the last column the products that follow find zeros, whatever x holds
#pragma unroll
          for (int e = 0; e < 8; e++)
            if (n0 + 16 * q + 8 * (e / 4) + 4 * half + e % 4 >= a.hidden) gv[e] = uv[e] = 0.f;
        if constexpr (!WHOLE)
#pragma unroll
          for (int e = 0; e < 2; e++) store_pack<TO, 4>(at + 32 * PO / (int)sizeof(TO) + 8 * e, uv + 4 * e);
      } else gate_all<N>(gv, uv, a.act);
      if constexpr (!WHOLE)
#pragma unroll
        for (int e = 0; e < N / 4; e++) store_pack<TO, 4>(at + 8 * e, gv + 4 * e);
    }
    if constexpr (WHOLE) {
      to_units(all_g, a.range, my_row / 32, n0 / 32);
      to_units(all_u, a.range, my_row / 32, (a.pad + n0) / 32);
      TO *at = reinterpret_cast<TO *>(s_own + (l % 32) * PO) + 4 * half;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        store_pack<TO, 4>(at + 8 * e, all_g + 4 * e);
        store_pack<TO, 4>(at + 32 * PO / (int)sizeof(TO) + 8 * e, all_u + 4 * e);
      }
    }
    const int64_t next = min(t + plan.row_groups, last);
    put(buffer ^ 1);
    fetch(min(t + 2 * plan.row_groups, last));
    // a last tile that is not full is asked for once more behind the loop, row by row; here this one stands in for it
    fetch_more(!PLAIN || (next + 1) * MR <= a.rows ? next : t, plain);
    wave_order();
    char *base = reinterpret_cast<char *>(static_cast<TO *>(a.out) + my_row * a.ld_out + n0);
    const char *mine = s_own + orow * PO + l % OP * 16;
    const int64_t left = a.rows - my_row;
#pragma unroll
    for (int j = 0; j < (GRAD ? 2 : 1) * NO; j++) {
      TO *to = reinterpret_cast<TO *>(base + ((int64_t)(j % NO) * OROWS * a.ld_out + j / NO * a.pad) * (int)sizeof(TO) + o_at);
      const Piece v = *reinterpret_cast<const Piece *>(mine + j * OROWS * PO);
      if constexpr (PLAIN) *reinterpret_cast<PieceAny *>(to) = v;
      else {
        if (orow + j % NO * OROWS >= left) continue;
        if (GRAD || n0 + ocol + OE <= a.hidden) *reinterpret_cast<PieceAny *>(to) = v;
        else
          for (int e = 0; n0 + ocol + e < a.hidden; e++) to[e] = reinterpret_cast<const TO *>(mine + j * OROWS * PO)[e];
      }
    }
    wave_order();
  };
  put(0);
  fetch(min(t + plan.row_groups, last));
  int buffer = 0;
  if (n0 >= (GRAD ? a.pad : a.hidden)) {     // a wave without columns loads rows with the others
    for (; t <= last; t += plan.row_groups, buffer ^= 1) {
      __syncthreads();
      put(buffer ^ 1);
      fetch(min(t + 2 * plan.row_groups, last));
    }
    return;
  }
  fetch_more(t, std::false_type());
  if (GRAD || whole)
    for (; t < last; t += plan.row_groups, buffer ^= 1) tile(t, buffer, std::true_type());
  else
    for (; t < last; t += plan.row_groups, buffer ^= 1) tile(t, buffer, std::false_type());
  fetch_more(t, std::false_type());
  tile(t, buffer, std::false_type());
}

// ------------------------------------------------------------------------------------ gradient
// dx = dg Wg^T + du Wu^T of the rows of one part: 128 rows by 128 columns a workgroup, 64 by 64 a wave.  (128 by 64 a wave reads a quarter less
// of LDS, but leaves room for two workgroups a CU instead of three: 233k x 256 x 683 347 us instead of 366, 100k x 602 x 1605 633 instead of 588.)
struct GatedDxArgs {
  const void *d, *gate, *up;                 // [rows][2 pad] of dg and du
  void *dx;
  int64_t rows, ld_gate, ld_up, ld_dx;
  int cols, hidden, pad;
  GatedRange range;
};
template <class T, bool SHORT>
__global__ __launch_bounds__(256, 2) void k_gated_dx(GatedDxArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int RI = 2, WM = 2, WN = 2, THREADS = 256, KC = kChunkK<T>, PE = 16 / sizeof(T), BM = 32 * RI * WM, BN = 64 * WN, P = kChunkPitch;
  constexpr int ND = BM * 8 / THREADS, NW = BN * 8 / THREADS, RS = THREADS / 8;
  constexpr int PO = BN * (int)sizeof(T) + 16, HALF = 16 * RI, kLoop = (BM + BN) * P, kEnd = HALF * WM * PO;      // results leave in two halves of a wave's rows
  __shared__ __align__(16) char s_mem[kLoop > kEnd ? kLoop : kEnd];
  char *s_d = s_mem, *s_w = s_mem + BM * P;
  const int tid = threadIdx.x, l = lane_id(), half = l / 32, wave = __builtin_amdgcn_readfirstlane(tid / kWave), wm = wave / WN, wn = wave % WN;
  const int gy = (a.cols + BN - 1) / BN, id = blockIdx.x / 8;
  const int64_t m0 = ((int64_t)(id / gy) * 8 + blockIdx.x % 8) * BM;
  const int n0 = id % gy * BN;
  if (m0 >= a.rows) return;
  Piece d[ND], w[NW];
  constexpr bool RANGED = kRanged<T>;
  int unit[RI][2], next_unit[RI][2], was[RI], was_code[RI];            // of a lane's row, and as the blocks have them
  int64_t blocks[RI];
  if constexpr (RANGED)
#pragma unroll
    for (int i = 0; i < RI; i++) {
      blocks[i] = min(m0 / 32 + wm * RI + i, (a.rows - 1) / 32) * a.range.across;
      was[i] = was_code[i] = 0;
    }
  const int at = tid % 8 * PE, row = tid / 8;
  const T *dp = static_cast<const T *>(a.d) + m0 * 2 * a.pad + at;
  uint32_t d_row[ND];
#pragma unroll
  for (int j = 0; j < ND; j++) d_row[j] = (uint32_t)(min((int64_t)(row + RS * j), a.rows - 1 - m0) * 2 * a.pad);
  auto fetch = [&](int k0) {
#pragma unroll
    for (int j = 0; j < ND; j++) d[j] = *reinterpret_cast<const Piece *>(dp + d_row[j] + k0);
    const bool second = k0 + at >= a.pad;
    const int k = k0 + at - (second ? a.pad : 0);
    const T *from = static_cast<const T *>(second ? a.up : a.gate);
    const int64_t ld = second ? a.ld_up : a.ld_gate;
#pragma unroll
    for (int j = 0; j < NW; j++) w[j] = raw_piece<T, T, SHORT>(from + (int64_t)min(n0 + row + RS * j, a.cols - 1) * ld, k, a.hidden);
    if constexpr (RANGED)
#pragma unroll
      for (int i = 0; i < RI; i++)
#pragma unroll
        for (int h = 0; h < 2; h++) next_unit[i][h] = a.range.unit[blocks[i] + k0 / 32 + h];
  };
  auto put = [&](int k0) {
    const int k = k0 + at - (k0 + at >= a.pad ? a.pad : 0);
#pragma unroll
    for (int j = 0; j < ND; j++) *reinterpret_cast<Piece *>(s_d + (row + RS * j) * P + tid % 8 * 16) = d[j];
#pragma unroll
    for (int j = 0; j < NW; j++) *reinterpret_cast<Piece *>(s_w + (row + RS * j) * P + tid % 8 * 16) = piece_of<T, T, SHORT>(w[j], k, a.hidden);
  };
  f32x16 acc[RI][2];
#pragma unroll
  for (int i = 0; i < RI; i++) acc[i][0] = acc[i][1] = f32x16{};
  fetch(0);
  put(0);
  __syncthreads();
  for (int k0 = 0; k0 < 2 * a.pad; k0 += KC) {
    const bool more = k0 + KC < 2 * a.pad;
    if constexpr (RANGED)
#pragma unroll
      for (int i = 0; i < RI; i++) { unit[i][0] = next_unit[i][0]; unit[i][1] = next_unit[i][1]; }
    if (more) fetch(k0 + KC);
#pragma unroll
    for (int s = 0; s < 4; s++) {
      V ds[RI], ws[2];
      if constexpr (RANGED)
        if (s % 2 == 0)                        // 32 columns of d: a block
#pragma unroll
          for (int i = 0; i < RI; i++) {
            const int code = unit[i][s / 2];
            if (code == was_code[i] && !(code & 1)) continue;
            int now = code >> 1;
            if (code & 1) now -= a.range.finer[(blocks[i] + k0 / 32 + s / 2) * 32 + l % 32];
            change_units(acc[i], was[i], now);
            was[i] = now;
            was_code[i] = code;
          }
#pragma unroll
      for (int n = 0; n < 2; n++) ws[n] = rows_frag<T>(s_w + (wn * 2 + n) * 32 * P, P, s);
#pragma unroll
      for (int i = 0; i < RI; i++) ds[i] = rows_frag<T>(s_d + (wm * RI + i) * 32 * P, P, s);
      mma_block<T>(ws, ds, acc);
    }
    __syncthreads();
    if (more) put(k0 + KC);
    __syncthreads();
  }
  if constexpr (RANGED)
#pragma unroll
    for (int i = 0; i < RI; i++)
      if (was_code[i]) change_units(acc[i], was[i], 0);
  constexpr int OP = BN / PE;
#pragma unroll
  for (int h = 0; h < 2; h++) {
#pragma unroll
    for (int i = 0; i < RI / 2; i++)
#pragma unroll
      for (int n = 0; n < 2; n++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float v[4] = {acc[RI / 2 * h + i][n][4 * e], acc[RI / 2 * h + i][n][4 * e + 1], acc[RI / 2 * h + i][n][4 * e + 2], acc[RI / 2 * h + i][n][4 * e + 3]};
          store_pack<T, 4>(reinterpret_cast<T *>(s_mem + (wm * HALF + i * 32 + l % 32) * PO) + (wn * 2 + n) * 32 + 8 * e + 4 * half, v);
        }
    __syncthreads();
    for (int i = tid; i < WM * HALF * OP; i += THREADS) {
      const int r_in = i / OP, c = i % OP, n = n0 + c * PE;
      const int64_t r = m0 + r_in / HALF * (32 * RI) + h * HALF + r_in % HALF;
      if (r >= a.rows || n >= a.cols) continue;
      T *to = static_cast<T *>(a.dx) + r * a.ld_dx + n;
      if (n + PE <= a.cols) *reinterpret_cast<PieceAny *>(to) = *reinterpret_cast<const Piece *>(s_mem + r_in * PO + c * 16);
      else {
        const T *from = reinterpret_cast<const T *>(s_mem + r_in * PO) + c * PE;
        for (int e = 0; n + e < a.cols; e++) to[e] = from[e];
      }
    }
    __syncthreads();
  }
}

// The same where tiles of 128 by 128 would leave most of the card without work: 32 rows by 32 columns a workgroup, whose eight waves share the depth and
// take their fragments straight from memory (200 x 256 x 683 bf16: 20 us in tiles).
template <class T, bool SHORT>
__global__ __launch_bounds__(512) void k_gated_dx_small(GatedDxArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int VK = kVec<T>, KS = kStep<T>, WAVES = 8;
  __shared__ float s_acc[WAVES][32][36];
  const int wave = threadIdx.x / kWave, l = lane_id(), half = l / 32;
  const int64_t r0 = (int64_t)blockIdx.x * 32, r = min(r0 + l % 32, a.rows - 1);
  const int n0 = blockIdx.y * 32, n = min(n0 + l % 32, a.cols - 1);
  const T *d = static_cast<const T *>(a.d) + r * 2 * a.pad, *gate = static_cast<const T *>(a.gate) + n * a.ld_gate, *up = static_cast<const T *>(a.up) + n * a.ld_up;
  f32x16 acc[1] = {f32x16{}};
  const int64_t blocks = kRanged<T> ? r0 / 32 * a.range.across : 0;
  int was = 0;
#pragma unroll 4
  for (int k0 = wave * KS; k0 < 2 * a.pad; k0 += WAVES * KS) {
    const int at = k0 + half * VK, k = at - (at >= a.pad ? a.pad : 0);
    const Piece dv = *reinterpret_cast<const Piece *>(d + at);
    const Piece wv = piece_of<T, T, SHORT>(raw_piece<T, T, SHORT>(at >= a.pad ? up : gate, k, a.hidden), k, a.hidden);
    if constexpr (kRanged<T>) {                // under no condition: sixteen instructions, where the step waits for its loads
      const int code = a.range.unit[blocks + k0 / 32], finer = a.range.finer[(blocks + k0 / 32) * 32 + l % 32];
      const int now = (code >> 1) - (code & 1 ? finer : 0);
      change_units(acc, was, now);
      was = now;
    }
    acc[0] = mma(__builtin_bit_cast(V, wv), __builtin_bit_cast(V, dv), acc[0]);
  }
  if constexpr (kRanged<T>) change_units(acc, was, 0);
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const F4 v = {acc[0][4 * e], acc[0][4 * e + 1], acc[0][4 * e + 2], acc[0][4 * e + 3]};
    *reinterpret_cast<F4 *>(&s_acc[wave][l % 32][8 * e + 4 * half]) = v;
  }
  __syncthreads();
  if (threadIdx.x >= 256) return;
  const int row = threadIdx.x / 8, c = threadIdx.x % 8 * 4;
  F4 t = F4{};
#pragma unroll
  for (int i = 0; i < WAVES; i++) t += *reinterpret_cast<F4 *>(&s_acc[i][row][c]);
  const float v[4] = {t[0], t[1], t[2], t[3]};
  if (r0 + row < a.rows && n0 + c < a.cols) store4(static_cast<T *>(a.dx) + (r0 + row) * a.ld_dx, n0 + c, a.cols, v);
}

// Sums over the rows of one part, x^T [dg du]: 128 WM columns of x by 64 WN of dg and du a workgroup, 128 by 64 a wave, over a slice of the rows.  The sums of
// the slice go to, or are added to, its partial matrix, in the fragments' order.  The tiles of one slice run on one chiplet: they read the same rows.
struct GatedDwArgs {
  const void *x, *d;
  float *part;                               // [slices][tiles of d][tiles of x][RI WM][2 WN] fragments
  int64_t rows, ld_x, slice;
  int cols, pad, add, slices, tiles_c, tiles_n;
  GatedRange range;
};
template <class T, int RI, int WM, int WN, bool SHORT>
__global__ __launch_bounds__(kWave * WM * WN, 2) void k_gated_dw(GatedDwArgs a) {
  typedef typename Frag<T>::V V;
  constexpr int THREADS = kWave * WM * WN, KR = kChunkK<T>, PE = 16 / sizeof(T), STEPS = KR / kStep<T>;       // rows at a time
  constexpr int BM = 32 * RI * WM, BN = 64 * WN, PX = BM * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 144), PD = BN * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 144), CX = BM / PE, CD = BN / PE;
  constexpr int NX = KR * CX / THREADS, ND = KR * CD / THREADS, RX = THREADS / CX, RD = THREADS / CD;
  __shared__ __align__(16) char s_x[KR * PX], s_d[KR * PD];
  const int tid = threadIdx.x, l = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / kWave), wm = wave / WN, wn = wave % WN;
  const int tiles = a.tiles_c * a.tiles_n, id = blockIdx.x / 8;
  const bool spread = a.slices % 8 != 0;     // few slices: over all chiplets
  const int slice = spread ? blockIdx.x / tiles : id / tiles * 8 + blockIdx.x % 8, tile = spread ? blockIdx.x % tiles : id % tiles;
  const int c0 = tile % a.tiles_c * BM, n0 = tile / a.tiles_c * BN;
  const int64_t r_begin = slice * a.slice, r_end = min(r_begin + a.slice, a.rows);
  const int blocks = max(0, min(RI, (a.cols - c0 - wm * 32 * RI + 31) / 32)), wide = n0 + wn * 64 < 2 * a.pad;      // of x that there are; whether there are any of d
  float *part = a.part + ((int64_t)slice * tiles + tile) * (BM * BN);
  f32x16 acc[RI][2];
#pragma unroll
  for (int i = 0; i < RI; i++)
#pragma unroll
    for (int n = 0; n < 2; n++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        F4 v = F4{};
        if (a.add) v = reinterpret_cast<const F4 *>(part)[(((wm * RI + i) * 2 * WN + wn * 2 + n) * 4 + e) * 64 + l];
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][n][4 * e + j] = v[j];
      }
  Piece x[NX], d[ND];
  const int xc = c0 + tid % CX * PE, dc = n0 + tid % CD * PE;
  const int dc_in = min(dc, 2 * a.pad - PE);
  // float16: units of the two blocks of rows of a chunk, of this wave's columns of d and of this thread's pieces
  constexpr bool RANGED = kRanged<T>;
  static_assert(!RANGED || (KR == 64 && 32 % RD == 0), "a chunk is two blocks of rows");
  int unit[2][2], next_unit[2][2], piece_unit[2], was[2] = {0, 0};
  int64_t row_block[2];
  const int wave_block = min(n0 / 32 + wn * 2, 2 * a.pad / 32 - 2);
  auto fetch = [&](int64_t r0) {             // of the last chunk the last row stands in for those past the slice's end
    const int left = (int)max((int64_t)1, min(r_end - r0, (int64_t)KR));
    const T *xp = static_cast<const T *>(a.x) + min(r0, a.rows - 1) * a.ld_x, *dp = static_cast<const T *>(a.d) + min(r0, a.rows - 1) * 2 * a.pad + dc_in;
#pragma unroll
    for (int j = 0; j < NX; j++) x[j] = raw_piece<T, T, SHORT>(xp + min(tid / CX + RX * j, left - 1) * a.ld_x, xc, a.cols);
#pragma unroll
    for (int j = 0; j < ND; j++) d[j] = *reinterpret_cast<const Piece *>(dp + (uint32_t)(min(tid / CD + RD * j, left - 1) * 2 * a.pad));
    if constexpr (RANGED)
#pragma unroll
      for (int q = 0; q < 2; q++) {
        row_block[q] = min(r0 / 32 + q, (a.rows - 1) / 32) * a.range.across;
        piece_unit[q] = a.range.unit[row_block[q] + dc_in / 32];
#pragma unroll
        for (int n = 0; n < 2; n++) next_unit[q][n] = a.range.unit[row_block[q] + wave_block + n];
      }
  };
  auto put = [&](int64_t r0) {
    const int left = (int)min(r_end - r0, (int64_t)KR);
#pragma unroll
    for (int j = 0; j < NX; j++) {
      Piece v = piece_of<T, T, SHORT>(x[j], xc, a.cols);
      if (left < KR && tid / CX + RX * j >= left) v = Piece{};
      *reinterpret_cast<Piece *>(s_x + (tid / CX + RX * j) * PX + tid % CX * 16) = v;
    }
#pragma unroll
    for (int j = 0; j < ND; j++) {
      Piece v = d[j];
      if constexpr (RANGED)
        if (piece_unit[RD * j / 32] & 1) {     // to the block's units
          const int finer = a.range.finer[(row_block[RD * j / 32] + dc_in / 32) * 32 + tid / CD + RD * j % 32];
          V t = __builtin_bit_cast(V, v);
#pragma unroll
          for (int e = 0; e < 8; e++) t[e] = (T)__builtin_amdgcn_ldexpf((float)t[e], -finer);
          v = __builtin_bit_cast(Piece, t);
        }
      if (left < KR && tid / CD + RD * j >= left) v = Piece{};
      *reinterpret_cast<Piece *>(s_d + (tid / CD + RD * j) * PD + tid % CD * 16) = v;
    }
  };
  fetch(r_begin);
  put(r_begin);
  __syncthreads();
  for (int64_t r0 = r_begin; r0 < r_end; r0 += KR) {
    const bool more = r0 + KR < r_end;
    if constexpr (RANGED)
#pragma unroll
      for (int q = 0; q < 4; q++) unit[q / 2][q % 2] = next_unit[q / 2][q % 2] >> 1;
    if (more) fetch(r0 + KR);
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      V xs[RI], ds[2];
      if constexpr (RANGED)
        if (s % 2 == 0)
#pragma unroll
          for (int n = 0; n < 2; n++)
            if (unit[s / 2][n] != was[n]) {
#pragma unroll
              for (int i = 0; i < RI; i++) change_units(reinterpret_cast<f32x16 (&)[1]>(acc[i][n]), was[n], unit[s / 2][n]);
              was[n] = unit[s / 2][n];
            }
#pragma unroll
      for (int n = 0; n < 2; n++) ds[n] = columns_frag<T>(s_d, PD, s, wn * 2 + n);
#pragma unroll
      for (int i = 0; i < RI; i++) xs[i] = columns_frag<T>(s_x, PX, s, wm * RI + i);
      mma_block<T>(ds, xs, acc);
    }
    __syncthreads();
    if (more) put(r0 + KR);
    __syncthreads();
  }
  if (!wide) return;
#pragma unroll
  for (int i = 0; i < RI; i++) {
    if (i >= blocks) continue;
#pragma unroll
    for (int n = 0; n < 2; n++) {
      if (kRanged<T> && was[n]) change_units(reinterpret_cast<f32x16 (&)[1]>(acc[i][n]), was[n], 0);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const F4 v = {acc[i][n][4 * e], acc[i][n][4 * e + 1], acc[i][n][4 * e + 2], acc[i][n][4 * e + 3]};
        reinterpret_cast<F4 *>(part)[(((wm * RI + i) * 2 * WN + wn * 2 + n) * 4 + e) * 64 + l] = v;
      }
    }
  }
}

// Partial matrices to the weights' gradients: 64 elements, four by four, a workgroup; 16 threads share a sum, in the slices' order.
struct GatedSumArgs {
  const float *part;
  void *d_gate, *d_up;
  int64_t ld_gate, ld_up;
  int slices, type, cols, hidden, pad, tiles_c, tiles_n, kt, nt;             // kt by nt fragments a tile
};
__global__ __launch_bounds__(256) void k_gated_sum(GatedSumArgs a) {
  __shared__ F4 s[16][17];
  const int x = threadIdx.x % 16, y = threadIdx.x / 16, per = a.kt * a.nt * 1024;
  const int64_t n = (int64_t)a.tiles_c * a.tiles_n * per, i = ((int64_t)blockIdx.x * 16 + x) * 4;
  const int tile = (int)(i / per), f = (int)(i % per), frag = f / 1024, e = f / 256 % 4, lane = f / 4 % 64;
  const int c = (tile % a.tiles_c * a.kt + frag / a.nt) * 32 + lane % 32;
  int h = (tile / a.tiles_c * a.nt + frag % a.nt) * 32 + 8 * e + 4 * (lane / 32);
  const bool up = h >= a.pad;
  if (up) h -= a.pad;
  void *out = up ? a.d_up : a.d_gate;
  const bool wanted = c < a.cols && h < a.hidden && out;     // (fragments beside the matrix are not written either)
  F4 t = F4{};
  if (wanted)
#pragma unroll 4
    for (int p = y; p < a.slices; p += 16) t += *reinterpret_cast<const F4 *>(a.part + p * n + i);
  s[y][x] = t;
  __syncthreads();
  if (y || !wanted) return;
  t = F4{};
#pragma unroll
  for (int p = 0; p < 16; p++) t += s[p][x];
  for (int j = 0; j < 4; j++)
    if (h + j < a.hidden) store_any(out, (int64_t)c * (up ? a.ld_up : a.ld_gate) + h + j, a.type, t[j]);
}

// ------------------------------------------------------------------------------------ a few rows
// One row and 32 columns of h a workgroup: lanes side by side take 16 bytes of a row of Wg and of Wu, the rest of the workgroup splits the depth.
// GRAD: dg and du in 32 bits go to `out`, [rows][2 hidden] of float.
template <class T, bool GRAD>
__global__ __launch_bounds__(kHeadThreads) void k_gated_few(GatedArgs a) {
  constexpr int VK = kVec<T>, CL = 32 / VK, SL = kHeadThreads / CL, W = kHeadThreads / kWave;
  __shared__ float s_sum[2][W][32];
  const int cl = threadIdx.x % CL, sl = threadIdx.x / CL, n0 = blockIdx.x * 32, n = n0 + cl * VK;
  const int64_t r = blockIdx.y;
  const T *x = static_cast<const T *>(a.x) + r * a.ld_x, *wg = static_cast<const T *>(a.gate), *wu = static_cast<const T *>(a.up);
  float g[VK], u[VK];
#pragma unroll
  for (int j = 0; j < VK; j++) g[j] = u[j] = 0.f;
  if (n < a.hidden)
#pragma unroll 4
    for (int k = sl; k < a.cols; k += SL) {
      const float xv = (float)x[k];
      const typename Frag<T>::V vg = row_frag<T>(wg + (int64_t)k * a.ld_gate, n, a.hidden), vu = row_frag<T>(wu + (int64_t)k * a.ld_up, n, a.hidden);
#pragma unroll
      for (int j = 0; j < VK; j++) {
        g[j] = fmaf(xv, (float)vg[j], g[j]);
        u[j] = fmaf(xv, (float)vu[j], u[j]);
      }
    }
#pragma unroll
  for (int j = 0; j < VK; j++) {
#pragma unroll
    for (int o = CL; o < kWave; o <<= 1) { g[j] += __shfl_xor(g[j], o, kWave); u[j] += __shfl_xor(u[j], o, kWave); }
    if (lane_id() < CL) { s_sum[0][threadIdx.x / kWave][cl * VK + j] = g[j]; s_sum[1][threadIdx.x / kWave][cl * VK + j] = u[j]; }
  }
  __syncthreads();
  const int c = n0 + threadIdx.x;
  if (threadIdx.x >= 32 || c >= a.hidden) return;
  float gv = 0.f, uv = 0.f;
#pragma unroll
  for (int i = 0; i < W; i++) { gv += s_sum[0][i][threadIdx.x]; uv += s_sum[1][i][threadIdx.x]; }
  if constexpr (GRAD) {
    const float dh = (float)static_cast<const T *>(a.dh)[r * a.ld_dh + c];
    gate_grad_all<1>(&gv, &uv, &dh, a.act);
    float *out = static_cast<float *>(a.out) + r * 2 * a.hidden + c;
    out[0] = gv;
    out[a.hidden] = uv;
  } else static_cast<T *>(a.out)[r * a.ld_out + c] = (T)((a.act == INK_ACT_GELU ? gelu(gv) : activate(gv, a.act)) * uv);
}

// Gradients of a few rows from dg and du in 32 bits.  dx: a row and 16 columns a workgroup, a wave takes four of them, its lanes side by side along
// the weights' rows.  dWg and dWu: a thread has 16 bytes of a row of each.  In 32 bits because so few numbers do not even out what rounding
// them first would cost, and because these launches are latency alone.
struct GatedFewArgs {
  const float *d;
  const void *x, *gate, *up;
  void *dx, *d_gate, *d_up;
  int64_t rows, ld_x, ld_gate, ld_up, ld_dx, ld_dg, ld_du;
  int cols, hidden;
};
template <class T>
__global__ __launch_bounds__(kHeadThreads) void k_gated_dx_few(GatedFewArgs a) {
  constexpr int VK = kVec<T>;
  const int64_t r = blockIdx.y;
  const int l = lane_id(), c0 = blockIdx.x * 16 + threadIdx.x / kWave * 4;
  float t[4] = {0.f, 0.f, 0.f, 0.f};
  for (int part = 0; part < 2; part++) {
    const float *d = a.d + (r * 2 + part) * a.hidden;
    const T *w = static_cast<const T *>(part ? a.up : a.gate);
    const int64_t ld = part ? a.ld_up : a.ld_gate;
    for (int n = l * VK; n < a.hidden; n += kWave * VK) {
      float dv[VK];
      if (n + VK <= a.hidden) load_pack<float, VK>(d + n, dv);
      else
#pragma unroll
        for (int j = 0; j < VK; j++) dv[j] = n + j < a.hidden ? d[n + j] : 0.f;
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const typename Frag<T>::V v = row_frag<T>(w + (int64_t)min(c0 + q, a.cols - 1) * ld, n, a.hidden);
#pragma unroll
        for (int j = 0; j < VK; j++) t[q] = fmaf(dv[j], (float)v[j], t[q]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 4; q++) {
    t[q] = group_sum<kWave>(t[q]);
    if (l == 0 && c0 + q < a.cols) static_cast<T *>(a.dx)[r * a.ld_dx + c0 + q] = (T)t[q];
  }
}
template <class T>
__global__ __launch_bounds__(kHeadThreads) void k_gated_dw_few(GatedFewArgs a) {
  constexpr int VK = kVec<T>;
  const int pieces = (a.hidden + VK - 1) / VK;
  const int64_t i = (int64_t)blockIdx.x * kHeadThreads + threadIdx.x;
  const int c = (int)(i / pieces), n = max(0, min((int)(i % pieces) * VK, a.hidden - VK));       // a last piece that is cut starts earlier: the same numbers
  if (c >= a.cols) return;
  float g[VK], u[VK];
#pragma unroll
  for (int j = 0; j < VK; j++) g[j] = u[j] = 0.f;
  const T *x = static_cast<const T *>(a.x) + c;
  if (a.hidden >= VK) {
    constexpr int R = 8;                     // rows under way
    for (int64_t r0 = 0; r0 < a.rows; r0 += R) {
      float xv[R], dg[R][VK], du[R][VK];
#pragma unroll
      for (int q = 0; q < R; q++) {
        const int64_t r = min(r0 + q, a.rows - 1);
        xv[q] = (float)x[r * a.ld_x];
        load_pack<float, VK>(a.d + r * 2 * a.hidden + n, dg[q]);
        load_pack<float, VK>(a.d + (r * 2 + 1) * a.hidden + n, du[q]);
      }
#pragma unroll
      for (int q = 0; q < R; q++)
        if (r0 + q < a.rows)
#pragma unroll
          for (int j = 0; j < VK; j++) {
            g[j] = fmaf(xv[q], dg[q][j], g[j]);
            u[j] = fmaf(xv[q], du[q][j], u[j]);
          }
    }
  } else
    for (int64_t r = 0; r < a.rows; r++)
#pragma unroll
      for (int j = 0; j < VK; j++)
        if (j < a.hidden) {
          g[j] = fmaf((float)x[r * a.ld_x], a.d[r * 2 * a.hidden + j], g[j]);
          u[j] = fmaf((float)x[r * a.ld_x], a.d[(r * 2 + 1) * a.hidden + j], u[j]);
        }
  for (int part = 0; part < 2; part++) {
    T *out = static_cast<T *>(part ? a.d_up : a.d_gate);
    if (!out) continue;
    out += c * (part ? a.ld_du : a.ld_dg) + n;
    const float *v = part ? u : g;
    if (n + VK <= a.hidden) store_pack<T, VK>(out, v);
    else
#pragma unroll
      for (int j = 0; j < VK; j++)
        if (n + j < a.hidden) out[j] = (T)v[j];
  }
}

// ------------------------------------------------------------------------------------ host side
// As ink_linear: each workgroup asks for its columns of both matrices again for every row, which the caches serve while the weights fit them.  us a call of 16 rows one by one,
// and of 17 in a tile, bf16: x 256 x 683 8.5 and 8.4 (the binding's time), x 602 x 1605 11.6 and 13.5, x 4096 x 4096 96 and 88, x 16384 x 4096 448 and 329; of one row 8.5, 8.8, 18, 55.
constexpr int64_t kFewRows = 16, kFewResults = 64 * 1024;

// rows of x or of the weights that hold no whole piece of 16 bytes
template <class T> static bool is_short(int cols, int hidden) { return std::min(cols, hidden) < 16 / (int)sizeof(T); }
// Many rows, and a depth whose weights fit the registers: workgroups for the whole card, each with a stream of row tiles.  us a call, stream and tiles:
// bf16 x 128 x 344 16384 rows 11.5 and 9.9, 32700 rows 14.9 and 16.5; x 256 x 683 8192 rows 17.5 and 16.2, 16384 rows 23 and 27; f32 x 128 x 344 16384
// rows 38 and 37, 32700 rows 63 and 68.
constexpr int64_t kStreamRows = 32 * 1024;
template <class T, class TO, int KS, int WN, int WM, int PER, bool GRAD> static void stream_launch(const GatedArgs &a, Launches &run) {
  constexpr int MR = 32 * WM, P = KS * kTypeStep<T> * (int)sizeof(T) + 16, OWN = 32 * (32 * (int)sizeof(TO) + 16) * (GRAD ? 2 : 1), WAVES = WN * WM;
  constexpr int lds = 2 * MR * P + WAVES * (OWN + (sizeof(T) == 1 ? 256 : 0)), per_cu = std::max(1, std::min((160 << 10) / lds, 4 * PER / WAVES));
  static_assert(lds <= 160 << 10, "LDS holds two tiles of rows and the waves' results");
  const int wide = GRAD ? a.pad : a.hidden;
  StreamPlan p;
  p.groups = (wide + 32 * WN - 1) / (32 * WN);
  const int64_t tiles = (a.rows + MR - 1) / MR;
  p.row_groups = (int)std::min<int64_t>((tiles + 7) / 8 * 8, std::max(8, 256 * per_cu / p.groups / 8 * 8));
  run.lds = lds;
  run(k_gated_stream<T, TO, KS, WN, WM, PER, GRAD>, dim3((unsigned)(p.groups * p.row_groups)), dim3(kWave * WAVES), a, p);
  run.lds = 0;
}
// Four waves a workgroup, one on every SIMD of its CU (workgroups of six leave no room for a second one although its registers are there), or, where the
// columns fill them about as well, twelve, three on every SIMD: rows of results then leave a workgroup whole, which counts where they are no multiple of
// whole lines (2.45M x 128 x 341 bf16 722 us with twelve waves, 872 with three workgroups of four; x 344 660 and 765; x 384 654 and 692).  With one or two
// waves side by side a thread has more of the rows under way and registers spill, as in linear.hip: up to 85 (16 bits, 16 steps), 98 (32 bits), 151 (8 bits, 8 steps), all with one wave;
// their calls wait for the rows.  Of the others the forms of 8-bit rows with 4 steps spill four.
template <class T, class TO, int KS, int PER, bool GRAD> static void stream_waves(const GatedArgs &a, Launches &run) {
  const int tiles = ((GRAD ? a.pad : a.hidden) + 31) / 32;
  if (tiles == 1) return stream_launch<T, TO, KS, 1, sizeof(T) == 4 ? 2 : 4, PER, GRAD>(a, run);
  if (tiles == 2 || tiles == 5 || tiles == 6) return stream_launch<T, TO, KS, 2, 2, PER, GRAD>(a, run);
  if constexpr (PER == 3)
    if (tiles > 8 && (tiles + 11) / 12 * 12 <= (tiles + 3) / 4 * 4 + 1) return stream_launch<T, TO, KS, 12, 1, PER, GRAD>(a, run);
  stream_launch<T, TO, KS, 4, 1, PER, GRAD>(a, run);
}
template <class T, class TO, bool GRAD> static bool stream_run(const GatedArgs &a, Launches &run) {
  const int steps = (a.cols + kTypeStep<T> - 1) / kTypeStep<T>;
  if (a.rows < (sizeof(T) == 2 && steps > 8 ? kStreamRows / 2 : kStreamRows)) return false;
  if (is_short<T>(a.cols, sizeof(T) == 1 ? a.cols : a.hidden) || a.hidden < 16 / (int)sizeof(TO)) return false;
  for (const int64_t ld : {a.ld_x, a.ld_out, a.ld_dh})
    if (ld >= 1 << 22) return false;         // offsets within a tile are 32-bit
  if constexpr (sizeof(T) == 4) {
    if (steps <= 8) stream_waves<T, TO, 8, 3, GRAD>(a, run);
    else if (steps <= 16) stream_waves<T, TO, 16, 2, GRAD>(a, run);
    else return false;
  } else if constexpr (sizeof(T) == 2) {
    if (steps <= 8) stream_waves<T, TO, 8, 3, GRAD>(a, run);
    else if (steps <= 16) stream_waves<T, TO, 16, 2, GRAD>(a, run);
    else return false;
  } else {
    if (steps <= 2) stream_waves<T, TO, 2, 3, GRAD>(a, run);
    else if (steps <= 4) stream_waves<T, TO, 4, 3, GRAD>(a, run);
    else if (steps <= 8) stream_waves<T, TO, 8, 2, GRAD>(a, run);
    else return false;
  }
  return true;
}

constexpr int64_t kLaunchRows = 1 << 21;     // a launch has fewer than 2^32 threads: so many rows by INK_MAX_IN_DIM columns are 2^30
template <class TL, class T, class TO> static void gated_tiles(const GatedArgs &a, Launches &run) {
  const int gy = (a.hidden + kTileHidden - 1) / kTileHidden;
  for (int64_t r0 = 0; r0 < a.rows; r0 += kLaunchRows) {
    GatedArgs b = a;
    b.rows = std::min(kLaunchRows, a.rows - r0);
    b.x = static_cast<const TL *>(a.x) + r0 * a.ld_x;
    b.out = static_cast<TO *>(a.out) + r0 * a.ld_out;
    if (a.x_scale) b.x_scale = a.x_scale + r0;
    const int64_t tiles = (b.rows + 127) / 128;
    run(is_short<T>(a.cols, a.hidden) ? k_gated_tile<TL, T, TO, false, true> : k_gated_tile<TL, T, TO, false, false>, dim3((unsigned)((tiles + 7) / 8 * 8 * gy)), dim3(256), b);
  }
}
template <class T, class TO> static void gated_run(const GatedArgs &a, Launches &run) {
  if constexpr (sizeof(T) != 1)
    if (a.rows <= kFewRows && a.rows * a.hidden <= kFewResults)
      return run(k_gated_few<T, false>, dim3((a.hidden + 31) / 32, (unsigned)a.rows), dim3(kHeadThreads), a);
  if constexpr (sizeof(T) != 1 || sizeof(TO) != 4)
    if (stream_run<T, TO, false>(a, run)) return;
  gated_tiles<T, std::conditional_t<sizeof(T) == 1 && sizeof(TO) == 4, bf16, T>, TO>(a, run);
}

// The gradient takes the rows in parts whose dg and du (2 pad columns) have up to 1 GB, so that the work memory does not grow with the rows.  (Parts of
// 128 MB, which the cache behind the L2s would hold, cost more in launches and partial sums than they save: 233k x 256 x 683 bf16 1123 us instead of 1022,
// 353k x 78 x 208 f32 1467 instead of 1227.)
// Few rows in the gradient, or so few numbers in dg that the errors of rounding them would not even out (3 x 602 x 62 bf16: 0.0025 from 64 bits, where
// rounding the results alone gives 0.0017).
static bool grad_of_few(int64_t rows, int hidden) { return rows * hidden <= (rows <= 2 * kFewRows ? kFewResults : rows <= 64 ? 4096 : 0); }
constexpr int64_t kFullTiles = 64;           // tiles of 128 by 128 from which on they are faster than small ones
struct GatedPlan { int pad, ri, wm, wn, tiles_c, tiles_n, slices; int64_t part_rows, slice, d_bytes, range_bytes, part_bytes; };
static GatedPlan gated_plan(int64_t rows, int cols, int hidden, int type) {
  GatedPlan p{};
  p.pad = (hidden + 31) / 32 * 32;
  const int64_t row_bytes = 2ll * p.pad * type_size(type);
  p.part_rows = std::min((rows + 255) / 256 * 256, std::max<int64_t>(1024, (1ll << 30) / row_bytes / 1024 * 1024));
  // the weights' gradients: 128 columns of x by 128 of dg and du; by 256, 128 by 64 a wave, where 16-bit rows are many and have no more columns
  // (1M x 128 x 344 398 us instead of 436, but 100k x 602 x 1605 1006 instead of 833: two workgroups a CU instead of three)
  const bool wide = type != INK_F32 && p.part_rows >= 8192 && cols <= 128;
  p.ri = wide ? 4 : 2;
  p.wm = wide ? 1 : 2;
  p.wn = 4 / p.wm;
  p.tiles_c = (cols + 127) / 128;
  p.tiles_n = (2 * p.pad + 64 * p.wn - 1) / (64 * p.wn);
  // Slices: eight (one a chiplet) times a number that leaves few of a chiplet's 64 or 96 places for workgroups empty (20k x 1024 x 4096
  // in one slice 1586 us, in 8 579; 100k x 602 x 1605 in 7 808, in 16 664); fewer where the rows are few or
  // the partial matrices would have more than 1 GB.
  const int64_t steps = p.part_rows / 64, tiles = (int64_t)p.tiles_c * p.tiles_n, places = wide ? 64 : 96;          // 64 rows: whole chunks of every type
  int64_t best = 1;
  auto used = [&](int64_t k) { return (double)(k * tiles) / (double)((k * tiles + places - 1) / places * places); };
  for (int64_t k = 2; k <= std::max<int64_t>(8, places / tiles) && k * tiles <= 4 * places; k++)
    if (used(k) > used(best) + 0.02) best = k;
  const int64_t tile_bytes = 128 * 64 * p.wn * 4;
  const int64_t slices = std::max<int64_t>(1, std::min({steps / 2, 8 * best, (int64_t)(1 << 30) / (tiles * tile_bytes)}));
  p.slice = (steps + slices - 1) / slices * 64;
  p.slices = (int)(slices >= 8 ? slices : (p.part_rows + p.slice - 1) / p.slice);
  p.d_bytes = p.part_rows * row_bytes;
  p.range_bytes = type == INK_F16 ? p.part_rows / 32 * (2 * p.pad / 32) * (32 + 4) : 0;
  p.part_bytes = (int64_t)p.slices * tiles * tile_bytes;
  return p;
}

template <class T> static void gated_grad(GatedArgs a, const GatedPlan &p, void *work, void *dx, int64_t ld_dx, bool weights, Launches &run) {
  const int64_t rows = a.rows;
  if (p.range_bytes) {
    const int64_t blocks = p.range_bytes / 36;
    a.range.unit = reinterpret_cast<int32_t *>(static_cast<char *>(work) + p.d_bytes);
    a.range.finer = reinterpret_cast<uint8_t *>(a.range.unit + blocks);
    a.range.across = 2 * p.pad / 32;
  }
  const bool brief = is_short<T>(a.cols, a.hidden);
  a.out = work; a.ld_out = 2 * p.pad; a.pad = p.pad;
  for (int64_t r0 = 0; r0 < rows; r0 += p.part_rows) {
    GatedArgs b = a;
    b.rows = std::min(p.part_rows, rows - r0);
    b.x = static_cast<const T *>(a.x) + r0 * a.ld_x;
    b.dh = static_cast<const T *>(a.dh) + r0 * a.ld_dh;
    const int64_t tiles = (b.rows + 127) / 128;
    if (!stream_run<T, T, true>(b, run)) run(brief ? k_gated_tile<T, T, T, true, true> : k_gated_tile<T, T, T, true, false>, dim3((unsigned)((tiles + 7) / 8 * 8 * ((a.hidden + kTileHidden - 1) / kTileHidden))), dim3(256), b);
    if (dx) {
      GatedDxArgs q{work, a.gate, a.up, static_cast<T *>(dx) + r0 * ld_dx, b.rows, a.ld_gate, a.ld_up, ld_dx, a.cols, a.hidden, p.pad, a.range};
      const int gy = (a.cols + 127) / 128;
      if (tiles * gy < kFullTiles) run(brief ? k_gated_dx_small<T, true> : k_gated_dx_small<T, false>, dim3((unsigned)((b.rows + 31) / 32), (a.cols + 31) / 32), dim3(512), q);
      else run(brief ? k_gated_dx<T, true> : k_gated_dx<T, false>, dim3((unsigned)((tiles + 7) / 8 * 8 * gy)), dim3(256), q);
    }
    if (weights) {
      GatedDwArgs q{b.x, work, reinterpret_cast<float *>(static_cast<char *>(work) + p.d_bytes + p.range_bytes), b.rows, a.ld_x, p.slice, a.cols, p.pad, r0 > 0, p.slices,
                    p.tiles_c, p.tiles_n, a.range};
      auto kernel = brief ? k_gated_dw<T, 2, 2, 2, true> : k_gated_dw<T, 2, 2, 2, false>;
      if constexpr (sizeof(T) == 2)
        if (p.ri == 4) kernel = brief ? k_gated_dw<T, 4, 1, 4, true> : k_gated_dw<T, 4, 1, 4, false>;
      run(kernel, dim3((unsigned)(p.slices * p.tiles_c * p.tiles_n)), dim3(256), q);
    }
  }
}

template <class T> static void gated_grad_few(GatedArgs a, GatedFewArgs f, void *work, Launches &run) {
  a.out = work;
  run(k_gated_few<T, true>, dim3((a.hidden + 31) / 32, (unsigned)a.rows), dim3(kHeadThreads), a);
  f.d = static_cast<const float *>(work);
  if (f.dx) run(k_gated_dx_few<T>, dim3((a.cols + 15) / 16, (unsigned)a.rows), dim3(kHeadThreads), f);
  const int64_t pieces = (int64_t)a.cols * ((a.hidden + kVec<T> - 1) / kVec<T>);
  if (f.d_gate || f.d_up) run(k_gated_dw_few<T>, dim3((unsigned)((pieces + kHeadThreads - 1) / kHeadThreads)), dim3(kHeadThreads), f);
}

static const char *gated_check(int64_t rows, int32_t cols, int32_t hidden, int32_t act) {
  if (act < INK_ACT_NONE || act > INK_ACT_SILU) return "unknown activation";
  if (rows < 0 || rows > kMaxHeadRows) return "rows out of range";
  if (cols < 1 || cols > INK_MAX_IN_DIM || hidden < 1 || hidden > INK_MAX_IN_DIM) return "cols and hidden must be 1 .. INK_MAX_IN_DIM";
  return nullptr;
}

}  // namespace ink

using namespace ink;

extern "C" ink_status ink_gated(const void *x, int64_t ld_x, const float *x_scale, const void *w_gate, int64_t ld_gate, const void *w_up,
                                int64_t ld_up, const float *gate_scale, const float *up_scale, int64_t rows, int32_t cols, int32_t hidden,
                                int32_t type, int32_t out_type, int32_t act, void *h, int64_t ld_h, void *hip_stream) {
  const char *who = "ink_gated";
  const bool eight = type == INK_E4M3;
  if (!known_type(type) && !eight) return fail_call(INK_E_ARG, "%s: unknown type", who);
  if (eight ? !known_type(out_type) : out_type != type) return fail_call(INK_E_ARG, "%s: the results' type must be the rows' type, of INK_E4M3 rows one of the others", who);
  if (const char *why = gated_check(rows, cols, hidden, act)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  const int w_rows = eight ? hidden : cols, w_cols = eight ? cols : hidden;
  if (!good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "%s: x is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(w_gate, w_rows, w_cols, ld_gate, type, false)) return fail_call(INK_E_ARG, "%s: w_gate is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(w_up, w_rows, w_cols, ld_up, type, false)) return fail_call(INK_E_ARG, "%s: w_up is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(h, rows, hidden, ld_h, out_type, true)) return fail_call(INK_E_ARG, "%s: h is NULL, not aligned to its type or has rows that overlap", who);
  if (eight && ((rows > 0 && !x_scale) || !gate_scale || !up_scale || !aligned_to(x_scale, 4) || !aligned_to(gate_scale, 4) || !aligned_to(up_scale, 4)))
    return fail_call(INK_E_ARG, "%s: a scale is NULL or not aligned", who);
  if (rows == 0) return INK_OK;
  GatedArgs a{};
  a.x = x; a.gate = w_gate; a.up = w_up; a.x_scale = x_scale; a.gate_scale = gate_scale; a.up_scale = up_scale; a.out = h;
  a.rows = rows; a.ld_x = ld_x; a.ld_gate = ld_gate; a.ld_up = ld_up; a.ld_out = ld_h; a.cols = cols; a.hidden = hidden; a.act = act;
  Launches run(hip_stream);
  if (eight) out_type == INK_F32 ? gated_run<e4m3, float>(a, run) : out_type == INK_BF16 ? gated_run<e4m3, bf16>(a, run) : gated_run<e4m3, f16>(a, run);
  else if (type == INK_F32) gated_run<float, float>(a, run);
  else type == INK_BF16 ? gated_run<bf16, bf16>(a, run) : gated_run<f16, f16>(a, run);
  return run.done(who);
}

extern "C" size_t ink_gated_backward_work(int64_t rows, int32_t cols, int32_t hidden, int32_t type) {
  if (!known_type(type) || rows < 1 || gated_check(rows, cols, hidden, INK_ACT_NONE)) return 0;
  if (grad_of_few(rows, hidden)) return (size_t)rows * 2 * hidden * sizeof(float);
  const GatedPlan p = gated_plan(rows, cols, hidden, type);
  return (size_t)(p.d_bytes + p.range_bytes + p.part_bytes);
}

extern "C" size_t ink_gated_backward_work_dx(int64_t rows, int32_t hidden, int32_t type) {
  if (!known_type(type) || rows < 1 || gated_check(rows, 1, hidden, INK_ACT_NONE)) return 0;
  if (grad_of_few(rows, hidden)) return (size_t)rows * 2 * hidden * sizeof(float);
  const GatedPlan p = gated_plan(rows, 1, hidden, type);         // (parts of the rows do not depend on the columns)
  return (size_t)(p.d_bytes + p.range_bytes);
}

extern "C" ink_status ink_gated_backward(const void *dh, int64_t ld_dh, const void *x, int64_t ld_x, const void *w_gate, int64_t ld_gate,
                                         const void *w_up, int64_t ld_up, int64_t rows, int32_t cols, int32_t hidden, int32_t type, int32_t act,
                                         void *dx, int64_t ld_dx, void *dw_gate, int64_t ld_dg, void *dw_up, int64_t ld_du, void *work,
                                         size_t work_bytes, void *hip_stream) {
  const char *who = "ink_gated_backward";
  if (!known_type(type)) return fail_call(INK_E_ARG, "%s: unknown type", who);
  if (const char *why = gated_check(rows, cols, hidden, act)) return fail_call(INK_E_ARG, "%s: %s", who, why);
  if (!good_matrix(dh, rows, hidden, ld_dh, type, false)) return fail_call(INK_E_ARG, "%s: dh is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(x, rows, cols, ld_x, type, false)) return fail_call(INK_E_ARG, "%s: x is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(w_gate, cols, hidden, ld_gate, type, false)) return fail_call(INK_E_ARG, "%s: w_gate is NULL, not aligned to its type or has rows that overlap", who);
  if (!good_matrix(w_up, cols, hidden, ld_up, type, false)) return fail_call(INK_E_ARG, "%s: w_up is NULL, not aligned to its type or has rows that overlap", who);
  if (dx && !good_matrix(dx, rows, cols, ld_dx, type, true)) return fail_call(INK_E_ARG, "%s: dx is not aligned to its type or has rows that overlap", who);
  if (dw_gate && !good_matrix(dw_gate, cols, hidden, ld_dg, type, true)) return fail_call(INK_E_ARG, "%s: dw_gate is not aligned to its type or has rows that overlap", who);
  if (dw_up && !good_matrix(dw_up, cols, hidden, ld_du, type, true)) return fail_call(INK_E_ARG, "%s: dw_up is not aligned to its type or has rows that overlap", who);
  const bool weights = dw_gate || dw_up;
  const size_t needed = weights ? ink_gated_backward_work(rows, cols, hidden, type) : ink_gated_backward_work_dx(rows, hidden, type);
  if (rows > 0 && (dx || weights) && (!work || !aligned_to(work, 16) || work_bytes < needed))
    return fail_call(INK_E_ARG, "%s: work holds less than ink_gated_backward_work%s bytes or is not aligned to 16", who, weights ? "" : "_dx");
  Launches run(hip_stream);
  GatedArgs a{};
  a.x = x; a.gate = w_gate; a.up = w_up; a.dh = dh;
  a.rows = rows; a.ld_x = ld_x; a.ld_gate = ld_gate; a.ld_up = ld_up; a.ld_dh = ld_dh; a.cols = cols; a.hidden = hidden; a.act = act;
  if (rows > 0 && (dx || weights) && grad_of_few(rows, hidden)) {
    const GatedFewArgs f{nullptr, x, w_gate, w_up, dx, dw_gate, dw_up, rows, ld_x, ld_gate, ld_up, ld_dx, ld_dg, ld_du, cols, hidden};
    if (type == INK_F32) gated_grad_few<float>(a, f, work, run);
    else type == INK_BF16 ? gated_grad_few<bf16>(a, f, work, run) : gated_grad_few<f16>(a, f, work, run);
    return run.done(who);
  }
  GatedPlan p = gated_plan(std::max<int64_t>(rows, 1), cols, hidden, type);
  if (rows > 0 && (dx || weights)) {
    if (type == INK_F32) gated_grad<float>(a, p, work, dx, ld_dx, weights, run);
    else type == INK_BF16 ? gated_grad<bf16>(a, p, work, dx, ld_dx, weights, run) : gated_grad<f16>(a, p, work, dx, ld_dx, weights, run);
  }
  if (weights) {                             // no rows: zeros
    GatedSumArgs s{};
    s.part = reinterpret_cast<const float *>(static_cast<const char *>(work) + p.d_bytes + p.range_bytes);
    s.d_gate = dw_gate; s.d_up = dw_up; s.ld_gate = ld_dg; s.ld_up = ld_du; s.slices = rows > 0 ? p.slices : 0; s.type = type;
    s.cols = cols; s.hidden = hidden; s.pad = p.pad; s.tiles_c = p.tiles_c; s.tiles_n = p.tiles_n; s.kt = 4; s.nt = 2 * p.wn;
    run(k_gated_sum, dim3((unsigned)((int64_t)p.tiles_c * p.tiles_n * s.kt * s.nt * 16)), dim3(256), s);
  }
  return run.done(who);
}
