// What the operators of an answer head (norm.hip, linear.hip, probs.hip) share: element types, vectors of them at any
// address, sums and maxima over groups of lanes, and the checks of their arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ink.h"
#include "prim.h"

namespace ink {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kHeadThreads = 256;

// V elements at an address that is a multiple of the element's size only: the hardware loads 16 bytes at any address, so
// rows of an odd number of elements need no variant of their own.
template <class T, int V> struct Pack { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <class T> struct Pack<T, 1> { typedef T type; };

template <class T, int V> __device__ __forceinline__ void load_pack(const T *p, float out[V]) {
  const typename Pack<T, V>::type v = *reinterpret_cast<const typename Pack<T, V>::type *>(p);
  if constexpr (V == 1) out[0] = (float)v;
  else
#pragma unroll
    for (int j = 0; j < V; j++) out[j] = (float)v[j];
}

// float -> T rounds to nearest, ties to even; NaN stays NaN
template <class T, int V> __device__ __forceinline__ void store_pack(T *p, const float in[V]) {
  typename Pack<T, V>::type v;
  if constexpr (V == 1) v = (T)in[0];
  else
#pragma unroll
    for (int j = 0; j < V; j++) v[j] = (T)in[j];
  *reinterpret_cast<typename Pack<T, V>::type *>(p) = v;
}

// element i of an array whose type is known at run time (weights, biases: read once per launch, not per row)
__device__ __forceinline__ float load_any(const void *p, int64_t i, int type) {
  if (type == INK_F32) return static_cast<const float *>(p)[i];
  return type == INK_BF16 ? (float)static_cast<const bf16 *>(p)[i] : (float)static_cast<const f16 *>(p)[i];
}
__device__ __forceinline__ void store_any(void *p, int64_t i, int type, float v) {
  if (type == INK_F32) static_cast<float *>(p)[i] = v;
  else if (type == INK_BF16) static_cast<bf16 *>(p)[i] = (bf16)v;
  else static_cast<f16 *>(p)[i] = (f16)v;
}

// Reduction over groups of L neighbouring lanes (L a power of two up to 64); every lane gets the result, and every lane of the
// wave has to be there.  Up to 16 lanes by data-parallel moves (a mirrored row does for an exchange once the quads agree), 16 and
// 32 lanes apart by the two swaps of gfx950: no step goes through LDS.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xf, 0xf, false);
}
template <int L, class U, class F> __device__ __forceinline__ U group_all(U x, F f) {
  static_assert(sizeof(U) == 4 && L <= kWave && (L & (L - 1)) == 0, "groups of lanes");
  auto bits = [](U v) { return __builtin_bit_cast(uint32_t, v); };
  auto val = [](uint32_t v) { return __builtin_bit_cast(U, v); };
  if constexpr (L >= 2) x = f(x, val(dpp<0xb1>(bits(x))));         // lane ^ 1
  if constexpr (L >= 4) x = f(x, val(dpp<0x4e>(bits(x))));         // lane ^ 2
  if constexpr (L >= 8) x = f(x, val(dpp<0x141>(bits(x))));        // 7 - lane within eight
  if constexpr (L >= 16) x = f(x, val(dpp<0x140>(bits(x))));       // 15 - lane within sixteen
  if constexpr (L >= 32) { const auto r = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false); x = f(val(r[0]), val(r[1])); }
  if constexpr (L >= 64) { const auto r = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false); x = f(val(r[0]), val(r[1])); }
  return x;
}
template <int L> __device__ __forceinline__ float group_sum(float x) { return group_all<L>(x, [](float a, float b) { return a + b; }); }

// The same over a workgroup of L > 64 threads: through LDS, s holds L / 64 floats and may be used again after the call.
template <int L> __device__ __forceinline__ float block_sum(float x, float *s) {
  constexpr int W = L / kWave;
  x = group_sum<kWave>(x);
  if (lane_id() == 0) s[threadIdx.x / kWave] = x;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < W; i++) t += s[i];
  __syncthreads();
  return t;
}

// ------------------------------------------------------------------------------------ host side
// Sets the message that ink_last_error(NULL) returns on this thread.
ink_status fail_call(ink_status st, const char *fmt, ...) noexcept __attribute__((format(printf, 2, 3)));

inline int type_size(int type) { return type == INK_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == INK_F32 || type == INK_BF16 || type == INK_F16; }
inline bool aligned_to(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// a matrix that is read: rows `ld` elements apart, or one row for all of them (ld = 0); one that is written: no two rows share memory
inline bool good_matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, int type, bool written) {
  if (rows == 0) return true;
  return p && aligned_to(p, type_size(type)) && (ld >= cols || rows == 1 || (!written && ld == 0)) && ld >= 0 && ld < (1ll << 40);
}
constexpr int64_t kMaxHeadRows = (1ll << 31) - 1;

// The kernels of one call: enqueued in order on its stream until one is refused.  The error is the launch's own; one that an
// earlier call of another library left behind is neither reported nor cleared.
struct Launches {
  hipStream_t stream;
  hipError_t error = hipSuccess;
  int lds = 0;                               // bytes of LDS that the next kernels get on top of their own
  explicit Launches(void *hip_stream) : stream((hipStream_t)hip_stream) {}
  template <class... P, class... A> void operator()(void (*kernel)(P...), dim3 grid, dim3 block, A... args) {
    if (error != hipSuccess) return;
    enqueue(kernel, grid, block, static_cast<P>(args)...);
  }
  ink_status done(const char *who) const {
    return error == hipSuccess ? INK_OK : fail_call(INK_E_DEVICE, "%s: %s", who, hipGetErrorString(error));
  }

 private:
  template <class... P> void enqueue(void (*kernel)(P...), dim3 grid, dim3 block, P... args) {
    void *ptrs[] = {(void *)&args...};
    error = hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, ptrs, (size_t)lds, stream);
  }
};

}  // namespace ink
