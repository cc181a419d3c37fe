// One step of AdamW over many tensors.
//
//   g = grad * grad_scale,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: some fifteen operations an element against 28 bytes (32-bit parameters and moments, 16-bit gradient and copy) or 16 (moments in
// 8 bits), at the rate of a copy (5.09 TB/s): 186M elements in 259 tensors 1025 us (5.20 GB), 27.7M with moments in 8 bits 94 us (448 MB).  One launch takes
// up to kAdamTensors tensors, whose addresses are its arguments, so that nothing is copied to the device ahead; workgroups take kAdamTile elements
// or several times that of one tensor and find it by a search over the tensors' first workgroups.  A thread has eight neighbouring elements.
//
// Moments in 8 bits: of 128 neighbouring elements each has an e4m3 code and all share a scale (their largest magnitude / 448), m as it is, of v
// the root, whose logarithm spans half the range.  Sixteen lanes hold such a block; the new scale is their maximum.  A moving average changes by 0.1 % a
// step, and the numbers of e4m3 lie 6 to 12 % apart: rounded to the nearest it would never move.  So a number between two codes goes to
// either with the probability of its nearness (the expectation is the number itself), by a random number that is a hash of seed, step, tensor and
// element.  The root never becomes 0 unless it is: where sqrt(v) in the denominator vanished, the step would be m / eps.  So a root below the smallest code, 2^-9 of
// the scale, is held there, not rounded by chance: from 1/229376 of the block's largest root down the steps are too small, and never too large.  Parameters in bfloat16 are rounded the
// same way, for the same reason; a copy in 16 bits, which no step reads again, to the nearest.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "head.h"

namespace ink {

constexpr int kAdamTensors = 32, kAdamEach = 8, kAdamTile = kHeadThreads * kAdamEach, kAdamBlock = INK_ADAMW_BLOCK;
static_assert(kAdamBlock == 16 * kAdamEach, "sixteen lanes hold a block");

struct AdamArgs {
  ink_adamw_tensor tensor[kAdamTensors];
  int32_t first[kAdamTensors];             // of a tensor's workgroups; behind the last tensor INT32_MAX
  int32_t tiles;                           // tiles a workgroup takes, one after another
  const int64_t *step_at;                  // the step's number on the device, or NULL
  const float *scale_at;                   // a factor of the gradient on the device, or NULL
  double log_b1, log_b2, lr;
  int64_t step;
  uint64_t seed;
  float b1, b2, new1, new2, by_m, by_v, eps, keep, grad_scale;
};

// A 32-bit number of a 32-bit number, every bit of it depending on every bit: two multiplications (odd numbers: the golden
// ratio's and the root of 3's fraction) between shifts.
__host__ __device__ inline uint32_t mix_bits(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9e3779b1u;
  x ^= x >> 15;
  x *= 0xbb67ae85u;
  return x ^ x >> 16;
}
constexpr uint32_t kMixNext = 0x6a09e667u;     // the root of 2's fraction

__device__ __forceinline__ uint32_t adam_key(uint32_t id, int64_t step, uint64_t seed, uint32_t high) {
  uint32_t k = 0;
  for (const uint32_t part : {id, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed, (uint32_t)(seed >> 32)}) k = mix_bits(k + part + kMixNext);
  return mix_bits(k + high);
}

// e4m3 code of 0 <= a <= 448: the 20 bits of `random` decide between the codes around a.  Below 2^-6 the numbers are multiples of
// 2^-9, above they have 3 bits behind the first: 20 of a float's bits are the rest.
__device__ __forceinline__ uint32_t code_by_chance(float a, uint32_t random) {
  const uint32_t low = ((uint32_t)(a * 536870912.f) + random) >> 20, high = ((__float_as_uint(a) + random) >> 20) - (120u << 3);
  return min(a < 0.015625f ? low : high, 0x7eu);
}

// Eight numbers of a block to codes and the block's scale, which all sixteen lanes of the block get.  With a number that is
// none the scale is none.
template <bool ROOT> __device__ __forceinline__ float to_codes(const float x[8], const uint32_t random[8], uint32_t code[2]) {
#pragma clang fp contract(off)
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; j++) top = fmaxf(top, fabsf(x[j]) <= 3.4028235e38f ? fabsf(x[j]) : INFINITY);
  top = group_all<16>(top, [](float a, float b) { return fmaxf(a, b); });
  const float scale = top == INFINITY ? NAN : top < 448.f * 1.17549435e-38f ? 0.f : top * (1.f / 448.f);
  const float by = scale > 0.f ? 1.f / scale : 0.f;
  code[0] = code[1] = 0;
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const float a = fabsf(x[j]) * by;
    uint32_t c = code_by_chance(a, random[j] & 0xfffffu);
    if (ROOT) c = a > 0.f ? max(c, 1u) : 0u;
    else c |= __float_as_uint(x[j]) >> 31 << 7;
    code[j / 4] |= c << 8 * (j % 4);
  }
  return scale;
}

__device__ __forceinline__ void from_codes(const uint32_t code[2], float scale, float x[8]) {
#pragma unroll
  for (int j = 0; j < 2; j++) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[j], true);
    x[4 * j] = lo[0] * scale; x[4 * j + 1] = lo[1] * scale; x[4 * j + 2] = hi[0] * scale; x[4 * j + 3] = hi[1] * scale;
  }
}

template <class T> __device__ __forceinline__ void load8(const T *p, int n, float v[8]) {
  if (n >= 8) return load_pack<T, 8>(p, v);
#pragma unroll
  for (int j = 0; j < 8; j++) v[j] = j < n ? (float)p[j] : 0.f;
}
template <class T> __device__ __forceinline__ void store8(T *p, int n, const float v[8]) {
  if (n >= 8) return store_pack<T, 8>(p, v);
#pragma unroll
  for (int j = 0; j < 8; j++)
    if (j < n) p[j] = (T)v[j];
}
__device__ __forceinline__ void load_codes(const uint8_t *p, int n, uint32_t code[2]) {
  typedef uint32_t W __attribute__((ext_vector_type(2), aligned(1)));
  code[0] = code[1] = 0;
  if (n >= 8) { const W w = *reinterpret_cast<const W *>(p); code[0] = w[0]; code[1] = w[1]; return; }
#pragma unroll
  for (int j = 0; j < 8; j++)
    if (j < n) code[j / 4] |= (uint32_t)p[j] << 8 * (j % 4);
}
__device__ __forceinline__ void store_codes8(uint8_t *p, int n, const uint32_t code[2]) {
  typedef uint32_t W __attribute__((ext_vector_type(2), aligned(1)));
  if (n >= 8) { *reinterpret_cast<W *>(p) = W{code[0], code[1]}; return; }
#pragma unroll
  for (int j = 0; j < 8; j++)
    if (j < n) p[j] = (uint8_t)(code[j / 4] >> 8 * (j % 4));
}

struct None {};                            // no copy

template <class TP, class TG, class TC, bool EIGHT>
__global__ __launch_bounds__(kHeadThreads) void k_adamw(AdamArgs a) {
  // Every operation is rounded by itself, none fused: a plain program of the same formulas then has the same bits, and the same codes (a number
  // that differs in its last bit falls on the other side of a random number now and then).  Memory bounds the kernel either way.
#pragma clang fp contract(off)
  constexpr bool CHANCE = EIGHT || sizeof(TP) == 2;
  int k = 0;
#pragma unroll
  for (int o = kAdamTensors / 2; o; o >>= 1)
    if ((int)blockIdx.x >= a.first[k + o]) k += o;             // no workgroup belongs to places behind the last tensor
  const ink_adamw_tensor t = a.tensor[k];
  const int64_t at = (int64_t)((int)blockIdx.x - a.first[k]) * a.tiles * kAdamTile;
  float by_m = a.by_m, by_v = a.by_v, grad_scale = a.grad_scale;
  int64_t step = a.step;
  if (a.step_at) {
    step = max(*a.step_at, (int64_t)1);
    by_m = (float)(a.lr / -expm1((double)step * a.log_b1));
    by_v = (float)(1.0 / sqrt(-expm1((double)step * a.log_b2)));
  }
  if (a.scale_at) grad_scale *= *a.scale_at;
  const uint32_t key = CHANCE ? adam_key((uint32_t)t.id, step, a.seed, (uint32_t)(at >> 32)) : 0;
  for (int i = 0; i < a.tiles; i++) {
    const int64_t e = at + (int64_t)i * kAdamTile + threadIdx.x * kAdamEach;
    if (at + (int64_t)i * kAdamTile >= t.n) break;
    const int n = (int)max((int64_t)0, min((int64_t)kAdamEach, t.n - e));
    float p[8], g[8], m[8], v[8];
    load8(static_cast<const TP *>(t.param) + e, n, p);
    load8(static_cast<const TG *>(t.grad) + e, n, g);
    if constexpr (EIGHT) {
      uint32_t cm[2], cv[2];
      load_codes(static_cast<const uint8_t *>(t.m) + e, n, cm);
      load_codes(static_cast<const uint8_t *>(t.v) + e, n, cv);
      const float sm = n ? t.m_scale[e / kAdamBlock] : 0.f, sv = n ? t.v_scale[e / kAdamBlock] : 0.f;
      from_codes(cm, sm, m);
      from_codes(cv, sv, v);
#pragma unroll
      for (int j = 0; j < 8; j++) v[j] *= v[j];
    } else {
      load8(static_cast<const float *>(t.m) + e, n, m);
      load8(static_cast<const float *>(t.v) + e, n, v);
    }
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      g[j] *= grad_scale;
      m[j] = a.b1 * m[j] + a.new1 * g[j];
      v[j] = a.b2 * v[j] + a.new2 * (g[j] * g[j]);
      root[j] = sqrtf(v[j]);
      p[j] = p[j] * a.keep - by_m * m[j] / (root[j] * by_v + a.eps);
    }
    uint32_t first[8], second[8];
    if constexpr (CHANCE)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        first[j] = mix_bits((uint32_t)(e + j) ^ key);
        second[j] = mix_bits(first[j] + kMixNext);
      }
    if constexpr (sizeof(TP) == 2) {
#pragma unroll
      for (int j = 0; j < 8; j++)              // the result is a number of 16 bits: the store does not round it again
        if (fabsf(p[j]) <= 3.4028235e38f) p[j] = __uint_as_float((__float_as_uint(p[j]) + (first[j] >> 20) + ((second[j] >> 20 & 15u) << 12)) & 0xffff0000u);
    }
    store8(static_cast<TP *>(t.param) + e, n, p);
    if constexpr (!__is_same(TC, None)) store8(static_cast<TC *>(t.copy) + e, n, p);
    if constexpr (EIGHT) {
      uint32_t cm[2], cv[2];
      const float sm = to_codes<false>(m, first, cm), sv = to_codes<true>(root, second, cv);
      store_codes8(static_cast<uint8_t *>(t.m) + e, n, cm);
      store_codes8(static_cast<uint8_t *>(t.v) + e, n, cv);
      if (n > 0 && threadIdx.x % 16 == 0) { t.m_scale[e / kAdamBlock] = sm; t.v_scale[e / kAdamBlock] = sv; }
    } else {
      store8(static_cast<float *>(t.m) + e, n, m);
      store8(static_cast<float *>(t.v) + e, n, v);
    }
  }
}

typedef void (*AdamKernel)(AdamArgs);
template <class TP, class TG, class TC> static AdamKernel adam_bits(bool eight) { return eight ? k_adamw<TP, TG, TC, true> : k_adamw<TP, TG, TC, false>; }
template <class TG> static AdamKernel adam_params(int param_type, int copy_type, bool eight) {
  if (param_type == INK_BF16) return adam_bits<bf16, TG, None>(eight);
  return copy_type == INK_BF16 ? adam_bits<float, TG, bf16>(eight) : copy_type == INK_F16 ? adam_bits<float, TG, f16>(eight) : adam_bits<float, TG, None>(eight);
}
static AdamKernel adam_kernel(int param_type, int grad_type, int copy_type, bool eight) {
  if (grad_type == INK_F32) return adam_params<float>(param_type, copy_type, eight);
  return grad_type == INK_BF16 ? adam_params<bf16>(param_type, copy_type, eight) : adam_params<f16>(param_type, copy_type, eight);
}

static const char *adam_tensor_check(const ink_adamw_tensor &t, int param_type, int grad_type, int copy_type, bool eight) {
  if (t.n < 0 || t.n >= 1ll << 40) return "elements out of range";
  if (t.n == 0) return nullptr;
  if (!t.param || !t.grad || !t.m || !t.v || (copy_type != INK_NO_TYPE && !t.copy) || (eight && (!t.m_scale || !t.v_scale))) return "a pointer is NULL";
  if (!aligned_to(t.param, type_size(param_type)) || !aligned_to(t.grad, type_size(grad_type)) || (copy_type != INK_NO_TYPE && !aligned_to(t.copy, type_size(copy_type))) ||
      (!eight && (!aligned_to(t.m, 4) || !aligned_to(t.v, 4))) || (eight && (!aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))))
    return "a pointer is not aligned to its type";
  return nullptr;
}

struct Extent { uintptr_t begin, end; };
// Whether a step over these tensors changes memory twice, or reads what it changes: workgroups would do so in no order.  What it changes, sorted; the
// rest is looked up in it.
static const char *adam_overlap(const ink_adamw_tensor *tensors, int n_tensors, int param_type, int grad_type, int copy_type, bool eight, const int64_t *step_at,
                                const float *scale_at, Extent *changed) {
  int n = 0;
  auto add = [&](const void *p, int64_t bytes) { changed[n++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes}; };
  for (int i = 0; i < n_tensors; i++) {
    const ink_adamw_tensor &t = tensors[i];
    if (!t.n) continue;
    add(t.param, t.n * type_size(param_type));
    add(t.m, t.n * (eight ? 1 : 4));
    add(t.v, t.n * (eight ? 1 : 4));
    if (copy_type != INK_NO_TYPE) add(t.copy, t.n * type_size(copy_type));
    if (eight) {
      add(t.m_scale, (t.n + kAdamBlock - 1) / kAdamBlock * 4);
      add(t.v_scale, (t.n + kAdamBlock - 1) / kAdamBlock * 4);
    }
  }
  std::sort(changed, changed + n, [](const Extent &a, const Extent &b) { return a.begin < b.begin; });
  for (int i = 1; i < n; i++)
    if (changed[i].begin < changed[i - 1].end) return "memory that the step changes stands in the call twice";
  auto apart = [&](const void *p, int64_t bytes) {               // of disjoint extents in order the last that begins before p + bytes decides
    const Extent *e = std::lower_bound(changed, changed + n, (uintptr_t)p + (uintptr_t)bytes, [](const Extent &a, uintptr_t at) { return a.begin < at; });
    return e == changed || e[-1].end <= (uintptr_t)p;
  };
  for (int i = 0; i < n_tensors; i++)
    if (tensors[i].n && !apart(tensors[i].grad, tensors[i].n * type_size(grad_type))) return "a gradient stands in memory that the step changes";
  if ((step_at && !apart(step_at, 8)) || (scale_at && !apart(scale_at, 4))) return "step_at or grad_scale_at stands in memory that the step changes";
  return nullptr;
}

}  // namespace ink

using namespace ink;

extern "C" ink_status ink_adamw(const ink_adamw_tensor *tensors, int32_t n_tensors, int32_t param_type, int32_t grad_type, int32_t copy_type,
                                int32_t moment_bits, double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                                const int64_t *step_at, double grad_scale, const float *grad_scale_at, uint64_t seed, void *hip_stream) {
  const char *who = "ink_adamw";
  auto refuse = [&](const char *why) { return fail_call(INK_E_ARG, "%s: %s", who, why); };
  if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return refuse("tensors is NULL or their number negative");
  if (param_type != INK_F32 && param_type != INK_BF16) return refuse("parameters are INK_F32 or INK_BF16");
  if (!known_type(grad_type)) return refuse("unknown type of the gradients");
  if (copy_type != INK_NO_TYPE && ((copy_type != INK_BF16 && copy_type != INK_F16) || param_type != INK_F32)) return refuse("a copy is INK_BF16 or INK_F16, of INK_F32 parameters");
  if (moment_bits != 32 && moment_bits != 8) return refuse("moments have 32 or 8 bits");
  if (!(lr >= 0 && lr <= 1e18)) return refuse("lr must be 0 .. 1e18");        // its product with 1 / (1 - beta1), or with the decay, is a float
  if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1)) return refuse("the betas must lie in [0, 1)");
  if (!(eps >= 1.2e-38 && eps < 1e30)) return refuse("eps must be positive, a normal float and finite");
  if (!(weight_decay >= 0 && weight_decay <= 1e18)) return refuse("weight_decay must be 0 .. 1e18");
  if (!(std::fabs(grad_scale) < 3e38)) return refuse("grad_scale must be finite");
  if (!step_at && step < 1) return refuse("steps count from 1");
  if (!aligned_to(step_at, 8) || !aligned_to(grad_scale_at, 4)) return refuse("step_at or grad_scale_at is not aligned");
  const bool eight = moment_bits == 8;
  for (int i = 0; i < n_tensors; i++)
    if (const char *why = adam_tensor_check(tensors[i], param_type, grad_type, copy_type, eight)) return fail_call(INK_E_ARG, "%s: tensor %d: %s", who, i, why);
  const std::unique_ptr<Extent[]> extents(new (std::nothrow) Extent[6 * (size_t)n_tensors + 1]);
  if (!extents) return fail_call(INK_E_OOM, "%s: no memory to look for tensors that overlap", who);
  if (const char *why = adam_overlap(tensors, n_tensors, param_type, grad_type, copy_type, eight, step_at, grad_scale_at, extents.get())) return refuse(why);
  AdamArgs a{};
  a.step_at = step_at; a.scale_at = grad_scale_at; a.step = step_at ? 1 : step; a.seed = seed; a.lr = lr;
  a.log_b1 = std::log(beta1); a.log_b2 = std::log(beta2);
  a.b1 = (float)beta1; a.b2 = (float)beta2; a.new1 = (float)(1 - beta1); a.new2 = (float)(1 - beta2);
  a.eps = (float)eps; a.keep = (float)(1 - lr * weight_decay); a.grad_scale = (float)grad_scale;
  a.by_m = (float)(lr / -std::expm1((double)a.step * a.log_b1));
  a.by_v = (float)(1 / std::sqrt(-std::expm1((double)a.step * a.log_b2)));
  const AdamKernel kernel = adam_kernel(param_type, grad_type, copy_type, eight);
  Launches run(hip_stream);
  for (int i = 0; i < n_tensors;) {
    int n = 0;
    int64_t tiles = 0;
    for (; i < n_tensors && n < kAdamTensors; i++)
      if (tensors[i].n) {
        a.tensor[n++] = tensors[i];
        tiles += (tensors[i].n + kAdamTile - 1) / kAdamTile;
      }
    if (!n) break;
    // tiles a workgroup: one until the card is full several times over; a power of two, so that none crosses a multiple of 2^32 elements
    for (a.tiles = 1; a.tiles < 1 << 20 && tiles / a.tiles >= 2 * 16384; a.tiles *= 2) {}
    int64_t groups = 0;
    for (int k = 0; k < kAdamTensors; k++) {
      a.first[k] = k < n ? (int32_t)groups : INT32_MAX;
      if (k < n) groups += (a.tensor[k].n + (int64_t)a.tiles * kAdamTile - 1) / ((int64_t)a.tiles * kAdamTile);
    }
    run(kernel, dim3((unsigned)groups), dim3(kHeadThreads), a);
  }
  return run.done(who);
}
