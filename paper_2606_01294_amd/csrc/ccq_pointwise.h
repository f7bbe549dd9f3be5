// ccq_pointwise.h -- device helpers of the operators around the recurrence: vectors of
// channels, sums over lanes, activations.
#pragma once
#include "ccq_device.h"
#include "ccq_kernels.h"

namespace ccq {

// Eight (N) consecutive channels of one row, 16-byte loads and stores.
template <typename T, int N = 8>
struct VecN {
  typedef T raw __attribute__((ext_vector_type(N)));
  static __device__ __forceinline__ raw load(const T* p) { return *reinterpret_cast<const raw*>(p); }
  static __device__ __forceinline__ float get(const raw& v, int e) { return static_cast<float>(v[e]); }
  static __device__ __forceinline__ void store(T* p, const float (&x)[N]) {
    raw v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = static_cast<T>(x[e]);
    *reinterpret_cast<raw*>(p) = v;
  }
};
template <typename T> using Vec8 = VecN<T, 8>;

// x + the value of the lane that CTRL names within the row of 16.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Sum over aligned groups of N <= 16 lanes within the vector unit, where a step costs a
// few cycles instead of a trip through the LDS crossbar.
template <int N>
__device__ __forceinline__ float row_sum(float x) {
  if constexpr (N >= 2) x = dpp_add<0xB1>(x);    // lane ^ 1
  if constexpr (N >= 4) x = dpp_add<0x4E>(x);    // lane ^ 2
  if constexpr (N >= 8) x = dpp_add<0x141>(x);   // mirrored in 8: the other four
  if constexpr (N >= 16) x = dpp_add<0x140>(x);  // mirrored in 16: the other eight
  return x;
}

// act(z) and act'(z): none, silu (z sigmoid z), sigmoid.  bf16 io takes the
// hardware's exponential and reciprocal as they are (about 1e-6 relative, far
// below the 2^-9 of the rounding on store).  fp32 io adds what they lack: the
// rounding of z log2(e), which e^r = 1 + r takes back, and one Newton step of the
// reciprocal (a few 2^-24 in all, in ten instructions).  exp(-z) overflows to
// infinity for z < -88, where sigmoid is then an exact 0.
template <typename T>
struct Act {
  static __device__ __forceinline__ float sigmoid(float z) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.f + __expf(-z));
    const float t = -z * 1.44269504f;
    // -z log2(e) - t, with log2(e) to 48 bits
    float r = __builtin_fmaf(-z, 1.44269504f, -t);
    r = __builtin_fmaf(-z, 1.92596303e-8f, r);
    // (a t or e that overflows takes no correction: infinity times it is NaN)
    r = fabsf(t) < 1e30f ? r * 0.693147181f : 0.f;
    const float e = __builtin_amdgcn_exp2f(t);
    const float d = 1.f + (e < 3e38f ? __builtin_fmaf(e, r, e) : e);
    const float q = __builtin_amdgcn_rcpf(d);
    return d < 3e38f ? __builtin_fmaf(__builtin_fmaf(-d, q, 1.f), q, q) : q;
  }
  static __device__ __forceinline__ float value(int act, float z) {
    if (act == kActNone) return z;
    const float s = sigmoid(z);
    return act == kActSilu ? z * s : s;
  }
  static __device__ __forceinline__ void both(int act, float z, float& v, float& d) {
    if (act == kActNone) {
      v = z;
      d = 1.f;
      return;
    }
    const float s = sigmoid(z);
    if (act == kActSilu) {
      v = z * s;
      d = s * (1.f + z * (1.f - s));
    } else {
      v = s;
      d = s * (1.f - s);
    }
  }
};

}  // namespace ccq
