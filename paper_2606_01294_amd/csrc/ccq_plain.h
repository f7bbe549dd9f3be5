// ccq_plain.h -- device helpers of the plain delta rule's paths through the Gated
// DeltaNet kernels.
#pragma once
#include "ccq_device.h"

namespace ccq {

// Query/key heads of a tensor and the one that value head h (of H) reads: with HK
// query/key heads, consecutive H / HK value heads share one; HK = 0: every value
// head has its own.
struct KeyHead {
  int H, h;
};
__device__ __forceinline__ KeyHead key_head(int HK, int H, int h) {
  return HK ? KeyHead{HK, h / (H / HK)} : KeyHead{H, h};
}

// The value of the neighbouring lane (lane ^ 1).
__device__ __forceinline__ float lane_swap(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xf, 0xf, true));
}

}  // namespace ccq
