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

// The (value head, chunk) of workgroup x, of N chunks a sequence, in a packed batch.
// Consecutive workgroups go to the eight compute-unit clusters in turn: a (sequence,
// query/key head, chunk) goes to one cluster with all of its value heads one after the
// other, which find its q and k in the cluster's L2; the chunks of a sequence go to the
// clusters in turn, from another one for every head, so that the long sequences load all
// alike.  (8 sequences of 680 to 2048 tokens, 8 value heads on 4, dk = dv = 128, chunk
// gradients: 129 us, with whole sequences on a cluster 147, the longest one's time.  A
// batch of one length takes the same either way and keeps the plain order.)
struct ChunkOf {
  int bh, ci;
};
__device__ __forceinline__ ChunkOf chunk_of(int x, int B, int HK, int H, int N) {
  const int G = H / HK, units = B * HK * N, full = units & ~7;
  int u, g;
  if (x < full * G) {
    u = x / 8 / G * 8 + x % 8;
    g = x / 8 % G;
  } else {
    u = full + (x - full * G) / G;
    g = (x - full * G) % G;
  }
  const int bk = u / N, ci = (u % N + bk) % N;
  return ChunkOf{bk / HK * H + bk % HK * G + g, ci};
}

// The value of the neighbouring lane (lane ^ 1).
__device__ __forceinline__ float lane_swap(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xf, 0xf, true));
}

}  // namespace ccq
