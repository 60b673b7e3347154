// What the cross-attention kernels share: which keys of a source count, the
// places of rows, and the join of parts of a softmax.
#pragma once

#include "pa_layers.h"

namespace pa {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kDevBadSource = 4;  // an item's source outside [0, G): the item has no keys

// Keys of a source that count, in order. With a mask a list of them is made
// first (k_attn_keys), so that dropped keys are neither read nor multiplied:
// what lies there (infinities, NaN) cannot reach a result.
struct Keys {
  int K;
  const int32_t* len;
  const int32_t* n;     // [G] listed keys (NULL: no mask)
  const int32_t* list;  // [G][K]
  __device__ __forceinline__ int count(int g) const {
    if (n) return n[g];
    return len ? min(max(len[g], 0), K) : K;
  }
  __device__ __forceinline__ int at(int g, int i) const { return list ? list[(int64_t)g * K + i] : i; }
};

__device__ __forceinline__ int source_of(const int32_t* src, int64_t stride, int n, int G, int32_t* status) {
  const int g = src ? src[(int64_t)n * stride] : n;
  if ((unsigned)g < (unsigned)G) return g;
  atomicCAS(status, 0, kDevBadSource);
  return -1;
}
__device__ __forceinline__ int items_of(const int32_t* count, int N) { return count ? min(max(*count, 0), N) : N; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The list above (k_attn.cu).
cudaError_t launch_attn_keys(const AttnArgs& a, int32_t* n, int32_t* list, cudaStream_t st);

}  // namespace pa
