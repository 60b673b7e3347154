// What the cross-attention kernels share: which keys of a source count, the
// places of rows, and the join of parts of a softmax.
#pragma once

#include "pa_bulk.cuh"
#include "pa_layers.h"
#include "pa_tcgen05.cuh"

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

// ---- tensor-core kernels: operand tiles and their copies ---------------------
// A tile of rows [row][d] lies in shared memory as core matrices of 8 rows x 16
// bytes, those of eight rows side by side: one layout in which the rows are M or
// N and d is K, or d is N (or M) and the rows are K. d16: d rounded up to 16; the
// last eight columns of it are zeros where d % 16 == 8.
__device__ __forceinline__ uint64_t tile_desc_rows(uint32_t base, int d16) {  // rows: M or N; d: K
  return tc_smem_desc(base, 128, (uint32_t)d16 * 16);
}
__device__ __forceinline__ uint64_t tile_desc_cols(uint32_t base, int d16) {  // d: M or N; rows: K
  return tc_smem_desc(base, (uint32_t)d16 * 16, 128);
}

// Bounded wait (about a second); after a failure a thread no longer waits, runs
// on with accesses in bounds, and the call's results are not valid.
__device__ __forceinline__ void wait_or_bad(uint64_t* bar, uint32_t parity, bool& bad, int32_t* status) {
  if (bad || mbar_test(bar, parity)) return;
  const long long t0 = clock64();
  while (!mbar_try(bar, parity)) {
    if (clock64() - t0 > 2000000000ll) {
      bad = true;
      atomicCAS(status, 0, kDevTimeout);
      return;
    }
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// The loader threads' copies: a job is the copies behind one mbarrier. Up to
// three jobs are in flight; a job's barrier gets each thread's arrival when the
// thread's copies have landed and are visible to the tensor core.
struct Jobs {
  uint64_t *b0, *b1;
  int n;
  __device__ Jobs() : b0(nullptr), b1(nullptr), n(0) {}
  __device__ __forceinline__ void push(uint64_t* bar) {
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (n == 2) {
      asm volatile("cp.async.wait_group 2;" ::: "memory");
      fence_proxy_async_smem();
      mbar_arrive(b0);
      b0 = b1;
      b1 = bar;
    } else {
      if (n == 0) b0 = bar;
      else b1 = bar;
      ++n;
    }
  }
  __device__ __forceinline__ void flush() {
    if (n == 0) return;
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    fence_proxy_async_smem();
    mbar_arrive(b0);
    if (n == 2) mbar_arrive(b1);
    n = 0;
  }
  // A wait of a loader: what others wait for comes first.
  __device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, bool& bad, int32_t* status) {
    if (!bad && mbar_test(bar, parity)) return;
    flush();
    wait_or_bad(bar, parity, bad, status);
  }
};

constexpr int kLoadWarps = 3;  // with the warp that issues the MMAs a multiple of four: registers go by four warps
constexpr int kLoadThreads = kLoadWarps * 32;

// Copy `rows` (a multiple of 8) rows of a tile: row r from at(r), zeros where at
// gives NULL. `any`: an address that may be named. By kLoadThreads threads.
template <typename T, typename At>
__device__ __forceinline__ void copy_tile(uint32_t dst, int rows, int d, int d16, const T* any, int tid, At at) {
  const int nch = d >> 3, r = tid & 7;
  int c = tid >> 3, rg = 0;
  while (c >= nch) {
    c -= nch;
    ++rg;
  }
  const int dc = (kLoadThreads / 8) % nch, dg = (kLoadThreads / 8) / nch;
  for (; rg * 8 < rows;) {
    const T* p = at(rg * 8 + r);
    copy16(dst + (uint32_t)(rg * (d16 >> 3) + c) * 128 + r * 16, p ? p + c * 8 : any, p != nullptr);
    c += dc;
    rg += dg;
    if (c >= nch) {
      c -= nch;
      ++rg;
    }
  }
}

// The list above (k_attn.cu).
cudaError_t launch_attn_keys(const AttnArgs& a, int32_t* n, int32_t* list, int32_t* pos, cudaStream_t st);
// The forward pass on the tensor cores (k_attn_tc.cu); parts of the keys, 1:
// none, else po [row][part][D] and pl [row][part] are written for the join.
int attn_tc_splits(const AttnArgs& a);
cudaError_t launch_attn_tc(const AttnArgs& a, const Keys& keys, float* po, float* pl, cudaStream_t st);

}  // namespace pa
