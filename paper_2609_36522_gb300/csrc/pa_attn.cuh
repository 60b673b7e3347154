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

// Two fp32 values in one instruction.
struct F2 {
  uint64_t v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ F2(uint32_t a, uint32_t b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(a), "r"(b)); }
  __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// f(values, first column) over the n16 TMEM columns (a multiple of 16) of this
// thread's lane, W at a time, then 16. A load takes its latency whatever its width,
// so few wide ones: 16 at a time with the next 16 on their way were slower (100 x 4096
// tokens, 77 keys of 40: 214 us against 177).
template <int N, typename F>
__device__ __forceinline__ void column_block(uint32_t t, int c, F& f) {
  uint32_t r[N];
  tmem_ld(t + c, r);
  tmem_ld_wait();
  f(r, c);
}
template <int W, typename F>
__device__ __forceinline__ void columns(uint32_t t, int n16, F f) {
  int c = 0;
  for (; c + W <= n16; c += W) column_block<W>(t, c, f);
  if constexpr (W > 16)
    for (; c < n16; c += 16) column_block<16>(t, c, f);
}
// The same over two sets of columns.
template <int N, typename F>
__device__ __forceinline__ void column_block2(uint32_t t, uint32_t u, int c, F& f) {
  uint32_t r[N], d[N];
  tmem_ld(t + c, r);
  tmem_ld(u + c, d);
  tmem_ld_wait();
  f(r, d, c);
}
template <int W, typename F>
__device__ __forceinline__ void columns2(uint32_t t, uint32_t u, int n16, F f) {
  int c = 0;
  for (; c + W <= n16; c += W) column_block2<W>(t, u, c, f);
  if constexpr (W > 16)
    if (c < n16) column_block2<16>(t, u, c, f);
}

// A warp's 32 rows of a tile, `scale` times the D columns from t on, to memory in
// 16 bits: staged in shared memory (su 16-byte units of a row at a time, sstride
// units apart; usu = 65536 / su + 1), then neighbouring lanes write neighbouring
// units. off: where this lane's row goes, in elements (negative: nowhere). zero: zeros.
template <typename T>
__device__ __forceinline__ void rows_out(T* to, int64_t off, uint32_t t, int D, float scale, bool zero, unsigned char* stage,
                                         int su, int sstride, uint32_t usu, int lane) {
  for (int c0 = 0; c0 < D; c0 += su * 8) {
    const int cols = min(su * 8, D - c0);
    unsigned char* mine = stage + lane * sstride * 16;
    if (zero) {
      for (int u = 0; u < cols / 8; ++u) *reinterpret_cast<uint4*>(mine + u * 16) = make_uint4(0, 0, 0, 0);
    } else {
      columns<16>(t + c0, (cols + 15) & ~15, [&](auto& r, int c) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] = __uint_as_float(r[8 * h + q]) * scale;
          if (h == 0 || c + 8 < cols) *reinterpret_cast<uint4*>(mine + (c / 8 + h) * 16) = Elem<T>::pack(v);
        }
      });
    }
    __syncwarp();
    for (int q = 0; q < su; ++q) {
      const uint32_t e = q * 32 + lane, r = (e * usu) >> 16, u = e - r * su;
      const int64_t o = __shfl_sync(0xffffffffu, off, r);
      if (o >= 0 && (int)u * 8 < cols)
        *reinterpret_cast<uint4*>(to + o + c0 + u * 8) = *reinterpret_cast<const uint4*>(stage + (r * sstride + u) * 16);
    }
    __syncwarp();
  }
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

// n K steps of an MMA from descriptors whose start addresses move by `da`, `db`
// 16-byte units a step; one thread. With A in TMEM a step is eight columns.
__device__ __forceinline__ void mma_steps(uint32_t d, uint64_t a, uint32_t da, uint64_t b, uint32_t db, int n, uint32_t idesc,
                                          bool add) {
  for (int k = 0; k < n; ++k, a += da, b += db) tc_mma_f16(d, a, b, idesc, add || k > 0 ? 1u : 0u);
}
__device__ __forceinline__ void mma_steps_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t db, int n, uint32_t idesc, bool add) {
  for (int k = 0; k < n; ++k, a += 8, b += db) tc_mma_f16_ta(d, a, b, idesc, add || k > 0 ? 1u : 0u);
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

// The loader threads' copies of a job land some time later; its mbarrier then
// gets each thread's arrival. Whoever waits for them to issue MMAs makes them
// visible to the tensor core (landed).
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void copies_drain() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void landed(uint64_t* bar, uint32_t parity, bool& bad, int32_t* status) {
  wait_or_bad(bar, parity, bad, status);
  fence_proxy_async_smem();
}

// Copy `rows` (a multiple of 8) rows of a tile by LT threads, zeros from row
// `valid` on. Eight neighbouring threads fill a core matrix; neighbouring groups
// of eight take neighbouring 16-byte pieces of the same eight rows. Rows at one
// distance: pointers only ever step.
template <int LT, typename T>
__device__ __forceinline__ void copy_rows(uint32_t dst, int rows, int valid, int d, int d16, const T* base, int64_t stride,
                                          int tid) {
  const int nch = d >> 3;
  int c = tid >> 3, row = tid & 7;
  row += c / nch * 8;
  c %= nch;
  const T* p = base + row * stride + c * 8;
  dst += (uint32_t)(row >> 3) * d16 * 16 + c * 128 + (row & 7) * 16;
  const int dc = (LT / 8) % nch, dr = (LT / 8) / nch * 8;
  const int64_t dp = dr * stride + dc * 8, wp = 8 * stride - nch * 8;
  const uint32_t dd = (uint32_t)(dr >> 3) * d16 * 16 + dc * 128, wd = (uint32_t)d16 * 16 - nch * 128;
#pragma unroll 2
  while (row < rows) {
    copy16(dst, row < valid ? p : base, row < valid);
    c += dc;
    row += dr;
    p += dp;
    dst += dd;
    if (c >= nch) {
      c -= nch;
      row += 8;
      p += wp;
      dst += wd;
    }
  }
}
// Rows at offsets (in elements, negative: zeros) that a table in shared memory holds.
template <int LT, typename T>
__device__ __forceinline__ void copy_rows_at(uint32_t dst, int rows, int d, int d16, const T* base, const int64_t* off, int tid) {
  const int nch = d >> 3;
  int c = tid >> 3, row = tid & 7;
  row += c / nch * 8;
  c %= nch;
  dst += (uint32_t)(row >> 3) * d16 * 16 + c * 128 + (row & 7) * 16;
  const int dc = (LT / 8) % nch, dr = (LT / 8) / nch * 8;
  const uint32_t dd = (uint32_t)(dr >> 3) * d16 * 16 + dc * 128, wd = (uint32_t)d16 * 16 - nch * 128;
#pragma unroll 2
  while (row < rows) {
    const int64_t o = off[row];
    copy16(dst, base + (o < 0 ? 0 : o + c * 8), o >= 0);
    c += dc;
    row += dr;
    dst += dd;
    if (c >= nch) {
      c -= nch;
      row += 8;
      dst += wd;
    }
  }
}

// What the loader threads share: a table of row offsets, two in turn (a thread
// that fills one has seen every thread pass the barrier after the other's use).
template <int LT>
struct RowTables {
  int64_t (*at)[128];
  int turn;
  // off(r): element offset of row r, negative: zeros
  template <typename F>
  __device__ __forceinline__ const int64_t* fill(int rows, int tid, F off) {
    int64_t* t = at[turn ^= 1];
    for (int r = tid; r < rows; r += LT) t[r] = off(r);
    asm volatile("bar.sync 1, %0;" ::"n"(LT) : "memory");
    return t;
  }
};

// Rows m0 .. m0 + 127 of an item and key head (m = token x R + head of the key
// head), zeros past the last token; keys k0 .. k0 + n - 1 of a source's keys
// that count, zeros up to a multiple of 16.
template <int LT, typename T>
__device__ __forceinline__ void copy_queries(RowTables<LT>& tab, uint32_t dst, const T* base, const Strides& s, uint32_t m0,
                                             int R, int Q, int d, int d16, int tid) {
  if (R == 1) {
    copy_rows<LT, T>(dst, 128, min(128, Q - (int)m0), d, d16, base + m0 * s.token, s.token, tid);
    return;
  }
  const int64_t* off = tab.fill(128, tid, [&](int r) {
    const uint32_t m = m0 + r, t = m / (uint32_t)R;
    return t < (uint32_t)Q ? t * s.token + (m - t * R) * s.head : (int64_t)-1;
  });
  copy_rows_at<LT, T>(dst, 128, d, d16, base, off, tid);
}
template <int LT, typename T>
__device__ __forceinline__ void copy_keys(RowTables<LT>& tab, uint32_t dst, const T* base, int64_t stride, const Keys& keys, int g,
                                          int k0, int n, int rows, int d, int d16, int tid) {
  if (!keys.list) {
    copy_rows<LT, T>(dst, rows, n, d, d16, base + k0 * stride, stride, tid);
    return;
  }
  const int64_t* off = tab.fill(rows, tid, [&](int r) { return r < n ? keys.at(g, k0 + r) * stride : (int64_t)-1; });
  copy_rows_at<LT, T>(dst, rows, d, d16, base, off, tid);
}

// The list above (k_attn.cu).
cudaError_t launch_attn_keys(const AttnArgs& a, int32_t* n, int32_t* list, int32_t* pos, cudaStream_t st);
// The forward pass on the tensor cores (k_attn_tc.cu); parts of the keys, 1:
// none, else po [row][part][D] and pl [row][part] are written for the join.
int attn_tc_splits(const AttnArgs& a);
cudaError_t launch_attn_tc(const AttnArgs& a, const Keys& keys, float* po, float* pl, cudaStream_t st);

}  // namespace pa
