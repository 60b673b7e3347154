// Cross attention, backward:
//   p_ij = exp(s_ij - lse_i),  dp_ij = do_i . v_j,  delta_i = do_i . o_i,
//   ds_ij = p_ij (dp_ij - delta_i),
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,
// the last two over all rows of all items of the source and all heads that share
// the key head, always in the same order.
#include "pa_attn.cuh"

namespace pa {
namespace {

// dq: a warp per row; delta is kept for the kernel below. Lane groups as in the
// forward kernel.
template <typename T>
__global__ void __launch_bounds__(256) k_attn_dq(AttnArgs a, Keys keys, int gs, float* __restrict__ delta) {
  const int lane = threadIdx.x & 31, at = lane & (gs - 1), kpw = 32 / gs;
  pdl_wait();
  pdl_trigger();
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int h = (int)(row % a.H);
  const int64_t nt = row / a.H;
  const int t = (int)(nt % a.Q);
  const int64_t n = nt / a.Q;
  if (n >= items_of(a.count, a.N)) return;
  const int g = source_of(a.src, a.src_stride, (int)n, a.G, a.status);
  const int kn = g < 0 ? 0 : keys.count(g), j = h / (a.H / a.J);
  const bool col = at * 8 < a.D;
  float q[8] = {}, d[8] = {}, o[8] = {}, acc[8] = {};
  if (col) {
    Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.q + n * a.qs.item + t * a.qs.token + h * a.qs.head + at * 8), q);
    Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.dout + n * a.dos.item + t * a.dos.token + h * a.dos.head + at * 8), d);
    Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.o + n * a.os.item + t * a.os.token + h * a.os.head + at * 8), o);
  }
  float dl = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) dl = fmaf(d[i], o[i], dl);
  for (int w = gs >> 1; w > 0; w >>= 1) dl += __shfl_xor_sync(0xffffffffu, dl, w);
  if (lane == 0) delta[row] = dl;
  const float c2 = a.scale * kLog2e, l2 = kn ? a.lse[row] * kLog2e : 0.f;
  const T* kp = (const T*)a.k + (int64_t)max(g, 0) * a.ks.item + j * a.ks.head + at * 8;
  const T* vp = (const T*)a.v + (int64_t)max(g, 0) * a.vs.item + j * a.vs.head + at * 8;
  for (int k0 = 0; k0 < kn; k0 += kpw) {
    const int i = k0 + lane / gs;
    float kf[8] = {}, vf[8] = {}, s = 0.f, dp = 0.f;
    if (i < kn && col) {
      const int64_t key = keys.at(g, i);
      Elem<T>::open(*reinterpret_cast<const uint4*>(kp + key * a.ks.token), kf);
      Elem<T>::open(*reinterpret_cast<const uint4*>(vp + key * a.vs.token), vf);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s = fmaf(q[e], kf[e], s);
      dp = fmaf(d[e], vf[e], dp);
    }
    for (int w = gs >> 1; w > 0; w >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, w);
      dp += __shfl_xor_sync(0xffffffffu, dp, w);
    }
    const float ds = i < kn ? ex2(s * c2 - l2) * (dp - dl) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(ds, kf[e], acc[e]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    for (int w = gs; w < 32; w <<= 1) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], w);
    acc[e] *= a.scale;
  }
  if (lane < gs && col)
    *reinterpret_cast<uint4*>((T*)a.dq + n * a.dqs.item + t * a.dqs.token + h * a.dqs.head + at * 8) = Elem<T>::pack(acc);
}

// dk and dv: a warp per key and key head, over all rows of the source in order.
template <typename T>
__global__ void __launch_bounds__(256) k_attn_dkv(AttnArgs a, Keys keys, int gs, const float* __restrict__ delta) {
  const int lane = threadIdx.x & 31, at = lane & (gs - 1), rpw = 32 / gs, R = a.H / a.J;
  pdl_wait();
  pdl_trigger();
  const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (unit >= (int64_t)a.G * a.J * a.K) return;
  const int j = (int)(unit % a.J), key = (int)(unit / a.J % a.K), g = (int)(unit / a.J / a.K);
  const bool col = at * 8 < a.D;
  const bool in = (!a.len || key < a.len[g]) && (!a.mask || a.mask[g * a.mask_stride + key] != 0);
  float kf[8] = {}, vf[8] = {}, dk[8] = {}, dv[8] = {};
  if (in && col) {
    Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.k + g * a.ks.item + key * a.ks.token + j * a.ks.head + at * 8), kf);
    Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.v + g * a.vs.item + key * a.vs.token + j * a.vs.head + at * 8), vf);
  }
  const float c2 = a.scale * kLog2e;
  const int N = in ? items_of(a.count, a.N) : 0;
  for (int64_t n = 0; n < N; ++n) {
    if ((a.src ? a.src[n * a.src_stride] : n) != g) continue;
    for (int r0 = 0; r0 < a.Q * R; r0 += rpw) {
      const int r = r0 + lane / gs, t = r / R, h = j * R + r % R;
      const bool there = t < a.Q;
      float q[8] = {}, d[8] = {}, s = 0.f, dp = 0.f;
      if (there && col) {
        Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.q + n * a.qs.item + t * a.qs.token + h * a.qs.head + at * 8), q);
        Elem<T>::open(*reinterpret_cast<const uint4*>((const T*)a.dout + n * a.dos.item + t * a.dos.token + h * a.dos.head + at * 8), d);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s = fmaf(q[e], kf[e], s);
        dp = fmaf(d[e], vf[e], dp);
      }
      for (int w = gs >> 1; w > 0; w >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, w);
        dp += __shfl_xor_sync(0xffffffffu, dp, w);
      }
      float p = 0.f, ds = 0.f;
      if (there) {
        const int64_t row = (n * a.Q + t) * a.H + h;
        p = ex2(s * c2 - a.lse[row] * kLog2e);
        ds = p * (dp - delta[row]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dk[e] = fmaf(ds, q[e], dk[e]);
        dv[e] = fmaf(p, d[e], dv[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    for (int w = gs; w < 32; w <<= 1) {
      dk[e] += __shfl_xor_sync(0xffffffffu, dk[e], w);
      dv[e] += __shfl_xor_sync(0xffffffffu, dv[e], w);
    }
    dk[e] *= a.scale;
  }
  if (lane < gs && col) {
    *reinterpret_cast<uint4*>((T*)a.dk + g * a.dks.item + key * a.dks.token + j * a.dks.head + at * 8) = Elem<T>::pack(dk);
    *reinterpret_cast<uint4*>((T*)a.dv + g * a.dvs.item + key * a.dvs.token + j * a.dvs.head + at * 8) = Elem<T>::pack(dv);
  }
}

struct Plan {
  size_t n, list, delta, total;
};
Plan plan(const AttnArgs& a) {
  Plan p{};
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, kAlign); return at; };
  if (a.mask) {
    p.n = take((size_t)a.G * 4);
    p.list = take((size_t)a.G * a.K * 4);
  }
  p.delta = take((size_t)a.N * a.Q * a.H * 4);
  p.total = o;
  return p;
}

template <typename T>
cudaError_t run(const AttnArgs& a, cudaStream_t st) {
  const Plan p = plan(a);
  Keys keys{a.K, a.len, nullptr, nullptr};
  cudaError_t e = cudaSuccess;
  if (a.mask) {
    int32_t* n = reinterpret_cast<int32_t*>(a.ws + p.n);
    int32_t* list = reinterpret_cast<int32_t*>(a.ws + p.list);
    e = launch_attn_keys(a, n, list, st);
    if (e != cudaSuccess) return e;
    keys.n = n;
    keys.list = list;
  }
  int gs = 1;
  while (gs * 8 < a.D) gs <<= 1;
  float* delta = reinterpret_cast<float*>(a.ws + p.delta);
  const int64_t rows = (int64_t)a.N * a.Q * a.H, units = (int64_t)a.G * a.J * a.K;
  if (rows > 0) {
    e = launch_ex(k_attn_dq<T>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, 0, a, keys, gs, delta);
    if (e != cudaSuccess) return e;
  }
  if (units == 0) return cudaSuccess;
  return launch_ex(k_attn_dkv<T>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, st, 0, a, keys, gs, (const float*)delta);
}

}  // namespace

size_t attn_backward_workspace(const AttnArgs& a) { return plan(a).total; }

cudaError_t launch_attn_backward(const AttnArgs& a, cudaStream_t st) {
  return a.dtype == 1 ? run<__half>(a, st) : run<__nv_bfloat16>(a, st);
}

}  // namespace pa
