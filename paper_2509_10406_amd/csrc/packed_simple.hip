// Exact attention over packed sequences, one wave per row: online softmax over 64 keys at a time, a key
// per lane for the scores and D / 64 dims per lane for the sums.  Reads a key's row once per query, so it is bound by the caches.
#include <type_traits>

#include "packed.h"

namespace {

template <typename T, int D>
__device__ __forceinline__ float dot_row(const T* __restrict__ x, const float* y) {
  float a = 0.f;
  for (int d = 0; d < D; d += 4) {
    float v[4];
    ld4(x, d, v);
#pragma unroll
    for (int u = 0; u < 4; ++u) a = fmaf(v[u], y[d + u], a);
  }
  return a;
}

template <typename T, int D>
__device__ __forceinline__ void row_to_lds(const T* __restrict__ x, float* y) {
  for (int d = threadIdx.x; d < D; d += 64) y[d] = Elem<T>::ld(x, d);
}

template <typename T, int D>
__global__ void __launch_bounds__(64) k_packed_fwd_simple(PackedDims d, const T* __restrict__ Q, const T* __restrict__ K,
                                                          const T* __restrict__ V, const int32_t* __restrict__ cu, T* __restrict__ O,
                                                          float* __restrict__ LSE) {
  __shared__ float q[D];
  const int h = blockIdx.y, hk = h / (d.Hq / d.Hkv), lane = threadIdx.x;
  const SeqTile st = seq_tile(cu, d.S, d.T, 1, blockIdx.x);
  if (!st.ok) return;
  const int n = st.beg + st.t;
  row_to_lds<T, D>(Q + d.q.at(n, h), q);
  __syncthreads();
  float m = MUSE_NEG_INF, l = 0.f, o[D / 64] = {};
  for (int k0 = st.beg; k0 <= n; k0 += 64) {
    const int j = k0 + lane;
    const float s = j <= n ? d.scale * dot_row<T, D>(K + d.k.at(j, hk), q) : MUSE_NEG_INF;
    const float mn = fmaxf(m, wave_max(s)), ref = mn == MUSE_NEG_INF ? 0.f : mn, al = __expf(m - ref), p = __expf(s - ref);
    m = mn;
    l = l * al + wave_sum(p);
    for (int x = 0; x < D / 64; ++x) o[x] *= al;
    for (int i = 0; i < min(64, n + 1 - k0); ++i) {
      const float pi = __shfl(p, i, 64);
      for (int x = 0; x < D / 64; ++x) o[x] = fmaf(pi, Elem<T>::ld(V + d.v.at(k0 + i, hk), lane + 64 * x), o[x]);
    }
  }
  for (int x = 0; x < D / 64; ++x) Elem<T>::st(O + d.o.at(n, h), lane + 64 * x, o[x] / l);
  if (lane == 0) LSE[(size_t)h * d.T + n] = m + __logf(l);
}

template <typename T, typename OT, int D>
__global__ void __launch_bounds__(64) k_packed_dq_simple(PackedDims d, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                                         const int32_t* __restrict__ cu, const T* __restrict__ O, const float* __restrict__ LSE,
                                                         const T* __restrict__ dO, float* __restrict__ delta, OT* __restrict__ dQ) {
  __shared__ float q[D], g[D];
  const int h = blockIdx.y, hk = h / (d.Hq / d.Hkv), lane = threadIdx.x;
  const SeqTile st = seq_tile(cu, d.S, d.T, 1, blockIdx.x);
  if (!st.ok) return;
  const int n = st.beg + st.t;
  row_to_lds<T, D>(Q + d.q.at(n, h), q);
  row_to_lds<T, D>(dO + d.g.at(n, h), g);
  __syncthreads();
  float dl = 0.f, a[D / 64] = {};
  for (int x = 0; x < D / 64; ++x) dl = fmaf(g[lane + 64 * x], Elem<T>::ld(O + d.o.at(n, h), lane + 64 * x), dl);
  dl = wave_sum(dl);
  const float lse = LSE[(size_t)h * d.T + n];
  if (lane == 0) delta[(size_t)h * d.T + n] = dl;
  for (int k0 = st.beg; k0 <= n; k0 += 64) {
    const int j = k0 + lane;
    float ds = 0.f;
    if (j <= n) ds = __expf(d.scale * dot_row<T, D>(K + d.k.at(j, hk), q) - lse) * (dot_row<T, D>(V + d.v.at(j, hk), g) - dl);
    for (int i = 0; i < min(64, n + 1 - k0); ++i) {
      const float di = __shfl(ds, i, 64);
      for (int x = 0; x < D / 64; ++x) a[x] = fmaf(di, Elem<T>::ld(K + d.k.at(k0 + i, hk), lane + 64 * x), a[x]);
    }
  }
  for (int x = 0; x < D / 64; ++x) Elem<OT>::st(dQ + d.dq.at(n, h), lane + 64 * x, d.scale * a[x]);
}

template <typename T, typename OT, int D>
__global__ void __launch_bounds__(64) k_packed_dkv_simple(PackedDims d, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                                          const int32_t* __restrict__ cu, const float* __restrict__ LSE,
                                                          const T* __restrict__ dO, const float* __restrict__ delta, OT* __restrict__ dK,
                                                          OT* __restrict__ dV) {
  __shared__ float k[D], v[D];
  const int hk = blockIdx.y, G = d.Hq / d.Hkv, lane = threadIdx.x;
  const SeqTile st = seq_tile(cu, d.S, d.T, 1, blockIdx.x);
  if (!st.ok) return;
  const int m = st.beg + st.t;
  row_to_lds<T, D>(K + d.k.at(m, hk), k);
  row_to_lds<T, D>(V + d.v.at(m, hk), v);
  __syncthreads();
  float ak[D / 64] = {}, av[D / 64] = {};
  for (int h = hk * G; h < hk * G + G; ++h)
    for (int q0 = m; q0 < st.end; q0 += 64) {
      const int n = q0 + lane;
      float p = 0.f, ds = 0.f;
      if (n < st.end) {
        p = __expf(d.scale * dot_row<T, D>(Q + d.q.at(n, h), k) - LSE[(size_t)h * d.T + n]);
        ds = p * (dot_row<T, D>(dO + d.g.at(n, h), v) - delta[(size_t)h * d.T + n]);
      }
      for (int i = 0; i < min(64, st.end - q0); ++i) {
        const float pi = __shfl(p, i, 64), di = __shfl(ds, i, 64);
        for (int x = 0; x < D / 64; ++x) {
          ak[x] = fmaf(di, Elem<T>::ld(Q + d.q.at(q0 + i, h), lane + 64 * x), ak[x]);
          av[x] = fmaf(pi, Elem<T>::ld(dO + d.g.at(q0 + i, h), lane + 64 * x), av[x]);
        }
      }
    }
  for (int x = 0; x < D / 64; ++x) {
    Elem<OT>::st(dK + d.dk.at(m, hk), lane + 64 * x, d.scale * ak[x]);
    Elem<OT>::st(dV + d.dv.at(m, hk), lane + 64 * x, av[x]);
  }
}

}  // namespace

int muse_launch_packed_fwd(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, void* O, float* LSE, void* ws, hipStream_t st) {
  (void)ws;
  const dim3 g((unsigned)packed_slots(d.T, d.S, 1), d.Hq);
  MuseProf prof_("k_packed_fwd", st);
  auto go = [&](auto* kernel, auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    hipLaunchKernelGGL(kernel, g, dim3(64), 0, st, d, (const E*)Q, (const E*)K, (const E*)V, cu, (E*)O, LSE);
  };
  if (d.dtype == MUSE_DTYPE_BF16) d.D == 64 ? go(k_packed_fwd_simple<bf16_t, 64>, (bf16_t*)0) : go(k_packed_fwd_simple<bf16_t, 128>, (bf16_t*)0);
  else d.D == 64 ? go(k_packed_fwd_simple<float, 64>, (float*)0) : go(k_packed_fwd_simple<float, 128>, (float*)0);
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}

int muse_launch_packed_bwd(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, const void* O, const float* LSE,
                           const void* dO, void* dQ, void* dK, void* dV, void* ws, hipStream_t st) {
  const unsigned slots = (unsigned)packed_slots(d.T, d.S, 1);
  float* delta = (float*)ws;
  auto go = [&](auto* kq, auto* kkv, auto* t, auto* u) {
    using E = std::remove_pointer_t<decltype(t)>;
    using G = std::remove_pointer_t<decltype(u)>;
    { MuseProf prof_("k_packed_dq", st); hipLaunchKernelGGL(kq, dim3(slots, d.Hq), dim3(64), 0, st, d, (const E*)Q, (const E*)K, (const E*)V, cu, (const E*)O, LSE, (const E*)dO, delta, (G*)dQ); }
    { MuseProf prof_("k_packed_dkv", st); hipLaunchKernelGGL(kkv, dim3(slots, d.Hkv), dim3(64), 0, st, d, (const E*)Q, (const E*)K, (const E*)V, cu, LSE, (const E*)dO, delta, (G*)dK, (G*)dV); }
  };
#define GO(E, G) (d.D == 64 ? go(k_packed_dq_simple<E, G, 64>, k_packed_dkv_simple<E, G, 64>, (E*)0, (G*)0) : go(k_packed_dq_simple<E, G, 128>, k_packed_dkv_simple<E, G, 128>, (E*)0, (G*)0))
  if (d.dtype == MUSE_DTYPE_BF16) d.grad_dtype == MUSE_DTYPE_BF16 ? GO(bf16_t, bf16_t) : GO(bf16_t, float);
  else GO(float, float);
#undef GO
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}

size_t muse_packed_fwd_ws_bytes(const PackedDims&) { return 0; }
size_t muse_packed_bwd_ws_bytes(const PackedDims& d) { return (size_t)d.Hq * d.T * 4; }
