// New keys and values into the paged cache: a workgroup has one page of one key/value head, for keys or for values.
//   scale = max(the page's, 2^e) with the least e >= -100 for which the largest finite magnitude is at most 448 2^e
//   byte  = e4m3(x / scale), to nearest, ties to even; e4m3(byte old / scale) for tokens the page holds where the scale has grown
// A power of two: dividing by it is exact, so a value is rounded once (again where the scale grows: then only values whose
// bits fall below the least e4m3 step lose any).
//
// Bound by HBM: rows are read once (16 bytes a lane, kept in registers between the maximum and the rounding) and bytes written once.
// 21498 tokens, 8 heads, D = 128, bf16: 30 us for 132 MB, 4.4 TB/s.  Single tokens: latency, 9.1 us for 128 of them.
// Keys leave as they come, 8 (fp32: 4) a lane; values turn through LDS, since their dims come first in the cache.
#include <type_traits>

#include "packed.h"

namespace {

__device__ __forceinline__ float finite_abs(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? __uint_as_float(b) : 0.f;
}
// the least power of two by which values up to amax stay within 448 = 1.75 * 2^8
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}
// four values -> four bytes; what is not finite as NaN
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  const float nan = __builtin_nanf("");
  auto fin = [&](float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? x : nan; };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(fin(a), fin(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(fin(c), fin(d), w, true);
  return (uint32_t)w;
}
__device__ __forceinline__ uint32_t again_e4m3(uint32_t w, float mul) {
  typedef float f2_t __attribute__((ext_vector_type(2)));
  const f2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return to_e4m3(a.x * mul, a.y * mul, b.x * mul, b.y * mul);
}

template <typename T>
struct Chunk;  // 16 bytes of a row
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ float get(const uint4& v, int i) { return __uint_as_float((&v.x)[i]); }
};
template <>
struct Chunk<bf16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ float get(const uint4& v, int i) {
    const uint32_t w = (&v.x)[i / 2];
    return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
  }
};

// page `pid` of one head: its places lo .. hi - 1 from the new rows
template <typename T, int D, int PAGE>
__device__ __forceinline__ void append_page(const CacheDims& d, bool vals, int h, int beg, int L, int first, int col, int pid, const T* __restrict__ K,
                                            const T* __restrict__ V, uint8_t* __restrict__ kc, uint8_t* __restrict__ vc, float* __restrict__ ks,
                                            float* __restrict__ vs) {
  using C = Chunk<T>;
  constexpr int CPR = D / C::N, NP = (PAGE * CPR + 255) / 256, LD = PAGE + 4;  // chunks of a row, passes over a page
  __shared__ __attribute__((aligned(16))) uint8_t turn[D * LD];
  __shared__ float part[4];
  const int tid = threadIdx.x, x0 = col * PAGE, lo = max(max(first, 0), x0) - x0, hi = min(L - x0, PAGE);
  const int64_t step = vals ? d.v.token : d.k.token;
  const T* src = (vals ? V + d.v.at(beg, h) : K + d.k.at(beg, h)) + (int64_t)(x0 - first) * step;  // of place 0; read from lo on
  uint4 v[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = tid + 256 * i, row = c / CPR;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (row >= lo && row < hi) v[i] = *reinterpret_cast<const uint4*>(src + row * step + (c % CPR) * C::N);
  }
  if (pid < 0 || pid >= d.pages) return;  // asked for behind the rows: both are on their way together
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int e = 0; e < C::N; ++e) amax = fmaxf(amax, finite_abs(C::get(v[i], e)));
  amax = wave_max(amax);
  if (tid % 64 == 0) part[tid / 64] = amax;
  const size_t ph = (size_t)pid * d.Hkv + h;
  float* sp = (vals ? vs : ks) + ph;
  const float old = lo ? *sp : 0.f;
  __syncthreads();
  const float scale = fmaxf(scale_for(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]))), old), inv = 1.f / scale;
  const bool grown = lo > 0 && scale != old;
  const float ratio = old * inv;
  if (tid == 0) *sp = scale;
  if (!vals) {
    uint8_t* page = kc + ph * (PAGE * D);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = tid + 256 * i, row = c / CPR;
      if (row < lo || row >= hi) continue;
      uint32_t w[C::N / 4];
#pragma unroll
      for (int g = 0; g < C::N / 4; ++g)
        w[g] = to_e4m3(C::get(v[i], 4 * g) * inv, C::get(v[i], 4 * g + 1) * inv, C::get(v[i], 4 * g + 2) * inv, C::get(v[i], 4 * g + 3) * inv);
      if constexpr (C::N == 8) *reinterpret_cast<uint2*>(page + (size_t)c * C::N) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(page + (size_t)c * C::N) = w[0];
    }
    if (grown)
      for (int c = tid; c < lo * D / 4; c += 256) {
        uint32_t* w = reinterpret_cast<uint32_t*>(page) + c;
        *w = again_e4m3(*w, ratio);
      }
    return;
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int c = tid + 256 * i, row = c / CPR;
    if (row < lo || row >= hi) continue;
#pragma unroll
    for (int g = 0; g < C::N / 4; ++g) {
      const uint32_t w = to_e4m3(C::get(v[i], 4 * g) * inv, C::get(v[i], 4 * g + 1) * inv, C::get(v[i], 4 * g + 2) * inv, C::get(v[i], 4 * g + 3) * inv);
#pragma unroll
      for (int e = 0; e < 4; ++e) turn[((c % CPR) * C::N + 4 * g + e) * LD + row] = (uint8_t)(w >> (8 * e));
    }
  }
  __syncthreads();
  // words of four places: those that the call stores, and where the scale has grown those of the earlier tokens
  uint8_t* page = vc + ph * (PAGE * D);
  const int w0 = grown ? 0 : lo / 4, nw = (hi + 3) / 4 - w0;
  for (int c = tid; c < nw * D; c += 256) {
    const int dim = c / nw, x = 4 * (w0 + c % nw);
    uint8_t* at = page + dim * PAGE + x;
    uint32_t w = *reinterpret_cast<const uint32_t*>(turn + dim * LD + x);
    if (x >= lo && x + 4 <= hi) {
      *reinterpret_cast<uint32_t*>(at) = w;
      continue;
    }
    const uint32_t was = *reinterpret_cast<const uint32_t*>(at), held = grown ? again_e4m3(was, ratio) : was;
    uint32_t out = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) out |= (x + e < lo ? held : x + e < hi ? w : was) & (0xffu << (8 * e));
    *reinterpret_cast<uint32_t*>(at) = out;
  }
}

// `every` > 0: number x is page x % every of sequence x / every's new tokens, and the ones `every` further on; else seq_tile's numbers.
template <typename T, int D, int PAGE>
__global__ void __launch_bounds__(256) k_cache_append(CacheDims d, int every, const T* __restrict__ K, const T* __restrict__ V, const int32_t* __restrict__ cu,
                                                      const int32_t* __restrict__ lens, const int32_t* __restrict__ table, uint8_t* __restrict__ kc,
                                                      uint8_t* __restrict__ vc, float* __restrict__ ks, float* __restrict__ vs) {
  const bool vals = blockIdx.z != 0;
  const int h = blockIdx.y;
  SeqTile st;
  if (every > 0) {
    st.s = blockIdx.x / every;
    st.t = blockIdx.x % every;
    st.beg = seq_row(cu, st.s, d.T);
    st.end = max(seq_row(cu, st.s + 1, d.T), st.beg);
  } else {
    st = seq_tile(cu, d.S, d.T, PAGE, blockIdx.x, 1);
  }
  const int n = st.end - st.beg;
  if (n == 0 || st.t < 0) return;
  const int L = max(lens[st.s], 0), first = L - n, p0 = max(first, 0);
  for (int t = st.t;; t += every) {
    const int col = p0 / PAGE + t;
    if (col >= d.cols || (long long)col * PAGE >= L) return;
    append_page<T, D, PAGE>(d, vals, h, st.beg, L, first, col, table[(size_t)st.s * d.cols + col], K, V, kc, vc, ks, vs);
    if (every <= 0) return;
    __syncthreads();
  }
}

}  // namespace

int muse_launch_cache_append(const CacheDims& d, const void* K, const void* V, const int32_t* cu, const int32_t* lens, const int32_t* table,
                             void* kc, void* vc, float* ks, float* vs, hipStream_t st) {
  // Pages that new tokens may touch: all together by their rows, or sequence by sequence by the bound on them, whichever is fewer
  // (the second needs no search: 128 single tokens 11.3 -> 9.3 us).
  const long long all = packed_slots(d.T, d.S, d.page) + d.S, each = (d.max_new + d.page - 2) / d.page + 1;
  const int every = each * d.S <= all ? (int)each : 0;
  const dim3 g((unsigned)(every ? each * d.S : all), d.Hkv, 2);
  MuseProf prof_("k_cache_append", st);
  auto go = [&](auto* kernel, auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    hipLaunchKernelGGL(kernel, g, dim3(256), 0, st, d, every, (const E*)K, (const E*)V, cu, lens, table, (uint8_t*)kc, (uint8_t*)vc, ks, vs);
  };
#define PAGES(E, DD)                                                 \
  switch (d.page) {                                                  \
    case 16: go(k_cache_append<E, DD, 16>, (E*)0); break;            \
    case 32: go(k_cache_append<E, DD, 32>, (E*)0); break;            \
    case 64: go(k_cache_append<E, DD, 64>, (E*)0); break;            \
    default: go(k_cache_append<E, DD, 128>, (E*)0); break;           \
  }
  if (d.dtype == MUSE_DTYPE_BF16) {
    if (d.D == 64) PAGES(bf16_t, 64) else PAGES(bf16_t, 128)
  } else {
    if (d.D == 64) PAGES(float, 64) else PAGES(float, 128)
  }
#undef PAGES
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
