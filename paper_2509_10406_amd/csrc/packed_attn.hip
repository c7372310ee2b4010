// Launches of exact attention over packed sequences, and delta, the backward's row sums.
#include <type_traits>

#include "attn_bwd_wide.h"

int muse_launch_packed_fwd_mfma(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, void* O, float* LSE, hipStream_t st);
int muse_launch_packed_fwd_cols(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, void* O, float* LSE, hipStream_t st);
int muse_launch_packed_fwd_f32(const PackedDims& d, const float* Q, const float* K, const float* V, const int32_t* cu, float* O, float* LSE, hipStream_t st);
int muse_launch_packed_bwd_f32(const PackedDims& d, const float* Q, const float* K, const float* V, const int32_t* cu, const float* dO, const float* LSE,
                               const float* delta, float* dQ, float* dK, float* dV, hipStream_t st);
int muse_launch_packed_dkv_cols(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, const void* dO, const float* LSE,
                                const float* delta, void* dK, void* dV, hipStream_t st);
int muse_launch_packed_dq_narrow(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, const void* dO, const float* LSE,
                                 const float* delta, void* dQ, hipStream_t st);

namespace {

constexpr int FEW = 64;  // rows of a tile of delta, and keys that count as few

// delta_i = dO_i . O_i = sum_j P_ij dP_ij.  O has been rounded to bf16: dS = P (dP - delta) then is off by 2^-8 of dO . O, which does not
// matter where dP - delta is as large as dP.  For the first rows of a sequence it is not: with one key it is 0, with few keys the weights
// are large and so is their share in dK, dQ (relative error modelled in 64 bits on the host, random inputs, 20 tokens, D = 64: 2.75e-3,
// 2.35e-3 by the second sum, 1.67e-3 from the gradients' own rounding alone).  So the first 64 rows of every sequence have the second sum, from scores made again: one tile.
// A workgroup has 64 rows of a head; bound by the reads of O and dO.  16384 tokens, 32 heads, D = 128: 58 us, 4.6 TB/s; 16000 tokens in 40
// sequences, 16 heads, D = 64: 18 us, 3.7.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_packed_delta(PackedDims d, int slots, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                                      const int32_t* __restrict__ cu, const T* __restrict__ O, const float* __restrict__ LSE,
                                                      const T* __restrict__ dO, float* __restrict__ delta) {
  clear_stamp(delta);
  const SeqTile st = packed_tile(cu, d.S, d.T, FEW, d.Hq, slots);
  if (!st.ok) return;
  const int h = st.h, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, r0 = st.beg + st.t * FEW, end = min(r0 + FEW, st.end);
  float* out = delta + (size_t)h * d.T;
  if constexpr (sizeof(T) == 2) {
    if (st.t == 0) {  // a wave has 32 queries, one operand column each, and the keys up to its own
      if (wave >= 2 || r0 + 32 * wave >= end) return;
      const int hk = h / (d.Hq / d.Hkv), col = lane % 32, half = lane / 32, n = r0 + 32 * wave + col, nc = min(n, end - 1);
      const float c = d.scale * 1.4426950408889634f, lse = LSE[(size_t)h * d.T + nc] * 1.4426950408889634f;
      float sum = 0.f;
      for (int k = 0; k <= wave; ++k) {
        const int m = min(r0 + 32 * k + col, end - 1);
        f32x16_t s = zero16(), dp = zero16();
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
          const int at = 16 * x + 8 * half;
          auto op = [&](const T* p) { return *reinterpret_cast<const bf16x8_t*>(p + at); };
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op(K + d.k.at(m, hk)), op(Q + d.q.at(nc, h)), s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op(V + d.v.at(m, hk)), op(dO + d.g.at(nc, h)), dp, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = r0 + 32 * k + 8 * (e / 4) + 4 * half + e % 4;
          if (key <= n) sum = fmaf(fast_exp2(fmaf(s[e], c, -lse)), dp[e], sum);
        }
      }
      sum += __shfl_xor(sum, 32, 64);
      if (half == 0 && n < end) out[n] = sum;
      return;
    }
  }
  constexpr int LPR = D * sizeof(T) / 16, RPW = 64 / LPR, N = 16 / sizeof(T);  // lanes of a row, rows of a wave, elements of a lane
  const int lr = lane % LPR;
  for (int i = 0; i < FEW / 4; i += RPW) {
    const int n = r0 + wave * (FEW / 4) + i + lane / LPR, nc = min(n, end - 1);
    float a[N], b[N], sum = 0.f;
    const T *po = O + d.o.at(nc, h) + lr * N, *pg = dO + d.g.at(nc, h) + lr * N;
#pragma unroll
    for (int u = 0; u < N; u += 4) {
      ld4(po, u, *reinterpret_cast<float(*)[4]>(a + u));
      ld4(pg, u, *reinterpret_cast<float(*)[4]>(b + u));
    }
#pragma unroll
    for (int u = 0; u < N; ++u) sum = fmaf(a[u], b[u], sum);
    sum = group_sum<(LPR > 16 ? 16 : LPR)>(sum);
    if constexpr (LPR > 16) sum += __shfl_xor(sum, 16, 64);
    if (lr == 0 && n < end) out[n] = sum;
  }
}

}  // namespace

// Which kernels a call takes, by the bound on its lengths (the caller's, or all tokens).  us, tiles of 128 / of 256 rows, about 16k tokens:
//   forward  D = 64: 40 sequences of 400 49 / 64 with 16 heads, 70 / 115 with 32 of 8; 16 of 1024 74 / 82 and 127 / 140; 8 of 2048 126 / 119
//            and 209 / 198; 16 of 768 on average and up to 2235 76 / 77 and 108 / 130.  D = 128: 64 of up to 909 97 / 107 and 162 /
//            207; 16 of 1024 130 / 117 and 232 / 216; 16 of up to 2235 115 / 104 and 193 / 184.
//   dQ       (the whole backward) D = 64: 64 of up to 909 175 / 195 and 315 / 358; 16 of 1024 211 / 218 and 369 / 375; 8 of 2048 323 / 309 and
//            646 / 622.  D = 128: 335 / 359 and 573 / 613; 414 / 418 and 754 / 755; 616 / 594 and 1203 / 1167.
//   dK, dV   (the whole backward) D = 64, tiles of 128 / of 256 keys: 400 of 20 133 / 204 and 204 / 266; 200 of 60 106 / 140 and 154 / 182; 128 of
//            128 168 / 163 and 202 / 202; 64 of 256 125 / 131 and 179 / 170; 40 of 400 157 / 166 and 289 / 268; 25 of 640 153 / 156 and
//            273 / 264; 16 of 1024 209 / 208.
static bool fwd_in_cols(const PackedDims& d) { return d.max_len < (d.D == 128 ? 960 : d.Hq > d.Hkv ? 2560 : 2048); }
static bool dq_narrow(const PackedDims& d) { return d.max_len <= 4 * TR; }
static bool dkv_in_cols(const PackedDims& d) { return d.D == 64 && d.max_len <= (d.Hq > d.Hkv ? 192 : 640); }

size_t muse_packed_fwd_ws_bytes(const PackedDims&) { return 0; }
size_t muse_packed_bwd_ws_bytes(const PackedDims& d) { return kTagBytes + (size_t)d.Hq * d.T * 4; }

int muse_launch_packed_fwd(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, void* O, float* LSE, void*, hipStream_t st) {
  if (d.dtype == MUSE_DTYPE_FP32) return muse_launch_packed_fwd_f32(d, (const float*)Q, (const float*)K, (const float*)V, cu, (float*)O, LSE, st);
  return fwd_in_cols(d) ? muse_launch_packed_fwd_cols(d, Q, K, V, cu, O, LSE, st) : muse_launch_packed_fwd_mfma(d, Q, K, V, cu, O, LSE, st);
}

int muse_launch_packed_bwd(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, const void* O, const float* LSE,
                           const void* dO, void* dQ, void* dK, void* dV, void* ws, hipStream_t st) {
  float* delta = (float*)((char*)ws + kTagBytes);
  {
    const int slots = (int)packed_slots(d.T, d.S, FEW);
    const dim3 g((unsigned)packed_grid(d.Hq, slots));
    MuseProf prof_("k_packed_delta", st);
    auto go = [&](auto* kernel, auto* t) {
      using E = std::remove_pointer_t<decltype(t)>;
      hipLaunchKernelGGL(kernel, g, dim3(256), 0, st, d, slots, (const E*)Q, (const E*)K, (const E*)V, cu, (const E*)O, LSE, (const E*)dO, delta);
    };
    if (d.dtype == MUSE_DTYPE_BF16) d.D == 64 ? go(k_packed_delta<bf16_t, 64>, (bf16_t*)0) : go(k_packed_delta<bf16_t, 128>, (bf16_t*)0);
    else d.D == 64 ? go(k_packed_delta<float, 64>, (float*)0) : go(k_packed_delta<float, 128>, (float*)0);
    MUSE_LAUNCH_CHECK();
  }
  if (d.dtype == MUSE_DTYPE_FP32)
    return muse_launch_packed_bwd_f32(d, (const float*)Q, (const float*)K, (const float*)V, cu, (const float*)dO, LSE, delta, (float*)dQ, (float*)dK, (float*)dV, st);
  const float sl = d.scale * 1.4426950408889634f;
  auto lay = [&](int tr, const Rows& a, const Rows& b) {
    return PackedBwd{cu, d.S, d.T, d.Hq, d.Hkv, (int)packed_slots(d.T, d.S, tr), d.q, d.k, d.v, d.g, a, b};
  };
  if (dkv_in_cols(d)) {
    MuseProf prof_("k_packed_dkv", st);
    if (const int rc = muse_launch_packed_dkv_cols(d, Q, K, V, cu, dO, LSE, delta, dK, dV, st)) return rc;
  } else {
    MuseProf prof_("k_packed_dkv", st);
    auto go = [&](auto* kernel, int tr, auto* k, auto* v) {
      const PackedBwd l = lay(tr, d.dk, d.dv);
      hipLaunchKernelGGL(kernel, dim3((unsigned)packed_grid(d.Hkv, l.slots)), dim3(256), 0, st, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V,
                         (const bf16_t*)dO, LSE, delta, k, v, l, d.scale, sl);
    };
    auto as = [&](auto* k, auto* v) {
      using OT = std::remove_pointer_t<decltype(k)>;
      d.D == 64 ? go(k_flash_bwd_dkv_wide<OT, PackedBwd>, TR, k, v) : go(k_flash_bwd_dkv128_wide<OT, PackedBwd>, TR128, k, v);
    };
    if (d.grad_dtype == MUSE_DTYPE_BF16) as((bf16_t*)dK, (bf16_t*)dV);
    else as((float*)dK, (float*)dV);
    MUSE_LAUNCH_CHECK();
  }
  MuseProf prof_("k_packed_dq", st);
  if (dq_narrow(d)) return muse_launch_packed_dq_narrow(d, Q, K, V, cu, dO, LSE, delta, dQ, st);
  auto go = [&](auto* kernel, auto* out) {
    const PackedBwd l = lay(TR, d.dq, d.dq);
    hipLaunchKernelGGL(kernel, dim3((unsigned)packed_grid(d.Hq, l.slots)), dim3(256), 0, st, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V,
                       (const bf16_t*)dO, LSE, delta, out, l, d.scale, sl);
  };
  if (d.grad_dtype == MUSE_DTYPE_BF16) d.D == 64 ? go(k_flash_bwd_dq_wide<64, bf16_t, PackedBwd>, (bf16_t*)dQ) : go(k_flash_bwd_dq_wide<128, bf16_t, PackedBwd>, (bf16_t*)dQ);
  else d.D == 64 ? go(k_flash_bwd_dq_wide<64, float, PackedBwd>, (float*)dQ) : go(k_flash_bwd_dq_wide<128, float, PackedBwd>, (float*)dQ);
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
