// dK and dV of packed sequences at D = 64, for short ones: a workgroup of four waves has 128 keys, 32 to a wave as the columns of the matrix
// instructions, two workgroups a CU (attn_bwd_wide.h's kernel has 256 keys and a CU to itself).  Queries come in tiles of 64, the
// query heads of the group one after the other, two tiles in LDS and a third on its way in registers:
//   S = Q K^T, dP = dO V^T;  P = exp2(c S - LSE), dS = P (dP - delta);  dV += P^T dO, dK += dS^T Q
// scores' rows are queries, so P and dS go back from the accumulators as operands, and the tiles serve both operand forms.
// 40 sequences of 400, 16 heads: 83 us, 197 MB at 2.4 TB/s, 0.33 PFLOP/s: few steps per workgroup bound it.
#include "attn_cols.h"
#include "packed.h"
#include "row_stage.h"

namespace {

constexpr int D = 64, KS = D / 16, DT = D / 32;

template <typename OT>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) k_packed_dkv_cols(
    PackedDims d, int slots, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const int32_t* __restrict__ cu,
    const bf16_t* __restrict__ dO, const float* __restrict__ LSE, const float* __restrict__ delta, OT* __restrict__ dK, OT* __restrict__ dV) {
  __shared__ __attribute__((aligned(256))) bf16_t qs[2][BN * D];
  __shared__ __attribute__((aligned(256))) bf16_t gs[2][BN * D];
  __shared__ __attribute__((aligned(16))) float seeds[2][2][BN];  // LSE in log2 units, delta
  const SeqTile st = packed_tile(cu, d.S, d.T, 128, d.Hkv, slots, false);
  if (!st.ok) return;
  const int hk = st.h, G = d.Hq / d.Hkv, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 32, half = lane / 32;
  const int k0 = st.beg + st.t * 128, ka = k0 + 32 * wave, m = ka + col, mc = min(m, st.end - 1);
  const float zscale = d.scale * 1.4426950408889634f;
  bf16x8_t kf[KS], vf[KS];
#pragma unroll
  for (int x = 0; x < KS; ++x) {
    kf[x] = *reinterpret_cast<const bf16x8_t*>(K + d.k.at(mc, hk) + 16 * x + 8 * half);
    vf[x] = *reinterpret_cast<const bf16x8_t*>(V + d.v.at(mc, hk) + 16 * x + 8 * half);
  }
  f32x16_t dk[DT], dv[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) dk[t] = dv[t] = zero16();

  const int per = (st.end - k0 + BN - 1) / BN, steps = per * G;  // tiles of queries of a head, of all heads
  TileRegs qr, gr;
  float sr = 0.f;
  auto fetch = [&](int i) {
    const int h = hk * G + i / per, q0 = k0 + i % per * BN;
    fetch_rows<D>(Q + d.q.head * h, q0, st.end, qr, d.q.token);
    fetch_rows<D>(dO + d.g.head * h, q0, st.end, gr, d.g.token);
    if (tid < 2 * BN) sr = (tid < BN ? LSE : delta)[(size_t)h * d.T + min(q0 + tid % BN, st.end - 1)];
  };
  auto commit = [&](int buf) {
    commit_rows<D>(qr, qs[buf]);
    commit_rows<D>(gr, gs[buf]);
    if (tid < 2 * BN) seeds[buf][tid / BN][tid % BN] = tid < BN ? sr * 1.4426950408889634f : sr;
  };
  fetch(0);
  commit(0);
  if (steps > 1) fetch(1);
  int buf = 0, at = 0;
  for (int i = 0; i < steps; ++i, buf ^= 1, at = at + 1 == per ? 0 : at + 1) {
    __syncthreads();
    if (i + 1 < steps) commit(buf ^ 1);
    if (i + 2 < steps) fetch(i + 2);
    const int q0 = k0 + at * BN;
    if (ka >= st.end || q0 + BN <= ka) continue;  // no keys, or all queries in front of them: wave-uniform
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int r0 = q0 + 32 * hh;
      if (r0 + 32 <= ka) continue;
      f32x16_t s = zero16(), dp = zero16();
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_row<D>(qs[buf], 32 * hh + col, 2 * x + half), kf[x], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_row<D>(gs[buf], 32 * hh + col, 2 * x + half), vf[x], dp, 0, 0, 0);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 l4 = *reinterpret_cast<const float4*>(&seeds[buf][0][32 * hh + 8 * g + 4 * half]);
        const float4 d4 = *reinterpret_cast<const float4*>(&seeds[buf][1][32 * hh + 8 * g + 4 * half]);
        const float la[4] = {l4.x, l4.y, l4.z, l4.w}, da[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int e = 4 * g + u;
          s[e] = fast_exp2(fmaf(s[e], zscale, -la[u]));
          dp[e] = s[e] * (dp[e] - da[u]);
        }
      }
      if (r0 < ka + 31 || r0 + 32 > st.end) {  // wave-uniform: queries in front of a key, or behind the sequence
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int n = r0 + 8 * (e / 4) + 4 * half + e % 4;
          const bool seen = n >= m && n < st.end;
          s[e] = seen ? s[e] : 0.f;
          dp[e] = seen ? dp[e] : 0.f;
        }
      }
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const bf16x8_t pf = pack8(s, 2 * g, 2 * g + 1), df = pack8(dp, 2 * g, 2 * g + 1);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          dv[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_cols<D>(gs[buf], 32 * hh + 16 * g, t, lane), pf, dv[t], 0, 0, 0);
          dk[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_cols<D>(qs[buf], 32 * hh + 16 * g, t, lane), df, dk[t], 0, 0, 0);
        }
      }
    }
  }
  if (m >= st.end) return;
  OT *ok = dK + d.dk.at(m, hk), *ov = dV + d.dv.at(m, hk);
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float k4[4] = {d.scale * dk[t][4 * g], d.scale * dk[t][4 * g + 1], d.scale * dk[t][4 * g + 2], d.scale * dk[t][4 * g + 3]};
      const float v4[4] = {dv[t][4 * g], dv[t][4 * g + 1], dv[t][4 * g + 2], dv[t][4 * g + 3]};
      st4(ok, 32 * t + 8 * g + 4 * half, k4);
      st4(ov, 32 * t + 8 * g + 4 * half, v4);
    }
}

}  // namespace

int muse_launch_packed_dkv_cols(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, const void* dO, const float* LSE,
                                const float* delta, void* dK, void* dV, hipStream_t st) {
  const int slots = (int)packed_slots(d.T, d.S, 128);
  auto go = [&](auto* kernel, auto* k, auto* v) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)packed_grid(d.Hkv, slots)), dim3(256), 0, st, d, slots, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V, cu,
                       (const bf16_t*)dO, LSE, delta, k, v);
  };
  if (d.grad_dtype == MUSE_DTYPE_BF16) go(k_packed_dkv_cols<bf16_t>, (bf16_t*)dK, (bf16_t*)dV);
  else go(k_packed_dkv_cols<float>, (float*)dK, (float*)dV);
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
