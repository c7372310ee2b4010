// Attention of 32 query rows per wave, the columns of v_mfma_f32_32x32x16_bf16, to staged tiles of 64 keys: S^T = K Q^T, the running
// softmax, O^T += V^T P^T.  Accumulator element e of lane l is row 8 (e / 4) + 4 (l / 32) + e % 4, column l % 32, so a column's
// softmax lives in two lanes and the weights go from the accumulator straight back as an operand.
#pragma once
#include "ff_common.h"
#include "flash_tile.h"
#include "lds_tile.h"

template <int D>
struct Cols {
  static constexpr int KS = D / 16, DT = D / 32;
  bf16x8_t q[KS];
  f32x16_t o[DT];
  float m, l;  // the reference (log2) that o and l are relative to; the lane's own part of the normaliser
  __device__ __forceinline__ void start(const bf16_t* row, int half) {
#pragma unroll
    for (int x = 0; x < KS; ++x) q[x] = *reinterpret_cast<const bf16x8_t*>(row + 16 * x + 8 * half);
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = zero16();
    m = MUSE_NEG_INF;
    l = 0.f;
  }
  // 64 keys.  kf(h, x): the operand of keys 32 h .. and dims 16 x ..; vf(g, t): that of keys 16 g .. and dims 32 t ..; zs(g) > 0: what scores
  // of the keys 16 g .. are multiplied by (log2 units), vs(g) what their weights are; hide: keys behind `last` (counted in the tile) are not seen;
  // dead: bit g, nobody sees the keys 16 g ...
  template <typename KF, typename VF, typename ZS, typename VS>
  __device__ __forceinline__ void attend(KF kf, VF vf, ZS zs, VS vs, bool hide, int last, int half, uint32_t dead = 0) {
    f32x16_t s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = zero16();
#pragma unroll
      for (int x = 0; x < KS; ++x) s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf(h, x), q[x], s[h], 0, 0, 0);
    }
    if (hide) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[h][e] = 32 * h + 8 * (e / 4) + e % 4 <= last - 4 * half ? s[h][e] : MUSE_NEG_INF;
    }
    if (dead) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[g / 2][8 * (g % 2) + e] = dead >> g & 1 ? MUSE_NEG_INF : s[g / 2][8 * (g % 2) + e];
    }
    float top = MUSE_NEG_INF;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float x = s[g / 2][8 * (g % 2)];
#pragma unroll
      for (int e = 1; e < 8; ++e) x = fmaxf(x, s[g / 2][8 * (g % 2) + e]);
      top = fmaxf(top, x * zs(g));
    }
    typedef uint32_t u2_t __attribute__((ext_vector_type(2)));
    const u2_t x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    // the reference follows the maximum in steps of more than 2^8: most tiles rescale nothing
    if (__builtin_amdgcn_ballot_w64(top > m + 8.f)) {
      const float mn = top > m + 8.f ? top : m, al = mn == MUSE_NEG_INF ? 1.f : fast_exp2(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] *= al;
    }
    const float ref = m == MUSE_NEG_INF ? 0.f : m;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x16_t& p = s[g / 2];
      const int G = g % 2;
#pragma unroll
      for (int e = 8 * G; e < 8 * G + 8; ++e) {
        p[e] = fast_exp2(fmaf(p[e], zs(g), -ref));
        l += p[e];  // in 32 bits; the weights are rounded to bf16 below, half a step each
        p[e] *= vs(g);
      }
      const bf16x8_t pf = pack8(p, 2 * G, 2 * G + 1);
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf(g, t), pf, o[t], 0, 0, 0);
    }
  }
};
