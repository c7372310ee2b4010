// Exact attention over packed sequences, forward, for short ones: a workgroup of four waves has 128 rows of a key/value head's group (the
// tokens' query heads one after the other, so that grouped heads share the staged keys and fill the tiles of short
// sequences), two workgroups a CU (D = 64: three).  attn_fwd.hip's kernel has 256 rows of one head and a CU to itself: it wins where
// sequences are long (the line is in packed_attn.hip).
//
// Two tiles of 64 keys and values in LDS, a third on its way in registers; one barrier per step, the next tile is written in its middle.
// 40 sequences of 400, 16 heads, D = 64: 50 us, 131 MB at 2.6 TB/s, 0.27 PFLOP/s: few steps per workgroup bound it.
#include "attn_cols.h"
#include "packed.h"
#include "row_stage.h"

namespace {

template <int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2))) k_packed_fwd_cols(
    PackedDims d, int slots, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const int32_t* __restrict__ cu,
    bf16_t* __restrict__ O, float* __restrict__ LSE) {
  constexpr int DT = D / 32;
  __shared__ __attribute__((aligned(256))) bf16_t ks[2][BN * D];
  __shared__ __attribute__((aligned(256))) bf16_t vs[2][BN * D];
  const int G = d.Hq / d.Hkv;
  const SeqTile st = packed_tile(cu, d.S, d.T, 128, d.Hkv, slots, true, G);
  if (!st.ok) return;
  const int hk = st.h, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, col = lane % 32, half = lane / 32;
  const int rows = (st.end - st.beg) * G, x0 = st.t * 128, w0 = x0 + 32 * wave, x = w0 + col, y = min(x, rows - 1);
  const int i = y / G, h = hk * G + y - i * G, n = st.beg + i;
  const int first = min(w0, rows - 1) / G, last = min(w0 + 31, rows - 1) / G;  // the wave's tokens
  const int keys = min(x0 + 127, rows - 1) / G + 1;
  const bf16_t *Kh = K + d.k.head * hk, *Vh = V + d.v.head * hk;
  Cols<D> c;
  c.start(Q + d.q.at(n, h), half);
  TileRegs kreg, vreg;
  auto fetch = [&](int k0) {
    fetch_rows<D>(Kh, st.beg + k0, st.end, kreg, d.k.token);
    fetch_rows<D>(Vh, st.beg + k0, st.end, vreg, d.v.token);
  };
  auto commit = [&](int buf) {
    commit_rows<D>(kreg, ks[buf]);
    commit_rows<D>(vreg, vs[buf]);
  };
  const float zscale = d.scale * 1.4426950408889634f;
  fetch(0);
  commit(0);
  if (keys > BN) fetch(BN);
  int buf = 0;
  for (int k0 = 0; k0 < keys; k0 += BN, buf ^= 1) {
    __syncthreads();
    if (k0 + BN < keys) commit(buf ^ 1);
    if (k0 + 2 * BN < keys) fetch(k0 + 2 * BN);
    if (w0 < rows && k0 <= last)
      c.attend([&](int hh, int u) { return tile_row<D>(ks[buf], 32 * hh + col, 2 * u + half); },
               [&](int g, int t) { return tile_cols<D>(vs[buf], 16 * g, t, lane); }, [&](int) { return zscale; }, [](int) { return 1.f; },
               k0 + BN - 1 > first, i - k0, half);
  }
  if (x >= rows) return;
  const float l = c.l + __shfl_xor(c.l, 32, 64), inv = 1.f / l;
  bf16_t* to = O + d.o.at(n, h);
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float v[4] = {c.o[t][4 * g] * inv, c.o[t][4 * g + 1] * inv, c.o[t][4 * g + 2] * inv, c.o[t][4 * g + 3] * inv};
      st4(to, 32 * t + 8 * g + 4 * half, v);
    }
  if (half == 0) LSE[(size_t)h * d.T + n] = (c.m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

}  // namespace

int muse_launch_packed_fwd_cols(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, void* O, float* LSE, hipStream_t st) {
  const int slots = (int)packed_slots(d.T, d.S, 128, d.Hq / d.Hkv);
  MuseProf prof_("k_packed_fwd", st);
  auto go = [&](auto* kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)packed_grid(d.Hkv, slots)), dim3(256), 0, st, d, slots, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V, cu,
                       (bf16_t*)O, LSE);
  };
  if (d.D == 64) go(k_packed_fwd_cols<64>);
  else go(k_packed_fwd_cols<128>);
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
