// The launches of the bf16 backward in tiles of 256 rows (attn_bwd_wide.h), and where the line to the tiles of 128 is.
#include "attn_bwd_wide.h"

// Where a workgroup's fixed part (operands of 256 rows, the masked steps, 64 KB of results) shows, the kernels of 128 rows with two
// or three workgroups on a CU are better.  us, 128 rows / 256 rows:
//   dQ      blocks of 384 35 / 102 at 1024 groups, 22 / 29 at 256; of 640 138 / 187 at 1024, 44 / 51 at 256; of 1024 85 / 84 at 256
//           groups, 51 / 41 at 128, 33 / 28 at 64, 24 / 26 at 32 (128 tiles of 256 rows: half of the chip's CUs); of 2048 39 / 42 at
//           16 groups, 55 / 46 at 32.  D = 128: 81 / 86 (640, 256 groups), 164 / 147 (1024, 256), 37 / 41 (1024, 32), 65 / 67 (2048, 16).
//   dK/dV   blocks of 256 74 / 81 at 1024 groups, 15 / 16 at 64; of 320 110 / 98 and 18 / 18; of 128 37 / 41 and 12 / 11.  D = 128:
//           blocks of 384 223 / 255 at 1024 groups, 25 / 24 at 64; of 512 107 / 105 at 256, 31 / 29 at 64; of 640 454 / 459 and 45 / 35.
//           Few groups need no clause here, although the larger tiles halve the workgroups at D = 64: the longest tile sets the
//           time, and it has twice the keys but reads each query once for them.  At 1 group and at 16: blocks of 320 17 / 16 and 17 /
//           16, of 512 19 / 20 and 20 / 20, of 1024 31 / 30 and 31 / 31, of 2048 53 / 51 and 53 / 52, of 4096 98 / 92 and 140 / 98,
//           of 16k 574 / 386 and 1200 / 948; four query heads per group 56 / 51 and 57 / 52 (512), 2158 / 1412 and 5011 / 3717 (16k).
//           D = 128: of 512 26 / 25 and 27 / 26, of 2048 77 / 68 and 79 / 69, of 16k 1148 / 975 and 2673 / 2187.
bool muse_attn_dq_wide(const MuseDims& d, int Bs) {
  return Bs >= 4 * TR && (long long)((Bs + TR - 1) / TR) * d.B * d.Hq * (d.N / Bs) > 128;
}
bool muse_attn_dkv_wide(const MuseDims& d, int Bs) { return d.D == 64 ? Bs > TR : Bs >= 2 * TR; }

// Rows go from memory to LDS 16 bytes at a time, from 16-byte boundaries: tensors that begin elsewhere (a view one element into
// its storage) are read through registers by the kernels of 128 rows, where any address will do.
bool muse_attn_rows_to_lds(const void* Q, const void* K, const void* V, const void* dO) {
  return ((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)dO) % 16 == 0;
}

// the gradients may leave in bf16 (MuseDims::grads16): all of them come from the kernels of attn_bwd_wide.h
bool muse_attn_bwd_writes16(const MuseDims& d, int Bs, const void* Q, const void* K, const void* V, const void* dO) {
  return d.dtype == MUSE_DTYPE_BF16 && muse_attn_dq_wide(d, Bs) && muse_attn_dkv_wide(d, Bs) && muse_attn_rows_to_lds(Q, K, V, dO);
}

int muse_launch_attn_dq_wide(const MuseDims& d, int Bs, const void* Q, const void* K, const void* V, const void* dO, const float* LSE,
                             const float* delta, void* dQ, hipStream_t st) {
  const int tiles = (Bs + TR - 1) / TR, groups = d.B * d.Hq * (d.N / Bs);
  MuseProf prof_("k_flash_bwd_dq", st);
  auto go = [&](auto* kernel, auto* out) {
    hipLaunchKernelGGL(kernel, flash_grid_of(tiles, groups), dim3(256), 0, st, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V,
                       (const bf16_t*)dO, LSE, delta, out, DenseBwd{d.N, Bs, d.Hq, d.Hkv, d.B, chunk_groups(Bs, d.D, groups)}, d.scale, d.scale * 1.4426950408889634f);
  };
  if (d.grads16) d.D == 64 ? go(k_flash_bwd_dq_wide<64, bf16_t, DenseBwd>, (bf16_t*)dQ) : go(k_flash_bwd_dq_wide<128, bf16_t, DenseBwd>, (bf16_t*)dQ);
  else d.D == 64 ? go(k_flash_bwd_dq_wide<64, float, DenseBwd>, (float*)dQ) : go(k_flash_bwd_dq_wide<128, float, DenseBwd>, (float*)dQ);
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}

int muse_launch_attn_dkv_wide(const MuseDims& d, int Bs, const void* Q, const void* K, const void* V, const void* dO, const float* LSE,
                              const float* delta, void* dK, void* dV, hipStream_t st) {
  const int tr = d.D == 64 ? TR : TR128, tiles = (Bs + tr - 1) / tr, groups = d.B * d.Hkv * (d.N / Bs);
  MuseProf prof_("k_flash_bwd_dkv", st);
  auto go = [&](auto* kernel, auto* k, auto* v) {
    hipLaunchKernelGGL(kernel, flash_grid_of(tiles, groups), dim3(256), 0, st, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V,
                       (const bf16_t*)dO, LSE, delta, k, v, DenseBwd{d.N, Bs, d.Hq, d.Hkv, d.B, chunk_groups(Bs, d.D, groups)}, d.scale, d.scale * 1.4426950408889634f);
  };
  auto as = [&](auto* k, auto* v) {
    using OT = std::remove_pointer_t<decltype(k)>;
    d.D == 64 ? go(k_flash_bwd_dkv_wide<OT, DenseBwd>, k, v) : go(k_flash_bwd_dkv128_wide<OT, DenseBwd>, k, v);
  };
  if (d.grads16) as((bf16_t*)dK, (bf16_t*)dV);
  else as((float*)dK, (float*)dV);
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
