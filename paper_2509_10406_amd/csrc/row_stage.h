// Tiles of 64 rows from memory through registers into LDS (lds_tile.h), for workgroups of 256 threads.
#pragma once
#include "lds_tile.h"

constexpr int BN = 64;  // rows staged in LDS per step

// Staging of a tile through registers, so that the global loads of the next tile are in flight while the current one is
// consumed: fetch_rows into registers, commit_rows from registers into LDS.  The registers are named members,
// not an array: an array that is passed around and read through pointer casts ends up in memory (the compiler
// parks it in LDS), and the wait for its loads then comes right after they are issued.
struct TileRegs {
  uint4 a, b, c, d;
};

// A tile as it lies: chunk c = thread + 256 i is chunk c % (D / 8) of row c / (D / 8), so a load instruction takes whole rows,
// and the tile in LDS (lds_tile.h) serves rows and transposed operands alike.
template <int D>
__device__ __forceinline__ uint4 fetch_row_chunk(const bf16_t* __restrict__ src, int r0, int N, int i, size_t step) {
  const int c = threadIdx.x + 256 * i;
  return *reinterpret_cast<const uint4*>(src + min(r0 + c / (D / 8), N - 1) * step + c % (D / 8) * 8);
}
template <int D>
__device__ __forceinline__ void fetch_rows(const bf16_t* __restrict__ src, int r0, int N, TileRegs& r, size_t step = D) {
  static_assert(BN * (D / 8) / 256 == (D == 64 ? 2 : 4), "chunks per thread");
  r.a = fetch_row_chunk<D>(src, r0, N, 0, step);
  r.b = fetch_row_chunk<D>(src, r0, N, 1, step);
  if constexpr (D == 128) {
    r.c = fetch_row_chunk<D>(src, r0, N, 2, step);
    r.d = fetch_row_chunk<D>(src, r0, N, 3, step);
  }
}
template <int D>
__device__ __forceinline__ void commit_row_chunk(const uint4 v, int i, bf16_t* tile) {
  const int c = threadIdx.x + 256 * i;
  *reinterpret_cast<uint4*>(tile + tile_at<D>(c / (D / 8), c % (D / 8))) = v;
}
template <int D>
__device__ __forceinline__ void commit_rows(const TileRegs& r, bf16_t* tile) {
  commit_row_chunk<D>(r.a, 0, tile);
  commit_row_chunk<D>(r.b, 1, tile);
  if constexpr (D == 128) {
    commit_row_chunk<D>(r.c, 2, tile);
    commit_row_chunk<D>(r.d, 3, tile);
  }
}
