// Packed sequences and the paged cache: what the entry points' checks hand to the kernels, and how a workgroup finds its rows.
#pragma once
#include "common.h"

struct Rows {  // strides of a packed tensor, in elements
  int64_t token, head;
  __device__ __forceinline__ int64_t at(int t, int h) const { return t * token + h * head; }
};

struct PackedDims {
  int S, Hq, Hkv, D, T, max_len;
  int dtype, grad_dtype;
  float scale;
  Rows q, k, v, o, g, dq, dk, dv;
};

struct CacheDims {
  int S, Hq, Hkv, D, T, pages, page, cols, max_new;
  int dtype;
  float scale;
  Rows q, k, v, o;
};

// Tiles of `per` rows that never straddle two sequences.  Sequence s has the numbers from cu[s] / per + s on: that leaves it at
// least as many as it has tiles, and needs no sums over the lengths.  Of the packed_slots numbers a few have no tile.
static inline long long packed_slots(int T, int S, int per) { return (long long)T / per + S; }

struct SeqTile {
  int s, t, beg, end;  // sequence, its tile, its rows beg .. end - 1
  bool ok;
  int h;
};

// the rows of sequence s (cu NULL: row s alone)
__device__ __forceinline__ int seq_row(const int32_t* cu, int s, int T) { return cu ? min(max(cu[s], 0), T) : min(s, T); }

// Every wave looks for itself, 64 sequences at a time; extra: more numbers per sequence than the tiles need.
__device__ __forceinline__ SeqTile seq_tile(const int32_t* __restrict__ cu, int S, int T, int per, int slot, int extra = 0) {
  const int lane = threadIdx.x % 64;
  auto start = [&](int s) { return seq_row(cu, s, T) / per + s * (1 + extra); };
  int lo = 0, n = S;
  SeqTile r{0, 0, 0, 0, false, 0};
  while (n > 1) {
    const int step = (n + 63) / 64;
    const bool le = lane * step < n && start(lo + lane * step) <= slot;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(le));
    if (c == 0) return r;
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  r.s = __builtin_amdgcn_readfirstlane(lo);
  r.beg = __builtin_amdgcn_readfirstlane(seq_row(cu, r.s, T));
  r.end = max(r.beg, __builtin_amdgcn_readfirstlane(seq_row(cu, r.s + 1, T)));
  r.t = slot - (r.beg / per + r.s * (1 + extra));
  r.ok = r.t >= 0 && r.t < (r.end - r.beg + per - 1) / per;
  return r;
}

// The numbering of the packed attention kernels' workgroups.  The tiles of a head stream the keys and values of their sequences, so an
// XCD (workgroups go to the eight round-robin) has whole heads, neighbours where it has several, and takes their tiles in
// the order of the rows, `back`: from the last one on.  A sequence's long tiles come before its short ones that way (the last tiles of queries
// are the long ones, the first of keys), and what runs at the same time reads the same rows.  Heads that are no multiple of
// eight: 2, 4 or 8 XCDs take turns at the tiles of theirs.
__device__ __forceinline__ SeqTile packed_tile(const int32_t* __restrict__ cu, int S, int T, int per, int H, int slots, bool back = true) {
  const int xcd = blockIdx.x % 8, n = blockIdx.x / 8;
  const int turns = H % 8 == 0 ? 1 : H % 4 == 0 ? 2 : H % 2 == 0 ? 4 : 8, hx = H * turns / 8;
  const int i = xcd % turns + turns * (n / hx), slot = back ? slots - 1 - i : i;
  SeqTile r = seq_tile(cu, S, T, per, slot);
  r.h = xcd / turns * hx + n % hx;
  r.ok = r.ok && slot >= 0 && slot < slots;
  return r;
}
static inline long long packed_grid(int H, long long slots) {
  const int turns = H % 8 == 0 ? 1 : H % 4 == 0 ? 2 : H % 2 == 0 ? 4 : 8;
  return (slots + turns - 1) / turns * (H * turns);
}
