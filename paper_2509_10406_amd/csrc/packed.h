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
// least as many as it has tiles, and needs no sums over the lengths.  Of the packed_slots numbers a few have no tile.  A token may
// count as `mul` rows (those of the heads of a group).
static inline long long packed_slots(int T, int S, int per, int mul = 1) { return (long long)T * mul / per + S; }

struct SeqTile {
  int s, t, beg, end;  // sequence, its tile, its rows beg .. end - 1
  bool ok;
  int h;
};

// the rows of sequence s (cu NULL: row s alone)
__device__ __forceinline__ int seq_row(const int32_t* cu, int s, int T) { return cu ? min(max(cu[s], 0), T) : min(s, T); }

// Every wave looks for itself, 64 sequences at a time (up to 64 of them: one read); extra: more numbers per sequence than the tiles need.
__device__ __forceinline__ SeqTile seq_tile(const int32_t* __restrict__ cu, int S, int T, int per, int slot, int extra = 0, int mul = 1) {
  const int lane = threadIdx.x % 64;
  int lo = 0, n = S, step, c, beg, end;
  do {
    step = (n + 63) / 64;
    const int s = min(lo + lane * step, S - 1);
    beg = seq_row(cu, s, T);
    end = seq_row(cu, s + 1, T);
    c = __popcll(__builtin_amdgcn_ballot_w64(lane * step < n && beg * mul / per + s * (1 + extra) <= slot));
    if (c == 0) return SeqTile{0, 0, 0, 0, false, 0};
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  } while (step > 1);
  SeqTile r;
  r.s = lo;
  r.beg = __builtin_amdgcn_readlane(beg, c - 1);
  r.end = max(r.beg, __builtin_amdgcn_readlane(end, c - 1));
  r.t = slot - (r.beg * mul / per + r.s * (1 + extra));
  r.ok = r.t >= 0 && r.t < ((r.end - r.beg) * mul + per - 1) / per;
  r.h = 0;
  return r;
}

// sums over the lanes up to the own one
__device__ __forceinline__ int scan64(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8: inside a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15: rows 0, 2 -> 1, 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast 31: row 1 -> 2, 3
  return v;
}

// The x-th of all tiles, `back`: from the last one on; for up to 64 sequences, a lane each.
__device__ __forceinline__ SeqTile seq_tile_exact(const int32_t* __restrict__ cu, int S, int T, int per, int x, bool back, int mul) {
  const int lane = threadIdx.x % 64;
  int beg = 0, end = 0;
  if (lane < S) {
    beg = seq_row(cu, lane, T);
    end = max(seq_row(cu, lane + 1, T), beg);
  }
  const int upto = scan64(((end - beg) * mul + per - 1) / per), total = __builtin_amdgcn_readlane(upto, 63);
  SeqTile r{0, 0, 0, 0, false, 0};
  if (x >= total) return r;
  const int at = back ? total - 1 - x : x;
  r.s = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > at));
  r.beg = __builtin_amdgcn_readlane(beg, r.s);
  r.end = __builtin_amdgcn_readlane(end, r.s);
  r.t = at - (r.s ? __builtin_amdgcn_readlane(upto, r.s - 1) : 0);
  r.ok = true;
  return r;
}

// The numbering of the packed attention kernels' workgroups.  The tiles of a head stream the keys and values of their sequences, so an
// XCD (workgroups go to the eight round-robin) has whole heads, neighbours where it has several, and takes their tiles in
// the order of the rows, `back`: from the last one on.  A sequence's long tiles come before its short ones that way (the last tiles of queries
// are the long ones, the first of keys), and what runs at the same time reads the same rows.  Heads that are no multiple of
// eight: 2, 4 or 8 XCDs take turns at the tiles of theirs.
// Up to 64 sequences are numbered without gaps, which takes one sum over the lanes.  Gaps cost more than their own time: workgroups are dealt
// out in turns, and where every second number is empty some CUs get little else (the wide kernel at 64 sequences of 256, 16 heads, D =
// 128: 83 us without, 127 with gaps; 40 of 400, D = 64, in tiles of 128: 48 and 51).  More sequences would take several sums: 200 of
// 60, 32 heads of 8, D = 128 81 us with gaps 71.
// A list of the tiles, long sequences first, made by a launch in front, was no faster: 16 prompts of 1 to 2800 tokens, 32 heads, D = 128 282
// us against 288, 5 for the list; all tiles by their length alone slower, as a sequence's rows are then read again and again.
__device__ __forceinline__ SeqTile packed_tile(const int32_t* __restrict__ cu, int S, int T, int per, int H, int slots, bool back = true, int mul = 1) {
  const int xcd = blockIdx.x % 8, n = blockIdx.x / 8;
  const int turns = H % 8 == 0 ? 1 : H % 4 == 0 ? 2 : H % 2 == 0 ? 4 : 8, hx = H * turns / 8;
  const int i = xcd % turns + turns * (n / hx), slot = back ? slots - 1 - i : i;
  SeqTile r = S <= 64 ? seq_tile_exact(cu, S, T, per, i, back, mul) : seq_tile(cu, S, T, per, slot, 0, mul);
  r.h = xcd / turns * hx + n % hx;
  r.ok = r.ok && i < slots;
  return r;
}
// A call that writes to a workspace clears the stamp at its head: the first workgroup of a launch does, for a layout that starts at `behind`.
__device__ __forceinline__ void clear_stamp(float* behind) {
  if ((blockIdx.x | blockIdx.y | blockIdx.z) == 0 && threadIdx.x < 4) reinterpret_cast<uint64_t*>(behind - kTagBytes / 4)[threadIdx.x] = 0;
}

static inline long long packed_grid(int H, long long slots) {
  const int turns = H % 8 == 0 ? 1 : H % 4 == 0 ? 2 : H % 2 == 0 ? 4 : 8;
  return (slots + turns - 1) / turns * (H * turns);
}
