// Attention of new tokens to a paged cache of e4m3 keys and values with a scale per page and head (causal, grouped heads).
//
// Bound by HBM for the few rows of generation: every cached byte is read once per key/value head, all query heads of the group
// (and a sequence's new tokens) being the columns of the same matrix instructions.  e4m3 values are bf16 values, so one conversion
// instruction for two bytes makes exact operands; key scales are applied to the scores, value scales to the weights, in fp32.
// fp32 inputs: queries and weights go in as three bf16 terms each (24 bits), products and sums are those of fp32.
//
// A wave takes 64 keys at a time, straight from memory to the operands' registers:
//   S^T = K Q^T   16x16x32: row r of the t-th of four instructions is key 16 (r / 4) + 4 t + r % 4, so a lane of group g = lane / 16 has
//                 the scores of keys 16 g .. 16 g + 15 in order: one page, one scale
//   O^T += V^T P^T  the lane's operand is 16 keys of one dim, adjacent in the cache (values have their dims first), and its
//                 weights are in order already
// so neither K, V nor P goes through LDS, and pages of 16 tokens or more need no other code.  The next tile's keys are on
// their way from behind the scores on, its values from behind the products.
//
// Work is counted in units of 256 keys (four waves of a workgroup, a tile each), over all sequences in a row, and divided evenly among
// the workgroups of a (head, row tile): a long context is shared by many, a workgroup may have several short ones.  A
// sequence that lies inside one workgroup's share is finished there; of the others every workgroup leaves (sum, maximum,
// normaliser) and a second kernel joins them, in the order of the keys: results do not depend on timing.
// 32 heads of 8, D = 128: two contexts of 131072 99 us, 537 MB at 5.4 TB/s; 64 ragged ones of up to 8k 59 us, 304 MB at 5.2.
#include <type_traits>

#include "attn_cols.h"
#include "packed.h"

namespace {

constexpr int UNIT = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.f;  // the softmax reference follows the maximum in steps of more than 2^8

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

struct CacheWork {  // of one launch
  int W, R, rows;   // workgroups per (head, row tile), row tiles, rows of a tile
  int G, sh;        // query heads per key/value head, log2(page)
  int least;        // units of a share, at the least
  bool whole;       // sequences are not divided: workgroup w has those of the numbers w, w + W, ..
  int used, join;   // rows of a tile that sequences have by the caller's bound, rows of a workgroup of the joining kernel
  float *po, *pm;   // partial sums [R][Hkv][2 W][rows][D], (maximum, normaliser) [..][rows][2]
};

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// sequence s as row tile r sees it
struct Seg {
  int beg, n, first;  // first row, new tokens, position of the first of them
  int keys;           // keys that any row of the tile may see
  int units;          // 0: no rows in this tile
};
__device__ __forceinline__ Seg seg_of(const CacheDims& d, const CacheWork& w, const int32_t* cu, const int32_t* lens, int s, int r, int tile_last) {
  Seg g;
  g.beg = seq_row(cu, s, d.T);
  g.n = max(seq_row(cu, s + 1, d.T), g.beg) - g.beg;
  const int L = max(lens[s], 0);
  g.first = L - g.n;
  const int last = min(tile_last, g.n - 1);
  g.keys = max(min(min(L, d.cols << w.sh), g.first + last + 1), 0);
  g.units = r * w.rows < g.n * w.G ? max((g.keys + UNIT - 1) / UNIT, 1) : 0;
  return g;
}
// the new token that the last row of a tile is of
__device__ __forceinline__ int last_token(const CacheWork& w, int r) { return ((r + 1) * w.rows - 1) / w.G; }

// All units of a row tile in a row: their number; whether a sequence has rows in the tile w.R further on; and either where the first unit of workgroup x's
// share lies (its sequence, the units in front of that), or the units in front of sequence x.  Up to 64 sequences: every wave by
// itself, a lane each; else the 256 threads together, each with a run of the sequences.
struct Found {
  int total, before, s;
  bool more;
};
struct FindLds {
  int sum[4], before, s, more;
};
// The first unit of workgroup w's share, and whose share a unit is in.  A share has `least` units, so the last workgroups may have none.
__device__ __forceinline__ int shares(const CacheWork& w, int total) { return min(w.W, max(total / w.least, 1)); }
__device__ __forceinline__ int share(const CacheWork& w, int total, int wg) {
  const int n = shares(w, total);
  return wg >= n ? total : (int)((long long)total * wg / n);
}
__device__ __forceinline__ int owner(const CacheWork& w, int total, int unit) { return (int)((((long long)unit + 1) * shares(w, total) - 1) / total); }
__device__ __forceinline__ Found find_unit(const CacheDims& d, const CacheWork& w, const int32_t* cu, const int32_t* lens, int r, int tile_last, FindLds& lds, int x,
                                           bool by_seq = false) {
  if (d.S <= 64) {
    const int lane = threadIdx.x % 64;
    Seg g{};
    if (lane < d.S) g = seg_of(d, w, cu, lens, lane, r, tile_last);
    const int upto = scan64(g.units);
    Found f;
    f.total = __builtin_amdgcn_readlane(upto, 63);
    f.more = __builtin_amdgcn_ballot_w64(g.n * w.G > (r + w.R) * w.rows) != 0;
    const int a = share(w, f.total, x);
    f.s = by_seq ? x : a < f.total ? __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > a)) : 0;
    f.before = f.s ? __builtin_amdgcn_readlane(upto, f.s - 1) : 0;
    return f;
  }
  const int tid = threadIdx.x, lane = tid % 64, per = (d.S + 255) / 256, s0 = tid * per, s1 = min(s0 + per, d.S);
  int mine = 0;
  bool more = false;
  for (int s = s0; s < s1; ++s) {
    const Seg g = seg_of(d, w, cu, lens, s, r, tile_last);
    mine += g.units;
    more = more || g.n * w.G > (r + w.R) * w.rows;
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  __syncthreads();  // what an earlier call left has been read
  if (lane == 63) lds.sum[tid / 64] = upto;
  if (tid == 0) lds.s = lds.before = lds.more = 0;  // of a share that begins behind the last unit: no place, but an index
  __syncthreads();
  Found f;
  f.total = __builtin_amdgcn_readfirstlane(lds.sum[0] + lds.sum[1] + lds.sum[2] + lds.sum[3]);
  for (int i = 0; i < tid / 64; ++i) upto += lds.sum[i];
  if (more) lds.more = 1;
  const int a = share(w, f.total, x);
  if (by_seq ? s0 <= x && x < s1 : upto - mine <= a && a < upto) {
    int b = upto - mine;
    for (int s = s0; s < s1; ++s) {
      const int u = seg_of(d, w, cu, lens, s, r, tile_last).units;
      if (by_seq ? s == x : a < b + u) {
        lds.s = s;
        lds.before = b;
        break;
      }
      b += u;
    }
  }
  __syncthreads();
  f.s = __builtin_amdgcn_readfirstlane(lds.s);
  f.before = __builtin_amdgcn_readfirstlane(lds.before);
  f.more = __builtin_amdgcn_readfirstlane(lds.more) != 0;
  return f;
}

__device__ __forceinline__ bf16x8_t from_e4m3(uint32_t a, uint32_t b) {
  const bf16x2_t x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const bf16x2_t z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  return bf16x8_t{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// 8 adjacent elements as TERMS bf16 operands that add up to them
template <int TERMS>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8_t (&to)[TERMS]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rest[j] = x[j];
#pragma unroll
  for (int t = 0; t < TERMS; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      to[t][j] = (__bf16)rest[j];
      if (t + 1 < TERMS) rest[j] -= (float)to[t][j];
    }
}
__device__ __forceinline__ void load_q(const bf16_t* p, bf16x8_t (&to)[1]) { to[0] = *reinterpret_cast<const bf16x8_t*>(p); }
__device__ __forceinline__ void load_q(const float* p, bf16x8_t (&to)[3]) {
  float x[8];
  ld4(p, 0, *reinterpret_cast<float(*)[4]>(x));
  ld4(p, 4, *reinterpret_cast<float(*)[4]>(x + 4));
  split8<3>(x, to);
}

// What workgroup w of row tile r0 has, one sequence after the other: body(sequence's Seg, its number, row tile, first and last unit, the place
// of its part if it has only some of them).
template <typename F>
__device__ __forceinline__ void for_segments(const CacheDims& d, const CacheWork& wk, const int32_t* cu, const int32_t* lens, FindLds& find, F body) {
  const int w = blockIdx.x, hk = blockIdx.y, r0 = blockIdx.z;
  for (int r = r0;; r += wk.R) {
    const int tile_last = last_token(wk, r);
    const Found f = find_unit(d, wk, cu, lens, r, tile_last, find, w);
    // More rows than the caller's bound said: whole sequences, one by one, too, so that nothing is left to be joined.
    const bool over = wk.whole || r >= wk.R;
    int a = share(wk, f.total, w), before = f.before;
    const int b = share(wk, f.total, w + 1);
    int s = over ? w : f.s;
    while (over ? s < d.S : a < b) {
      const Seg sg = seg_of(d, wk, cu, lens, s, r, tile_last);
      const int u0 = over ? 0 : a - before, u1 = over ? sg.units : min(sg.units, b - before);
      if (sg.units > 0) body(sg, s, r, u0, u1, (((size_t)r0 * d.Hkv + hk) * 2 * wk.W + 2 * w + (u0 == 0)) * wk.rows);
      if (over) {
        s += wk.W;
      } else {
        before += sg.units;
        a = max(a, before);
        ++s;
      }
    }
    if (!f.more) break;
  }
}

template <typename T, int D, int RT>
__global__ void __launch_bounds__(256, RT > 1 ? 1 : D == 64 && sizeof(T) == 2 ? 3 : 2) k_cache_fwd(CacheDims d, CacheWork wk, const T* __restrict__ Q, const int32_t* __restrict__ cu,
                                                   const int32_t* __restrict__ lens, const int32_t* __restrict__ table,
                                                   const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc, const float* __restrict__ ks,
                                                   const float* __restrict__ vs, T* __restrict__ O, float* __restrict__ LSE) {
  constexpr int TERMS = sizeof(T) == 4 ? 3 : 1, KC = D / 64, NM = D / 32, DT = D / 16, ROWS = 16 * RT, LDO = D + 4;
  __shared__ FindLds find;
  __shared__ float ml[2][4][ROWS];
  __shared__ __attribute__((aligned(16))) float os[4][16][LDO];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 16, g = lane / 16;
  const int hk = blockIdx.y, G = wk.G, sh = wk.sh, inpage = d.page - 1;
  const float zscale = d.scale * kLog2e;

  for_segments(d, wk, cu, lens, find, [&](const Seg& sg, int s, int r, int u0, int u1, size_t slot) {
    // this lane's column of every row tile: new token, head, last key
    int row[RT], pos[RT];
    int64_t at[RT];
    const int rows = sg.n * G;
    bf16x8_t qf[RT][NM][TERMS];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int x = r * ROWS + 16 * t + col, y = min(x, rows - 1), i = y / G, h = hk * G + y - i * G;
      row[t] = sg.beg + i;
      pos[t] = x < rows ? sg.first + i : -1;
      at[t] = d.q.at(row[t], h);
#pragma unroll
      for (int m = 0; m < NM; ++m) load_q(Q + at[t] + 64 * (m / 2) + 16 * g + 8 * (m % 2), qf[t][m]);
    }
    const int least = sg.first + r * ROWS / G;  // the first row's last key: no row of the tile is masked up to there
    f32x4_t o[RT][DT];
    float mx[RT], l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      mx[t] = MUSE_NEG_INF;
      l[t] = 0.f;
#pragma unroll
      for (int x = 0; x < DT; ++x) o[t][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t* tab = table + (size_t)s * d.cols;
    // the page of 16 keys, -1 if there are none
    auto page_of = [&](int key) {
      int p = -1;
      if (key < sg.keys) p = tab[key >> sh];
      return p >= 0 && p < d.pages ? p : -1;
    };
    u32x4_t kr[4][KC], vr[DT];
    auto load_k = [&](int k0, int pid) {
      const uint8_t* p = kc + (((size_t)max(pid, 0) * d.Hkv + hk) << sh) * D + (((k0 + 16 * (col / 4)) & inpage) + col % 4) * D + 16 * g;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int c = 0; c < KC; ++c) kr[t][c] = *reinterpret_cast<const u32x4_t*>(p + 4 * t * D + 64 * c);
    };
    auto load_v = [&](int k0, int pid) {
      const uint8_t* p = vc + ((((size_t)max(pid, 0) * d.Hkv + hk) * D + col) << sh) + ((k0 + 16 * g) & inpage);
#pragma unroll
      for (int x = 0; x < DT; ++x) vr[x] = *reinterpret_cast<const u32x4_t*>(p + ((16 * x) << sh));
    };
    const int kend = min(u1 * UNIT, sg.keys);
    int k0 = u0 * UNIT + 64 * wave;
    int pk = page_of(k0 + 16 * (col / 4)), pv = page_of(k0 + 16 * g);
    float ksc = 0.f, vsc = 0.f;
    if (k0 < kend) {
      load_k(k0, pk);
      load_v(k0, pv);
      ksc = ks[(size_t)max(pv, 0) * d.Hkv + hk];
      vsc = vs[(size_t)max(pv, 0) * d.Hkv + hk];
    }
    int npk = page_of(k0 + UNIT + 16 * (col / 4)), npv = page_of(k0 + UNIT + 16 * g);
    for (; k0 < kend; k0 += UNIT) {
      f32x4_t sc[RT][4];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) sc[t][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          const bf16x8_t kf = from_e4m3(kr[x][m / 2][2 * (m % 2)], kr[x][m / 2][2 * (m % 2) + 1]);
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int u = TERMS - 1; u >= 0; --u) sc[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][m][u], sc[t][x], 0, 0, 0);
        }
      const bool more = k0 + UNIT < kend;
      const bool live = pv >= 0;
      const float c = (live ? ksc : 0.f) * zscale, pvs = live ? vsc : 0.f;
      if (more) {
        load_k(k0 + UNIT, npk);
        ksc = ks[(size_t)max(npv, 0) * d.Hkv + hk];
        vsc = vs[(size_t)max(npv, 0) * d.Hkv + hk];
      }
      const bool edge = k0 + 63 > least || __builtin_amdgcn_ballot_w64(!live) != 0;  // wave-uniform
      bf16x8_t pf[RT][2][TERMS];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float z[16], top = MUSE_NEG_INF;
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = sc[t][e / 4][e % 4] * c;
        if (edge) {
#pragma unroll
          for (int e = 0; e < 16; ++e) z[e] = live && k0 + 16 * g + e <= pos[t] ? z[e] : MUSE_NEG_INF;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, z[e]);
        {
          typedef uint32_t u2_t __attribute__((ext_vector_type(2)));
          const u2_t x = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
          top = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
          const u2_t y = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
          top = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
        }
        if (__builtin_amdgcn_ballot_w64(top > mx[t] + kLazy)) {
          const float mn = top > mx[t] + kLazy ? top : mx[t], al = mn == MUSE_NEG_INF ? 1.f : exp2_(mx[t] - mn);
          mx[t] = mn;
          l[t] *= al;
#pragma unroll
          for (int x = 0; x < DT; ++x) o[t][x] *= al;
        }
        const float ref = mx[t] == MUSE_NEG_INF ? 0.f : mx[t];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          float p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float e = exp2_(z[8 * m + j] - ref);
            l[t] += e;
            p[j] = e * pvs;
          }
          split8<TERMS>(p, pf[t][m]);
        }
      }
      if (edge) {  // bytes behind the last key may be anything, and 0 * NaN is NaN
        const int nb = live ? min(max(sg.keys - (k0 + 16 * g), 0), 16) : 0;
        u32x4_t mask;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = nb - 4 * i;
          mask[i] = k >= 4 ? 0xffffffffu : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
        }
#pragma unroll
        for (int x = 0; x < DT; ++x) vr[x] &= mask;
      }
#pragma unroll
      for (int x = 0; x < DT; ++x)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const bf16x8_t vf = from_e4m3(vr[x][2 * m], vr[x][2 * m + 1]);
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int u = TERMS - 1; u >= 0; --u) o[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t][m][u], o[t][x], 0, 0, 0);
        }
      pv = npv;
      if (more) {
        load_v(k0 + UNIT, npv);
        npk = page_of(k0 + 2 * UNIT + 16 * (col / 4));
        npv = page_of(k0 + 2 * UNIT + 16 * g);
      }
    }
    // the four waves' parts
    const bool whole = u0 == 0 && u1 == sg.units;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
      if (g == 0) {
        ml[0][wave][16 * t + col] = mx[t];
        ml[1][wave][16 * t + col] = l[t];
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (r * ROWS + 16 * t >= rows) break;  // the same for all
#pragma unroll
      for (int x = 0; x < DT; ++x) *reinterpret_cast<f32x4_t*>(&os[wave][col][16 * x + 4 * g]) = o[t][x];
      __syncthreads();
      const int rr = tid / 16, y = r * ROWS + 16 * t + rr, d0 = tid % 16 * (D / 16);
      float M = MUSE_NEG_INF, lt = 0.f, v[D / 16];
#pragma unroll
      for (int i = 0; i < 4; ++i) M = fmaxf(M, ml[0][i][16 * t + rr]);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) v[j] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float fw = M == MUSE_NEG_INF ? 0.f : exp2_(ml[0][i][16 * t + rr] - M);
        lt += fw * ml[1][i][16 * t + rr];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) v[j] = fmaf(fw, os[i][rr][d0 + j], v[j]);
      }
      if (whole) {
        if (y < rows) {
          const int i = y / G, h = hk * G + y - i * G;
          const float inv = lt == 0.f ? 0.f : 1.f / lt;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) v[j] *= inv;
          T* to = O + d.o.at(sg.beg + i, h) + d0;
#pragma unroll
          for (int j = 0; j < D / 64; ++j) st4(to, 4 * j, v + 4 * j);
          if (LSE && tid % 16 == 0) LSE[(size_t)h * d.T + sg.beg + i] = (M + __builtin_amdgcn_logf(lt)) * kLn2;
        }
      } else {
        float* to = wk.po + (slot + 16 * t + rr) * D + d0;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) st4(to, 4 * j, v + 4 * j);
        if (tid % 16 == 0) *reinterpret_cast<float2*>(wk.pm + (slot + 16 * t + rr) * 2) = make_float2(M, lt);
      }
      __syncthreads();
    }
  });
}

// Many rows (pieces of prompts): a workgroup has 128 rows, 32 to a wave, and its four waves share the staged tiles: 64 keys and
// values as bf16 in LDS, converted once for all rows (k_cache_fwd would convert them again for every 16 to 64).  Keys lie row by row (lds_tile.h);
// values as they come, dims first, a dim's 16 keys in the order of the weights' operand (accumulator rows 4 h .. and 8 + 4 h .. of half
// h side by side), the 16-byte chunks of a dim's 64 keys changed places by bits of the dim so that 16 dims reach all banks.
// 8 pieces of up to 289 tokens on contexts of up to 3.5k, 16 heads of 4, D = 128: 55 us, bound by conversions and vector work.
template <int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) k_cache_fwd_cols(
    CacheDims d, CacheWork wk, const bf16_t* __restrict__ Q, const int32_t* __restrict__ cu, const int32_t* __restrict__ lens,
    const int32_t* __restrict__ table, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc, const float* __restrict__ ks,
    const float* __restrict__ vs, bf16_t* __restrict__ O, float* __restrict__ LSE) {
  constexpr int DT = D / 32, NC = D / 64;  // 16-byte pieces of keys, and of values, that a thread brings in
  __shared__ FindLds find;
  __shared__ __attribute__((aligned(256))) bf16_t kt[2][64 * D];
  __shared__ __attribute__((aligned(256))) bf16_t vt[2][64 * D];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, col = lane % 32, half = lane / 32;
  const int hk = blockIdx.y, G = wk.G, sh = wk.sh, inpage = d.page - 1;
  const float zscale = d.scale * kLog2e;
  auto vt_at = [](int dim, int chunk) { return dim * 64 + ((chunk ^ ((dim >> 1) & 7)) << 3); };
  for_segments(d, wk, cu, lens, find, [&](const Seg& sg, int s, int r, int u0, int u1, size_t slot) {
    const int rows = sg.n * G, w0 = r * 128 + 32 * wave, x = w0 + col, y = min(x, rows - 1), i = y / G, h = hk * G + y - i * G;
    const int first = sg.first + min(w0, rows - 1) / G, last = sg.first + min(w0 + 31, rows - 1) / G;  // the wave's positions
    Cols<D> c;
    c.start(Q + d.q.at(sg.beg + i, h), half);
    const int32_t* tab = table + (size_t)s * d.cols;
    struct Tile {  // what belongs to 64 keys: pages of 16 keys each, and their scales
      int pid[4];
      float zs[4], vs[4];
    };
    auto pages_of = [&](int k0) {
      Tile t;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        int p = -1;
        if (k0 + 16 * j < sg.keys) p = __builtin_amdgcn_readfirstlane(tab[(k0 + 16 * j) >> sh]);
        t.pid[j] = p >= 0 && p < d.pages ? p : -1;
      }
      return t;
    };
    u32x4_t kr[NC], vr[NC];
    auto fetch = [&](int k0, Tile& t) {
#pragma unroll
      for (int u = 0; u < NC; ++u) {
        const int cc = tid + 256 * u, row = cc / (D / 16), j = row / 16, dim = cc / 4, jv = cc % 4;
        const int pk = max(j == 0 ? t.pid[0] : j == 1 ? t.pid[1] : j == 2 ? t.pid[2] : t.pid[3], 0);
        const int pv = max(jv == 0 ? t.pid[0] : jv == 1 ? t.pid[1] : jv == 2 ? t.pid[2] : t.pid[3], 0);
        kr[u] = *reinterpret_cast<const u32x4_t*>(kc + ((((size_t)pk * d.Hkv + hk) << sh) + ((k0 + row) & inpage)) * D + cc % (D / 16) * 16);
        vr[u] = *reinterpret_cast<const u32x4_t*>(vc + ((((size_t)pv * d.Hkv + hk) * D + dim) << sh) + ((k0 + 16 * jv) & inpage));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const size_t at = (size_t)max(t.pid[j], 0) * d.Hkv + hk;
        t.zs[j] = t.pid[j] < 0 ? 1.f : fmaxf(ks[at] * zscale, 0x1p-126f);
        t.vs[j] = t.pid[j] < 0 ? 0.f : vs[at];
      }
    };
    auto commit = [&](int k0, const Tile& t, int buf) {
#pragma unroll
      for (int u = 0; u < NC; ++u) {
        const int cc = tid + 256 * u, row = cc / (D / 16), ch = cc % (D / 16) * 2, dim = cc / 4, jv = cc % 4;
        *reinterpret_cast<bf16x8_t*>(&kt[buf][tile_at<D>(row, ch)]) = from_e4m3(kr[u][0], kr[u][1]);
        *reinterpret_cast<bf16x8_t*>(&kt[buf][tile_at<D>(row, ch + 1)]) = from_e4m3(kr[u][2], kr[u][3]);
        // bytes behind the last key, or of no page, may be anything, and 0 * NaN is NaN
        const int pv = jv == 0 ? t.pid[0] : jv == 1 ? t.pid[1] : jv == 2 ? t.pid[2] : t.pid[3], nb = pv < 0 ? 0 : sg.keys - (k0 + 16 * jv);
        u32x4_t v = vr[u];
        if (nb < 16) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] &= nb >= 4 * e + 4 ? 0xffffffffu : nb <= 4 * e ? 0u : (1u << (8 * (nb - 4 * e))) - 1u;
        }
        *reinterpret_cast<bf16x8_t*>(&vt[buf][vt_at(dim, 2 * jv)]) = from_e4m3(v[0], v[2]);
        *reinterpret_cast<bf16x8_t*>(&vt[buf][vt_at(dim, 2 * jv + 1)]) = from_e4m3(v[1], v[3]);
      }
    };
    const int kbeg = u0 * UNIT, kend = min(u1 * UNIT, sg.keys);
    Tile now = pages_of(kbeg), next = pages_of(kbeg + 64);
    __syncthreads();  // nobody reads the tiles of the segment before
    if (kbeg < kend) {
      fetch(kbeg, now);
      commit(kbeg, now, 0);
      if (kbeg + 64 < kend) fetch(kbeg + 64, next);
    }
    int buf = 0;
    for (int k0 = kbeg; k0 < kend; k0 += 64, buf ^= 1) {
      __syncthreads();
      Tile after = pages_of(k0 + 128);
      if (k0 + 64 < kend) commit(k0 + 64, next, buf ^ 1);
      if (k0 + 128 < kend) fetch(k0 + 128, after);
      if (w0 < rows && k0 <= last) {
        const uint32_t dead = (now.pid[0] < 0 ? 1u : 0u) | (now.pid[1] < 0 ? 2u : 0u) | (now.pid[2] < 0 ? 4u : 0u) | (now.pid[3] < 0 ? 8u : 0u);
        c.attend([&](int hh, int u) { return tile_row<D>(kt[buf], 32 * hh + col, 2 * u + half); },
                 [&](int g, int t) { return *reinterpret_cast<const bf16x8_t*>(&vt[buf][vt_at(32 * t + col, 2 * g + half)]); },
                 [&](int g) { return now.zs[g]; }, [&](int g) { return now.vs[g]; }, k0 + 63 > first, sg.first + i - k0, half, dead);
      }
      now = next;
      next = after;
    }
    if (x >= rows) return;
    const float l = c.l + __shfl_xor(c.l, 32, 64);
    if (u0 == 0 && u1 == sg.units) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16_t* to = O + d.o.at(sg.beg + i, h);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float v[4] = {c.o[t][4 * g] * inv, c.o[t][4 * g + 1] * inv, c.o[t][4 * g + 2] * inv, c.o[t][4 * g + 3] * inv};
          st4(to, 32 * t + 8 * g + 4 * half, v);
        }
      if (LSE && half == 0) LSE[(size_t)h * d.T + sg.beg + i] = (c.m + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      const size_t at = slot + 32 * wave + col;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float v[4] = {c.o[t][4 * g], c.o[t][4 * g + 1], c.o[t][4 * g + 2], c.o[t][4 * g + 3]};
          st4(wk.po + at * D, 32 * t + 8 * g + 4 * half, v);
        }
      if (half == 0) *reinterpret_cast<float2*>(wk.pm + at * 2) = make_float2(c.m, l);
    }
  });
}

// Joins the parts of the sequences that several workgroups share.  Where there are fewer sequences than shares workgroup x has sequence x, else
// it looks at the border between the shares x and x + 1, and the first border inside a sequence has that sequence.
struct Parts {
  Seg sg;
  int w0, n;    // the sequence's parts are those of the workgroups w0 .. w0 + n - 1; n < 2: nothing to be done here
  size_t base;  // of the head's and row tile's parts
  __device__ __forceinline__ size_t at(int i, int rows) const { return (base + 2 * (w0 + i) + (i == 0)) * rows; }  // of the i-th part's first row
};
__device__ __forceinline__ Parts parts_of(const CacheDims& d, const CacheWork& wk, const int32_t* cu, const int32_t* lens, FindLds& find, int x, int hk, int r) {
  Parts p{};
  const bool by_seq = d.S < wk.W;
  const int tile_last = last_token(wk, r);
  const Found f = find_unit(d, wk, cu, lens, r, tile_last, find, by_seq ? x : x + 1, by_seq);
  if (!by_seq) {
    const int a = share(wk, f.total, x + 1);
    if (a >= f.total || share(wk, f.total, x) > f.before || a <= f.before) return p;
  }
  p.sg = seg_of(d, wk, cu, lens, f.s, r, tile_last);
  if (p.sg.units == 0) return p;
  p.w0 = owner(wk, f.total, f.before);
  p.n = owner(wk, f.total, f.before + p.sg.units - 1) - p.w0 + 1;
  p.base = ((size_t)r * d.Hkv + hk) * 2 * wk.W;
  return p;
}

// Few rows (tiles of 16): bound by the latency of its reads.  A workgroup has one row, and its waves a quarter of the parts each where there
// are many (joined in order, through LDS), or a row per wave.  5.4 us for two contexts of 131072, 6.1 for 64 ragged ones, 32 heads, D = 128.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_cache_join(CacheDims d, CacheWork wk, const int32_t* __restrict__ cu, const int32_t* __restrict__ lens,
                                                    T* __restrict__ O, float* __restrict__ LSE) {
  constexpr int DL = D / 64, FEW = 8;
  __shared__ FindLds find;
  __shared__ float part[4][D + 1];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
  const int groups = (wk.used + wk.join - 1) / wk.join, hk = blockIdx.y / groups, first = blockIdx.y % groups * wk.join, r = blockIdx.z;
  clear_stamp(wk.po);
  const Parts p = parts_of(d, wk, cu, lens, find, blockIdx.x, hk, r);
  if (p.n < 2) return;
  const int n = p.n;
  const bool together = wk.join == 1 && n > FEW;
  if (!together && wave >= wk.join) return;
  const int rows = min(16, p.sg.n * wk.G - r * 16);
  // join is 1 or 4; rows beyond the caller's bound (`used`) go round once more
  for (int q = first + (together ? 0 : wave % wk.join); q < rows; q += groups * wk.join) {
    const int i0 = together ? n * wave / 4 : 0, i1 = together ? n * (wave + 1) / 4 : n;
    float M = MUSE_NEG_INF;
    for (int i = lane; i < n; i += 64) M = fmaxf(M, wk.pm[(p.at(i, 16) + q) * 2]);
    M = wave_max(M);
    float l = 0.f, v[DL] = {};
    auto add = [&](auto batch, int i, float fw, int j0) {  // the parts i .. i + batch - 1, all asked for before the first is used
      constexpr int B = decltype(batch)::value;
      float x[B][DL];
#pragma unroll
      for (int u = 0; u < B; ++u)
#pragma unroll
        for (int j = 0; j < DL; ++j) x[u][j] = wk.po[(p.at(i + u, 16) + q) * D + lane * DL + j];
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const float fu = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, fw), i + u - j0));
#pragma unroll
        for (int j = 0; j < DL; ++j) v[j] = fmaf(fu, x[u][j], v[j]);
      }
    };
    for (int j0 = i0; j0 < i1; j0 += 64) {
      float fw = 0.f;
      if (j0 + lane < i1) {
        const float2 ml = *reinterpret_cast<const float2*>(wk.pm + (p.at(j0 + lane, 16) + q) * 2);
        fw = M == MUSE_NEG_INF ? 0.f : exp2_(ml.x - M);
        l += fw * ml.y;
      }
      int i = j0;
      const int end = min(j0 + 64, i1);
      for (; i + 8 <= end; i += 8) add(std::integral_constant<int, 8>(), i, fw, j0);
      for (; i + 2 <= end; i += 2) add(std::integral_constant<int, 2>(), i, fw, j0);
      if (i < end) add(std::integral_constant<int, 1>(), i, fw, j0);
    }
    l = wave_sum(l);
    if (together) {
      __syncthreads();  // the row before has been read
#pragma unroll
      for (int j = 0; j < DL; ++j) part[wave][lane * DL + j] = v[j];
      if (lane == 0) part[wave][D] = l;
      __syncthreads();
      if (wave != 0) continue;
      l = (part[0][D] + part[1][D]) + (part[2][D] + part[3][D]);
#pragma unroll
      for (int j = 0; j < DL; ++j) v[j] = (part[0][lane * DL + j] + part[1][lane * DL + j]) + (part[2][lane * DL + j] + part[3][lane * DL + j]);
    }
    const int y = r * 16 + q, i = y / wk.G, h = hk * wk.G + y - i * wk.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* to = O + d.o.at(p.sg.beg + i, h) + lane * DL;
#pragma unroll
    for (int j = 0; j < DL; ++j) Elem<T>::st(to, j, v[j] * inv);
    if (LSE && lane == 0) LSE[(size_t)h * d.T + p.sg.beg + i] = (M + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// Many rows (tiles of 32, 64 or 128, bf16): a workgroup has 32 rows, a thread four dims of D / 32 of them, whose parts it asks for together.
// 15.6 us for 1571 rows of 16 heads, D = 128, in 8 sequences.
template <int D>
__global__ void __launch_bounds__(256) k_cache_join_rows(CacheDims d, CacheWork wk, const int32_t* __restrict__ cu, const int32_t* __restrict__ lens,
                                                         bf16_t* __restrict__ O, float* __restrict__ LSE) {
  constexpr int TPR = D / 4, STEP = 256 / TPR, N = 32 / STEP;
  __shared__ FindLds find;
  const int tid = threadIdx.x, groups = wk.rows / 32, hk = blockIdx.y / groups, q0 = blockIdx.y % groups * 32 + tid / TPR, r = blockIdx.z;
  clear_stamp(wk.po);
  const Parts p = parts_of(d, wk, cu, lens, find, blockIdx.x, hk, r);
  if (p.n < 2) return;
  const int rows = p.sg.n * wk.G - r * wk.rows;
  if (q0 >= rows) return;
  float m[N], l[N], v[N][4] = {};
#pragma unroll
  for (int u = 0; u < N; ++u) {
    m[u] = MUSE_NEG_INF;
    l[u] = 0.f;
  }
  for (int i = 0; i < p.n; ++i) {
    const size_t at = p.at(i, wk.rows) + q0;
    float2 ml[N];
    float4 x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {  // rows of the tile that the sequence does not have were written too, or are not used
      ml[u] = *reinterpret_cast<const float2*>(wk.pm + (at + u * STEP) * 2);
      x[u] = *reinterpret_cast<const float4*>(wk.po + (at + u * STEP) * D + tid % TPR * 4);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float mn = fmaxf(m[u], ml[u].x), ref = mn == MUSE_NEG_INF ? 0.f : mn, fa = exp2_(m[u] - ref), fb = exp2_(ml[u].x - ref);
      m[u] = mn;
      l[u] = fa * l[u] + fb * ml[u].y;
      const float y[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) v[u][j] = fmaf(fb, y[j], fa * v[u][j]);
    }
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int q = q0 + u * STEP, y = r * wk.rows + q, i = y / wk.G, h = hk * wk.G + y - i * wk.G;
    if (q >= rows) continue;
    const float inv = l[u] == 0.f ? 0.f : 1.f / l[u];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[u][j] *= inv;
    st4(O + d.o.at(p.sg.beg + i, h), tid % TPR * 4, v[u]);
    if (LSE && tid % TPR == 0) LSE[(size_t)h * d.T + p.sg.beg + i] = (m[u] + __builtin_amdgcn_logf(l[u])) * kLn2;
  }
}

// The division of a launch.  16 rows to a tile where the new tokens' rows fit (fp32: always), else 64, 32 at D = 128: a tile's keys are
// read and converted once for all its rows.  More rows are more registers than there are: beyond 64, tiles of 128 by way of LDS.
struct Plan {
  CacheWork w;
  int rt;
  size_t sums, bytes;  // of the partial sums, of the workspace
};
Plan plan_of(const CacheDims& d) {
  Plan p{};
  p.w.G = d.Hq / d.Hkv;
  p.w.sh = __builtin_ctz((unsigned)d.page);
  const long long rows = (long long)d.max_new * p.w.G;
  p.rt = rows <= 16 || d.dtype == MUSE_DTYPE_FP32 ? 1 : rows > 64 ? 8 : d.D == 64 ? 4 : 2;  // 8: k_cache_fwd_cols
  p.w.rows = 16 * p.rt;
  p.w.R = (int)((rows + p.w.rows - 1) / p.w.rows);
  if (p.w.R > 65535) p.w.R = 65535;
  // As many workgroups as the chip holds at once, no more: all have the same work, and one that waits for a place doubles the time (64
  // ragged contexts up to 8k, D = 128: 59 us with 512 workgroups, 69 with 768).  Not more than there are units.
  const long long each = ((long long)d.cols * d.page + UNIT - 1) / UNIT, heads = (long long)d.Hkv * p.w.R;
  const int per_cu = p.rt == 8 ? 2 : p.rt > 1 ? 1 : d.D == 64 && d.dtype == MUSE_DTYPE_BF16 ? 3 : 2;
  long long W = 256 * per_cu / heads;
  // Short contexts are not divided where the chip is full without that, or where there are few rows: the second launch would take longer than
  // a workgroup does (one context of 1000, 8 heads: 9.2 us for 6.4 + 4.7).
  p.w.whole = each <= 4 && (p.rt == 1 || d.S * heads >= 256 * per_cu);
  const long long most = p.w.whole ? d.S : d.S * each;
  if (W > most) W = most;
  p.w.W = (int)(W < 1 ? 1 : W);
  p.w.least = p.rt == 8 ? 2 : 1;  // a part of 128 rows costs as much as half a unit (8 pieces of up to 300: 56 + 15.7 us; 1: 56 + 17, 3: 64 + 14)
  p.w.used = rows < p.w.rows && p.rt == 1 ? (int)rows : p.w.rows;
  p.w.join = p.rt > 1 ? 32 : p.w.W > 8 * d.S ? 1 : 4;
  if (p.w.W > 1 && !p.w.whole) {
    const size_t slots = (size_t)heads * 2 * p.w.W * p.w.rows;
    p.sums = slots * d.D * 4;
    p.bytes = kTagBytes + p.sums + slots * 8;
  }
  return p;
}

}  // namespace

size_t muse_cache_fwd_ws_bytes(const CacheDims& d) { return plan_of(d).bytes; }

int muse_launch_cache_fwd(const CacheDims& d, const void* Q, const int32_t* cu, const int32_t* lens, const int32_t* table, const void* kc, const void* vc,
                          const float* ks, const float* vs, void* O, float* LSE, void* ws, hipStream_t st) {
  Plan p = plan_of(d);
  p.w.po = (float*)((char*)ws + kTagBytes);
  p.w.pm = (float*)((char*)ws + kTagBytes + p.sums);
  auto go = [&](auto* kernel, auto* join, auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    {
      MuseProf prof_("k_cache_fwd", st);
      hipLaunchKernelGGL(kernel, dim3(p.w.W, d.Hkv, p.w.R), dim3(256), 0, st, d, p.w, (const E*)Q, cu, lens, table, (const uint8_t*)kc, (const uint8_t*)vc, ks,
                         vs, (E*)O, LSE);
    }
    if (p.bytes) {
      MuseProf prof_("k_cache_join", st);
      hipLaunchKernelGGL(join, dim3(d.S < p.w.W ? d.S : p.w.W - 1, d.Hkv * ((p.w.used + p.w.join - 1) / p.w.join), p.w.R), dim3(256), 0, st, d, p.w, cu, lens, (E*)O, LSE);
    }
  };
  if (d.dtype == MUSE_DTYPE_BF16) {
    if (p.rt == 8) d.D == 64 ? go(k_cache_fwd_cols<64>, k_cache_join_rows<64>, (bf16_t*)0) : go(k_cache_fwd_cols<128>, k_cache_join_rows<128>, (bf16_t*)0);
    else if (d.D == 64) p.rt == 1 ? go(k_cache_fwd<bf16_t, 64, 1>, k_cache_join<bf16_t, 64>, (bf16_t*)0) : go(k_cache_fwd<bf16_t, 64, 4>, k_cache_join_rows<64>, (bf16_t*)0);
    else p.rt == 1 ? go(k_cache_fwd<bf16_t, 128, 1>, k_cache_join<bf16_t, 128>, (bf16_t*)0) : go(k_cache_fwd<bf16_t, 128, 2>, k_cache_join_rows<128>, (bf16_t*)0);
  } else {
    d.D == 64 ? go(k_cache_fwd<float, 64, 1>, k_cache_join<float, 64>, (float*)0) : go(k_cache_fwd<float, 128, 1>, k_cache_join<float, 128>, (float*)0);
  }
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
