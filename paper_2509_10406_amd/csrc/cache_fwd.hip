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
#include <type_traits>

#include "packed.h"

namespace {

constexpr int UNIT = 256;
constexpr int JOIN = 8;  // rows of a workgroup of k_cache_join
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.f;  // the softmax reference follows the maximum in steps of more than 2^8

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

struct CacheWork {  // of one launch
  int W, R, rows;   // workgroups per (head, row tile), row tiles, rows of a tile
  int G, sh;        // query heads per key/value head, log2(page)
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

// All units of a row tile in a row: their number, the most new tokens of a sequence, and where the first unit of workgroup wg's share
// lies: its sequence and the units in front of that.  256 threads, each with a run of the sequences.
struct Found {
  int total, before, s, most;
};
struct FindLds {
  int sum[4], most[4], before, s;
};
// The first unit of workgroup w's share, and whose share a unit is in.  Where there are fewer units than workgroups, the first of these
// have one each: a share in the middle of a sequence is never empty.
__device__ __forceinline__ int share(int total, int w, int W) { return total <= W ? min(w, total) : (int)((long long)total * w / W); }
__device__ __forceinline__ int owner(int total, int unit, int W) { return total <= W ? unit : (int)((((long long)unit + 1) * W - 1) / total); }
__device__ __forceinline__ Found find_unit(const CacheDims& d, const CacheWork& w, const int32_t* cu, const int32_t* lens, int r, int tile_last, FindLds& lds, int wg) {
  const int tid = threadIdx.x, lane = tid % 64, per = (d.S + 255) / 256, s0 = tid * per, s1 = min(s0 + per, d.S);
  int mine = 0, most = 0;
  for (int s = s0; s < s1; ++s) {
    const Seg g = seg_of(d, w, cu, lens, s, r, tile_last);
    mine += g.units;
    most = max(most, g.n);
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto, o, 64);
    if (lane >= o) upto += x;
    most = max(most, __shfl_xor(most, o, 64));
  }
  __syncthreads();  // what an earlier call left has been read
  if (lane == 63) lds.sum[tid / 64] = upto;
  if (lane == 0) lds.most[tid / 64] = most;
  if (tid == 0) lds.s = lds.before = 0;  // of a share that begins behind the last unit: no place, but an index
  __syncthreads();
  Found f;
  f.total = __builtin_amdgcn_readfirstlane(lds.sum[0] + lds.sum[1] + lds.sum[2] + lds.sum[3]);
  f.most = __builtin_amdgcn_readfirstlane(max(max(lds.most[0], lds.most[1]), max(lds.most[2], lds.most[3])));
  for (int i = 0; i < tid / 64; ++i) upto += lds.sum[i];
  const int a = share(f.total, wg, w.W);
  if (upto - mine <= a && a < upto) {
    int b = upto - mine;
    for (int s = s0; s < s1; ++s) {
      const int u = seg_of(d, w, cu, lens, s, r, tile_last).units;
      if (a < b + u) {
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
  const int w = blockIdx.x, hk = blockIdx.y, r0 = blockIdx.z, G = wk.G, sh = wk.sh, inpage = d.page - 1;
  const float zscale = d.scale * kLog2e;

  for (int r = r0;; r += wk.R) {
    const int tile_last = last_token(wk, r);
    const Found f = find_unit(d, wk, cu, lens, r, tile_last, find, w);
    // More rows than the caller's bound said: whole sequences, one by one, so that nothing is left to be joined.
    const bool over = r >= wk.R;
    int a = share(f.total, w, wk.W), before = f.before;
    const int b = share(f.total, w + 1, wk.W);
    int s = over ? w : f.s;
    while (over ? s < d.S : a < b) {
      const Seg sg = seg_of(d, wk, cu, lens, s, r, tile_last);
      const int u0 = over ? 0 : a - before, u1 = over ? sg.units : min(sg.units, b - before);
      if (sg.units > 0) {
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
        const size_t slot = (((size_t)r0 * d.Hkv + hk) * 2 * wk.W + 2 * w + (u0 == 0)) * ROWS;
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
      }
      if (over) {
        s += wk.W;
      } else {
        before += sg.units;
        a = max(a, before);
        ++s;
      }
    }
    if ((r + wk.R) * ROWS >= f.most * G) break;
  }
}

// Joins the parts of the sequences that several workgroups share.  Workgroup x looks at the border between the shares x and x + 1: the first
// border inside a sequence has that sequence.  Bound by the latency of its reads, so a row's parts are asked for eight at a time and,
// where there are many, by the four waves together (a quarter of them each, joined in order through LDS); few parts: a wave per row.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_cache_join(CacheDims d, CacheWork wk, const int32_t* __restrict__ cu, const int32_t* __restrict__ lens,
                                                    T* __restrict__ O, float* __restrict__ LSE) {
  constexpr int DL = D / 64, FEW = 8;
  __shared__ FindLds find;
  __shared__ float part[4][D + 1];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, w = blockIdx.x + 1, hk = blockIdx.y / (wk.rows / JOIN),
            first = blockIdx.y % (wk.rows / JOIN) * JOIN, r = blockIdx.z;
  const int tile_last = last_token(wk, r);
  const Found f = find_unit(d, wk, cu, lens, r, tile_last, find, w);
  const int a = share(f.total, w, wk.W);
  if (a >= f.total || share(f.total, w - 1, wk.W) > f.before || a <= f.before) return;
  const Seg sg = seg_of(d, wk, cu, lens, f.s, r, tile_last);
  const int n = owner(f.total, f.before + sg.units - 1, wk.W) - (w - 1) + 1;  // parts: of the workgroups w - 1, w, ..
  const size_t base = ((size_t)r * d.Hkv + hk) * 2 * wk.W;
  auto slot = [&](int i) { return (base + (i == 0 ? 2 * (w - 1) + 1 : 2 * (w - 1 + i))) * wk.rows; };
  const bool together = n > FEW;
  const int rows = min(first + JOIN, sg.n * wk.G - r * wk.rows);
  for (int q = first + (together ? 0 : wave); q < rows; q += together ? 1 : 4) {
    const int i0 = together ? n * wave / 4 : 0, i1 = together ? n * (wave + 1) / 4 : n;
    float M = MUSE_NEG_INF;
    for (int i = lane; i < n; i += 64) M = fmaxf(M, wk.pm[(slot(i) + q) * 2]);
    M = wave_max(M);
    float l = 0.f, v[DL] = {};
    for (int j0 = i0; j0 < i1; j0 += 64) {
      float fw = 0.f;
      if (j0 + lane < i1) {
        const float2 p = *reinterpret_cast<const float2*>(wk.pm + (slot(j0 + lane) + q) * 2);
        fw = M == MUSE_NEG_INF ? 0.f : exp2_(p.x - M);
        l += fw * p.y;
      }
      const int m = min(64, i1 - j0);
      for (int k = 0; k < m; k += 8) {
        float x[8][DL];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float* p = wk.po + (slot(min(j0 + k + u, i1 - 1)) + q) * D + lane * DL;
#pragma unroll
          for (int j = 0; j < DL; ++j) x[u][j] = p[j];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float fu = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, fw), k + u));
#pragma unroll
          for (int j = 0; j < DL; ++j) v[j] = k + u < m ? fmaf(fu, x[u][j], v[j]) : v[j];
        }
      }
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
    const int y = r * wk.rows + q, i = y / wk.G, h = hk * wk.G + y - i * wk.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* to = O + d.o.at(sg.beg + i, h) + lane * DL;
#pragma unroll
    for (int j = 0; j < DL; ++j) Elem<T>::st(to, j, v[j] * inv);
    if (LSE && lane == 0) LSE[(size_t)h * d.T + sg.beg + i] = (M + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// The division of a launch.  16 rows to a tile where the new tokens' rows fit (fp32: always), else 64, 32 at D = 128: a tile's keys are
// read and converted once for all its rows.  More rows are more registers than there are.
struct Plan {
  CacheWork w;
  int rt;
  size_t po, bytes;
};
Plan plan_of(const CacheDims& d) {
  Plan p{};
  p.w.G = d.Hq / d.Hkv;
  p.w.sh = __builtin_ctz((unsigned)d.page);
  const long long rows = (long long)d.max_new * p.w.G;
  p.rt = rows <= 16 || d.dtype == MUSE_DTYPE_FP32 ? 1 : d.D == 64 ? 4 : 2;
  p.w.rows = 16 * p.rt;
  p.w.R = (int)((rows + p.w.rows - 1) / p.w.rows);
  if (p.w.R > 65535) p.w.R = 65535;
  // as many workgroups as stay on the chip at once; not more than there are units
  const long long units = (long long)d.S * (((long long)d.cols * d.page + UNIT - 1) / UNIT), heads = (long long)d.Hkv * p.w.R;
  long long W = (768 + heads - 1) / heads;
  if (W > units) W = units;
  p.w.W = (int)(W < 1 ? 1 : W);
  if (p.w.W > 1) {
    const size_t slots = (size_t)heads * 2 * p.w.W * p.w.rows;
    p.po = slots * d.D * 4;
    p.bytes = p.po + slots * 8;
  }
  return p;
}

}  // namespace

size_t muse_cache_fwd_ws_bytes(const CacheDims& d) { return plan_of(d).bytes; }

int muse_launch_cache_fwd(const CacheDims& d, const void* Q, const int32_t* cu, const int32_t* lens, const int32_t* table, const void* kc, const void* vc,
                          const float* ks, const float* vs, void* O, float* LSE, void* ws, hipStream_t st) {
  Plan p = plan_of(d);
  p.w.po = (float*)ws;
  p.w.pm = (float*)((char*)ws + p.po);
  auto go = [&](auto* kernel, auto* join, auto* t) {
    using E = std::remove_pointer_t<decltype(t)>;
    {
      MuseProf prof_("k_cache_fwd", st);
      hipLaunchKernelGGL(kernel, dim3(p.w.W, d.Hkv, p.w.R), dim3(256), 0, st, d, p.w, (const E*)Q, cu, lens, table, (const uint8_t*)kc, (const uint8_t*)vc, ks,
                         vs, (E*)O, LSE);
    }
    if (p.w.W > 1) {
      MuseProf prof_("k_cache_join", st);
      hipLaunchKernelGGL(join, dim3(p.w.W - 1, d.Hkv * (p.w.rows / JOIN), p.w.R), dim3(256), 0, st, d, p.w, cu, lens, (E*)O, LSE);
    }
  };
  if (d.dtype == MUSE_DTYPE_BF16) {
    if (d.D == 64) p.rt == 1 ? go(k_cache_fwd<bf16_t, 64, 1>, k_cache_join<bf16_t, 64>, (bf16_t*)0) : go(k_cache_fwd<bf16_t, 64, 4>, k_cache_join<bf16_t, 64>, (bf16_t*)0);
    else p.rt == 1 ? go(k_cache_fwd<bf16_t, 128, 1>, k_cache_join<bf16_t, 128>, (bf16_t*)0) : go(k_cache_fwd<bf16_t, 128, 2>, k_cache_join<bf16_t, 128>, (bf16_t*)0);
  } else {
    d.D == 64 ? go(k_cache_fwd<float, 64, 1>, k_cache_join<float, 64>, (float*)0) : go(k_cache_fwd<float, 128, 1>, k_cache_join<float, 128>, (float*)0);
  }
  MUSE_LAUNCH_CHECK();
  return MUSE_OK;
}
