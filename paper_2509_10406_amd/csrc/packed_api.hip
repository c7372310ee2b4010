// C entry points of the packed sequences and of the paged cache: checks on the host, then the launches.
#include <math.h>

#include <initializer_list>

#include "packed.h"

size_t muse_packed_fwd_ws_bytes(const PackedDims& d);
size_t muse_packed_bwd_ws_bytes(const PackedDims& d);
size_t muse_cache_fwd_ws_bytes(const CacheDims& d);
int muse_launch_packed_fwd(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, void* O, float* LSE, void* ws, hipStream_t st);
int muse_launch_packed_bwd(const PackedDims& d, const void* Q, const void* K, const void* V, const int32_t* cu, const void* O, const float* LSE,
                           const void* dO, void* dQ, void* dK, void* dV, void* ws, hipStream_t st);
int muse_launch_cache_append(const CacheDims& d, const void* K, const void* V, const int32_t* cu, const int32_t* lens, const int32_t* table,
                             void* kc, void* vc, float* ks, float* vs, hipStream_t st);
int muse_launch_cache_fwd(const CacheDims& d, const void* Q, const int32_t* cu, const int32_t* lens, const int32_t* table, const void* kc, const void* vc,
                          const float* ks, const float* vs, void* O, float* LSE, void* ws, hipStream_t st);

namespace {

constexpr int kMaxRows = 1 << 27;          // tokens; tile numbers and row indices then fit 32 bits
constexpr int64_t kMaxToken = 1 << 22;     // token stride: offsets inside a tile of rows are 32-bit
constexpr int64_t kMaxHead = 1ll << 40;

// a tensor of `heads` heads whose rows begin at 16-byte boundaries; out: no row twice
int make_rows(const muse_rows& r, int T, int heads, int D, int dtype, bool out, Rows* to) {
  const int64_t es = dtype == MUSE_DTYPE_BF16 ? 2 : 4;
  to->token = T > 1 ? r.token : 0;  // a stride along one element says nothing
  to->head = heads > 1 ? r.head : 0;
  if (to->token < 0 || to->head < 0 || to->token * es % 16 || to->head * es % 16) return MUSE_ERR_INVALID_ARG;
  if (to->token > kMaxToken || to->head > kMaxHead) return MUSE_ERR_UNSUPPORTED;
  if (out) {
    const int64_t t = to->token, h = to->head;
    const bool tokens_out = (T == 1 || t >= (heads - 1) * h + D) && (heads == 1 || h >= D);
    const bool heads_out = (heads == 1 || h >= (T - 1) * t + D) && (T == 1 || t >= D);
    if (!tokens_out && !heads_out) return MUSE_ERR_INVALID_ARG;
  }
  return MUSE_OK;
}

bool aligned16(std::initializer_list<const void*> p) {
  uintptr_t a = 0;
  for (const void* x : p) a |= (uintptr_t)x;
  return a % 16 == 0;
}

// what both kinds of params share
template <typename P>
int check_common(const P* p) {
  if (!p) return MUSE_ERR_INVALID_ARG;
  if (p->S < 1 || p->Hq < 1 || p->Hkv < 1 || p->T < 1 || p->Hq % p->Hkv || p->flags) return MUSE_ERR_INVALID_ARG;
  if (p->dtype != MUSE_DTYPE_FP32 && p->dtype != MUSE_DTYPE_BF16) return MUSE_ERR_INVALID_ARG;
  if (!(p->scale >= 0.f) || isinf(p->scale)) return MUSE_ERR_INVALID_ARG;
  if (p->D != 64 && p->D != 128) return MUSE_ERR_UNSUPPORTED;
  if (p->T > kMaxRows || p->S > (1 << 20) || p->Hq > 4096 || p->Hkv > 4096) return MUSE_ERR_UNSUPPORTED;
  return MUSE_OK;
}

int packed_dims(const muse_packed_params* p, bool bwd, PackedDims* d) {
  int rc = check_common(p);
  if (rc) return rc;
  if (p->grad_dtype != MUSE_DTYPE_FP32 && p->grad_dtype != p->dtype) return MUSE_ERR_INVALID_ARG;
  if (p->max_len < 0) return MUSE_ERR_INVALID_ARG;
  if (((long long)p->T / 64 + p->S + 8) * p->Hq > (1 << 23)) return MUSE_ERR_UNSUPPORTED;  // workgroups of a launch
  *d = PackedDims{p->S, p->Hq, p->Hkv, p->D, p->T, p->max_len > 0 && p->max_len < p->T ? p->max_len : p->T, p->dtype, p->grad_dtype,
                  p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->D), {}, {}, {}, {}, {}, {}, {}, {}};
  if ((rc = make_rows(p->q, p->T, p->Hq, p->D, p->dtype, false, &d->q)) || (rc = make_rows(p->k, p->T, p->Hkv, p->D, p->dtype, false, &d->k)) ||
      (rc = make_rows(p->v, p->T, p->Hkv, p->D, p->dtype, false, &d->v)) || (rc = make_rows(p->o, p->T, p->Hq, p->D, p->dtype, !bwd, &d->o)))
    return rc;
  if (!bwd) return MUSE_OK;
  if ((rc = make_rows(p->dout, p->T, p->Hq, p->D, p->dtype, false, &d->g)) || (rc = make_rows(p->dq, p->T, p->Hq, p->D, p->grad_dtype, true, &d->dq)) ||
      (rc = make_rows(p->dk, p->T, p->Hkv, p->D, p->grad_dtype, true, &d->dk)) || (rc = make_rows(p->dv, p->T, p->Hkv, p->D, p->grad_dtype, true, &d->dv)))
    return rc;
  return MUSE_OK;
}

int cache_dims(const muse_cache_params* p, CacheDims* d) {
  const int rc = check_common(p);
  if (rc) return rc;
  if (p->pages < 1 || p->table_cols < 1 || p->max_new < 0) return MUSE_ERR_INVALID_ARG;
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128) return MUSE_ERR_UNSUPPORTED;
  // Positions, rows of a group and units of work are int32; the attention rounds positions up to a unit of 256 keys and looks at
  // the table for up to two units further on, which has to stay within 31 bits too.
  if ((long long)p->table_cols * p->page > 0x80000000ll - 1024 || (long long)p->T * (p->Hq / p->Hkv) > (1 << 29) ||
      (long long)p->S * (((long long)p->table_cols * p->page + 255) / 256 + 1) > 0x7fffffffll)
    return MUSE_ERR_UNSUPPORTED;
  *d = CacheDims{p->S, p->Hq, p->Hkv, p->D, p->T, p->pages, p->page, p->table_cols, p->max_new > 0 && p->max_new < p->T ? p->max_new : p->T,
                 p->dtype, p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)p->D), {}, {}, {}, {}};
  return MUSE_OK;
}

}  // namespace

extern "C" {

int muse_packed_workspace_bytes(const muse_packed_params* p, int which, size_t* bytes) {
  if (!bytes || (which != MUSE_WS_EXACT_FWD && which != MUSE_WS_EXACT_BWD)) return MUSE_ERR_INVALID_ARG;
  PackedDims d;
  const int rc = packed_dims(p, which == MUSE_WS_EXACT_BWD, &d);
  if (rc) return rc;
  *bytes = which == MUSE_WS_EXACT_BWD ? muse_packed_bwd_ws_bytes(d) : muse_packed_fwd_ws_bytes(d);
  return MUSE_OK;
}

int exact_attn_packed_fwd(const muse_packed_params* p, const void* Q, const void* K, const void* V, const int32_t* cu_seqlens, void* O,
                          float* LSE, void* ws, size_t ws_bytes, void* stream) {
  PackedDims d;
  const int rc = packed_dims(p, false, &d);
  if (rc) return rc;
  if (!Q || !K || !V || !cu_seqlens || !O || !LSE || !aligned16({Q, K, V, O})) return MUSE_ERR_INVALID_ARG;
  const size_t need = muse_packed_fwd_ws_bytes(d);
  if (need && (!ws || (uintptr_t)ws % 256)) return MUSE_ERR_INVALID_ARG;
  if (ws_bytes < need) return MUSE_ERR_WORKSPACE_TOO_SMALL;
  return muse_launch_packed_fwd(d, Q, K, V, cu_seqlens, O, LSE, ws, (hipStream_t)stream);
}

int exact_attn_packed_bwd(const muse_packed_params* p, const void* Q, const void* K, const void* V, const int32_t* cu_seqlens, const void* O,
                          const float* LSE, const void* dO, void* dQ, void* dK, void* dV, void* ws, size_t ws_bytes, void* stream) {
  PackedDims d;
  const int rc = packed_dims(p, true, &d);
  if (rc) return rc;
  if (!Q || !K || !V || !cu_seqlens || !O || !LSE || !dO || !dQ || !dK || !dV || !ws || !aligned16({Q, K, V, O, dO, dQ, dK, dV})) return MUSE_ERR_INVALID_ARG;
  if ((uintptr_t)ws % 256) return MUSE_ERR_INVALID_ARG;
  if (ws_bytes < muse_packed_bwd_ws_bytes(d)) return MUSE_ERR_WORKSPACE_TOO_SMALL;
  return muse_launch_packed_bwd(d, Q, K, V, cu_seqlens, O, LSE, dO, dQ, dK, dV, ws, (hipStream_t)stream);
}

int exact_attn_cache_append(const muse_cache_params* p, const void* K, const void* V, const int32_t* cu_new, const int32_t* kv_lens,
                            const int32_t* table, void* k_cache, void* v_cache, float* k_scale, float* v_scale, void* stream) {
  CacheDims d;
  int rc = cache_dims(p, &d);
  if (rc) return rc;
  if ((rc = make_rows(p->k, p->T, p->Hkv, p->D, p->dtype, false, &d.k)) || (rc = make_rows(p->v, p->T, p->Hkv, p->D, p->dtype, false, &d.v))) return rc;
  if (!K || !V || !kv_lens || !table || !k_cache || !v_cache || !k_scale || !v_scale || !aligned16({K, V, k_cache, v_cache})) return MUSE_ERR_INVALID_ARG;
  if (!cu_new) {  // one new token per sequence, whatever the caller's bound says
    if (p->T != p->S) return MUSE_ERR_INVALID_ARG;
    d.max_new = 1;
  }
  return muse_launch_cache_append(d, K, V, cu_new, kv_lens, table, k_cache, v_cache, k_scale, v_scale, (hipStream_t)stream);
}

int muse_cache_workspace_bytes(const muse_cache_params* p, size_t* bytes) {
  if (!bytes) return MUSE_ERR_INVALID_ARG;
  CacheDims d;
  const int rc = cache_dims(p, &d);
  if (rc) return rc;
  *bytes = muse_cache_fwd_ws_bytes(d);
  if (p->T == p->S) {  // a call without cu_new takes the plan of single tokens
    d.max_new = 1;
    const size_t single = muse_cache_fwd_ws_bytes(d);
    if (single > *bytes) *bytes = single;
  }
  return MUSE_OK;
}

int exact_attn_cache_fwd(const muse_cache_params* p, const void* Q, const int32_t* cu_new, const int32_t* kv_lens, const int32_t* table,
                         const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, void* O, float* LSE, void* ws,
                         size_t ws_bytes, void* stream) {
  CacheDims d;
  int rc = cache_dims(p, &d);
  if (rc) return rc;
  if ((rc = make_rows(p->q, p->T, p->Hq, p->D, p->dtype, false, &d.q)) || (rc = make_rows(p->o, p->T, p->Hq, p->D, p->dtype, true, &d.o))) return rc;
  if (!Q || !kv_lens || !table || !k_cache || !v_cache || !k_scale || !v_scale || !O || !aligned16({Q, k_cache, v_cache, O})) return MUSE_ERR_INVALID_ARG;
  if (!cu_new) {  // one new token per sequence, whatever the caller's bound says
    if (p->T != p->S) return MUSE_ERR_INVALID_ARG;
    d.max_new = 1;
  }
  const size_t need = muse_cache_fwd_ws_bytes(d);
  if (need && (!ws || (uintptr_t)ws % 256)) return MUSE_ERR_INVALID_ARG;
  if (ws_bytes < need) return MUSE_ERR_WORKSPACE_TOO_SMALL;
  return muse_launch_cache_fwd(d, Q, cu_new, kv_lens, table, k_cache, v_cache, k_scale, v_scale, O, LSE, ws, (hipStream_t)stream);
}

}  // extern "C"
