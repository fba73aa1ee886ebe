// C ABI of the 4-bit key/value cache (see include/ll.h), the last part of ll_runtime.hip
#pragma once
#include "kv4_host.h"

extern "C" {

size_t ll_kv4_pool_bytes(const ll_kv4_cache* cache) {
  Kv4Pool p;
  return kv4_check_cache("ll_kv4_pool_bytes", cache, false, &p) == LL_OK ? 2 * (p.codes + p.params) : 0;
}

int ll_kv4_write(const ll_kv4_cache* cache, const ll_kv4_rows* rows, int32_t dtype, const ll_kv4_view* k, const ll_kv4_view* v,
                 void* hip_stream) {
  const char* who = "ll_kv4_write";
  Kv4Pool p;
  Kv4Rows r;
  Kv4View kk, vv;
  int rc;
  if ((rc = kv4_check_cache(who, cache, true, &p)) != LL_OK || (rc = kv4_check_rows(who, rows, true, &r)) != LL_OK ||
      (rc = kv4_check_type(who, dtype)) != LL_OK) return rc;
  if (r.n_seqs == 0 || r.n_rows == 0) return LL_OK;
  if ((rc = kv4_check_view(who, "k", k, rows, p.kv_heads, cache->head_dim, false, &kk)) != LL_OK ||
      (rc = kv4_check_view(who, "v", v, rows, p.kv_heads, cache->head_dim, false, &vv)) != LL_OK) return rc;
  kv4_launch_write(static_cast<hipStream_t>(hip_stream), dtype, cache->head_dim, p, r, kk, vv);
  HIPCHK(hipGetLastError());
  return LL_OK;
}

int ll_kv4_read(const ll_kv4_cache* cache, const ll_kv4_rows* rows, int32_t dtype, const ll_kv4_view* k, const ll_kv4_view* v,
                void* hip_stream) {
  const char* who = "ll_kv4_read";
  Kv4Pool p;
  Kv4Rows r;
  Kv4View kk, vv;
  int rc;
  if ((rc = kv4_check_cache(who, cache, true, &p)) != LL_OK || (rc = kv4_check_rows(who, rows, true, &r)) != LL_OK ||
      (rc = kv4_check_type(who, dtype)) != LL_OK) return rc;
  if (r.n_seqs == 0 || r.n_rows == 0) return LL_OK;
  if ((rc = kv4_check_view(who, "k", k, rows, p.kv_heads, cache->head_dim, true, &kk)) != LL_OK ||
      (rc = kv4_check_view(who, "v", v, rows, p.kv_heads, cache->head_dim, true, &vv)) != LL_OK) return rc;
  kv4_launch_read(static_cast<hipStream_t>(hip_stream), dtype, cache->head_dim, p, r, kk, vv);
  HIPCHK(hipGetLastError());
  return LL_OK;
}

size_t ll_kv4_attention_workspace_bytes(const ll_kv4_cache* cache, const ll_kv4_rows* rows, int32_t n_heads) {
  Kv4Pool p;
  Kv4Rows r;
  if (kv4_check_cache("ll_kv4_attention_workspace_bytes", cache, false, &p) != LL_OK ||
      kv4_check_rows("ll_kv4_attention_workspace_bytes", rows, false, &r) != LL_OK || n_heads < 1 || n_heads % p.kv_heads) return 0;
  return kv4_plan(p, r, rows->max_len, cache->head_dim, n_heads).bytes;
}

int ll_kv4_attention(const ll_kv4_cache* cache, const ll_kv4_rows* rows, int32_t dtype, int32_t n_heads, float scale,
                     const ll_kv4_view* q, const ll_kv4_view* k, const ll_kv4_view* v, const ll_kv4_view* out, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
  const char* who = "ll_kv4_attention";
  Kv4Pool p;
  Kv4Rows r;
  Kv4View qq, kk, vv, oo;
  int rc;
  if ((rc = kv4_check_cache(who, cache, true, &p)) != LL_OK || (rc = kv4_check_rows(who, rows, true, &r)) != LL_OK ||
      (rc = kv4_check_type(who, dtype)) != LL_OK) return rc;
  if (n_heads < 1 || n_heads > kKv4MaxHeads || n_heads % p.kv_heads)
    return fail(LL_E_BAD_CONFIG, "%s: n_heads = %d, need a multiple of n_kv_heads = %d up to %d", who, n_heads, p.kv_heads, kKv4MaxHeads);
  if (!(scale >= 0.f) || !(scale < INFINITY)) return fail(LL_E_BAD_ARG, "%s: scale = %g, need a finite value >= 0", who, (double)scale);
  if (!k != !v) return fail(LL_E_BAD_ARG, "%s: k and v come together", who);
  if ((int64_t)r.table_stride * p.page_tokens > kKv4MaxPositions)
    return fail(LL_E_BAD_ARG, "%s: a page table of %d pages of %d positions, at most %d positions", who, r.table_stride, p.page_tokens,
                kKv4MaxPositions);
  if ((int64_t)r.max_rows * (n_heads / p.kv_heads) > kKv4MaxPositions)
    return fail(LL_E_BAD_ARG, "%s: %d rows of %d heads a key head, at most %d", who, r.max_rows, n_heads / p.kv_heads, kKv4MaxPositions);
  if (r.n_seqs == 0 || r.n_rows == 0) return LL_OK;
  if ((rc = kv4_check_view(who, "q", q, rows, n_heads, cache->head_dim, false, &qq)) != LL_OK ||
      (rc = kv4_check_view(who, "out", out, rows, n_heads, cache->head_dim, true, &oo)) != LL_OK) return rc;
  if (k && ((rc = kv4_check_view(who, "k", k, rows, p.kv_heads, cache->head_dim, false, &kk)) != LL_OK ||
            (rc = kv4_check_view(who, "v", v, rows, p.kv_heads, cache->head_dim, false, &vv)) != LL_OK)) return rc;
  const Kv4Plan a = kv4_plan(p, r, rows->max_len, cache->head_dim, n_heads);
  const int most = a.many ? 1 << 23 : 1 << 24;      // of 512 or 256 threads, which stay inside 32 bits
  if (a.works * a.splits >= most)
    return fail(LL_E_BAD_ARG, "%s: %lld workgroups, a launch holds %d", who, (long long)(a.works * a.splits), most - 1);
  if (workspace_bytes < a.bytes || (a.bytes && !workspace))
    return fail(LL_E_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, a.bytes);
  if (a.bytes && reinterpret_cast<uintptr_t>(workspace) % kAlign)
    return fail(LL_E_WORKSPACE, "%s: workspace must be %zu-byte aligned", who, kAlign);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (scale == 0.f) scale = 1.0f / sqrtf((float)cache->head_dim);
  kv4_launch_attention(s, dtype, cache->head_dim, p, r, n_heads, scale, qq, k ? &kk : nullptr, k ? &vv : nullptr, oo, a,
                       static_cast<float*>(workspace));
  HIPCHK(hipGetLastError());
  return LL_OK;
}

}  // extern "C"
