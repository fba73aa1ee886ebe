// Host side of the 4-bit key/value cache's calls: checks, launch shapes, launches.
#pragma once
#include "kv4_kernels.h"

namespace {

constexpr int kKv4MaxRows = 1 << 26;     // pool rows: a row's byte offset within a head's codes stays inside 32 bits
constexpr int kKv4MaxHeads = 4096;

int kv4_check_cache(const char* who, const ll_kv4_cache* c, bool with_pool, Kv4Pool* out) {
  if (!c) return fail(LL_E_BAD_ARG, "%s: null cache", who);
  if (c->head_dim != 64 && c->head_dim != 128) return fail(LL_E_BAD_CONFIG, "%s: head_dim = %d, need 64 or 128", who, c->head_dim);
  if (c->n_kv_heads < 1 || c->n_kv_heads > kKv4MaxHeads)
    return fail(LL_E_BAD_CONFIG, "%s: n_kv_heads = %d outside [1, %d]", who, c->n_kv_heads, kKv4MaxHeads);
  if (c->page_tokens < 1 || c->n_pages < 1 || (int64_t)c->page_tokens * c->n_pages > kKv4MaxRows)
    return fail(LL_E_BAD_CONFIG, "%s: %d pages of %d positions, need one to %d positions", who, c->n_pages, c->page_tokens, kKv4MaxRows);
  Kv4Pool p{};
  p.base = static_cast<char*>(c->pool);
  p.kv_heads = c->n_kv_heads;
  p.page_tokens = c->page_tokens;
  p.pool_rows = c->page_tokens * c->n_pages;
  p.codes = align_up((size_t)c->n_kv_heads * p.pool_rows * (c->head_dim / 2));
  p.params = align_up((size_t)c->n_kv_heads * p.pool_rows * (c->head_dim / 8));
  while ((1 << p.shift) < c->page_tokens) ++p.shift;
  p.magic = (u32)(((1ull << (31 + p.shift)) + c->page_tokens - 1) / c->page_tokens);
  if (with_pool) {
    const size_t need = 2 * (p.codes + p.params);
    if (!c->pool) return fail(LL_E_BAD_ARG, "%s: null pool", who);
    if (c->pool_bytes < need) return fail(LL_E_WORKSPACE, "%s: pool has %zu bytes, %zu needed", who, c->pool_bytes, need);
    if (reinterpret_cast<uintptr_t>(c->pool) % kAlign) return fail(LL_E_WORKSPACE, "%s: pool must be %zu-byte aligned", who, kAlign);
  }
  if (out) *out = p;
  return LL_OK;
}

int kv4_check_rows(const char* who, const ll_kv4_rows* r, bool with_pointers, Kv4Rows* out) {
  if (!r) return fail(LL_E_BAD_ARG, "%s: null rows", who);
  if (r->n_seqs < 0 || r->n_rows < 0 || r->max_rows < 1 || r->table_stride < 1 || r->max_len < 0)
    return fail(LL_E_BAD_ARG, "%s: n_seqs = %d, n_rows = %d, max_rows = %d, table_stride = %d, max_len = %d", who, r->n_seqs,
                r->n_rows, r->max_rows, r->table_stride, r->max_len);
  if (!r->row_start && (int64_t)r->n_seqs * r->max_rows != r->n_rows && with_pointers)
    return fail(LL_E_BAD_ARG, "%s: without row_start n_rows = %d must be n_seqs * max_rows = %d * %d", who, r->n_rows, r->n_seqs, r->max_rows);
  if (r->n_seqs >= 1 << 24 || r->n_rows >= 1 << 24)      // threads of a launch along one dimension stay inside 32 bits
    return fail(LL_E_BAD_ARG, "%s: n_seqs = %d, n_rows = %d, at most %d", who, r->n_seqs, r->n_rows, (1 << 24) - 1);
  if (with_pointers && r->n_seqs > 0 && (!r->len || !r->page_table)) return fail(LL_E_BAD_ARG, "%s: null len or page_table", who);
  if (out) {
    *out = Kv4Rows{};
    out->row_start = r->row_start; out->len = r->len; out->table = r->page_table;
    out->n_seqs = r->n_seqs; out->n_rows = r->n_rows; out->table_stride = r->table_stride;
    out->max_rows = std::min(r->max_rows, std::max(r->n_rows, 1));      // no sequence has more rows than there are
  }
  return LL_OK;
}

int kv4_check_view(const char* who, const char* name, const ll_kv4_view* v, const ll_kv4_rows* r, int heads, int head_dim,
                   bool written, Kv4View* out) {
  if (!v || !v->data) return fail(LL_E_BAD_ARG, "%s: null %s", who, name);
  if (reinterpret_cast<uintptr_t>(v->data) % 2) return fail(LL_E_BAD_ARG, "%s: %s is not aligned to its elements", who, name);
  if (v->row_stride < 0 || v->head_stride < 0) return fail(LL_E_BAD_ARG, "%s: negative stride of %s", who, name);
  if (written) {      // no two elements of an output at one address: heads within a row, or rows within a head
    const int64_t row = v->row_stride, head = v->head_stride;
    const bool apart_heads = heads == 1 || head >= head_dim, apart_rows = r->n_rows <= 1 || row >= head_dim;
    const bool nested = heads == 1 || r->n_rows <= 1 || row >= (heads - 1) * head + head_dim ||
                        head >= (int64_t)(r->n_rows - 1) * row + head_dim;
    if (!apart_heads || !apart_rows || !nested)
      return fail(LL_E_BAD_ARG, "%s: strides %lld, %lld make elements of %s overlap", who, (long long)row, (long long)head, name);
  }
  out->data = v->data;
  out->row_stride = v->row_stride;
  out->head_stride = v->head_stride;
  out->wide = reinterpret_cast<uintptr_t>(v->data) % 16 == 0 && v->row_stride % 8 == 0 && v->head_stride % 8 == 0;
  return LL_OK;
}

int kv4_check_type(const char* who, int32_t dtype) {
  return dtype == LL_F16 || dtype == LL_BF16 ? LL_OK : fail(LL_E_BAD_ARG, "%s: dtype = %d, need LL_F16 or LL_BF16", who, dtype);
}

// go(type, head_dim) with the two as compile-time constants
template <int N> struct Kv4Dim { static constexpr int value = N; };
template <class F>
void kv4_dispatch(int32_t dtype, int head_dim, F&& go) {
  if (dtype == LL_F16) head_dim == 128 ? go(Kv4F16{}, Kv4Dim<128>{}) : go(Kv4F16{}, Kv4Dim<64>{});
  else head_dim == 128 ? go(Kv4Bf16{}, Kv4Dim<128>{}) : go(Kv4Bf16{}, Kv4Dim<64>{});
}

// Blocks of 8 rows where that leaves every CU with work of several workgroups; single rows, whose chain is shorter, else
constexpr int kKv4RowBlock = 8;
template <class F>
void kv4_row_blocks(const Kv4Pool& p, const Kv4Rows& r, int head_dim, F&& go) {
  const int units = p.kv_heads * (head_dim / 8), threads = std::min(256, (units + 63) / 64 * 64), parts = (units + threads - 1) / threads;
  if ((int64_t)r.n_rows * parts * 2 >= (int64_t)2 * kKv4RowBlock * num_cus())
    go(Kv4Dim<kKv4RowBlock>{}, dim3((r.n_rows + kKv4RowBlock - 1) / kKv4RowBlock, parts, 2), dim3(threads));
  else go(Kv4Dim<1>{}, dim3(r.n_rows, parts, 2), dim3(threads));
}

void kv4_launch_write(hipStream_t s, int32_t dtype, int head_dim, const Kv4Pool& p, const Kv4Rows& r, const Kv4View& k, const Kv4View& v) {
  kv4_dispatch(dtype, head_dim, [&](auto t, auto hd) {
    kv4_row_blocks(p, r, head_dim, [&](auto n, dim3 grid, dim3 threads) {
      hipLaunchKernelGGL((kv4_write_kernel<decltype(t), decltype(hd)::value, decltype(n)::value>), grid, threads, 0, s, p, r, k, v);
    });
  });
}

// How attention is cut into workgroups: blocks of query rows, and shares of the keys where that leaves CUs idle
struct Kv4Plan {
  bool many;                   // row blocks of 128, else of 16
  int row_blocks, splits;
  int64_t works;               // (row block, key head, sequence)
  size_t bytes;                // of workspace
};
#ifndef KV4_MANY_FROM
#define KV4_MANY_FROM 64
#endif
Kv4Plan kv4_plan(const Kv4Pool& p, const Kv4Rows& r, int max_len, int head_dim, int heads) {
  Kv4Plan a{};
  const int64_t rows = (int64_t)r.max_rows * (heads / p.kv_heads);
  a.many = rows > KV4_MANY_FROM;
  const int block = a.many ? KV4_MANY_ROWS : KV4_FEW_ROWS;
  a.row_blocks = (int)((rows + block - 1) / block);
  a.works = (int64_t)a.row_blocks * p.kv_heads * r.n_seqs;
  const int64_t most = (int64_t)r.table_stride * p.page_tokens;
  const int64_t len = max_len > 0 ? std::min<int64_t>(max_len, most) : most;
  const int64_t rounds = (len + KV4_TILE * KV4_WAVES - 1) / (KV4_TILE * KV4_WAVES);      // of the four waves over the keys
  const int64_t want = (2 * num_cus() + a.works - 1) / std::max<int64_t>(a.works, 1);
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, rounds / 4, 64}));       // (64: a wave's lanes, see the join)
  if (a.splits > 1) a.bytes = align_up((size_t)a.works * a.splits * block * (head_dim + 2) * sizeof(float));
  return a;
}

void kv4_launch_attention(hipStream_t s, int32_t dtype, int head_dim, const Kv4Pool& p, const Kv4Rows& r, int heads, float scale,
                          const Kv4View& q, const Kv4View* k, const Kv4View* v, const Kv4View& o, const Kv4Plan& a, float* part) {
  const bool fresh = k && r.max_rows == 1 && !a.many;
  if (k && !fresh) kv4_launch_write(s, dtype, head_dim, p, r, *k, *v);
  kv4_dispatch(dtype, head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    const dim3 grid((unsigned)(a.works * a.splits));
    const bool p16 = p.page_tokens % 16 == 0;
    if (a.many) {
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p, r, q, o, heads, scale, a.splits, a.row_blocks, part);
      };
      p16 ? go(kv4_attn_many_kernel<T, HD, true>) : go(kv4_attn_many_kernel<T, HD, false>);
      if (a.splits > 1)
        hipLaunchKernelGGL((kv4_join_kernel<T, HD, KV4_MANY_ROWS>), dim3((unsigned)a.works, KV4_MANY_ROWS / 4), dim3(256), 0, s, p, r, o,
                           heads, a.splits, a.row_blocks, part);
      return;
    }
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p, r, q, o, fresh ? *k : q, fresh ? *v : q, heads, scale, a.splits, a.row_blocks, part);
    };
    if (p16) fresh ? go(kv4_attn_few_kernel<T, HD, true, true>) : go(kv4_attn_few_kernel<T, HD, true, false>);
    else fresh ? go(kv4_attn_few_kernel<T, HD, false, true>) : go(kv4_attn_few_kernel<T, HD, false, false>);
    if (a.splits > 1)
      hipLaunchKernelGGL((kv4_join_kernel<T, HD, KV4_FEW_ROWS>), dim3((unsigned)a.works, KV4_FEW_ROWS / 4), dim3(256), 0, s, p, r, o, heads,
                         a.splits, a.row_blocks, part);
  });
}

}  // namespace

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
  kv4_dispatch(dtype, cache->head_dim, [&](auto t, auto hd) {
    kv4_row_blocks(p, r, cache->head_dim, [&](auto n, dim3 grid, dim3 threads) {
      hipLaunchKernelGGL((kv4_read_kernel<decltype(t), decltype(hd)::value, decltype(n)::value>), grid, threads, 0,
                         static_cast<hipStream_t>(hip_stream), p, r, kk, vv);
    });
  });
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
  if (r.n_seqs == 0 || r.n_rows == 0) return LL_OK;
  if ((rc = kv4_check_view(who, "q", q, rows, n_heads, cache->head_dim, false, &qq)) != LL_OK ||
      (rc = kv4_check_view(who, "out", out, rows, n_heads, cache->head_dim, true, &oo)) != LL_OK) return rc;
  if (k && ((rc = kv4_check_view(who, "k", k, rows, p.kv_heads, cache->head_dim, false, &kk)) != LL_OK ||
            (rc = kv4_check_view(who, "v", v, rows, p.kv_heads, cache->head_dim, false, &vv)) != LL_OK)) return rc;
  const Kv4Plan a = kv4_plan(p, r, rows->max_len, cache->head_dim, n_heads);
  if (a.works * a.splits >= 1 << 24)
    return fail(LL_E_BAD_ARG, "%s: %lld workgroups, a launch holds %d", who, (long long)(a.works * a.splits), (1 << 24) - 1);
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
