// Host side of the 4-bit key/value cache: checks, launch shapes, launches.  Part of ll_runtime.hip, in front of what uses it.
#pragma once
#include "kv4_kernels.h"

namespace {

constexpr int kKv4MaxRows = 1 << 26;     // pool rows: a row's byte offset within a head's codes stays inside 32 bits
constexpr int kKv4MaxHeads = 4096;
constexpr int kKv4MaxPositions = 1 << 30;      // of a page table that attention reads; query rows of a key head: positions and rows a
                                               // few tiles further on stay inside 32 bits

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
  if ((reinterpret_cast<uintptr_t>(r->row_start) | reinterpret_cast<uintptr_t>(r->len) | reinterpret_cast<uintptr_t>(r->page_table)) % 4)
    return fail(LL_E_BAD_ARG, "%s: row_start, len or page_table is not aligned to its elements", who);
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
  *out = Kv4View{};
  out->data = v->data;
  out->row_stride = v->row_stride;
  out->head_stride = v->head_stride;
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

// Blocks of 8 rows where they still give every CU two workgroups: reading 32 x 1 .. 1000 rows of 32 heads takes 77 us, row by
// row 134; writing 4 x 1 .. 8190 rows of 8 heads and reading them 61, row by row 67.  Single rows, whose chain is shorter, else:
// writing 16 rows 7.6 us, in blocks 15.3; 500 rows of 32 heads and reading them 13.8, 18.4.
constexpr int kKv4RowBlock = 8;
template <class F>
void kv4_row_blocks(const Kv4Pool& p, const Kv4Rows& r, int head_dim, int layers, F&& go) {
  const int units = p.kv_heads * (head_dim / 8), threads = std::min(256, (units + 63) / 64 * 64), parts = (units + threads - 1) / threads;
  if ((int64_t)r.n_rows * parts * 2 * layers >= (int64_t)2 * kKv4RowBlock * num_cus())
    go(Kv4Dim<kKv4RowBlock>{}, dim3((r.n_rows + kKv4RowBlock - 1) / kKv4RowBlock, parts, 2 * layers), dim3(threads));
  else go(Kv4Dim<1>{}, dim3(r.n_rows, parts, 2 * layers), dim3(threads));
}

void kv4_launch_write(hipStream_t s, int32_t dtype, int head_dim, const Kv4Pool& p, const Kv4Rows& r, const Kv4View& k, const Kv4View& v,
                      int layers = 1) {
  kv4_dispatch(dtype, head_dim, [&](auto t, auto hd) {
    kv4_row_blocks(p, r, head_dim, layers, [&](auto n, dim3 grid, dim3 threads) {
      hipLaunchKernelGGL((kv4_write_kernel<decltype(t), decltype(hd)::value, decltype(n)::value>), grid, threads, 0, s, p, r, k, v);
    });
  });
}

void kv4_launch_read(hipStream_t s, int32_t dtype, int head_dim, const Kv4Pool& p, const Kv4Rows& r, const Kv4View& k, const Kv4View& v) {
  kv4_dispatch(dtype, head_dim, [&](auto t, auto hd) {
    kv4_row_blocks(p, r, head_dim, 1, [&](auto n, dim3 grid, dim3 threads) {
      hipLaunchKernelGGL((kv4_read_kernel<decltype(t), decltype(hd)::value, decltype(n)::value>), grid, threads, 0, s, p, r, k, v);
    });
  });
}

// How attention is cut into workgroups: blocks of query rows, and shares of the keys where that leaves CUs idle
struct Kv4Plan {
  bool many;                   // row blocks of KV4_MANY_ROWS, else of KV4_FEW_ROWS
  int row_blocks, splits;
  int64_t works;               // (row block, key head, sequence)
  size_t bytes;                // of workspace
};
Kv4Plan kv4_plan(const Kv4Pool& p, const Kv4Rows& r, int max_len, int head_dim, int heads) {
  Kv4Plan a{};
  const int64_t rows = (int64_t)r.max_rows * (heads / p.kv_heads);
  const int64_t most = (int64_t)r.table_stride * p.page_tokens;
  const int64_t len = max_len > 0 ? std::min<int64_t>(max_len, most) : most;
  const int64_t rounds = (len + KV4_TILE * KV4_WAVES - 1) / (KV4_TILE * KV4_WAVES);      // of the four waves over the keys
  const int64_t shares = std::max<int64_t>(1, std::min<int64_t>(rounds / 4, 64));        // at most (64: a wave's lanes, see the join)
  // Blocks of 256 rows where they, times the shares, leave no CU idle: there a workgroup turns codes into operands once for 16
  // times as many rows.  1024 rows of 32 heads behind 7169 positions: 204 us, in blocks of 16 rows 391; six sequences of up to
  // 700 rows of 64 heads: 121, 164.  One sequence of 500 rows and 32 heads is 64 such blocks: 34 us, in blocks of 16 rows 22.
  const int64_t many = (rows + KV4_MANY_ROWS - 1) / KV4_MANY_ROWS * p.kv_heads * r.n_seqs;
  a.many = rows > 64 && many * shares >= num_cus();
  const int block = a.many ? KV4_MANY_ROWS : KV4_FEW_ROWS;
  a.row_blocks = (int)((rows + block - 1) / block);
  a.works = (int64_t)a.row_blocks * p.kv_heads * r.n_seqs;
  // Two workgroups a CU of the kernels for few rows (of which three or four fit), one of the other, which fills a CU's LDS.
  // 4, 6, 9 and 16 times as many shares for few rows gained nothing: what a workgroup saves comes back in the join.
  const int64_t want = ((a.many ? 1 : 2) * num_cus() + a.works - 1) / std::max<int64_t>(a.works, 1);
  a.splits = (int)std::min<int64_t>(want, shares);
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
        hipLaunchKernelGGL(kernel, grid, dim3(KV4_MANY_WAVES * 64), 0, s, p, r, q, o, heads, scale, a.splits, a.row_blocks, part);
      };
      p16 ? go(kv4_attn_many_kernel<T, HD, true>) : go(kv4_attn_many_kernel<T, HD, false>);
      if (a.splits > 1)
        hipLaunchKernelGGL((kv4_join_kernel<T, HD, KV4_MANY_ROWS>), dim3((unsigned)a.works, KV4_MANY_ROWS / 4 / KV4_JOIN_ROWS(KV4_MANY_ROWS)), dim3(256), 0, s, p, r, o,
                           heads, a.splits, a.row_blocks, part);
      return;
    }
    auto single = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p, r, q, o, fresh ? *k : q, fresh ? *v : q, heads, scale, a.splits, part);
    };
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p, r, q, o, fresh ? *k : q, fresh ? *v : q, heads, scale, a.splits, a.row_blocks, part);
    };
    // one query row a key head: 32 sequences of 1500 .. 2500 positions 75 us, by the kernel for up to 16 rows 93; 16 of 10 .. 560
    // 17, 21
    if (r.max_rows == 1 && heads == p.kv_heads) {
      if (p16) fresh ? single(kv4_attn_one_kernel<T, HD, true, true>) : single(kv4_attn_one_kernel<T, HD, true, false>);
      else fresh ? single(kv4_attn_one_kernel<T, HD, false, true>) : single(kv4_attn_one_kernel<T, HD, false, false>);
    } else if (p16) fresh ? go(kv4_attn_few_kernel<T, HD, true, true>) : go(kv4_attn_few_kernel<T, HD, true, false>);
    else fresh ? go(kv4_attn_few_kernel<T, HD, false, true>) : go(kv4_attn_few_kernel<T, HD, false, false>);
    if (a.splits > 1)
      hipLaunchKernelGGL((kv4_join_kernel<T, HD, KV4_FEW_ROWS>), dim3((unsigned)a.works, KV4_FEW_ROWS / 4 / KV4_JOIN_ROWS(KV4_FEW_ROWS)), dim3(256), 0, s, p, r, o, heads,
                         a.splits, a.row_blocks, part);
  });
}

}  // namespace
