// A key/value cache held in 4 bits: quantising rows into it, reading them back, and attention over it.
//
// A group is 32 consecutive elements of one head's key or value row and is held as 32 codes c in 0 .. 15 and two binary16
// numbers:  value = mid + s (c - 8).  s is the smallest binary16 number of at most 8 significant bits with 15 s >= max - min,
// mid is min + 8 s rounded to binary16, and c - 8 the element's distance from mid in steps of s, rounded to the nearest (half
// to even) and cut to -8 .. 7.  An element is then off by at most s / 2 and mid's own rounding.  8 bits for s, because
// s (c - 8) then has at most 11 and is a binary16 number itself: no kernel that feeds it to the matrix instructions rounds.
// A group with a NaN, an infinity or a span above 15 * 8160 (8 s would leave binary16) reads as NaN.
//
// Pool of one layer: [K codes][V codes][K parameters][V parameters], every region padded to 256 bytes; codes are
// [kv head][pool row][head_dim / 2] bytes, element 2 j in the low half of byte j; parameters are [kv head][pool row]
// [head_dim / 32] pairs (s, mid).  5 bits an element.  A page is page_tokens consecutive pool rows; page_table[b][i] is the
// first pool row of sequence b's page i.  An entry whose page does not lie within the pool is a page that is not there: its
// positions are not written, read as zeros and attended by nobody.
#pragma once
#include "ll_device.h"

#define KV4_GROUP 32
#define KV4_MAX_STEP 8160.0f     // largest number of 8 significant bits with 8 s inside binary16

typedef uint16_t u16;
typedef uint32_t u32;
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef u16 u16x8 __attribute__((ext_vector_type(8)));

// One layer's pool
struct Kv4Pool {
  char* base;
  size_t codes, params;      // bytes of a codes region and of a parameters region, padding included
  int kv_heads, pool_rows, page_tokens;
  u32 magic;                 // position / page_tokens = (2 u magic) >> 32 >> shift for 0 <= u < 2^31
  int shift;
};
// Rows of a call: sequence b has rows row_start[b] .. row_start[b + 1] - 1 (without row_start: max_rows each), the last
// of them at position len[b] - 1
struct Kv4Rows {
  const int *row_start, *len, *table;
  const int* active;         // optional: 0 = the sequence has no positions
  int len_add;               // added to len[b]
  int n_seqs, max_rows, n_rows, table_stride;
};
// [row][head][head_dim], the last dimension contiguous; strides in elements
struct Kv4View {
  void* data;
  long row_stride, head_stride;
  int wide;                  // rows of every head can be read and written 16 bytes at a time
};

template <int HD>
__device__ __forceinline__ char* kv4_codes(const Kv4Pool& p, int which, int head) {
  return p.base + which * p.codes + (size_t)head * p.pool_rows * (HD / 2);
}
template <int HD>
__device__ __forceinline__ char* kv4_params(const Kv4Pool& p, int which, int head) {
  return p.base + 2 * p.codes + which * p.params + (size_t)head * p.pool_rows * (HD / 8);
}

// Rows of sequence b that this call has: the first one's index, how many the sequence has (of which at most max_rows are
// looked at), and the sequence's length.  Bounds come from device memory: they are cut to what the tensors hold.
struct Kv4Seq {
  int first, rows, len;
};
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Rows& r, int b) {
  Kv4Seq s;
  s.first = b * r.max_rows;
  s.rows = r.max_rows;
  if (r.row_start) {
    const int from = r.row_start[b], to = r.row_start[b + 1];
    s.first = min(max(from, 0), r.n_rows);
    s.rows = min(max(to, s.first), r.n_rows) - s.first;
  }
  s.len = max(r.len[b], 0) + r.len_add;
  if (r.active && !r.active[b]) s.len = 0;
  return s;
}

// Sequence of row i, or -1: all 64 lanes of a wave look at a sequence each
__device__ __forceinline__ int kv4_find(const Kv4Rows& r, int i) {
  if (!r.row_start) return i / r.max_rows;
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < r.n_seqs; b0 += 64) {
    const int b = min(b0 + lane, r.n_seqs - 1);
    const unsigned long long hit = __ballot(i >= r.row_start[b] && i < r.row_start[b + 1]);
    if (hit) return b0 + __ffsll(hit) - 1;
  }
  return -1;
}

// Pool row of position u >= 0 of the sequence with this page-table row; -1 where there is none
__device__ __forceinline__ int kv4_row(const Kv4Pool& p, const int* table, int table_stride, int u) {
  const int page = (int)(__umulhi((u32)u << 1, p.magic) >> p.shift);
  if (page >= table_stride) return -1;
  const int at = table[page];
  return (u32)at <= (u32)(p.pool_rows - p.page_tokens) ? at + (u - page * p.page_tokens) : -1;
}

// ---- element types at the borders: binary16 and bfloat16 ----
struct Kv4F16 {
  static __device__ __forceinline__ float load(u16 v) { return (float)__builtin_bit_cast(half_t, v); }
  static __device__ __forceinline__ u16 store(float v) { return __builtin_bit_cast(u16, (half_t)v); }
};
struct Kv4Bf16 {
  static __device__ __forceinline__ float load(u16 v) { return __builtin_bit_cast(float, (u32)v << 16); }
  static __device__ __forceinline__ u16 store(float v) {      // to the nearest, half to even; NaN stays one
    const u32 b = __builtin_bit_cast(u32, v);
    return (u16)(v != v ? (b >> 16) | 0x40 : (b + 0x7fff + ((b >> 16) & 1)) >> 16);
  }
};
__device__ __forceinline__ u16x8 kv4_load8(const Kv4View& t, int row, int head, int e) {
  const u16* p = (const u16*)t.data + row * t.row_stride + head * t.head_stride + e;
  if (t.wide) return *as_global(reinterpret_cast<const u16x8*>(p));
  u16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = *as_global(p + i);
  return v;
}
__device__ __forceinline__ void kv4_store8(const Kv4View& t, int row, int head, int e, u16x8 v) {
  u16* p = (u16*)t.data + row * t.row_stride + head * t.head_stride + e;
  if (t.wide) {
    *as_global(reinterpret_cast<u16x8*>(p)) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) *as_global(p + i) = v[i];
  }
}

// A number that is a binary16 number of at most 8 significant bits: rounded up to the next one (x >= 0)
__device__ __forceinline__ float kv4_step_up(float x) {
  if (x < 0x1p-16f) return ceilf(x * 0x1p24f) * 0x1p-24f;          // binary16's smallest step
  return __builtin_bit_cast(float, (__builtin_bit_cast(u32, x) + 0xffff) & 0xffff0000u);
}
__device__ __forceinline__ float kv4_step_next(float s, int dir) {   // s > 0: its neighbour of that kind
  if (s < 0x1p-16f || (s == 0x1p-16f && dir < 0)) return s + dir * 0x1p-24f;
  return __builtin_bit_cast(float, __builtin_bit_cast(u32, s) + dir * 0x10000);
}

template <int CTRL>
__device__ __forceinline__ float kv4_quad_min(float v) { return fminf(v, dpp_mov<CTRL>(v)); }
template <int CTRL>
__device__ __forceinline__ float kv4_quad_max(float v) { return fmaxf(v, dpp_mov<CTRL>(v)); }

// Four neighbouring lanes hold a group, 8 elements each: the lane's 8 codes (element i in bits 4 i ..) and the group's
// parameters (s in the low half).  What a float cannot decide is decided in 64 bits: whether 15 s reaches the span, and the
// code of an element closer than the float's error to the border between two (some 1e-5 of them).
__device__ __forceinline__ u32 kv4_quantise(const float (&x)[8], u32& param) {
  float lo = x[0], hi = x[0];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    bad |= !(fabsf(x[i]) < INFINITY);
  }
  lo = kv4_quad_min<0x4E>(kv4_quad_min<0xB1>(lo));
  hi = kv4_quad_max<0x4E>(kv4_quad_max<0xB1>(hi));
  const double span = (double)hi - (double)lo;
  float s = 0.f;
  if (hi > lo) {
    s = kv4_step_up((hi - lo) * (1.0f / 15.0f));
    if (15.0 * (double)s < span) s = kv4_step_next(s, 1);
    const float below = kv4_step_next(s, -1);
    if (15.0 * (double)below >= span) s = below;
  }
  const half_t mid_h = (half_t)(float)((double)lo + 8.0 * (double)s);
  float mid = (float)mid_h;
  float flag = bad || !(s <= KV4_MAX_STEP) || !(fabsf(mid) < INFINITY) ? 1.f : 0.f;
  flag = kv4_quad_max<0x4E>(kv4_quad_max<0xB1>(flag));
  if (flag != 0.f) {
    param = 0x7e007e00u;
    return 0;
  }
  param = (u32)__builtin_bit_cast(u16, (half_t)s) | (u32)__builtin_bit_cast(u16, mid_h) << 16;
  const float inv = s > 0.f ? 1.0f / s : 0.f;
  int c[8];
  bool near = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = (x[i] - mid) * inv, n = rintf(y);
    near |= fabsf(fabsf(y - n) - 0.5f) < 1e-5f;
    c[i] = (int)fminf(fmaxf(n, -8.f), 7.f) + 8;
  }
  if (__any(near) && s > 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double n = rint(((double)x[i] - (double)mid) / (double)s);
      c[i] = (int)fmin(fmax(n, -8.0), 7.0) + 8;
    }
  }
  u32 w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) w |= (u32)c[i] << (4 * i);
  return w;
}

// Rows of k and v into the cache.  A thread takes 8 elements, four threads a group.  grid = (rows, parts of a row's
// 2 kv_heads HD / 8 threads).
template <class T, int HD>
__global__ __launch_bounds__(256) void kv4_write_kernel(Kv4Pool p, Kv4Rows r, Kv4View k, Kv4View v) {
  constexpr int UPR = HD / 8;
  const int b = kv4_find(r, blockIdx.x);
  if (b < 0) return;
  const Kv4Seq s = kv4_seq(r, b);
  const int j = blockIdx.x - s.first, pos = s.len - s.rows + j;
  if (j >= r.max_rows || pos < 0) return;
  const int row = kv4_row(p, r.table + (size_t)b * r.table_stride, r.table_stride, pos);
  if (row < 0) return;
  const int units = p.kv_heads * UPR, t = blockIdx.y * 256 + threadIdx.x;
  if (t >= 2 * units) return;
  const int which = t >= units, unit = which ? t - units : t, head = unit / UPR, oct = unit % UPR;
  const u16x8 in = kv4_load8(which ? v : k, s.first + j, head, oct * 8);
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = T::load(in[i]);
  u32 param;
  const u32 w = kv4_quantise(x, param);
  *(u32*)(kv4_codes<HD>(p, which, head) + (size_t)row * (HD / 2) + oct * 4) = w;
  if (oct % 4 == 0) *(u32*)(kv4_params<HD>(p, which, head) + (size_t)row * (HD / 8) + oct) = param;
}

__device__ __forceinline__ float kv4_value(u32 w, int i, float s, float mid) {
  return fmaf(s, (float)((w >> (4 * i)) & 15) - 8.0f, mid);
}

// The same rows out of the cache.  Rows of positions that are not there are zeros; grid as kv4_write_kernel's.
template <class T, int HD>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Pool p, Kv4Rows r, Kv4View k, Kv4View v) {
  constexpr int UPR = HD / 8;
  const int b = kv4_find(r, blockIdx.x);
  if (b < 0) return;
  const Kv4Seq s = kv4_seq(r, b);
  const int j = blockIdx.x - s.first, pos = s.len - s.rows + j;
  if (j >= r.max_rows) return;
  const int row = pos < 0 ? -1 : kv4_row(p, r.table + (size_t)b * r.table_stride, r.table_stride, pos);
  const int units = p.kv_heads * UPR, t = blockIdx.y * 256 + threadIdx.x;
  if (t >= 2 * units) return;
  const int which = t >= units, unit = which ? t - units : t, head = unit / UPR, oct = unit % UPR;
  u16x8 out{};
  if (row >= 0) {
    const u32 w = *(const u32*)(kv4_codes<HD>(p, which, head) + (size_t)row * (HD / 2) + oct * 4);
    const u32 param = *(const u32*)(kv4_params<HD>(p, which, head) + (size_t)row * (HD / 8) + oct / 4 * 4);
    const float sc = Kv4F16::load(param & 0xffff), mid = Kv4F16::load(param >> 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = T::store(kv4_value(w, i, sc, mid));
  }
  kv4_store8(which ? v : k, s.first + j, head, oct * 8, out);
}

// Attention of one row and head per wave: HD / 8 lanes hold a row of the cache, the wave's lane groups take every 64 / (HD / 8)-th
// key, each with a running maximum and sum.  grid = (rows, ceil(heads / 4)).
template <class T, int HD>
__global__ __launch_bounds__(256) void kv4_attn_simple_kernel(Kv4Pool p, Kv4Rows r, Kv4View q, Kv4View o, int heads,
                                                              float scale) {
  constexpr int LPR = HD / 8, GPW = 64 / LPR;
  const int b = kv4_find(r, blockIdx.x);
  const int lane = threadIdx.x & 63, h = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int gi = lane / LPR, li = lane % LPR;
  if (h >= heads || b < 0) return;
  const Kv4Seq s = kv4_seq(r, b);
  const int j = blockIdx.x - s.first;
  if (j >= r.max_rows) return;
  const int kh = h / (heads / p.kv_heads), n_keys = s.len - s.rows + j + 1;
  const int* table = r.table + (size_t)b * r.table_stride;
  const u16x8 qin = kv4_load8(q, s.first + j, h, li * 8);
  float qv[8], acc[8], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) { qv[e] = T::load(qin[e]) * scale; acc[e] = 0.f; }
  for (int u = gi; u < n_keys; u += GPW) {
    const int row = kv4_row(p, table, r.table_stride, u);
    if (row < 0) continue;
    const u32 kw = *(const u32*)(kv4_codes<HD>(p, 0, kh) + (size_t)row * (HD / 2) + li * 4);
    const u32 vw = *(const u32*)(kv4_codes<HD>(p, 1, kh) + (size_t)row * (HD / 2) + li * 4);
    const u32 kp = *(const u32*)(kv4_params<HD>(p, 0, kh) + (size_t)row * (HD / 8) + li / 4 * 4);
    const u32 vp = *(const u32*)(kv4_params<HD>(p, 1, kh) + (size_t)row * (HD / 8) + li / 4 * 4);
    float dot = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) dot += qv[e] * kv4_value(kw, e, Kv4F16::load(kp & 0xffff), Kv4F16::load(kp >> 16));
    dot = group_sum<LPR>(dot);
    const float mn = fmaxf(m, dot), corr = m == mn ? 1.f : __expf(m - mn), pr = __expf(dot - mn);
    l = l * corr + pr;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      acc[e] = acc[e] * corr + pr * kv4_value(vw, e, Kv4F16::load(vp & 0xffff), Kv4F16::load(vp >> 16));
    m = mn;
  }
  float M = m;
#pragma unroll
  for (int off = LPR; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
  const float w = M > -INFINITY ? __expf(m - M) : 0.f;
  l *= w;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] *= w;
#pragma unroll
  for (int off = LPR; off < 64; off <<= 1) {
    l += __shfl_xor(l, off);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], off);
  }
  if (gi == 0) {
    u16x8 out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = T::store(l != 0.f ? acc[e] / l : 0.f);
    kv4_store8(o, s.first + j, h, li * 8, out);
  }
}
