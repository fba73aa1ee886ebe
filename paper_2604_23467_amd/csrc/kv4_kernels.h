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
typedef u32 u32x8 __attribute__((ext_vector_type(8)));
typedef u16 u16x8 __attribute__((ext_vector_type(8)));
typedef u16 u16x8u __attribute__((ext_vector_type(8), aligned(2)));      // anywhere in memory: one access of 16 bytes all the same

// One layer's pool
struct Kv4Pool {
  char* base;
  size_t codes, params;      // bytes of a codes region and of a parameters region, padding included
  size_t layer;              // bytes from one layer's pool to the next, for calls on several layers
  int kv_heads, pool_rows, page_tokens;
  u32 magic;                 // position / page_tokens = (2 u magic) >> 32 >> shift for 0 <= u < 2^31
  int shift;
};
// Rows of a call: sequence b has rows row_start[b] .. row_start[b + 1] - 1 (without row_start: max_rows each), the last
// of them at position len[b] - 1
struct Kv4Rows {
  const int *row_start, *len, *table;
  const int* active;         // optional: 0 = the sequence has no positions
  const int* order;          // optional: sequences in the order in which attention's workgroups take them
  int len_add;               // added to len[b]
  int n_seqs, max_rows, n_rows, table_stride;
};
// [row][head][head_dim], the last dimension contiguous; strides in elements
struct Kv4View {
  void* data;
  long row_stride, head_stride;
  long layer_stride;         // from one layer to the next
  int frag_k, frag_tb;       // frag_tb > 0: rows of frag_k elements in the projections' operand order (act_offset)
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
// A word at an address that all lanes share, by a scalar load (for what no kernel of this file writes)
__device__ __forceinline__ int kv4_scalar(const int* p) { return *(const __attribute__((address_space(4))) int*)p; }

__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Rows& r, int b) {
  Kv4Seq s;
  s.first = b * r.max_rows;
  s.rows = r.max_rows;
  const int len = kv4_scalar(r.len + b);
  if (r.row_start) {
    const int from = kv4_scalar(r.row_start + b), to = kv4_scalar(r.row_start + b + 1);
    s.first = min(max(from, 0), r.n_rows);
    s.rows = min(max(to, s.first), r.n_rows) - s.first;
  }
  s.len = max(len, 0) + r.len_add;
  if (r.active && !kv4_scalar(r.active + b)) s.len = 0;
  return s;
}

// Sequences of the rows from i0 on, -1 where a row has none: all 64 lanes of a wave look at a sequence each
template <int N>
__device__ __forceinline__ void kv4_find(const Kv4Rows& r, int i0, int (&b)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) b[n] = r.row_start || i0 + n >= r.n_rows ? -1 : (i0 + n) / r.max_rows;
  if (!r.row_start) return;
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < r.n_seqs; b0 += 64) {
    const int mine = min(b0 + lane, r.n_seqs - 1), from = r.row_start[mine], to = min(r.row_start[mine + 1], r.n_rows);
    int missing = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const unsigned long long hit = __ballot(i0 + n >= from && i0 + n < to);
      if (b[n] < 0 && hit) b[n] = b0 + __ffsll(hit) - 1;
      missing |= b[n] < 0;
    }
    if (!missing) return;
  }
}

// Pool row of position u >= 0 of the sequence with this page-table row; -1 where there is none
__device__ __forceinline__ int kv4_row(const Kv4Pool& p, const int* table, int table_stride, int u) {
  const int page = (int)(__umulhi((u32)u << 1, p.magic) >> p.shift);
  if (page >= table_stride) return -1;
  const int at = table[page];
  return (u32)at <= (u32)(p.pool_rows - p.page_tokens) ? at + (u - page * p.page_tokens) : -1;
}

// Pool rows of the call's rows from i0 on: -1 where a row's position has none, -2 where the row is none of the call's.  A lane
// looks after a row: with scalar registers alone the rows would be worked out one after the other, in as many instructions as
// quantising them takes.
template <int N>
__device__ __forceinline__ void kv4_places(const Kv4Pool& p, const Kv4Rows& r, int i0, int (&row)[N]) {
  int b[N];
  kv4_find<N>(r, i0, b);
  const int i = threadIdx.x & (N - 1);
  int mine = b[0];
#pragma unroll
  for (int n = 1; n < N; ++n) mine = i == n ? b[n] : mine;
  const int at = max(mine, 0), len = max(r.len[at], 0) + r.len_add;
  int first = at * r.max_rows, rows = r.max_rows;
  if (r.row_start) {
    first = min(max(r.row_start[at], 0), r.n_rows);
    rows = min(max(r.row_start[at + 1], first), r.n_rows) - first;
  }
  const int j = i0 + i - first, pos = (r.active && !r.active[at] ? 0 : len) - rows + j;
  const int page = (int)(__umulhi((u32)max(pos, 0) << 1, p.magic) >> p.shift);
  const int entry = r.table[(size_t)at * r.table_stride + min(page, r.table_stride - 1)];
  const bool ok = pos >= 0 && page < r.table_stride && (u32)entry <= (u32)(p.pool_rows - p.page_tokens);
  const int found = mine < 0 || j >= r.max_rows ? -2 : ok ? entry + (pos - page * p.page_tokens) : -1;
#pragma unroll
  for (int n = 0; n < N; ++n) row[n] = __builtin_amdgcn_readlane(found, n);
}

// ---- element types at the borders: binary16 and bfloat16 ----
struct Kv4F16 {
  static constexpr int bits = 11;
  static __device__ __forceinline__ float load(u16 v) { return (float)__builtin_bit_cast(half_t, v); }
  static __device__ __forceinline__ u16 store(float v) { return __builtin_bit_cast(u16, (half_t)v); }
};
struct Kv4Bf16 {
  static constexpr int bits = 8;
  static __device__ __forceinline__ float load(u16 v) { return __builtin_bit_cast(float, (u32)v << 16); }
  static __device__ __forceinline__ u16 store(float v) {      // to the nearest, half to even; NaN stays one
    const u32 b = __builtin_bit_cast(u32, v);
    return (u16)(v != v ? (b >> 16) | 0x40 : (b + 0x7fff + ((b >> 16) & 1)) >> 16);
  }
};
__device__ __forceinline__ u16x8 kv4_load8(const Kv4View& t, int row, int head, int e) {
  return *(const LL_GLOBAL u16x8u*)((const u16*)t.data + row * t.row_stride + (head * t.head_stride + e));
}
template <int HD>
__device__ __forceinline__ u16* kv4_element(const Kv4View& t, int row, int head, int e) {      // of an output
  if (t.frag_tb) return (u16*)t.data + act_offset(row, head * HD + e, t.frag_k, t.frag_tb);
  return (u16*)t.data + row * t.row_stride + (head * t.head_stride + e);
}
template <int HD>
__device__ __forceinline__ void kv4_store8(const Kv4View& t, int row, int head, int e, u16x8 v) {
  *(LL_GLOBAL u16x8u*)kv4_element<HD>(t, row, head, e) = v;
}

// A number that is a binary16 number of at most 8 significant bits: rounded up to the next one (x >= 0)
__device__ __forceinline__ float kv4_step_up(float x) {
  const float few = ceilf(x * 0x1p24f) * 0x1p-24f;                 // below, binary16's smallest step is the coarser one
  const float many = __builtin_bit_cast(float, (__builtin_bit_cast(u32, x) + 0xffff) & 0xffff0000u);
  return x < 0x1p-16f ? few : many;
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
// parameters (s in the low half).  Whether 15 s reaches the span is decided in 64 bits.  A code is the nearest whole number to
// the correctly rounded quotient (x - mid) / s, which is halfway between two whole numbers only where the exact one is, as long
// as x and mid are multiples of s / 2^20 and x - mid is exact: true but for numbers 2^9 times smaller than s.  Where there are
// such and an element lies near a border, 64 bits decide.
__device__ __forceinline__ u32 kv4_quantise(const float (&x)[8], u32& param) {
  float lo = fminf(x[0], x[1]), hi = fmaxf(x[0], x[1]);
  bool nan = __builtin_isunordered(x[0], x[1]);        // (an infinity shows in the span)
#pragma unroll
  for (int i = 2; i < 8; i += 2) {
    lo = fminf(lo, fminf(x[i], x[i + 1]));
    hi = fmaxf(hi, fmaxf(x[i], x[i + 1]));
    nan |= __builtin_isunordered(x[i], x[i + 1]);
  }
  lo = kv4_quad_min<0x4E>(kv4_quad_min<0xB1>(lo));
  hi = kv4_quad_max<0x4E>(kv4_quad_max<0xB1>(hi));
  const unsigned long long nans = __ballot(nan);
  const double span = (double)hi - (double)lo;
  float s = kv4_step_up((hi - lo) * (1.0f / 15.0f));
  if (15.0 * (double)s < span) s = kv4_step_next(s, 1);
  const float below = kv4_step_next(s, -1);
  if (s > 0.f && 15.0 * (double)below >= span) s = below;
  const half_t mid_h = (half_t)sk_fp32((float)fma(8.0, (double)s, (double)lo));      // by way of 32 bits, in two instructions
  const float mid = (float)mid_h;
  if ((nans && (nans >> (threadIdx.x & 60) & 15)) || !(s <= KV4_MAX_STEP) || !(fabsf(mid) < INFINITY)) {
    param = 0x7e007e00u;
    return 0;
  }
  param = (u32)__builtin_bit_cast(u16, (half_t)s) | (u32)__builtin_bit_cast(u16, mid_h) << 16;
  const float inv = s > 0.f ? __builtin_amdgcn_rcpf(s) : 0.f;
  auto quotient = [&](float v) {
    const float d = v - mid, y = d * inv;
    return fmaf(fmaf(-y, s, d), inv, y);
  };
  float c[8], least = fabsf(mid);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    least = fminf(least, fabsf(x[i]));
    c[i] = __builtin_amdgcn_fmed3f(rintf(quotient(x[i])), -8.f, 7.f);
  }
  if (__any(least < s * 0x1p-9f)) {      // (few rows get here; fewer go on)
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) off = fmaxf(off, fabsf(quotient(x[i]) - rintf(quotient(x[i]))));
    if (__any(off > 0.49999f && least < s * 0x1p-9f) && s > 0.f) {
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        float v = x[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) v = k == i ? x[k] : v;
        v = __builtin_amdgcn_fmed3f((float)rint(((double)v - (double)mid) / (double)s), -8.f, 7.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = k == i ? v : c[k];
      }
    }
  }
  auto four = [](float a, float b, float d, float e) {   // c + 8 of four elements in 16 bits: whole numbers, exact
    return (u32)fmaf(fmaf(e, 16.f, d), 256.f, fmaf(b, 16.f, a + 34952.f));
  };
  return four(c[0], c[1], c[2], c[3]) | four(c[4], c[5], c[6], c[7]) << 16;
}

// Rows of k and v into the cache, of several layers at once where grid.z = 2 x layers.  A thread takes 8 elements of N
// consecutive rows, four threads a group.  grid = (blocks of N rows, parts of a row's kv_heads HD / 8 threads, keys and values).
// The cache has a head's rows side by side, so the rows of a block share lines of it: written one by one from different XCDs, a
// line of parameters (8 rows) would leave eight L2s in parts.
// Reads 2 bytes an element and writes 5 / 8.  Four sequences of 1 .. 8190 rows of 8 heads of 128: 34 us (row by row 52), with
// the vector unit busy half of it (23 operations an element, a quarter of them for the group's parameters) and waiting for memory
// the rest: rows are requested in front of the look-up of their places, which takes three dependent loads (behind it: 35 us).
template <class T, int HD, int N>
__global__ __launch_bounds__(256) void kv4_write_kernel(Kv4Pool p, Kv4Rows r, Kv4View k, Kv4View v) {
  constexpr int UPR = HD / 8;
  const int i0 = blockIdx.x * N, unit = blockIdx.y * blockDim.x + threadIdx.x, which = blockIdx.z & 1;
  const int head = unit / UPR, oct = unit % UPR;
  Kv4View from = which ? v : k;
  from.data = (u16*)from.data + (blockIdx.z >> 1) * from.layer_stride;
  p.base += (blockIdx.z >> 1) * p.layer;
  u16x8 in[N];                                         // also of rows that have no place, in front of what says so
#pragma unroll
  for (int n = 0; n < N; ++n) in[n] = kv4_load8(from, min(i0 + n, r.n_rows - 1), min(head, p.kv_heads - 1), oct * 8);
  __builtin_amdgcn_sched_barrier(0);
  int row[N];
  kv4_places<N>(p, r, i0, row);
  if (head >= p.kv_heads) return;
  char *codes = kv4_codes<HD>(p, which, head) + oct * 4, *params = kv4_params<HD>(p, which, head) + oct;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (row[n] < 0) continue;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = T::load(in[n][i]);
    u32 param;
    const u32 w = kv4_quantise(x, param);
    *as_global(reinterpret_cast<u32*>(codes + (size_t)(u32)row[n] * (HD / 2))) = w;
    if (oct % 4 == 0) *as_global(reinterpret_cast<u32*>(params + (size_t)(u32)row[n] * (HD / 8))) = param;
  }
}

__device__ __forceinline__ float kv4_value(u32 w, int i, float s, float mid) {
  return fmaf(s, (float)((w >> (4 * i)) & 15) - 8.0f, mid);
}

// The same rows out of the cache.  Rows of positions that are not there are zeros; grid and blocks as kv4_write_kernel's.
// Bound by memory: 32 sequences of 1 .. 1000 rows of 32 heads of 128, 344 MB, in 74 us, 4.7 TB/s, where a copy moves 5.0 (row by
// row: 128 us).
template <class T, int HD, int N>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Pool p, Kv4Rows r, Kv4View k, Kv4View v) {
  constexpr int UPR = HD / 8;
  const int i0 = blockIdx.x * N, unit = blockIdx.y * blockDim.x + threadIdx.x, which = blockIdx.z;
  const int head = unit / UPR, oct = unit % UPR;
  int row[N];
  kv4_places<N>(p, r, i0, row);
  if (head >= p.kv_heads) return;
  const Kv4View to = which ? v : k;
  const char *codes = kv4_codes<HD>(p, which, head) + oct * 4, *params = kv4_params<HD>(p, which, head) + oct / 4 * 4;
  u32 w[N], param[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    w[n] = *as_global(reinterpret_cast<const u32*>(codes + (size_t)(u32)max(row[n], 0) * (HD / 2)));
    param[n] = *as_global(reinterpret_cast<const u32*>(params + (size_t)(u32)max(row[n], 0) * (HD / 8)));
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (row[n] == -2) continue;
    const float sc = Kv4F16::load(param[n] & 0xffff), mid = Kv4F16::load(param[n] >> 16);
    u16x8 out;
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = row[n] < 0 ? (u16)0 : T::store(kv4_value(w[n], i, sc, mid));
    kv4_store8<HD>(to, i0 + n, head, oct * 8, out);
  }
}

// ---- attention ----
//
// Scores and outputs of up to 16 query rows (rows of a sequence times the heads that share a key head) run on the matrix
// instructions, also where there is one row only: a code costs the vector unit 1.6 operations on its way into an operand and
// nothing more, where a product of its own would cost two.
//
//   S^T [32 keys][16 queries]   = K Q^T:    16x16x32 products, keys as rows, queries as columns
//   O^T [head_dim][16 queries] += V^T P^T:  the values' elements as rows
//
// Both contract over an order of their own choosing, so every operand is built in the registers of the lane that loaded it,
// without LDS.  With lane = 16 h + c:
//  * K: the lane loads a quarter (HD / 4 elements) of key c; product s takes its 8 elements 8 s .. of all four quarters.
//    q is laid out to match.  The middles enter by a product of their own: the lane's mid against the sum of q over the
//    quarter, which is split into three binary16 numbers.
//  * S^T leaves the lane with keys 4 h + i and 16 + 4 h + i (i < 4) of query c: exactly the 8 keys that the lane feeds to
//    the second product as P^T.
//  * V: for these 8 keys the lane loads elements (HD / 16) c ..; a permutation of half words pairs two keys, and every
//    nibble position e is then the operand of the HD / 16 elements' e-th row block: row c of product e is element
//    (HD / 16) c + e.  A further product's rows are the middles of the groups (row 4 g'), ones (row 1: the sum of the
//    weights) and where a group is NaN (rows 4 g' + 2); a lane's outputs then all belong to one group, whose sum is in its
//    own registers.
// s (c - 8) is exact in binary16 (see above).  Weights are at most 2^15 (the maximum is taken off in front of the exponential);
// they enter as two binary16 numbers, which is 22 bits, where outputs are binary16 themselves, and as one, 11 bits, where these
// have 8; sums are 32 bits wide.

typedef half_t h2 __attribute__((ext_vector_type(2)));

#define KV4_WAVES 4              // of a workgroup; they take every fourth tile
#define KV4_TILE 32              // keys of a tile
#define KV4_FEW_ROWS 16
#define KV4_SHIFT 15.0f          // log2 of the largest weight

__device__ __forceinline__ h2 kv4_h2(u32 v) { return __builtin_bit_cast(h2, v); }
__device__ __forceinline__ u32 kv4_u32(h2 v) { return __builtin_bit_cast(u32, v); }
__device__ __forceinline__ u32 kv4_lo16(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ u32 kv4_hi16(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Nibbles 0 and 4, 1 and 5, 2 and 6, 3 and 7 of w as pairs of c - 8: a code set into the mantissa of 1024 (or, four bits
// higher, of 64) is that number plus c.
// The constants are hidden from the compiler, in registers of the two kinds that v_and_or_b32 takes together: it would write
// two instructions with a literal each.
struct Kv4Bits {
  u32 low, high, k1024, k64;
  __device__ __forceinline__ Kv4Bits() : low(0x000f000fu), high(0x00f000f0u), k1024(0x64006400u), k64(0x54005400u) {
    asm("" : "+s"(low), "+s"(high));
    asm("" : "+v"(k1024), "+v"(k64));
  }
  __device__ __forceinline__ void unpack(u32 w, h2 (&d)[4]) const {
    const u32 y = w >> 8;
    d[0] = kv4_h2((w & low) | k1024) - h2{1032, 1032};
    d[1] = kv4_h2((w & high) | k64) - h2{72, 72};
    d[2] = kv4_h2((y & low) | k1024) - h2{1032, 1032};
    d[3] = kv4_h2((y & high) | k64) - h2{72, 72};
  }
};

__device__ __forceinline__ float kv4_max_over_quarters(float v) {      // lanes c, c + 16, c + 32, c + 48
  const u32 b = __builtin_bit_cast(u32, v);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  const float a = fmaxf(__builtin_bit_cast(float, (u32)r[0]), __builtin_bit_cast(float, (u32)r[1]));
  const u32 d = __builtin_bit_cast(u32, a);
  const auto t = __builtin_amdgcn_permlane16_swap(d, d, false, false);
  return fmaxf(__builtin_bit_cast(float, (u32)t[0]), __builtin_bit_cast(float, (u32)t[1]));
}

__device__ __forceinline__ f4 kv4_mfma(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// What a workgroup works on: row block rb of key head `head` of sequence b, and a share of its keys
struct Kv4Work {
  int b, rb, head, split;
};
__device__ __forceinline__ Kv4Work kv4_work(const Kv4Rows& r, int id, int splits, int kv_heads, int row_blocks) {
  Kv4Work w;
  w.split = id % splits;
  id /= splits;
  w.head = id % kv_heads;
  id /= kv_heads;
  w.rb = id % row_blocks;
  w.b = r.order ? kv4_scalar(r.order + id / row_blocks) : id / row_blocks;
  return w;
}
// Positions that the sequence's row j sees: none behind what the page table has entries for (at most 2^30, the host's check),
// however large the length that lies in memory
__device__ __forceinline__ int kv4_keys(const Kv4Pool& p, const Kv4Rows& r, const Kv4Seq& s, int j) {
  return max(min(s.len - s.rows + j + 1, r.table_stride * p.page_tokens), 0);
}
// Tiles of a share when `tiles` of them are dealt to `splits` workgroups: whole rounds of the waves
__device__ __forceinline__ int kv4_share(int tiles, int splits) {
  return ((tiles + splits - 1) / splits + KV4_WAVES - 1) / KV4_WAVES * KV4_WAVES;
}

// Queries of a row block as the second operand, in K's order: lane (h, c) has quarter h of query c's row, scaled by a power of
// two to a largest element of 1 .. 2 (bfloat16's 8 bits then fit binary16, whatever their exponent); and what scores have to be
// multiplied by for a softmax to the base 2.
template <int HD>
struct Kv4Query {
  h8 q[HD / 32];
  h8 sums;
  float scale;
};
template <class T, int HD>
__device__ __forceinline__ void kv4_query(const u16x8 (&in)[HD / 32], float scale, Kv4Query<HD>& out) {
  float x[HD / 32][8], top = 0.f;
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[s][i] = T::load(in[s][i]);
      top = fmaxf(top, fabsf(x[s][i]));
    }
  }
  top = kv4_max_over_quarters(top);
  int e = 0;
  if (top > 0.f && top < INFINITY) e = ilogbf(top);
  float sum = 0.f;
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {          // pairs (i, i + 4), as a word of codes unpacks
      const half_t a = (half_t)ldexpf(x[s][i], -e), b = (half_t)ldexpf(x[s][i + 4], -e);
      out.q[s][2 * i] = a;
      out.q[s][2 * i + 1] = b;
      sum += (float)a + (float)b;
    }
  }
  const half_t s1 = (half_t)sum, s2 = (half_t)(sum - (float)s1), s3 = (half_t)(sum - (float)s1 - (float)s2);
  out.sums = h8{s1, s2, s3, 0, 0, 0, 0, 0};
  out.scale = fmaxf(ldexpf(scale * 1.44269504088896340736f, e), 0x1p-126f);
}

// A tile of 32 keys as it lies in the pool: the lane's part of keys c and 16 + c, and of its 8 values
template <int HD>
struct Kv4Tile {
  u32x4 k0, k1;                 // (head_dim 64: the first two words)
  u32x2 kp;
  u32x8 v, vp;
};

// Tiles come into LDS by direct loads, which cost no registers while they are under way: a wave has two slots of its own, one
// of which is filled while the other is used.  A half of a slot (keys or values) is 32 rows of codes in pieces of 16 bytes and
// their parameters.  Pieces are stored in an order in which neither the keys' reads (a piece of each of 16 rows) nor the
// values' (a word each of rows 4 h + i) meet in a bank: head_dim 128, piece x of row 4 b + a of a block of 16 rows at
// 16 b + 4 (a ^ b) + (x ^ b); head_dim 64, piece x of row y at 2 y + (x ^ bit 3 of y).
template <int HD>
struct Kv4Ring {
  static constexpr int CODES = KV4_TILE * HD / 2, PARAMS = KV4_TILE * HD / 8, HALF = CODES + PARAMS, SLOT = 2 * HALF;
  static constexpr int LOADS = HD == 128 ? 4 : 2;      // direct loads of a half (all lanes take part in each)
  const char *kc, *kp, *vc, *vp;      // codes and parameters of the key head
  char* slots;                        // the wave's two slots
  int lane, h, c;
  u32 code_row, code_at, param_row, param_at;      // row (of 16, or of 32 with head_dim 64) and bytes in it that the lane brings in

  __device__ __forceinline__ Kv4Ring(const Kv4Pool& p, int head, char* lds, int lane_) : slots(lds), lane(lane_) {
    h = lane >> 4;
    c = lane & 15;
    kc = kv4_codes<HD>(p, 0, head);
    kp = kv4_params<HD>(p, 0, head);
    vc = kv4_codes<HD>(p, 1, head);
    vp = kv4_params<HD>(p, 1, head);
    if (HD == 128) {
      code_row = 4 * h + (((lane >> 2) & 3) ^ h);
      code_at = ((lane & 3) ^ h) * 16;
      param_row = lane >> 2;
      param_at = (lane & 3) * 4;
    } else {
      code_row = lane >> 1;
      code_at = ((lane & 1) ^ (lane >> 4 & 1)) * 16;
      param_row = lane >> 1;
      param_at = (lane & 1) * 4;
    }
  }
  static __device__ __forceinline__ int piece(int row, int x) {
    return HD == 128 ? (row & 16) * 64 + ((row >> 2 & 3) * 16 + ((row ^ row >> 2) & 3) * 4 + (x ^ (row >> 2 & 3))) * 16
                     : (2 * row + (x ^ (row >> 3 & 1))) * 16;
  }
  template <int SIZE>
  static __device__ __forceinline__ void bring(const char* from, char* to) {
    if constexpr (SIZE == 16) __builtin_amdgcn_global_load_lds((const LL_GLOBAL void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    else __builtin_amdgcn_global_load_lds((const LL_GLOBAL void*)from, (__attribute__((address_space(3))) void*)to, 4, 0, 0);
  }
  // where: says where the tile's rows are in the pool
  template <class Where>
  __device__ __forceinline__ void fetch(const char* codes, const char* params, char* to, const Where& where) const {
    if (HD == 128) {
      bring<16>(where.at(codes, HD / 2, 0, code_row) + code_at, to);
      bring<16>(where.at(codes, HD / 2, 1, code_row) + code_at, to + CODES / 2);
      bring<4>(where.at(params, HD / 8, 0, param_row) + param_at, to + CODES);
      bring<4>(where.at(params, HD / 8, 1, param_row) + param_at, to + CODES + PARAMS / 2);
    } else {
      bring<16>(where.split(codes, HD / 2, code_row) + code_at, to);
      bring<4>(where.split(params, HD / 8, param_row) + param_at, to + CODES);
    }
  }
  template <class Where>
  __device__ __forceinline__ void fetch_keys(int slot, const Where& where) const { fetch(kc, kp, slots + slot * SLOT, where); }
  template <class Where>
  __device__ __forceinline__ void fetch_values(int slot, const Where& where) const { fetch(vc, vp, slots + slot * SLOT + HALF, where); }

  __device__ __forceinline__ void read_keys(int slot, Kv4Tile<HD>& t) const {
    const char* s = slots + slot * SLOT;
    if (HD == 128) {
      t.k0 = *reinterpret_cast<const u32x4*>(s + piece(c, h));
      t.k1 = *reinterpret_cast<const u32x4*>(s + piece(16 + c, h));
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(s + piece(c, h >> 1) + (h & 1) * 8);
      const u32x2 y = *reinterpret_cast<const u32x2*>(s + piece(16 + c, h >> 1) + (h & 1) * 8);
      t.k0 = u32x4{x[0], x[1], 0, 0};
      t.k1 = u32x4{y[0], y[1], 0, 0};
    }
    const u32* q = reinterpret_cast<const u32*>(s + CODES);
    const int g = HD == 128 ? h : h >> 1;
    t.kp = u32x2{q[c * (HD / 32) + g], q[(16 + c) * (HD / 32) + g]};
  }
  __device__ __forceinline__ void read_values(int slot, Kv4Tile<HD>& t) const {
    const char* s = slots + slot * SLOT + HALF;
    const u32* q = reinterpret_cast<const u32*>(s + CODES);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int row = (j & 3) + 4 * h + 16 * (j >> 2);
      if (HD == 128) t.v[j] = *reinterpret_cast<const u32*>(s + piece(row, c >> 2) + (c & 3) * 4);
      else t.v[j] = *reinterpret_cast<const u16*>(s + piece(row, c >> 3) + (c & 7) * 2);
      t.vp[j] = q[row * (HD / 32) + c * (HD / 16) / KV4_GROUP];
    }
  }
};
// Where a tile's rows are: 16 consecutive pool rows each from two scalar rows on ...
struct Kv4Halves {
  u32x2 row;
  __device__ __forceinline__ const char* at(const char* base, int bytes, int half, u32 i) const {
    return base + (size_t)row[half] * bytes + i * bytes;
  }
  __device__ __forceinline__ const char* split(const char* base, int bytes, u32 i) const {
    const u32 a = row[0], b = row[1];
    return base + (size_t)(((i & 16) ? b : a) + (i & 15)) * bytes;
  }
};
// ... or anywhere, as 32 words in LDS say
struct Kv4Listed {
  const u32* rows;
  __device__ __forceinline__ const char* at(const char* base, int bytes, int half, u32 i) const {
    return base + (size_t)rows[16 * half + i] * bytes;
  }
  __device__ __forceinline__ const char* split(const char* base, int bytes, u32 i) const { return base + (size_t)rows[i] * bytes; }
};

// Keys of a tile against the queries: S^T of keys 16 j + 4 h + i
template <int HD>
__device__ __forceinline__ void kv4_scores(const Kv4Tile<HD>& t, const Kv4Query<HD>& q, const Kv4Bits& bits, f4& s0, f4& s1) {
  auto one = [&](u32x4 w, u32 param) {
    const half_t mid = kv4_h2(param)[1];
    f4 s = kv4_mfma(h8{mid, mid, mid, 0, 0, 0, 0, 0}, q.sums, f4{0.f, 0.f, 0.f, 0.f});
    const h2 step = kv4_h2(kv4_lo16(param, param));
#pragma unroll
    for (int n = 0; n < HD / 32; ++n) {
      h2 d[4];
      bits.unpack(w[n], d);
      const u32x4 a{kv4_u32(d[0] * step), kv4_u32(d[1] * step), kv4_u32(d[2] * step), kv4_u32(d[3] * step)};
      s = kv4_mfma(__builtin_bit_cast(h8, a), q.q[n], s);
    }
    return s;
  };
  s0 = one(t.k0, t.kp[0]);
  s1 = one(t.k1, t.kp[1]);
}

// Bit of the lane's i-th key (keys 4 h .. and 16 + 4 h ..) in a word with a bit for each of a tile's keys
__device__ __forceinline__ int kv4_key(int i, int h) { return (i & 3) + 4 * h + 16 * (i >> 2); }

// Operand of the block of middles, ones and NaN marks.  there: which of the tile's keys have a row.  Keys that have none, and
// groups that are NaN, must not meet a weight of zero: their parameters become zero.  Both are rare and found for the whole wave
// at once: a sum of all middles is NaN if one is.
template <int HD>
__device__ __forceinline__ h8 kv4_middles(Kv4Tile<HD>& t, u32 there, int c, int h, u32 mid_row, u32 one_row) {
  u32 marks = 0;
  h2 all = kv4_h2(t.vp[0]);
#pragma unroll
  for (int j = 1; j < 8; ++j) all += kv4_h2(t.vp[j]);
  if (~there || __any(!(all[1] == all[1]))) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const half_t mid = kv4_h2(t.vp[j])[1];
      const bool gone = !(there >> kv4_key(j, h) & 1), nan = !(mid == mid);
      if (nan && !gone) marks |= 1u << j;
      if (gone || nan) t.vp[j] = 0;
    }
  }
  u32x4 w;
#pragma unroll
  for (int a = 0; a < 4; ++a) w[a] = (kv4_hi16(t.vp[2 * a], t.vp[2 * a + 1]) & mid_row) | one_row;
  if (__any(marks)) {
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const u32 mark = (marks >> (2 * a) & 1 ? 0x3c00u : 0u) | (marks >> (2 * a + 1) & 1 ? 0x3c000000u : 0u);
      w[a] = (c & 3) == 2 ? mark : w[a];
    }
  }
  return __builtin_bit_cast(h8, w);
}

// Values of a tile as operands: o[i] is row block 4 PART + i (element (HD / 16) c + 4 PART + i of the lane's 8 keys)
template <int HD, int PART>
__device__ __forceinline__ void kv4_values(const Kv4Tile<HD>& t, const Kv4Bits& bits, h8 (&o)[4]) {
  u32x4 w[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const h2 step = kv4_h2(kv4_lo16(t.vp[2 * a], t.vp[2 * a + 1]));
    h2 d[4];
    bits.unpack(PART ? kv4_hi16(t.v[2 * a], t.v[2 * a + 1]) : kv4_lo16(t.v[2 * a], t.v[2 * a + 1]), d);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i][a] = kv4_u32(d[i] * step);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __builtin_bit_cast(h8, w[i]);
}

// Up to 16 query rows of one key head.  grid = splits * kv_heads * row blocks * sequences workgroups (kv4_work's order) of four
// waves; the waves take every fourth tile of the workgroup's share and keep a softmax of their own, which meet in LDS.
// P16: page_tokens is a multiple of 16, so that halves of a tile are consecutive pool rows and their addresses scalar.
// NEW: knew and vnew hold the sequences' last rows (one row each), which the workgroup that has the last key quantises into
// the pool and attends from LDS.  part: with more than one split, the shares' results ([work][16][HD + 2] floats).
// Four sequences of 30000 positions, 8 key heads of 128 and 4 query heads each: 41 us, 4.0 TB/s of the cache.  What bounds it is
// a wave's chain of loads, codes to operands (420 vector instructions for 32 keys), products and softmax: the vector unit is
// busy 46 % of the time, the matrix cores 9 %.  Four workgroups a CU would need 128 registers a lane, and spill: 32 sequences of
// 2000 positions then take 125 us instead of 92.
template <class T, int HD, bool P16, bool NEW>
__global__ __launch_bounds__(256, 3) void kv4_attn_few_kernel(Kv4Pool p, Kv4Rows r, Kv4View q, Kv4View o, Kv4View knew, Kv4View vnew,
                                                           int heads, float scale, int splits, int row_blocks, float* part) {
  constexpr int NE = HD / 16;
  constexpr bool TWO = T::bits > 8;
  using Ring = Kv4Ring<HD>;
  constexpr int RING = KV4_WAVES * 2 * Ring::SLOT, MEET = KV4_WAVES * (NE + 1) * 64 * 16;
  __shared__ __attribute__((aligned(16))) char s_mem[RING > MEET ? RING : MEET];      // the tiles, then what the waves hand in
  __shared__ __attribute__((aligned(16))) u32 s_rows[P16 ? 1 : KV4_WAVES][KV4_TILE];
  __shared__ float s_m[KV4_WAVES][16];
  __shared__ __attribute__((aligned(16))) u32 s_new[2][HD / 8], s_newp[2][HD / 32];
  const Kv4Work w = kv4_work(r, blockIdx.x, splits, p.kv_heads, row_blocks);
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Kv4Seq s = kv4_seq(r, w.b);
  const int share_heads = heads / p.kv_heads, rows = min(s.rows, r.max_rows) * share_heads;
  const int f0 = w.rb * KV4_FEW_ROWS;
  if (f0 >= rows) return;
  const int first_limit = s.len - s.rows + f0 / share_heads;               // last position that the first query sees
  const int n_keys = kv4_keys(p, r, s, min(f0 + KV4_FEW_ROWS - 1, rows - 1) / share_heads);
  const int tiles = (n_keys + KV4_TILE - 1) / KV4_TILE, share = kv4_share(tiles, splits);
  const int t0 = w.split * share, t1 = min(t0 + share, tiles);
  if (w.split > 0 && t0 >= tiles) return;
  const int* table = r.table + (size_t)w.b * r.table_stride;

  // requested in front of everything that waits for the page table
  const int f = f0 + c, j = f / share_heads, qhead = w.head * share_heads + f - j * share_heads;
  const bool there = f < rows;
  const int limit = there ? s.len - s.rows + j : -1;                       // last position that the lane's query sees
  u16x8 qin[HD / 32], nin{};
#pragma unroll
  for (int n = 0; n < HD / 32; ++n) {
    qin[n] = u16x8{};
    if (there) qin[n] = kv4_load8(q, s.first + j, qhead, h * (HD / 4) + n * 8);
  }
  if (NEW && wave < 2 && lane < HD / 8) nin = kv4_load8(wave ? vnew : knew, s.first, w.head, lane * 8);
  __builtin_amdgcn_sched_barrier(0);

  // Pool rows of a tile: the page table's entries are requested a tile ahead of the tile's own loads.  place() then says where
  // the rows are, and which of the tile's keys have one (others: row 0).  Without P16 a lane looks after a key, and the rows go
  // through LDS.
  const Ring ring(p, w.head, s_mem + wave * 2 * Ring::SLOT, lane);
  const int ahead = P16 ? 0 : lane & (KV4_TILE - 1);
  auto page = [&](int u) { return (int)(__umulhi((u32)u << 1, p.magic) >> p.shift); };
  auto look = [&](int t) {
    const int last = r.table_stride - 1, u = t * KV4_TILE + ahead;
    if constexpr (P16) return u32x2{(u32)kv4_scalar(table + min(page(u), last)), (u32)kv4_scalar(table + min(page(u + 16), last))};
    else return u32x2{(u32)*as_global(table + min(page(u), last)), 0};
  };
  auto row = [&](int u, u32 at) {                                          // -1: none
    const int pg = page(u);
    return u < n_keys && pg < r.table_stride && at <= (u32)(p.pool_rows - p.page_tokens) ? (int)(at + (u - pg * p.page_tokens)) : -1;
  };
  auto place = [&](int t, u32x2 at, u32& has) {
    const int u = t * KV4_TILE + ahead;
    if constexpr (P16) {
      const int a = row(u, at[0]), b = row(u + 16, at[1]);
      const u32 one = a >= 0 ? 0xffffu >> max(u + 16 - n_keys, 0) : 0u, two = b >= 0 ? 0xffffu >> max(u + 32 - n_keys, 0) : 0u;
      has = one | two << 16;
      return Kv4Halves{u32x2{(u32)max(a, 0), (u32)max(b, 0)}};
    } else {
      const int a = row(u, at[0]);
      has = (u32)__ballot(a >= 0);
      s_rows[wave][ahead] = max(a, 0);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      return Kv4Listed{s_rows[wave]};
    }
  };
  int t = t0 + wave;
  u32x2 at{0, 0};
  u32 has = 0, has1 = 0;                                                   // keys of this tile and the next that have a row
  if (t < t1) {
    const u32x2 at0 = look(t), at1 = look(t + KV4_WAVES);
    at = look(t + 2 * KV4_WAVES);
    {
      const auto where = place(t, at0, has);
      ring.fetch_keys(0, where);
      ring.fetch_values(0, where);
    }
    __builtin_amdgcn_sched_barrier(0);
    {
      const auto where = place(t + KV4_WAVES, at1, has1);
      ring.fetch_keys(1, where);
      ring.fetch_values(1, where);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  Kv4Query<HD> query;
  kv4_query<T, HD>(qin, scale, query);
  const int pnew = NEW ? s.len - s.rows : -1;
  if (NEW && pnew >= 0 && pnew / KV4_TILE >= t0 && pnew / KV4_TILE < t1) {
    if (wave < 2 && lane < HD / 8) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = T::load(nin[i]);
      u32 param;
      const u32 code = kv4_quantise(x, param);
      s_new[wave][lane] = code;
      s_newp[wave][lane >> 2] = param;
      const int to = kv4_row(p, table, r.table_stride, pnew);
      if (to >= 0) {
        *(u32*)(kv4_codes<HD>(p, wave, w.head) + (size_t)to * (HD / 2) + lane * 4) = code;
        if (lane % 4 == 0) *(u32*)(kv4_params<HD>(p, wave, w.head) + (size_t)to * (HD / 8) + lane) = param;
      }
    }
    wait_lgkm_at_most<0>();
    __builtin_amdgcn_s_barrier();                                          // (__syncthreads would wait for the tiles, too)
    asm volatile("" ::: "memory");
  }

  f4 acc[NE + 1];
#pragma unroll
  for (int e = 0; e <= NE; ++e) acc[e] = f4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY;

  // Loads of a wave land in the order in which they were issued: keys and values of a tile, then those of the next.  A wait
  // leaves what is younger than its half of a tile in flight, and a half is fetched anew once its reads have arrived.
  const Kv4Bits bits;
  const u32 mid_row = (c & 3) == 0 ? ~0u : 0u, one_row = c == 1 ? 0x3c003c00u : 0u;
  Kv4Tile<HD> tile;
  for (int slot = 0; t < t1; t += KV4_WAVES, slot ^= 1) {
    const int u0 = t * KV4_TILE;
    u32 has2;
    const auto where = place(t + 2 * KV4_WAVES, at, has2);
    at = look(t + 3 * KV4_WAVES);
    wait_vm_at_most<3 * Ring::LOADS>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    ring.read_keys(slot, tile);
    if (NEW && pnew >= u0 && pnew < u0 + KV4_TILE) {
      const int n0 = pnew - u0;
      const u32x4 code = HD == 128 ? *reinterpret_cast<const u32x4*>(&s_new[0][h * (HD / 32)])
                                   : u32x4{s_new[0][2 * h], s_new[0][2 * h + 1], 0, 0};
      const u32 param = s_newp[0][HD == 128 ? h : h >> 1];
      if (n0 == c) { tile.k0 = code; tile.kp[0] = param; }
      if (n0 == 16 + c) { tile.k1 = code; tile.kp[1] = param; }
    }
    wait_lgkm_at_most<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    ring.fetch_keys(slot, where);
    __builtin_amdgcn_sched_barrier(0);
    f4 s0, s1;
    kv4_scores<HD>(tile, query, bits, s0, s1);
    s0 *= query.scale;
    s1 *= query.scale;
    if (u0 + KV4_TILE - 1 > first_limit || ~has) {                         // some query does not see some key
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int a = kv4_key(i, h), b = kv4_key(4 + i, h);
        if (!(has >> a & 1) || u0 + a > limit) s0[i] = -INFINITY;
        if (!(has >> b & 1) || u0 + b > limit) s1[i] = -INFINITY;
      }
    }
    float top = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
    top = fmaxf(kv4_max_over_quarters(top), m);
    if (__any(top > m)) {
      const float corr = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
      m = top;
#pragma unroll
      for (int e = 0; e <= NE; ++e) acc[e] *= corr;
    }
    const float base = KV4_SHIFT - (m > -INFINITY ? m : 0.f);
    u32x4 ph, pl;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f4& x = i < 2 ? s0 : s1;
      const float a = __builtin_amdgcn_exp2f(x[2 * (i & 1)] + base);
      const float b = __builtin_amdgcn_exp2f(x[2 * (i & 1) + 1] + base);
      if (TWO) {                                                           // cut to 11 bits, and what that leaves, cut likewise
        const auto hi = __builtin_amdgcn_cvt_pkrtz(a, b);
        ph[i] = __builtin_bit_cast(u32, hi);
        pl[i] = __builtin_bit_cast(u32, __builtin_amdgcn_cvt_pkrtz(fmaf((float)hi[0], -1.0f, a), fmaf((float)hi[1], -1.0f, b)));
      } else {
        ph[i] = kv4_u32(h2{(half_t)a, (half_t)b});
      }
    }
    auto add = [&](int e, h8 o) {
      acc[e] = kv4_mfma(o, __builtin_bit_cast(h8, ph), acc[e]);
      if (TWO) acc[e] = kv4_mfma(o, __builtin_bit_cast(h8, pl), acc[e]);
    };
    __builtin_amdgcn_sched_barrier(0);
    wait_vm_at_most<3 * Ring::LOADS>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    ring.read_values(slot, tile);
    if (NEW && pnew >= u0 && pnew < u0 + KV4_TILE) {
      const int n0 = pnew - u0;
      const u32 code = HD == 128 ? s_new[1][c] : (s_new[1][c >> 1] >> (16 * (c & 1))) & 0xffff;
      const u32 param = s_newp[1][c * (HD / 16) / KV4_GROUP];
#pragma unroll
      for (int n = 0; n < 8; ++n)
        if (n0 == kv4_key(n, h)) { tile.v[n] = code; tile.vp[n] = param; }
    }
    wait_lgkm_at_most<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    ring.fetch_values(slot, where);
    __builtin_amdgcn_sched_barrier(0);
    add(NE, kv4_middles<HD>(tile, has, c, h, mid_row, one_row));
    h8 op[4];
    kv4_values<HD, 0>(tile, bits, op);
#pragma unroll
    for (int i = 0; i < 4; ++i) add(i, op[i]);
    if (HD == 128) {
      kv4_values<HD, 1>(tile, bits, op);
#pragma unroll
      for (int i = 0; i < 4; ++i) add(4 * (HD / 128) + i, op[i]);
    }
    has = has1;
    has1 = has2;
  }
  wait_vm_at_most<0>();                                                    // the loads ahead must not land in what follows

  // the waves' softmaxes meet
  if (h == 0) s_m[wave][c] = m;
  __syncthreads();
  typedef float Meet[NE + 1][64][4];
  Meet* meet = reinterpret_cast<Meet*>(s_mem);
  float top = s_m[0][c];
#pragma unroll
  for (int i = 1; i < KV4_WAVES; ++i) top = fmaxf(top, s_m[i][c]);
  const float weight = m > -INFINITY ? __builtin_amdgcn_exp2f(m - top) : 0.f;
#pragma unroll
  for (int e = 0; e <= NE; ++e)
    *reinterpret_cast<f4*>(meet[wave][e][lane]) = acc[e] * weight;
  __syncthreads();
  f4 sums[NE / KV4_WAVES], extra{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = 0; n < NE / KV4_WAVES; ++n) {
    sums[n] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KV4_WAVES; ++i) sums[n] += *reinterpret_cast<const f4*>(meet[i][wave * (NE / KV4_WAVES) + n][lane]);
  }
#pragma unroll
  for (int i = 0; i < KV4_WAVES; ++i) extra += *reinterpret_cast<const f4*>(meet[i][NE][lane]);
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < KV4_WAVES; ++i) l += meet[i][NE][c][1];
  __syncthreads();
  typedef float Out[HD + 4];
  Out* out = reinterpret_cast<Out*>(s_mem);
  const float mid = extra[2] != 0.f ? NAN : extra[0];                      // a NaN mark with any weight
  const float inv = splits > 1 ? 1.0f : l != 0.f ? 1.0f / l : 0.f;
#pragma unroll
  for (int n = 0; n < NE / KV4_WAVES; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {                                          // element (HD / 16) (4 h + i) + e
      const int e = (HD / 16) * (4 * h + i) + wave * (NE / KV4_WAVES) + n;
      out[c][e] = (sums[n][i] + mid) * inv;
    }
  __syncthreads();
  if (splits == 1) {
    for (int i = tid; i < 16 * (HD / 8); i += 256) {
      const int row = i / (HD / 8), oct = i % (HD / 8), ff = f0 + row, jj = ff / share_heads;
      if (ff >= rows) break;
      u16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = T::store(out[row][oct * 8 + e]);
      kv4_store8<HD>(o, s.first + jj, w.head * share_heads + ff - jj * share_heads, oct * 8, v);
    }
  } else {
    float* to = part + (size_t)blockIdx.x * 16 * (HD + 2);
    for (int i = tid; i < min(16, rows - f0) * (HD / 4); i += 256) {
      const int row = i / (HD / 4), x = i % (HD / 4);
      *reinterpret_cast<f4*>(to + row * HD + x * 4) = *reinterpret_cast<const f4*>(&out[row][x * 4]);
    }
    if (tid < 16) {
      to[16 * HD + tid] = top;
      to[16 * HD + 16 + tid] = l;
    }
  }
}

// all of a workgroup's waves, without waiting for loads in flight
__device__ __forceinline__ void kv4_barrier() {
  wait_lgkm_at_most<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- one query row a key head ----
//
// A single row leaves fifteen of sixteen columns of the matrix instructions empty, and their operands cost the vector unit more
// than the products themselves: a code takes 1.1 operations for the score (half words set into 1024 + c, as above, then two at
// a time into v_dot2_f32_f16; what 1024 and 64 add up to is taken off in front, as the start of the sum) and 2.1 for the output
// (c - 8, then a multiply-add from a half word to 32 bits).  HD / 32 lanes hold a key, a group of 32 elements each, so that a lane
// has one step and one middle.  All of a wave's lanes share the running maximum; weights stay in 32 bits.
// 32 sequences of 1500 .. 2500 positions of 32 heads: 67 us, 4.9 TB/s of the cache; a kernel that only loads the same bytes in
// this pattern takes 57 .. 60, whatever the loads' width.
#define KV4_ONE_STEPS 2          // keys of a lane in a trip: 4 of them leave registers for three workgroups a CU only (77 -> 79 us)

template <class T, int HD, bool P16, bool NEW>
__global__ __launch_bounds__(256, 4) void kv4_attn_one_kernel(Kv4Pool p, Kv4Rows r, Kv4View q, Kv4View o, Kv4View knew, Kv4View vnew,
                                                              int heads, float scale, int splits, float* part) {
  constexpr int U = KV4_ONE_STEPS, LPK = HD / 32, KPS = 64 / LPK, TRIP = U * KPS, NEXT = KV4_WAVES * TRIP;
  __shared__ float s_acc[KV4_WAVES * 4][HD], s_part[KV4_WAVES * 4][LPK], s_m[KV4_WAVES], s_l[KV4_WAVES];
  __shared__ __attribute__((aligned(16))) u32 s_new[2][HD / 8], s_newp[2][LPK];
  const Kv4Work w = kv4_work(r, blockIdx.x, splits, p.kv_heads, 1);
  const int tid = threadIdx.x, lane = tid & 63, g = lane % LPK;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Kv4Seq s = kv4_seq(r, w.b);
  if (s.rows < 1) return;
  const int n_keys = kv4_keys(p, r, s, 0);
  const int tiles = (n_keys + KV4_TILE - 1) / KV4_TILE, share = kv4_share(tiles, splits);
  const int t0 = w.split * share, end = min((t0 + share) * KV4_TILE, n_keys);
  if (w.split > 0 && t0 >= tiles) return;
  const int* table = r.table + (size_t)w.b * r.table_stride;

  // requested in front of everything that waits for the page table
  u16x8 qin[4], nin{};
#pragma unroll
  for (int n = 0; n < 4; ++n) qin[n] = kv4_load8(q, s.first, w.head, g * 32 + n * 8);
  if (NEW && wave < 2 && lane < HD / 8) nin = kv4_load8(wave ? vnew : knew, s.first, w.head, lane * 8);
  __builtin_amdgcn_sched_barrier(0);

  // pool rows of a trip's keys (or, with P16, of the first of every 16 keys); entries are requested a trip ahead
  constexpr int PER = P16 ? KPS / 16 : 1, ENTRIES = U * PER;
  auto page = [&](int u) { return (int)(__umulhi((u32)u << 1, p.magic) >> p.shift); };
  auto look = [&](int k, u32 (&at)[ENTRIES]) {
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
      const int u = P16 ? k + 16 * i : k + KPS * i + lane / LPK;
      const int* e = table + min(page(u), r.table_stride - 1);
      at[i] = P16 ? (u32)kv4_scalar(e) : (u32)*as_global(e);
    }
  };
  auto place = [&](int k, const u32 (&at)[ENTRIES], int (&row)[ENTRIES]) {      // -1: none
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
      const int u = P16 ? k + 16 * i : k + KPS * i + lane / LPK, pg = page(u);
      row[i] = u < n_keys && pg < r.table_stride && at[i] <= (u32)(p.pool_rows - p.page_tokens) ? (int)(at[i] + (u - pg * p.page_tokens)) : -1;
    }
  };
  const char *kc = kv4_codes<HD>(p, 0, w.head), *kp = kv4_params<HD>(p, 0, w.head);
  const char *vc = kv4_codes<HD>(p, 1, w.head), *vp = kv4_params<HD>(p, 1, w.head);
  auto fetch = [&](const char* codes, const char* params, const int (&row)[ENTRIES], u32x4 (&c)[U], u32 (&par)[U]) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (P16 && PER == 1) {                           // a scalar row, and a lane's place behind it
        const u32 at = max(row[i], 0), x = lane / LPK;
        c[i] = *as_global(reinterpret_cast<const u32x4*>(codes + (size_t)at * (HD / 2) + (x * (HD / 2) + g * 16)));
        par[i] = *as_global(reinterpret_cast<const u32*>(params + (size_t)at * (HD / 8) + (x * (HD / 8) + g * 4)));
      } else {
        const int first = row[i * PER], last = row[i * PER + PER - 1];
        const u32 at = P16 ? (u32)max(lane & 32 ? last : first, 0) + (lane / LPK & 15) : (u32)max(first, 0);
        c[i] = *as_global(reinterpret_cast<const u32x4*>(codes + (size_t)(at * (HD / 2) + g * 16)));
        par[i] = *as_global(reinterpret_cast<const u32*>(params + (size_t)(at * (HD / 8) + g * 4)));
      }
    }
  };
  // which of the lane's keys exist (a bit each)
  auto exist = [&](int k, const int (&row)[ENTRIES]) {
    u32 m = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int first = row[i * PER], last = row[i * PER + PER - 1], at = PER == 2 && (lane & 32) ? last : first;
      if (at >= 0 && k + KPS * i + lane / LPK < end) m |= 1u << i;
    }
    return m;
  };
  u32x4 kk[U], vv[U];
  u32 kq[U], vq[U], at[ENTRIES];
  u32 has = 0;
  int k = t0 * KV4_TILE + wave * TRIP;
  if (k < end) {
    u32 now[ENTRIES];
    int row[ENTRIES];
    look(k, now);
    look(k + NEXT, at);
    place(k, now, row);
    has = exist(k, row);
    fetch(kc, kp, row, kk, kq);
    fetch(vc, vp, row, vv, vq);
  }

  // The lane's group of the query, in the order in which codes unpack, scaled by a power of two to a largest element of
  // 2^14 .. 2^15 (far from binary16's subnormal numbers, which the product may pass over)
  h2 qf[16];
  float qsum = 0.f, start = 0.f, qscale;
  {
    float x[32], top = 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[8 * n + i] = T::load(qin[n][i]);
        top = fmaxf(top, fabsf(x[8 * n + i]));
      }
    }
    top = fmaxf(top, dpp_mov<0xB1>(top));
    if (LPK == 4) top = fmaxf(top, dpp_mov<0x4E>(top));
    const int e = top > 0.f && top < INFINITY ? ilogbf(top) - 14 : 0;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const half_t a = (half_t)ldexpf(x[8 * n + i], -e), b = (half_t)ldexpf(x[8 * n + i + 4], -e);
        qf[4 * n + i] = h2{a, b};
        const float ab = (float)a + (float)b;
        qsum += ab;
        start -= ab * (i & 1 ? 72.f : 1032.f);
      }
    qscale = fmaxf(ldexpf(scale * 1.44269504088896340736f, e), 0x1p-126f);
  }
  const int pnew = NEW ? s.len - s.rows : -1;
  const bool mine = NEW && pnew >= t0 * KV4_TILE && pnew < end;
  if (mine) {
    if (wave < 2 && lane < HD / 8) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = T::load(nin[i]);
      u32 param;
      const u32 code = kv4_quantise(x, param);
      s_new[wave][lane] = code;
      s_newp[wave][lane >> 2] = param;
      const int to = kv4_row(p, table, r.table_stride, pnew);
      if (to >= 0) {
        *(u32*)(kv4_codes<HD>(p, wave, w.head) + (size_t)to * (HD / 2) + lane * 4) = code;
        if (lane % 4 == 0) *(u32*)(kv4_params<HD>(p, wave, w.head) + (size_t)to * (HD / 8) + lane) = param;
      }
    }
    kv4_barrier();
  }

  const Kv4Bits bits;
  float acc[32], sum_mid = 0.f, l = 0.f, m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[i] = 0.f;
  for (; k < end; k += NEXT) {
    const bool more = k + NEXT < end;
    int row[ENTRIES];
    u32 has_next = 0;
    if (more) {
      place(k + NEXT, at, row);
      has_next = exist(k + NEXT, row);
      look(k + 2 * NEXT, at);
    }
    const bool fresh = mine && pnew >= k && pnew < k + TRIP;
    const int fresh_step = (pnew - k) / KPS, fresh_lane = (pnew - k) % KPS;
    if (fresh && lane / LPK == fresh_lane) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (i == fresh_step) {
          kk[i] = *reinterpret_cast<const u32x4*>(&s_new[0][4 * g]);
          kq[i] = s_newp[0][g];
          vv[i] = *reinterpret_cast<const u32x4*>(&s_new[1][4 * g]);
          vq[i] = s_newp[1][g];
        }
    }
    float x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float dot = start;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const u32 c = kk[i][n], y = c >> 8;
        dot = __builtin_amdgcn_fdot2(kv4_h2((c & bits.low) | bits.k1024), qf[4 * n], dot, false);
        dot = __builtin_amdgcn_fdot2(kv4_h2((c & bits.high) | bits.k64), qf[4 * n + 1], dot, false);
        dot = __builtin_amdgcn_fdot2(kv4_h2((y & bits.low) | bits.k1024), qf[4 * n + 2], dot, false);
        dot = __builtin_amdgcn_fdot2(kv4_h2((y & bits.high) | bits.k64), qf[4 * n + 3], dot, false);
      }
      const h2 par = kv4_h2(kq[i]);
      float t = fmaf((float)par[0], dot, (float)par[1] * qsum);
      t += dpp_mov<0xB1>(t);
      if (LPK == 4) t += dpp_mov<0x4E>(t);
      x[i] = t * qscale;
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) fetch(kc, kp, row, kk, kq);
    if (__any(has != (1u << U) - 1)) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (!(has >> i & 1)) {                         // no weight, and nothing that a weight of zero could meet
          x[i] = -INFINITY;
          vq[i] = 0;
        }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < U; ++i) top = fmaxf(top, x[i]);
    if (LPK == 2) top = fmaxf(top, dpp_mov<0x4E>(top));
    top = fmaxf(top, dpp_mov<0x124>(top));             // row_ror:4, row_ror:8: a row of 16 lanes
    top = fmaxf(top, dpp_mov<0x128>(top));
    top = fmaxf(kv4_max_over_quarters(top), m);
    if (top > m) {                                     // the same for all lanes
      const float corr = __builtin_amdgcn_exp2f(m - top);
      m = top;
      l *= corr;
      sum_mid *= corr;
#pragma unroll
      for (int i = 0; i < 32; ++i) acc[i] *= corr;
    }
    const float base = m > -INFINITY ? m : 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float w1 = __builtin_amdgcn_exp2f(x[i] - base);
      const h2 par = kv4_h2(vq[i]);
      const float ws = w1 * (float)par[0];
      l += w1;
      sum_mid = fmaf(w1, (float)par[1], sum_mid);
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        h2 d[4];
        bits.unpack(vv[i][n], d);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[8 * n + e] = fmaf(ws, (float)d[e][0], acc[8 * n + e]);
          acc[8 * n + e + 4] = fmaf(ws, (float)d[e][1], acc[8 * n + e + 4]);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) fetch(vc, vp, row, vv, vq);
    has = has_next;
  }

  // the lanes of a group within rows of 16 lanes, then the rows of all waves, meet
  if (lane == 0) s_m[wave] = m;
  __syncthreads();
  float top = s_m[0];
#pragma unroll
  for (int i = 1; i < KV4_WAVES; ++i) top = fmaxf(top, s_m[i]);
  const float weight = m > -INFINITY ? __builtin_amdgcn_exp2f(m - top) : 0.f;
  auto row_sum = [&](float v) {
    if (LPK == 2) v += dpp_mov<0x4E>(v);
    v += dpp_mov<0x124>(v);
    return v + dpp_mov<0x128>(v);
  };
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[i] = row_sum(acc[i] * weight);
  sum_mid = row_sum(sum_mid * weight);
  l = row_sum(l * weight);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lane == 0) s_l[wave] = l;
  if ((lane & 15) < LPK) {
    const int at_row = wave * 4 + (lane >> 4);
    s_part[at_row][g] = sum_mid;
#pragma unroll
    for (int n = 0; n < 8; ++n)
      *reinterpret_cast<f4*>(&s_acc[at_row][g * 32 + n * 4]) = f4{acc[4 * n], acc[4 * n + 1], acc[4 * n + 2], acc[4 * n + 3]};
  }
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < KV4_WAVES; ++i) l += s_l[i];
  if (tid < HD) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < KV4_WAVES * 4; ++i) v += s_acc[i][tid] + s_part[i][tid / 32];
    if (splits == 1) *kv4_element<HD>(o, s.first, w.head, tid) = T::store(l != 0.f ? v / l : 0.f);
    else part[(size_t)blockIdx.x * KV4_FEW_ROWS * (HD + 2) + tid] = v;
  }
  if (splits > 1 && tid == 0) {
    float* to = part + (size_t)blockIdx.x * KV4_FEW_ROWS * (HD + 2) + KV4_FEW_ROWS * HD;
    to[0] = top;
    to[KV4_FEW_ROWS] = l;
  }
}

// ---- many query rows ----
//
// 256 query rows of one key head, 32 a wave.  Here the products count, and the 32x32x16 form has the higher rate; codes are
// turned into operands once for all eight waves, as fragments in LDS, 16 bytes a lane and side by side as the waves read them:
// waves 0 .. 3 make 32 keys each of a tile of 128, waves 4 .. 7 their values.  LDS holds two tiles, so that one barrier a tile
// is enough, and the makers of keys do so in front of their products, those of values behind them: a SIMD has one wave of
// either kind, whose vector and matrix instructions then overlap.  With lane = 32 h + c, a product's rows and columns c and its
// contraction 8 h + i, the operands follow the same ideas as above:
//  * K: half h of key c's row, 8 elements a product, and a product of the middles (two groups a half with head_dim 128);
//  * S^T leaves the lane with keys 8 a + 4 h + b (a, b < 4) of query c; product n of V^T P^T contracts over a = 2 n and 2 n + 1;
//  * V: row c of block e is element (HD / 32) c + e, and the lane's outputs are HD / 8 elements in a row for every a, of group a
//    (head_dim 64: a / 2).  Rows of the further block: 4 x the group's middle, 4 x + 1 ones, 4 x + 2 the group's NaN marks.
// Weights enter as one binary16 number here: a relative 2^-11 each, independent of the others', as large as a binary16 output's
// own rounding; a second one would be another KV4_MANY_ROWS x keys x head_dim product.
// 1024 rows of 32 heads behind 7169 positions: 190 us and a join of 12, 0.64 PFLOP/s of 1.15 that a large library product
// reaches; blocks of 128 rows took 205.  The vector unit (weights, operands) is busy 44 % of the time, the matrix cores
// 32 %, and a wave reads 19 KB of LDS for 32 keys; they overlap only across a SIMD's two waves.  64 rows a wave, which would
// halve the LDS reads, needs more than a lane's 512 registers: 532 us with the spills.
#define KV4_MANY_ROWS 256
#define KV4_MANY_WAVES 8

__device__ __forceinline__ f16v kv4_mfma(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float kv4_max_over_halves(float v) {
  const u32 b = __builtin_bit_cast(u32, v);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__builtin_bit_cast(float, (u32)r[0]), __builtin_bit_cast(float, (u32)r[1]));
}
template <int HD>
struct Kv4Operands {
  static constexpr int KS = HD / 16, NE = HD / 32;            // products of a score; row blocks of elements
  static constexpr int FRAGS = KS + 1 + 2 * (NE + 1);         // fragments of 32 keys
};

template <class T, int HD, bool P16>
__global__ __launch_bounds__(KV4_MANY_WAVES * 64, 2) void kv4_attn_many_kernel(Kv4Pool p, Kv4Rows r, Kv4View q, Kv4View o, int heads,
                                                                               float scale, int splits, int row_blocks, float* part) {
  using Op = Kv4Operands<HD>;
  constexpr int KS = Op::KS, NE = Op::NE;
  __shared__ __attribute__((aligned(16))) h8 s_frag[2][KV4_WAVES][Op::FRAGS][64];
  __shared__ __attribute__((aligned(16))) u32 s_rows[P16 ? 1 : KV4_MANY_WAVES][KV4_TILE];
  __shared__ u32 s_has[2][KV4_WAVES];
  Kv4Work w = kv4_work(r, blockIdx.x, splits, p.kv_heads, row_blocks);
  w.rb = row_blocks - 1 - w.rb;                                            // the longest first
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int sub = wave & 3;                                                // the wave makes the operands of this part of a tile
  const bool makes_keys = wave < 4;
  const Kv4Seq s = kv4_seq(r, w.b);
  const int share_heads = heads / p.kv_heads, rows = min(s.rows, r.max_rows) * share_heads;
  const int f0 = w.rb * KV4_MANY_ROWS;
  if (f0 >= rows) return;
  const int n_keys = kv4_keys(p, r, s, min(f0 + KV4_MANY_ROWS - 1, rows - 1) / share_heads);
  const int tiles = (n_keys + KV4_TILE - 1) / KV4_TILE, share = kv4_share(tiles, splits);
  const int t0 = w.split * share, t1 = min(t0 + share, tiles);
  if (w.split > 0 && t0 >= tiles) return;
  const int* table = r.table + (size_t)w.b * r.table_stride;

  const int fw = f0 + wave * 32, f = fw + c, j = f / share_heads, qhead = w.head * share_heads + f - j * share_heads;
  const bool there = f < rows;
  const int limit = there ? s.len - s.rows + j : -1;
  const int first_limit = s.len - s.rows + fw / share_heads;               // of the wave's queries
  const int last_limit = fw < rows ? s.len - s.rows + min(fw + 31, rows - 1) / share_heads : -1;

  // Pool rows of the wave's part (32 keys) of a tile
  const int ahead = P16 ? 0 : c;
  auto page = [&](int u) { return (int)(__umulhi((u32)u << 1, p.magic) >> p.shift); };
  auto look = [&](int t) {
    const int last = r.table_stride - 1, u = t * KV4_TILE + ahead;
    if constexpr (P16) return u32x2{(u32)kv4_scalar(table + min(page(u), last)), (u32)kv4_scalar(table + min(page(u + 16), last))};
    else return u32x2{(u32)*as_global(table + min(page(u), last)), 0};
  };
  auto row = [&](int u, u32 at) {
    const int pg = page(u);
    return u < n_keys && pg < r.table_stride && at <= (u32)(p.pool_rows - p.page_tokens) ? (int)(at + (u - pg * p.page_tokens)) : -1;
  };
  auto place = [&](int t, u32x2 at, u32& has) {
    const int u = t * KV4_TILE + ahead;
    if constexpr (P16) {
      const int a = row(u, at[0]), b = row(u + 16, at[1]);
      const u32 one = a >= 0 ? 0xffffu >> max(u + 16 - n_keys, 0) : 0u, two = b >= 0 ? 0xffffu >> max(u + 32 - n_keys, 0) : 0u;
      has = one | two << 16;
      return Kv4Halves{u32x2{(u32)max(a, 0), (u32)max(b, 0)}};
    } else {
      const int a = row(u, at[0]);
      has = (u32)__ballot(a >= 0);
      s_rows[wave][ahead] = max(a, 0);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      return Kv4Listed{s_rows[wave]};
    }
  };
  // 32 keys as they lie in the pool: half h of key c's row; or the lane's HD / 32 elements of 16 values
  u32 raw[32];               // K: codes, then 2 parameters; V: codes, then parameters (the same registers for either)
  u32 has = 0;
  auto fetch = [&](const auto& where) {
    const char *codes = kv4_codes<HD>(p, makes_keys ? 0 : 1, w.head), *params = kv4_params<HD>(p, makes_keys ? 0 : 1, w.head);
    if (makes_keys) {
      const char* a = where.split(codes, HD / 2, c) + h * (HD / 4);
#pragma unroll
      for (int n = 0; n < HD / 64; ++n) {
        const u32x4 x = *as_global(reinterpret_cast<const u32x4*>(a + 16 * n));
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[4 * n + i] = x[i];
      }
      const char* b = where.split(params, HD / 8, c) + h * (HD / 16);
      raw[8] = *as_global(reinterpret_cast<const u32*>(b));
      if (HD == 128) raw[9] = *as_global(reinterpret_cast<const u32*>(b + 4));
    } else {
#pragma unroll
      for (int n = 0; n < 16; ++n) {                   // key 16 (n / 8) + 8 (n / 4 % 2) + 4 h + n % 4
        const u32 i = 8 * (n >> 2 & 1) + 4 * h + (n & 3);
        const char* x = where.at(codes, HD / 2, n >> 3, i) + c * (HD / 64);
        raw[n] = HD == 128 ? (u32)*as_global(reinterpret_cast<const u16*>(x)) : (u32)*as_global(reinterpret_cast<const unsigned char*>(x));
        raw[16 + n] = *as_global(reinterpret_cast<const u32*>(where.at(params, HD / 8, n >> 3, i) + (c * (HD / 32) / KV4_GROUP) * 4));
      }
    }
  };
  const Kv4Bits bits;
  const u32 mid_row = (c & 3) == 0 ? ~0u : 0u, one_row = (c & 3) == 1 ? 0x3c003c00u : 0u;
  // 32 keys as fragments: K's KS, their middles, then for either half of the keys V's NE and theirs
  auto produce = [&](int buf) {
    h8(*out)[64] = s_frag[buf][sub];
    if (makes_keys) {
#pragma unroll
      for (int n = 0; n < KS; ++n) {
        const u32 g = raw[8 + (HD == 128 ? n >> 2 : 0)];
        const h2 step = kv4_h2(kv4_lo16(g, g));
        h2 d[4];
        bits.unpack(raw[n], d);
        out[n][lane] = __builtin_bit_cast(h8, u32x4{kv4_u32(d[0] * step), kv4_u32(d[1] * step), kv4_u32(d[2] * step), kv4_u32(d[3] * step)});
      }
      const half_t m0 = kv4_h2(raw[8])[1], m1 = HD == 128 ? kv4_h2(raw[9])[1] : (half_t)0;
      out[KS][lane] = h8{m0, m0, m0, m1, m1, m1, 0, 0};
      if (lane == 0) s_has[buf][sub] = has;
      return;
    }
    u32 marks = 0;
    h2 all = kv4_h2(raw[16]);
#pragma unroll
    for (int n = 1; n < 16; ++n) all += kv4_h2(raw[16 + n]);
    if (~has || __any(!(all[1] == all[1]))) {
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        const half_t mid = kv4_h2(raw[16 + n])[1];
        const int key = 16 * (n >> 3) + 8 * (n >> 2 & 1) + 4 * h + (n & 3);
        const bool gone = !(has >> key & 1), nan = !(mid == mid);
        if (nan && !gone) marks |= 1u << n;
        if (gone || nan) raw[16 + n] = 0;
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u32x4 w4[4], mids;
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int n = 8 * t + 2 * a;
        const h2 step = kv4_h2(kv4_lo16(raw[16 + n], raw[17 + n]));
        h2 d[4];
        bits.unpack(raw[n] | raw[n + 1] << 16, d);
#pragma unroll
        for (int i = 0; i < NE; ++i) w4[i][a] = kv4_u32(d[i] * step);
        mids[a] = (kv4_hi16(raw[16 + n], raw[17 + n]) & mid_row) | one_row;
      }
      if (__any(marks)) {
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int n = 8 * t + 2 * a;
          const u32 mark = (marks >> n & 1 ? 0x3c00u : 0u) | (marks >> (n + 1) & 1 ? 0x3c000000u : 0u);
          mids[a] = (c & 3) == 2 ? mark : mids[a];
        }
      }
#pragma unroll
      for (int i = 0; i < NE; ++i) out[KS + 1 + t * (NE + 1) + i][lane] = __builtin_bit_cast(h8, w4[i]);
      out[KS + 1 + t * (NE + 1) + NE][lane] = __builtin_bit_cast(h8, mids);
    }
  };

  u32x2 at{0, 0};
  if (t0 < t1) {
    const u32x2 at0 = look(t0 + sub);
    at = look(t0 + KV4_WAVES + sub);
    fetch(place(t0 + sub, at0, has));
  }
  // queries, in K's order and scaled as above
  h8 qf[KS], sums;
  float qscale;
  {
    float x[KS][8], top = 0.f;
#pragma unroll
    for (int n = 0; n < KS; ++n) {
      u16x8 in{};
      if (there) in = kv4_load8(q, s.first + j, qhead, h * (HD / 2) + n * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[n][i] = T::load(in[i]);
        top = fmaxf(top, fabsf(x[n][i]));
      }
    }
    top = kv4_max_over_halves(top);
    int e = 0;
    if (top > 0.f && top < INFINITY) e = ilogbf(top);
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < KS; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const half_t a = (half_t)ldexpf(x[n][i], -e), b = (half_t)ldexpf(x[n][i + 4], -e);
        qf[n][2 * i] = a;
        qf[n][2 * i + 1] = b;
        sum[n >> 2] += (float)a + (float)b;
      }
    half_t y[2][3];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      y[g][0] = (half_t)sum[g];
      y[g][1] = (half_t)(sum[g] - (float)y[g][0]);
      y[g][2] = (half_t)(sum[g] - (float)y[g][0] - (float)y[g][1]);
    }
    sums = h8{y[0][0], y[0][1], y[0][2], y[1][0], y[1][1], y[1][2], 0, 0};
    qscale = fmaxf(ldexpf(scale * 1.44269504088896340736f, e), 0x1p-126f);
  }

  f16v acc[NE + 1];
#pragma unroll
  for (int e = 0; e <= NE; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[e][i] = 0.f;
  float m = -INFINITY;
  // the next tile's operands into the other buffer, and the request for the one behind it
  auto prepare = [&](int t, int buf) {
    produce(buf);
    if (t + KV4_WAVES < t1) {
      const u32x2 now = at;
      at = look(t + 2 * KV4_WAVES + sub);
      fetch(place(t + KV4_WAVES + sub, now, has));
    }
  };
  if (t0 < t1) prepare(t0, 0);
  kv4_barrier();
  for (int t = t0, buf = 0; t < t1; t += KV4_WAVES, buf ^= 1) {
    const bool more = t + KV4_WAVES < t1;
    if (makes_keys && more) prepare(t + KV4_WAVES, buf ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    for (int n = 0; n < KV4_WAVES; ++n) {
      const int u0 = (t + n) * KV4_TILE;
      if (u0 > last_limit || u0 >= n_keys) break;
      const u32 there_mask = __builtin_amdgcn_readfirstlane(s_has[buf][n]);
      const h8(*in)[64] = s_frag[buf][n];
      f16v sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
      sc = kv4_mfma(in[KS][lane], sums, sc);
#pragma unroll
      for (int i = 0; i < KS; ++i) sc = kv4_mfma(in[i][lane], qf[i], sc);
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = sc[i] * qscale;
      if (u0 + KV4_TILE - 1 > first_limit || ~there_mask) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 8 * (i >> 2) + 4 * h + (i & 3);
          if (!(there_mask >> key & 1) || u0 + key > limit) x[i] = -INFINITY;
        }
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
      top = fmaxf(kv4_max_over_halves(top), m);
      if (__any(top > m)) {
        const float corr = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
        m = top;
#pragma unroll
        for (int e = 0; e <= NE; ++e) acc[e] *= corr;
      }
      const float base = KV4_SHIFT - (m > -INFINITY ? m : 0.f);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        h8 pr;
#pragma unroll
        for (int i = 0; i < 8; ++i) pr[i] = (half_t)__builtin_amdgcn_exp2f(x[8 * k + i] + base);
#pragma unroll
        for (int e = 0; e <= NE; ++e) acc[e] = kv4_mfma(in[KS + 1 + k * (NE + 1) + e][lane], pr, acc[e]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!makes_keys && more) prepare(t + KV4_WAVES, buf ^ 1);
    kv4_barrier();
  }

  // outputs: element (HD / 32) (8 a + 4 h + b) + e is register 4 a + b of block e
  if (!there) return;
  const float l = acc[NE][1], inv = splits > 1 ? 1.0f : l != 0.f ? 1.0f / l : 0.f;
  float* to = part + (size_t)blockIdx.x * KV4_MANY_ROWS * (HD + 2);
  const int at_row = wave * 32 + c;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const float mid = acc[NE][4 * a + 2] != 0.f ? NAN : acc[NE][4 * a];
    float y[HD / 8];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int e = 0; e < NE; ++e) y[b * NE + e] = (acc[e][4 * a + b] + mid) * inv;
    const int e0 = (HD / 32) * (8 * a + 4 * h);
#pragma unroll
    for (int n = 0; n < HD / 64; ++n) {
      if (splits == 1) {
        u16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = T::store(y[8 * n + i]);
        kv4_store8<HD>(o, s.first + j, qhead, e0 + 8 * n, v);
      } else {
        *reinterpret_cast<f4*>(to + at_row * HD + e0 + 8 * n) = f4{y[8 * n], y[8 * n + 1], y[8 * n + 2], y[8 * n + 3]};
        *reinterpret_cast<f4*>(to + at_row * HD + e0 + 8 * n + 4) = f4{y[8 * n + 4], y[8 * n + 5], y[8 * n + 6], y[8 * n + 7]};
      }
    }
  }
  if (splits > 1 && h == 0) {
    to[KV4_MANY_ROWS * HD + at_row] = m;
    to[KV4_MANY_ROWS * HD + KV4_MANY_ROWS + at_row] = l;
  }
}

// The shares of a query row together: a wave a row (of many rows: four), a lane a share for the weights, then HD / 64 elements a
// lane.  grid = (kv_heads * row blocks * sequences, ROWS / 4 / rows of a wave).
// Rows of a block that the sequence has not got are read, within the block's part, and not used.
// Bound by its chain (place, shares' maxima, store) and, for many rows, by the instructions around 16 bytes a lane: 32768 rows
// of 2 shares, 34 MB, 12 us (a wave a row, requested in front of the weights 18.6, behind them 20.4); 128 rows of 16 shares 4.7
// (a workgroup a row block: 10.5).
#define KV4_JOIN_ROWS(block) ((block) > KV4_FEW_ROWS ? 4 : 1)
template <class T, int HD, int ROWS>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4Pool p, Kv4Rows r, Kv4View o, int heads, int splits, int row_blocks,
                                                       const float* part) {
  typedef float vec __attribute__((ext_vector_type(HD / 64)));
  constexpr size_t PART = ROWS * (HD + 2);
  constexpr int R = KV4_JOIN_ROWS(ROWS), B = ROWS > KV4_FEW_ROWS ? 2 : 16;      // rows of a wave, shares requested at once
  Kv4Work w = kv4_work(r, blockIdx.x, 1, p.kv_heads, row_blocks);
  if (ROWS > KV4_FEW_ROWS) w.rb = row_blocks - 1 - w.rb;
  const Kv4Seq s = kv4_seq(r, w.b);
  const int share_heads = heads / p.kv_heads, rows = min(s.rows, r.max_rows) * share_heads;
  const int lane = threadIdx.x & 63, row0 = (blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * R;
  const int f0 = w.rb * ROWS;
  if (f0 + row0 >= rows) return;
  const int n_keys = kv4_keys(p, r, s, min(f0 + ROWS - 1, rows - 1) / share_heads);
  const int tiles = (n_keys + KV4_TILE - 1) / KV4_TILE, share = kv4_share(tiles, splits);
  const int n = tiles ? (tiles + share - 1) / share : 1;
  const float* from = part + (size_t)blockIdx.x * splits * PART;
  vec v[R][B], a[R];
  float m[R], weight[R], inv[R];
  auto load = [&](int k) {
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
      for (int i = 0; i < B; ++i)
        v[q][i] = *as_global(reinterpret_cast<const vec*>(from + (row0 + q) * HD + lane * (HD / 64) + min(k + i, n - 1) * PART));
  };
#pragma unroll
  for (int q = 0; q < R; ++q) {
    m[q] = lane < n ? from[lane * PART + ROWS * HD + row0 + q] : -INFINITY;
    inv[q] = lane < n ? from[lane * PART + ROWS * HD + ROWS + row0 + q] : 0.f;
  }
  load(0);
#pragma unroll
  for (int q = 0; q < R; ++q) {
    float top = m[q];
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    weight[q] = m[q] > -INFINITY ? __builtin_amdgcn_exp2f(m[q] - top) : 0.f;
    const float sum = wave_sum(weight[q] * inv[q]);
    inv[q] = sum != 0.f ? 1.0f / sum : 0.f;
    a[q] = vec{};
  }
  for (int k = 0;;) {
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
      for (int i = 0; i < B; ++i)
        if (k + i < n) a[q] += v[q][i] * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight[q]), k + i));
    if ((k += B) >= n) break;
    load(k);
  }
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int f = f0 + row0 + q, j = f / share_heads;
    if (f >= rows) break;
    u16* to = kv4_element<HD>(o, s.first + j, w.head * share_heads + f - j * share_heads, lane * (HD / 64));
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) to[i] = T::store(a[q][i] * inv[q]);
  }
}
