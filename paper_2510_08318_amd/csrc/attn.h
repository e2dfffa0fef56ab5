// Softmax attention with a sliding window and first tokens that stay visible, over token tensors (linattn_window_*) and over a
// paged cache (linattn_cache_*): what the host dispatch and the kernels agree on.
#pragma once
#include "kernels.h"

namespace linattn {
namespace attn {

// Which keys the query at position p sees of a sequence of `len` tokens: j < len, j <= p + right (right >= 0), and j >= p - left
// (left >= 0) or j < sinks.  As ranges: the first tokens [0, first) and the window [lo, hi), first <= lo.
// left, right: -1 (no limit) or below 2^30; positions below 2^30, so that the sums fit 32 bits.
struct Sight {
  int left, right, sinks;
};
__host__ __device__ inline int key_lo(const Sight& s, int p) { return s.left < 0 || p < s.left ? 0 : p - s.left; }
__host__ __device__ inline int key_hi(const Sight& s, int p, int len) { return s.right < 0 || p + s.right >= len ? len : p + s.right + 1; }
__host__ __device__ inline bool sees(const Sight& s, int p, int j, int len) {
  return j < len && (s.right < 0 || j <= p + s.right) && (s.left < 0 || j >= p - s.left || j < s.sinks);
}
// The queries that see key j: [query_lo, query_hi).
__host__ __device__ inline int query_lo(const Sight& s, int j) { return s.right < 0 || j < s.right ? 0 : j - s.right; }
__host__ __device__ inline int query_hi(const Sight& s, int j, int len) {
  return s.left < 0 || j < s.sinks || j + s.left >= len ? len : j + s.left + 1;
}

__host__ __device__ inline int clamp_length(const int* lengths, int b, int n) {
  if (!lengths) return n;
  const int x = lengths[b];
  return x < 0 ? 0 : x < n ? x : n;
}

// One call of linattn_window_fwd / linattn_window_bwd.
struct WindowArgs {
  const void *q, *k, *v, *out, *dout;
  void *o, *dq, *dk, *dv;
  float* lse;               // written by the forward, read by the backward
  float* delta;             // fp32 [B*H][n], workspace of the backward
  const int* lengths;       // nullable
  int B, H, HK, n, d;
  Rows qr, kr;              // rows of q, out, dout, dq and of k, v, dk, dv
  Sight sight;
  float scale;
  hipStream_t stream;
};

// The pool of a paged cache and who owns which page.  Rows are [pages][HK][page][d].
struct Pool {
  void *k, *v;
  uint8_t *k_exp, *v_exp;   // e4m3: biased exponent of a row's scale, [pages][HK][page]
  const int* table;         // [B][width]
  const int* lengths;       // [B]
  const int* counts;        // [B], nullable
  int B, HK, d, page, pages, width;
  uint32_t magic, shift;    // of page_of
};
// Division by a page size that only the call knows: m = ceil(2^(31 + s) / page), s = ceil(log2(page)), gives the quotient of every j
// below 2^31 as (j * m) >> (31 + s), and m is below 2^32.
inline void set_divisor(Pool* p) {
  uint32_t s = 0;
  while ((1u << s) < (uint32_t)p->page) ++s;
  p->shift = s;
  p->magic = (uint32_t)((((uint64_t)1 << (31 + s)) + p->page - 1) / p->page);
}
__host__ __device__ inline int page_of(const Pool& p, int j) { return (int)(((uint64_t)(uint32_t)j * p.magic) >> (31 + p.shift)); }
// Row of key j of sequence b in the pool, in rows of one head: -1 where the table names no page of the pool.  j >= 0.
__device__ __forceinline__ long long pool_row(const Pool& p, int b, int h, int j) {
  const int i = page_of(p, j);
  const int at = i < p.width ? p.table[(size_t)b * p.width + i] : -1;
  if ((unsigned)at >= (unsigned)p.pages) return -1;
  return ((long long)at * p.HK + h) * p.page + (j - i * p.page);
}
__device__ __forceinline__ int pool_length(const Pool& p, int b) { return clamp_length(p.lengths, b, p.width * p.page); }

// One call of linattn_cache_attn.
struct CacheArgs {
  Pool pool;
  const void* q;
  void* o;
  float* lse;               // nullable
  float* work;
  int H, n;
  Rows qr;
  Sight sight;
  float scale;
  hipStream_t stream;
};

hipError_t launch_window_fwd(const WindowArgs& a, int dtype);
hipError_t launch_window_bwd(const WindowArgs& a, int dtype);
hipError_t launch_cache_write(const Pool& p, bool e4m3, const void* k, const void* v, int n, const Rows& r, hipStream_t s);
hipError_t launch_cache_read(const Pool& p, bool e4m3, void* k, void* v, int n, const Rows& r, hipStream_t s);
hipError_t launch_cache_attn(const CacheArgs& a, bool e4m3);

}  // namespace attn
}  // namespace linattn
