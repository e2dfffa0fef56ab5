// Rows of a paged cache's pool: e4m3 codes and exponents, and access by key.
// A quantised row is e4m3 codes and one exponent: x ~ code 2^e, e the least integer with max|x| 2^-e <= 448 and at least kLeastExp.  With a power of
// two for a scale the codes' rounding is the only one: code 2^e has 4 significant bits and (e >= kLeastExp) the exponent of a normal bf16, so
// that what is read back, as bf16 or by the attention, is the same value without another rounding.
#pragma once
#include "attn_plain.h"

namespace linattn {
namespace attn {

constexpr int kExpBias = 127;
constexpr int kMostExp = 120;         // of rows with entries from 448 2^119 on
constexpr int kLeastExp = -117;      // 2^-9, the smallest code, times 2^-117 is 2^-126, the smallest normal bf16

__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }      // -126 <= e <= 127
__device__ __forceinline__ float row_scale(uint8_t byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }      // 2^e of a stored exponent

// Four codes -> values times s.
__device__ __forceinline__ void decode4(uint32_t codes, float s, float* f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  f[0] = lo[0] * s; f[1] = lo[1] * s; f[2] = hi[0] * s; f[3] = hi[1] * s;
}
// Eight codes -> eight bf16, times the power of two s (exact).
__device__ __forceinline__ uint4 decode8(uint2 c, float s) {
  auto two = [&](uint32_t w, auto hi) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, s, decltype(hi)::value)); };
  return make_uint4(two(c.x, std::false_type{}), two(c.x, std::true_type{}), two(c.y, std::false_type{}), two(c.y, std::true_type{}));
}

// Rows of one head of the pool, for the sequence b.
template <bool E4M3>
struct PoolKeys {
  const Pool* pool;
  int b, h, d;
  __device__ __forceinline__ bool there(int j) const { return pool_row(*pool, b, h, j) >= 0; }
  __device__ __forceinline__ void row8(const void* base, const uint8_t* exps, int j, int c, float* f) const {
    const long long r = pool_row(*pool, b, h, j);
    if constexpr (E4M3) {
      const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(base) + r * d + c);
      const float s = row_scale(exps[r]);
      decode4(x.x, s, f); decode4(x.y, s, f + 4);
    } else load8(static_cast<const uint16_t*>(base) + r * d + c, f);
  }
  __device__ __forceinline__ float row1(const void* base, const uint8_t* exps, int j, int c) const {
    const long long r = pool_row(*pool, b, h, j);
    if constexpr (E4M3) {
      float f[4];
      decode4(static_cast<const uint8_t*>(base)[r * d + c], row_scale(exps[r]), f);
      return f[0];
    } else return f32::ldf(static_cast<const uint16_t*>(base), (size_t)(r * d + c));
  }
  __device__ __forceinline__ void k8(int j, int c, float* f) const { row8(pool->k, pool->k_exp, j, c, f); }
  __device__ __forceinline__ void v8(int j, int c, float* f) const { row8(pool->v, pool->v_exp, j, c, f); }
  __device__ __forceinline__ float k1(int j, int c) const { return row1(pool->k, pool->k_exp, j, c); }
  __device__ __forceinline__ float v1(int j, int c) const { return row1(pool->v, pool->v_exp, j, c); }
};

// The pool's rows of a tile's keys, lane by lane (key j0 + lane, the last key again from `end` on): a row, and which keys have one.  A key without a page takes the row of
// the tile's first key that has one: its weight is 0, and 0 times an infinity or NaN in some other sequence's row, or in one that was never written, would have
// the queries' rows done again key by key.  (A tile in which no key has a page is not looked at.)
// The table is read through the scalar cache, an entry at a time (a tile has two pages at most where they are no smaller): a vector load's answer could not be
// waited for without all the loads that were asked for before it, a tile that is on its way among them.
struct PoolRows {
  long long row;           // of this lane's key
  unsigned long long there;
  template <int KT>
  __device__ __forceinline__ void find(const Pool& p, int b, int h, int j0, int end, int lane) {
    const int last = j0 + KT < end ? j0 + KT - 1 : end - 1, j = j0 + lane < last ? j0 + lane : last, mine = page_of(p, j);
    typedef __attribute__((address_space(4))) const int* Table;
    const Table table = (Table)(uintptr_t)p.table;
    const int i1 = __builtin_amdgcn_readfirstlane(page_of(p, last));
    int entry = -1;
    for (int i = __builtin_amdgcn_readfirstlane(page_of(p, j0)); i <= i1; ++i) {
      const int e = table[(size_t)b * p.width + i];
      entry = mine == i ? e : entry;
    }
    const bool ok = (unsigned)entry < (unsigned)p.pages;
    there = __ballot(ok);
    row = ok ? ((long long)entry * p.HK + h) * p.page + (j - mine * p.page) : 0;
    if (there != ~0ull && there != 0) {
      const long long other = of(__ffsll(there) - 1);
      row = ok ? row : other;
    }
  }
  __device__ __forceinline__ long long of(int i) const {
    return (long long)((unsigned long long)(uint32_t)__shfl((int)row, i) | (unsigned long long)(uint32_t)__shfl((int)(row >> 32), i) << 32);
  }
};

}  // namespace attn
}  // namespace linattn
