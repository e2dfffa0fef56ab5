// The paged cache: linattn_cache_write, linattn_cache_read, linattn_cache_attn.
#include "../../include/linattn.h"
#include "attn_keys.h"

namespace linattn {
namespace attn {

// e of a row whose largest finite magnitude is amax: 448 = 1.75 2^8.
__device__ __forceinline__ int row_exponent(float amax) {
  const uint32_t u = __builtin_bit_cast(uint32_t, amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000);
  return e < kLeastExp ? kLeastExp : e;
}

// ---- write --------------------------------------------------------------------------------

__device__ __forceinline__ float max_over(float x, int lanes) {
  for (int o = lanes / 2; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
// 448 is the largest code: a magnitude beyond it can only be an infinity here, which e4m3 does not have; it becomes NaN, as a NaN does.
// most: 448, or 240 in the rows of the largest exponent, whose code 256 would be 2^128.
__device__ __forceinline__ uint32_t encode4(const float* f, float s, float most) {
  float x[4], y[4];
  for (int i = 0; i < 4; ++i) {
    y[i] = f[i] * s;
    x[i] = __builtin_amdgcn_fmed3f(y[i], -most, most);
  }
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
  uint32_t u = (uint32_t)r;
  for (int i = 0; i < 4; ++i)
    if (!(fabsf(y[i]) <= 448.f)) u |= 0x7fu << (8 * i);
  return u;
}

// A row of d bf16 to d / 8 lanes.  A chunk of 4680 x 12 x 128 takes 12 us quantised (43 MB, 3.6 TB/s: a row of k and of v a thread in flight, and its maximum before
// anything is stored) and 10.6 as it is (57 MB, 5.4 TB/s), a token of each of 64 sequences 3.2 us, a launch.
template <int D, bool E4M3>
__device__ __forceinline__ void write_row(const uint16_t* src, void* pool, uint8_t* exps, long long row, int part) {
  const uint4 x = *reinterpret_cast<const uint4*>(src + 8 * part);
  if constexpr (!E4M3) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(pool) + row * D + 8 * part) = x;
  } else {
    float f[8], amax = 0.f;
    unpack_bf16x8(x, f);
    for (int i = 0; i < 8; ++i)
      if (fabsf(f[i]) < INFINITY) amax = fmaxf(amax, fabsf(f[i]));
    const int e = row_exponent(max_over(amax, D / 8));
    const float s = pow2(-e), most = e == kMostExp ? 240.f : 448.f;
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + row * D + 8 * part) = make_uint2(encode4(f, s, most), encode4(f + 4, s, most));
    if (part == 0) exps[row] = (uint8_t)(e + kExpBias);
  }
}

template <int D, bool E4M3, bool HEADS_INNER>
__global__ __launch_bounds__(256) void cache_write_kernel(Pool p, const uint16_t* k, const uint16_t* v, int n, Rows r) {
  constexpr int LANES = D / 8;
  const int part = threadIdx.x % LANES, b = blockIdx.y;
  const long long item = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int t = (int)(HEADS_INNER ? item / p.HK : item % n), h = (int)(HEADS_INNER ? item % p.HK : item / n);
  const int count = clamp_length(p.counts, b, n), length = p.lengths[b];
  if (item >= (long long)n * p.HK || t >= count) return;
  // (places go by lengths as it is: a token past the table has none, and must not take an earlier one's)
  const int j = (length < 0 ? 0 : length) - count + t;
  if (j < 0) return;
  const long long row = pool_row(p, b, h, j);
  if (row < 0) return;
  const size_t at = (size_t)b * r.sb + (size_t)h * r.sh + (size_t)t * r.sn;
  write_row<D, E4M3>(k + at, p.k, p.k_exp, row, part);
  write_row<D, E4M3>(v + at, p.v, p.v_exp, row, part);
}

// ---- read ---------------------------------------------------------------------------------

// A thread has 16 bytes of a row of k and of v in the tensors, for kReadItems rows: their loads are in flight together.  Bound by memory: 4 x 32760 x
// 12 x 128 e4m3 (a third of it behind the sequences' ends), 287 MB read and 805 written in 195 us = 5.6 TB/s; with a row a thread 257.
constexpr int kReadItems = 4;
template <int D, bool E4M3, bool HEADS_INNER>
__global__ __launch_bounds__(256) void cache_read_kernel(Pool p, uint16_t* k, uint16_t* v, int n, Rows r) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  const int part = threadIdx.x % LANES, b = blockIdx.y, len = pool_length(p, b);
  const long long item0 = (long long)blockIdx.x * (ROWS * kReadItems) + threadIdx.x / LANES, items = (long long)n * p.HK;
  size_t at[kReadItems];
  long long row[kReadItems];
  typename std::conditional<E4M3, u32x2, u32x4>::type ck[kReadItems], cv[kReadItems];
  uint8_t ek[kReadItems], ev[kReadItems];
#pragma unroll
  for (int i = 0; i < kReadItems; ++i) {
    const long long item = item0 + i * ROWS < items ? item0 + i * ROWS : items - 1;
    const int t = (int)(HEADS_INNER ? item / p.HK : item % n), h = (int)(HEADS_INNER ? item % p.HK : item / n);
    at[i] = (size_t)b * r.sb + (size_t)h * r.sh + (size_t)t * r.sn + 8 * part;
    row[i] = t < len ? pool_row(p, b, h, t) : -1;
  }
#pragma unroll
  for (int i = 0; i < kReadItems; ++i) {
    using C = decltype(ck[0] + ck[0]);
    const size_t from = (size_t)(row[i] < 0 ? 0 : row[i]) * LANES + part;
    ck[i] = __builtin_nontemporal_load(static_cast<const C*>(p.k) + from);
    cv[i] = __builtin_nontemporal_load(static_cast<const C*>(p.v) + from);
    if constexpr (E4M3) { ek[i] = p.k_exp[row[i] < 0 ? 0 : row[i]]; ev[i] = p.v_exp[row[i] < 0 ? 0 : row[i]]; }
  }
#pragma unroll
  for (int i = 0; i < kReadItems; ++i) {
    if (item0 + i * ROWS >= items) break;
    uint4 x, y;
    if constexpr (E4M3) {
      x = decode8(make_uint2(ck[i][0], ck[i][1]), row_scale(ek[i]));
      y = decode8(make_uint2(cv[i][0], cv[i][1]), row_scale(ev[i]));
    } else {
      x = __builtin_bit_cast(uint4, ck[i]);
      y = __builtin_bit_cast(uint4, cv[i]);
    }
    if (row[i] < 0) x = y = make_uint4(0, 0, 0, 0);
    st_nt(reinterpret_cast<uint4*>(k + at[i]), x);
    st_nt(reinterpret_cast<uint4*>(v + at[i]), y);
  }
}

static dim3 copy_grid(const Pool& p, int n, int items) {      // items: rows of a thread
  const int rows = 2048 / p.d * items;
  return dim3((unsigned)(((long long)n * p.HK + rows - 1) / rows), p.B);
}

hipError_t launch_cache_write(const Pool& p, bool e4m3, const void* k, const void* v, int n, const Rows& r, hipStream_t s) {
  auto go = [&](auto d, auto quantised) {
    constexpr int D = decltype(d)::value;
    constexpr bool E = decltype(quantised)::value;
    const auto *kk = static_cast<const uint16_t*>(k), *vv = static_cast<const uint16_t*>(v);
    if (r.sh < r.sn) cache_write_kernel<D, E, true><<<copy_grid(p, n, 1), 256, 0, s>>>(p, kk, vv, n, r);
    else cache_write_kernel<D, E, false><<<copy_grid(p, n, 1), 256, 0, s>>>(p, kk, vv, n, r);
  };
  using std::integral_constant;
  if (p.d == 64) e4m3 ? go(integral_constant<int, 64>{}, std::true_type{}) : go(integral_constant<int, 64>{}, std::false_type{});
  else e4m3 ? go(integral_constant<int, 128>{}, std::true_type{}) : go(integral_constant<int, 128>{}, std::false_type{});
  return hipGetLastError();
}
hipError_t launch_cache_read(const Pool& p, bool e4m3, void* k, void* v, int n, const Rows& r, hipStream_t s) {
  auto go = [&](auto d, auto quantised) {
    constexpr int D = decltype(d)::value;
    constexpr bool E = decltype(quantised)::value;
    auto *kk = static_cast<uint16_t*>(k), *vv = static_cast<uint16_t*>(v);
    if (r.sh < r.sn) cache_read_kernel<D, E, true><<<copy_grid(p, n, kReadItems), 256, 0, s>>>(p, kk, vv, n, r);
    else cache_read_kernel<D, E, false><<<copy_grid(p, n, kReadItems), 256, 0, s>>>(p, kk, vv, n, r);
  };
  using std::integral_constant;
  if (p.d == 64) e4m3 ? go(integral_constant<int, 64>{}, std::true_type{}) : go(integral_constant<int, 64>{}, std::false_type{});
  else e4m3 ? go(integral_constant<int, 128>{}, std::true_type{}) : go(integral_constant<int, 128>{}, std::false_type{});
  return hipGetLastError();
}

// ---- attention ----------------------------------------------------------------------------

hipError_t launch_cache_attn(const CacheArgs& a, bool e4m3) {
  const Pool& p = a.pool;
  RowsArgs r{a.q, a.o, a.lse, a.work, p.B, a.H, p.HK, a.H / p.HK, a.n, 0, 1, a.qr, a.sight, a.scale * kLog2e};
  const KeyParts parts = cache_splits(p.B, a.H, p.HK, a.n, p.d, e4m3, reach_of(a));
  r.splits = parts.splits;
  if (few_rows(a.H, p.HK, a.n)) {
    if (p.d == 64) return e4m3 ? launch_keys<64, KeysOfPool<64, true>>(r, p, a.stream) : launch_keys<64, KeysOfPool<64, false>>(r, p, a.stream);
    return e4m3 ? launch_keys<128, KeysOfPool<128, true>>(r, p, a.stream) : launch_keys<128, KeysOfPool<128, false>>(r, p, a.stream);
  }
  if (parts.splits > 1) {
    r.part_keys = parts.keys; r.reach = (int)reach_of(a); r.lengths = p.lengths;
  }
  if (p.d == 64) return e4m3 ? launch_rows<64, 64, PoolSource<64, 64, true>>(r, p, a.stream) : launch_rows<64, 64, PoolSource<64, 64, false>>(r, p, a.stream);
  return e4m3 ? launch_rows<128, 64, PoolSource<128, 64, true>>(r, p, a.stream) : launch_rows<128, 64, PoolSource<128, 64, false>>(r, p, a.stream);
}

}  // namespace attn
}  // namespace linattn
