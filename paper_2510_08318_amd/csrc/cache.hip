// The paged cache: linattn_cache_write, linattn_cache_read, linattn_cache_attn.
// A quantised row is e4m3 codes and one exponent: x ~ code 2^e, e the least integer with max|x| 2^-e <= 448 and at least kLeastExp.  With a power of
// two for a scale the codes' rounding is the only one: code 2^e has 4 significant bits and (e >= kLeastExp) the exponent of a normal bf16, so
// that what is read back, as bf16 or by the attention, is the same value without another rounding.
#include "../../include/linattn.h"
#include "attn_plain.h"

namespace linattn {
namespace attn {

constexpr int kExpBias = 127;
constexpr int kMostExp = 120;         // of rows with entries from 448 2^119 on
constexpr int kLeastExp = -117;      // 2^-9, the smallest code, times 2^-117 is 2^-126, the smallest normal bf16

// e of a row whose largest finite magnitude is amax: 448 = 1.75 2^8.
__device__ __forceinline__ int row_exponent(float amax) {
  const uint32_t u = __builtin_bit_cast(uint32_t, amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000);
  return e < kLeastExp ? kLeastExp : e;
}
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }      // -126 <= e <= 127

// Four codes -> values times s.
__device__ __forceinline__ void decode4(uint32_t codes, float s, float* f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  f[0] = lo[0] * s; f[1] = lo[1] * s; f[2] = hi[0] * s; f[3] = hi[1] * s;
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
      const float s = pow2((int)exps[r] - kExpBias);
      decode4(x.x, s, f); decode4(x.y, s, f + 4);
    } else load8(static_cast<const uint16_t*>(base) + r * d + c, f);
  }
  __device__ __forceinline__ float row1(const void* base, const uint8_t* exps, int j, int c) const {
    const long long r = pool_row(*pool, b, h, j);
    if constexpr (E4M3) {
      float f[4];
      decode4(static_cast<const uint8_t*>(base)[r * d + c], pow2((int)exps[r] - kExpBias), f);
      return f[0];
    } else return f32::ldf(static_cast<const uint16_t*>(base), (size_t)(r * d + c));
  }
  __device__ __forceinline__ void k8(int j, int c, float* f) const { row8(pool->k, pool->k_exp, j, c, f); }
  __device__ __forceinline__ void v8(int j, int c, float* f) const { row8(pool->v, pool->v_exp, j, c, f); }
  __device__ __forceinline__ float k1(int j, int c) const { return row1(pool->k, pool->k_exp, j, c); }
  __device__ __forceinline__ float v1(int j, int c) const { return row1(pool->v, pool->v_exp, j, c); }
};

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

// A row of d bf16 to d / 8 lanes.
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
  const int count = clamp_length(p.counts, b, n), j = pool_length(p, b) - count + t;
  if (item >= (long long)n * p.HK || t >= count || j < 0) return;
  const long long row = pool_row(p, b, h, j);
  if (row < 0) return;
  const size_t at = (size_t)b * r.sb + (size_t)h * r.sh + (size_t)t * r.sn;
  write_row<D, E4M3>(k + at, p.k, p.k_exp, row, part);
  write_row<D, E4M3>(v + at, p.v, p.v_exp, row, part);
}

// ---- read ---------------------------------------------------------------------------------

template <int D, bool E4M3, bool HEADS_INNER>
__global__ __launch_bounds__(256) void cache_read_kernel(Pool p, uint16_t* k, uint16_t* v, int n, Rows r) {
  constexpr int LANES = D / 8;
  const int part = threadIdx.x % LANES, b = blockIdx.y;
  const long long item = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (item >= (long long)n * p.HK) return;
  const int t = (int)(HEADS_INNER ? item / p.HK : item % n), h = (int)(HEADS_INNER ? item % p.HK : item / n);
  const size_t at = (size_t)b * r.sb + (size_t)h * r.sh + (size_t)t * r.sn + 8 * part;
  float fk[8] = {}, fv[8] = {};
  if (t < pool_length(p, b) && pool_row(p, b, h, t) >= 0) {
    const PoolKeys<E4M3> keys{&p, b, h, D};
    keys.k8(t, 8 * part, fk);
    keys.v8(t, 8 * part, fv);
  }
  *reinterpret_cast<uint4*>(k + at) = make_uint4(pack_bf16x2(fk[0], fk[1]), pack_bf16x2(fk[2], fk[3]), pack_bf16x2(fk[4], fk[5]), pack_bf16x2(fk[6], fk[7]));
  *reinterpret_cast<uint4*>(v + at) = make_uint4(pack_bf16x2(fv[0], fv[1]), pack_bf16x2(fv[2], fv[3]), pack_bf16x2(fv[4], fv[5]), pack_bf16x2(fv[6], fv[7]));
}

template <int D, bool E4M3>
static dim3 copy_grid(const Pool& p, int n) { return dim3((unsigned)(((long long)n * p.HK + 2048 / D - 1) / (2048 / D)), p.B); }

hipError_t launch_cache_write(const Pool& p, bool e4m3, const void* k, const void* v, int n, const Rows& r, hipStream_t s) {
  auto go = [&](auto d, auto quantised) {
    constexpr int D = decltype(d)::value;
    constexpr bool E = decltype(quantised)::value;
    const auto *kk = static_cast<const uint16_t*>(k), *vv = static_cast<const uint16_t*>(v);
    if (r.sh < r.sn) cache_write_kernel<D, E, true><<<copy_grid<D, E>(p, n), 256, 0, s>>>(p, kk, vv, n, r);
    else cache_write_kernel<D, E, false><<<copy_grid<D, E>(p, n), 256, 0, s>>>(p, kk, vv, n, r);
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
    if (r.sh < r.sn) cache_read_kernel<D, E, true><<<copy_grid<D, E>(p, n), 256, 0, s>>>(p, kk, vv, n, r);
    else cache_read_kernel<D, E, false><<<copy_grid<D, E>(p, n), 256, 0, s>>>(p, kk, vv, n, r);
  };
  using std::integral_constant;
  if (p.d == 64) e4m3 ? go(integral_constant<int, 64>{}, std::true_type{}) : go(integral_constant<int, 64>{}, std::false_type{});
  else e4m3 ? go(integral_constant<int, 128>{}, std::true_type{}) : go(integral_constant<int, 128>{}, std::false_type{});
  return hipGetLastError();
}

// ---- attention ----------------------------------------------------------------------------

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void cache_attn_plain_kernel(CacheArgs a) {
  __shared__ float sq[4][D], sp[4][64];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  const int t = blockIdx.x * 4 + w;
  if (t >= a.n) return;
  const int len = pool_length(a.pool, b), count = clamp_length(a.pool.counts, b, a.n), pos = len - count + t;
  const size_t at = head_base(a.qr, bh, a.H) + (size_t)t * a.qr.sn;
  float m = -INFINITY, l = 0.f, acc[D / 64] = {};
  if (t < count && pos >= 0) {
    for (int x = lane; x < D; x += 64) sq[w][x] = f32::ldf(static_cast<const uint16_t*>(a.q), at + x);
    __builtin_amdgcn_wave_barrier();
    const PoolKeys<E4M3> keys{&a.pool, b, h / (a.H / a.pool.HK), D};
    plain_row<D>(keys, sq[w], sp[w], pos, len, a.sight, a.scale * kLog2e, lane, m, l, acc);
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  for (int x = 0; x < D / 64; ++x) store1(static_cast<uint16_t*>(a.o) + at + lane + 64 * x, acc[x] * inv);
  if (a.lse && lane == 0) a.lse[(size_t)bh * a.n + t] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

hipError_t launch_cache_attn(const CacheArgs& a, bool e4m3) {
  const dim3 grid((a.n + 3) / 4, a.pool.B * a.H);
  if (a.pool.d == 64) {
    if (e4m3) cache_attn_plain_kernel<64, true><<<grid, 256, 0, a.stream>>>(a);
    else cache_attn_plain_kernel<64, false><<<grid, 256, 0, a.stream>>>(a);
  } else {
    if (e4m3) cache_attn_plain_kernel<128, true><<<grid, 256, 0, a.stream>>>(a);
    else cache_attn_plain_kernel<128, false><<<grid, 256, 0, a.stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace attn
}  // namespace linattn
