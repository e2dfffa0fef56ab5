// Rows of softmax attention one at a time, a wavefront to a row, in fp32 FMAs: for each 64 keys a lane takes the scores of one, then
// the lanes take the channels.  Only what a row sees is touched, so an infinity or NaN elsewhere does not reach it.
#pragma once
#include "attn.h"
#include "f32_split.h"

namespace linattn {
namespace attn {

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float wave_sum(float x) {
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f) {
  if constexpr (sizeof(T) == 2) unpack_bf16x8(*reinterpret_cast<const uint4*>(p), f);
  else { f32::unpack_f32x4(*reinterpret_cast<const uint4*>(p), f); f32::unpack_f32x4(*reinterpret_cast<const uint4*>(p + 4), f + 4); }
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = (uint16_t)pack_bf16x2(v, v); }

// Rows of a token tensor: there(j), the eight values from channel c of row j, one value.
template <typename T>
struct TokenKeys {
  const T *k, *v;
  size_t sn;
  __device__ __forceinline__ bool there(int) const { return true; }
  __device__ __forceinline__ void k8(int j, int c, float* f) const { load8(k + (size_t)j * sn + c, f); }
  __device__ __forceinline__ float k1(int j, int c) const { return f32::ldf(k, (size_t)j * sn + c); }
  __device__ __forceinline__ void v8(int j, int c, float* f) const { load8(v + (size_t)j * sn + c, f); }
  __device__ __forceinline__ float v1(int j, int c) const { return f32::ldf(v, (size_t)j * sn + c); }
};

// x . row j, x in LDS
template <int D, typename L8>
__device__ __forceinline__ float dot_row(const float* x, L8 l8) {
  float s = 0.f;
  for (int c = 0; c < D; c += 8) {
    float f[8];
    l8(c, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[c + e], f[e], s);
  }
  return s;
}

// o of a row, not yet divided by the sum l; m: the largest score (base 2).  sq: the query's D values, sp: 64 floats, both in LDS and the wavefront's own.
template <int D, typename Keys>
__device__ void plain_row(const Keys& keys, const float* sq, float* sp, int p, int len, const Sight& sight, float scale2, int lane,
                          float& m, float& l, float (&acc)[D / 64]) {
  m = -INFINITY; l = 0.f;
  for (int i = 0; i < D / 64; ++i) acc[i] = 0.f;
  const int lo = key_lo(sight, p), hi = key_hi(sight, p, len), first = sight.sinks < lo ? sight.sinks : lo;
  for (int part = 0; part < 2; ++part)
    for (int j0 = part ? lo : 0, end = part ? hi : (first < hi ? first : hi); j0 < end; j0 += 64) {
      const int j = j0 + lane;
      const bool on = j < end && keys.there(j);
      const float s = on ? scale2 * dot_row<D>(sq, [&](int c, float* f) { keys.k8(j, c, f); }) : -INFINITY;
      const float mn = fmaxf(m, wave_max(s));
      const float pr = on && s != -INFINITY ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l = l * alpha + wave_sum(pr);
      const unsigned long long mask = __ballot(on);
      __builtin_amdgcn_wave_barrier();
      sp[lane] = pr;
      __builtin_amdgcn_wave_barrier();
      for (int i = 0; i < D / 64; ++i) acc[i] *= alpha;
      for (int t = 0; t < 64; ++t)
        if (mask >> t & 1)
          for (int i = 0; i < D / 64; ++i) acc[i] = fmaf(sp[t], keys.v1(j0 + t, lane + 64 * i), acc[i]);
    }
}

}  // namespace attn
}  // namespace linattn
