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

// o of a row, not yet divided by the sum l; m: the largest score (base 2).  The keys are those of [a0, a1) and [b0, b1) that position p sees.  sq: the
// query's D values, sp: 64 floats, both in LDS and the wavefront's own.
template <int D, typename Keys>
__device__ void plain_row(const Keys& keys, const float* sq, float* sp, int p, int len, const Sight& sight, int a0, int a1, int b0, int b1,
                          float scale2, int lane, float& m, float& l, float (&acc)[D / 64]) {
  m = -INFINITY; l = 0.f;
  for (int i = 0; i < D / 64; ++i) acc[i] = 0.f;
  for (int part = 0; part < 2; ++part)
    for (int j0 = part ? b0 : a0, end = part ? b1 : a1; j0 < end; j0 += 64) {
      const int j = j0 + lane;
      const bool on = j < end && sees(sight, p, j, len) && keys.there(j);
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

// Sum over the keys of ds_j k_j of the query at position p, in sq, with upstream gradient in sg.  p = 2^(scale2 s + nl nl2), delta: dout . o.
template <int D, typename Keys>
__device__ void plain_dq_row(const Keys& keys, const float* sq, const float* sg, float* sp, int p, int len, const Sight& sight, float scale2, float nl,
                             float nl2, float delta, int lane, float (&acc)[D / 64]) {
  for (int x = 0; x < D / 64; ++x) acc[x] = 0.f;
  if (nl == -INFINITY) return;
  const int lo = key_lo(sight, p), hi = key_hi(sight, p, len), first = sight.sinks < lo ? sight.sinks : lo;
  for (int part = 0; part < 2; ++part)
    for (int j0 = part ? lo : 0, end = part ? hi : first; j0 < end; j0 += 64) {
      const int j = j0 + lane;
      float ds = 0.f;
      if (j < end) {
        const float s = dot_row<D>(sq, [&](int c, float* f) { keys.k8(j, c, f); });
        const float dp = dot_row<D>(sg, [&](int c, float* f) { keys.v8(j, c, f); });
        ds = __builtin_amdgcn_exp2f(fmaf(s, scale2, nl * nl2)) * (dp - delta);
      }
      __builtin_amdgcn_wave_barrier();
      sp[lane] = ds;
      __builtin_amdgcn_wave_barrier();
      const int cnt = end - j0 < 64 ? end - j0 : 64;
      for (int t = 0; t < cnt; ++t)
        for (int x = 0; x < D / 64; ++x) acc[x] = fmaf(sp[t], keys.k1(j0 + t, lane + 64 * x), acc[x]);
    }
}

// The part of dk (before the scale) and dv of a key, in sk and sv, that the queries i0 .. i1-1 of one head give; rows: their q (as k) and dout (as v).
template <int D, typename Rows_>
__device__ void plain_dkv_row(const Rows_& rows, const float* sk, const float* sv, float* sp, float* ss, int i0, int i1, float scale2, float nl2,
                              const float* nl, const float* nd, int lane, float (&dk)[D / 64], float (&dv)[D / 64]) {
  for (; i0 < i1; i0 += 64) {
    const int i = i0 + lane;
    float p = 0.f, ds = 0.f;
    const float l = i < i1 ? nl[i] : -INFINITY;
    const bool on = l != -INFINITY;
    if (on) {
      const float s = dot_row<D>(sk, [&](int c, float* f) { rows.k8(i, c, f); });
      const float dp = dot_row<D>(sv, [&](int c, float* f) { rows.v8(i, c, f); });
      p = __builtin_amdgcn_exp2f(fmaf(s, scale2, l * nl2));
      ds = p * (dp + nd[i]);
    }
    const unsigned long long mask = __ballot(on);
    __builtin_amdgcn_wave_barrier();
    sp[lane] = p;
    ss[lane] = ds;
    __builtin_amdgcn_wave_barrier();
    for (int t = 0; t < 64; ++t)
      if (mask >> t & 1)
        for (int x = 0; x < D / 64; ++x) {
          dk[x] = fmaf(ss[t], rows.k1(i0 + t, lane + 64 * x), dk[x]);
          dv[x] = fmaf(sp[t], rows.v1(i0 + t, lane + 64 * x), dv[x]);
        }
  }
}

// A wavefront's LDS for these.
template <int D>
struct PlainScratch {
  float a[D], b[D], p[64], s[64];
  template <typename T>
  __device__ __forceinline__ void put(float* to, const T* row, int lane) {
    for (int x = lane; x < D; x += 64) to[x] = f32::ldf(row, x);
    __builtin_amdgcn_wave_barrier();
  }
};

}  // namespace attn
}  // namespace linattn
