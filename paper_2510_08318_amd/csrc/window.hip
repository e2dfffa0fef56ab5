// Softmax attention with a sliding window and first tokens: linattn_window_fwd, linattn_window_bwd.
#include "../../include/linattn.h"
#include "attn_plain.h"

namespace linattn {
namespace attn {

template <int D>
struct WaveScratch {
  float a[D], b[D], p[64], s[64];
};

template <int D, typename T>
__global__ __launch_bounds__(256) void window_fwd_plain_kernel(WindowArgs a) {
  __shared__ WaveScratch<D> ws[4];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  const int i = blockIdx.x * 4 + w;
  if (i >= a.n) return;
  const int len = clamp_length(a.lengths, b, a.n);
  const T* q = static_cast<const T*>(a.q) + head_base(a.qr, bh, a.H) + (size_t)i * a.qr.sn;
  T* o = static_cast<T*>(a.o) + head_base(a.qr, bh, a.H) + (size_t)i * a.qr.sn;
  const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
  float m = -INFINITY, l = 0.f, acc[D / 64] = {};
  if (i < len) {
    for (int x = 0; x < D / 64; ++x) ws[w].a[lane + 64 * x] = f32::ldf(q, lane + 64 * x);
    __builtin_amdgcn_wave_barrier();
    const TokenKeys<T> keys{static_cast<const T*>(a.k) + kv, static_cast<const T*>(a.v) + kv, a.kr.sn};
    plain_row<D>(keys, ws[w].a, ws[w].p, i, len, a.sight, a.scale * kLog2e, lane, m, l, acc);
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  for (int x = 0; x < D / 64; ++x) store1(o + lane + 64 * x, acc[x] * inv);
  if (a.lse && lane == 0) a.lse[(size_t)bh * a.n + i] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

template <int D, typename T>
__global__ __launch_bounds__(256) void window_delta_kernel(WindowArgs a) {
  const int lane = threadIdx.x % 64, bh = blockIdx.y, i = blockIdx.x * 4 + threadIdx.x / 64;
  if (i >= a.n) return;
  const size_t at = head_base(a.qr, bh, a.H) + (size_t)i * a.qr.sn;
  float s = 0.f;
  if (i < clamp_length(a.lengths, bh / a.H, a.n))
    for (int x = lane; x < D; x += 64) s = fmaf(f32::ldf(static_cast<const T*>(a.out), at + x), f32::ldf(static_cast<const T*>(a.dout), at + x), s);
  s = wave_sum(s);
  if (lane == 0) a.delta[(size_t)bh * a.n + i] = s;
}

template <int D, typename T>
__global__ __launch_bounds__(256) void window_dq_plain_kernel(WindowArgs a) {
  __shared__ WaveScratch<D> ws[4];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  const int i = blockIdx.x * 4 + w;
  if (i >= a.n) return;
  const int len = clamp_length(a.lengths, b, a.n);
  const size_t at = head_base(a.qr, bh, a.H) + (size_t)i * a.qr.sn;
  const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
  float acc[D / 64] = {};
  const float lse = i < len ? a.lse[(size_t)bh * a.n + i] : -INFINITY;
  if (lse != -INFINITY) {
    const float delta = a.delta[(size_t)bh * a.n + i], scale2 = a.scale * kLog2e, lse2 = lse * kLog2e;
    for (int x = lane; x < D; x += 64) {
      ws[w].a[x] = f32::ldf(static_cast<const T*>(a.q), at + x);
      ws[w].b[x] = f32::ldf(static_cast<const T*>(a.dout), at + x);
    }
    __builtin_amdgcn_wave_barrier();
    const TokenKeys<T> keys{static_cast<const T*>(a.k) + kv, static_cast<const T*>(a.v) + kv, a.kr.sn};
    const int lo = key_lo(a.sight, i), hi = key_hi(a.sight, i, len), first = a.sight.sinks < lo ? a.sight.sinks : lo;
    for (int part = 0; part < 2; ++part)
      for (int j0 = part ? lo : 0, end = part ? hi : first; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        float ds = 0.f;
        if (j < end) {
          const float s = dot_row<D>(ws[w].a, [&](int c, float* f) { keys.k8(j, c, f); });
          const float dp = dot_row<D>(ws[w].b, [&](int c, float* f) { keys.v8(j, c, f); });
          ds = __builtin_amdgcn_exp2f(fmaf(s, scale2, -lse2)) * (dp - delta);
        }
        __builtin_amdgcn_wave_barrier();
        ws[w].p[lane] = ds;
        __builtin_amdgcn_wave_barrier();
        const int cnt = end - j0 < 64 ? end - j0 : 64;
        for (int t = 0; t < cnt; ++t)
          for (int x = 0; x < D / 64; ++x) acc[x] = fmaf(ws[w].p[t], keys.k1(j0 + t, lane + 64 * x), acc[x]);
      }
  }
  for (int x = 0; x < D / 64; ++x) store1(static_cast<T*>(a.dq) + at + lane + 64 * x, a.scale * acc[x]);
}

template <int D, typename T>
__global__ __launch_bounds__(256) void window_dkv_plain_kernel(WindowArgs a) {
  __shared__ WaveScratch<D> ws[4];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bk = blockIdx.y, b = bk / a.HK, hk = bk % a.HK, G = a.H / a.HK;
  const int j = blockIdx.x * 4 + w;
  if (j >= a.n) return;
  const int len = clamp_length(a.lengths, b, a.n);
  const size_t at = head_base(a.kr, bk, a.HK) + (size_t)j * a.kr.sn;
  float dk[D / 64] = {}, dv[D / 64] = {};
  if (j < len) {
    for (int x = lane; x < D; x += 64) {
      ws[w].a[x] = f32::ldf(static_cast<const T*>(a.k), at + x);
      ws[w].b[x] = f32::ldf(static_cast<const T*>(a.v), at + x);
    }
    __builtin_amdgcn_wave_barrier();
    const float scale2 = a.scale * kLog2e;
    for (int g = 0; g < G; ++g) {
      const int bh = b * a.H + hk * G + g;
      const size_t base = head_base(a.qr, bh, a.H);
      const TokenKeys<T> rows{static_cast<const T*>(a.q) + base, static_cast<const T*>(a.dout) + base, a.qr.sn};
      const int end = query_hi(a.sight, j, len);
      for (int i0 = query_lo(a.sight, j); i0 < end; i0 += 64) {
        const int i = i0 + lane;
        float p = 0.f, ds = 0.f;
        bool on = i < end;
        const float lse = on ? a.lse[(size_t)bh * a.n + i] : -INFINITY;
        on = lse != -INFINITY;
        if (on) {
          const float s = dot_row<D>(ws[w].a, [&](int c, float* f) { rows.k8(i, c, f); });
          const float dp = dot_row<D>(ws[w].b, [&](int c, float* f) { rows.v8(i, c, f); });
          p = __builtin_amdgcn_exp2f(fmaf(s, scale2, -lse * kLog2e));
          ds = p * (dp - a.delta[(size_t)bh * a.n + i]);
        }
        const unsigned long long mask = __ballot(on);
        __builtin_amdgcn_wave_barrier();
        ws[w].p[lane] = p;
        ws[w].s[lane] = ds;
        __builtin_amdgcn_wave_barrier();
        for (int t = 0; t < 64; ++t)
          if (mask >> t & 1)
            for (int x = 0; x < D / 64; ++x) {
              dk[x] = fmaf(ws[w].s[t], rows.k1(i0 + t, lane + 64 * x), dk[x]);
              dv[x] = fmaf(ws[w].p[t], rows.v1(i0 + t, lane + 64 * x), dv[x]);
            }
      }
    }
  }
  for (int x = 0; x < D / 64; ++x) {
    store1(static_cast<T*>(a.dk) + at + lane + 64 * x, a.scale * dk[x]);
    store1(static_cast<T*>(a.dv) + at + lane + 64 * x, dv[x]);
  }
}

template <int D, typename T>
static hipError_t fwd_as(const WindowArgs& a) {
  window_fwd_plain_kernel<D, T><<<dim3((a.n + 3) / 4, a.B * a.H), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}
template <int D, typename T>
static hipError_t bwd_as(const WindowArgs& a) {
  const dim3 rows((a.n + 3) / 4, a.B * a.H), keys((a.n + 3) / 4, a.B * a.HK);
  window_delta_kernel<D, T><<<rows, 256, 0, a.stream>>>(a);
  window_dq_plain_kernel<D, T><<<rows, 256, 0, a.stream>>>(a);
  window_dkv_plain_kernel<D, T><<<keys, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_window_fwd(const WindowArgs& a, int dtype) {
  if (dtype == LINATTN_F32) return a.d == 64 ? fwd_as<64, float>(a) : fwd_as<128, float>(a);
  return a.d == 64 ? fwd_as<64, uint16_t>(a) : fwd_as<128, uint16_t>(a);
}
hipError_t launch_window_bwd(const WindowArgs& a, int dtype) {
  if (dtype == LINATTN_F32) return a.d == 64 ? bwd_as<64, float>(a) : bwd_as<128, float>(a);
  return a.d == 64 ? bwd_as<64, uint16_t>(a) : bwd_as<128, uint16_t>(a);
}

}  // namespace attn
}  // namespace linattn
