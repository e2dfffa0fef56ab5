// Softmax attention with a sliding window and first tokens: linattn_window_fwd, linattn_window_bwd.
#include "../../include/linattn.h"
#include "attn_bwd.h"
#include "attn_f32.h"

namespace linattn {
namespace attn {

template <int D, typename T>
__global__ __launch_bounds__(256) void window_fwd_plain_kernel(WindowArgs a) {
  __shared__ PlainScratch<D> ws[4];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  const int i = blockIdx.x * 4 + w;
  if (i >= a.n) return;
  const int len = clamp_length(a.lengths, b, a.n);
  const size_t at = head_base(a.qr, bh, a.H) + (size_t)i * a.qr.sn;
  const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
  float m = -INFINITY, l = 0.f, acc[D / 64] = {};
  if (i < len) {
    ws[w].put(ws[w].a, static_cast<const T*>(a.q) + at, lane);
    const TokenKeys<T> keys{static_cast<const T*>(a.k) + kv, static_cast<const T*>(a.v) + kv, a.kr.sn};
    const int lo = key_lo(a.sight, i), hi = key_hi(a.sight, i, len);
    plain_row<D>(keys, ws[w].a, ws[w].p, i, len, a.sight, 0, a.sight.sinks < lo ? a.sight.sinks : lo, lo, hi, a.scale * kLog2e, lane, m, l, acc);
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  for (int x = 0; x < D / 64; ++x) store1(static_cast<T*>(a.o) + at + lane + 64 * x, acc[x] * inv);
  if (a.lse && lane == 0) a.lse[(size_t)bh * a.n + i] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D, typename T>
__global__ __launch_bounds__(256) void window_dq_plain_kernel(WindowArgs a) {
  __shared__ PlainScratch<D> ws[4];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  const int i = blockIdx.x * 4 + w;
  if (i >= a.n) return;
  const int len = clamp_length(a.lengths, b, a.n);
  const size_t at = head_base(a.qr, bh, a.H) + (size_t)i * a.qr.sn;
  const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
  float acc[D / 64] = {}, nl = -INFINITY, delta = 0.f;
  if (i < len) {
    const float lse = a.lse[(size_t)bh * a.n + i];
    nl = lse == -INFINITY ? lse : -lse / a.scale;
    ws[w].put(ws[w].a, static_cast<const T*>(a.q) + at, lane);
    ws[w].put(ws[w].b, static_cast<const T*>(a.dout) + at, lane);
    for (int x = lane; x < D; x += 64) delta = fmaf(f32::ldf(static_cast<const T*>(a.out), at + x), ws[w].b[x], delta);
    delta = wave_sum(delta);
    const TokenKeys<T> keys{static_cast<const T*>(a.k) + kv, static_cast<const T*>(a.v) + kv, a.kr.sn};
    plain_dq_row<D>(keys, ws[w].a, ws[w].b, ws[w].p, i, len, a.sight, a.scale * kLog2e, nl, a.scale * kLog2e, delta, lane, acc);
  }
  if (lane == 0) {
    a.nl[(size_t)bh * a.n + i] = nl;
    a.nd[(size_t)bh * a.n + i] = -delta;
  }
  for (int x = 0; x < D / 64; ++x) store1(static_cast<T*>(a.dq) + at + lane + 64 * x, a.scale * acc[x]);
}

template <int D, typename T>
__global__ __launch_bounds__(256) void window_dkv_plain_kernel(WindowArgs a) {
  __shared__ PlainScratch<D> ws[4];
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64, bk = blockIdx.y, b = bk / a.HK, hk = bk % a.HK, G = a.H / a.HK;
  const int j = blockIdx.x * 4 + w;
  if (j >= a.n) return;
  const int len = clamp_length(a.lengths, b, a.n);
  const size_t at = head_base(a.kr, bk, a.HK) + (size_t)j * a.kr.sn;
  float dk[D / 64] = {}, dv[D / 64] = {};
  if (j < len) {
    ws[w].put(ws[w].a, static_cast<const T*>(a.k) + at, lane);
    ws[w].put(ws[w].b, static_cast<const T*>(a.v) + at, lane);
    for (int g = 0; g < G; ++g) {
      const int bh = b * a.H + hk * G + g;
      const size_t base = head_base(a.qr, bh, a.H);
      const TokenKeys<T> rows{static_cast<const T*>(a.q) + base, static_cast<const T*>(a.dout) + base, a.qr.sn};
      plain_dkv_row<D>(rows, ws[w].a, ws[w].b, ws[w].p, ws[w].s, query_lo(a.sight, j), query_hi(a.sight, j, len), a.scale * kLog2e, a.scale * kLog2e,
                       a.nl + (size_t)bh * a.n, a.nd + (size_t)bh * a.n, lane, dk, dv);
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
  window_dq_plain_kernel<D, T><<<rows, 256, 0, a.stream>>>(a);
  window_dkv_plain_kernel<D, T><<<keys, 256, 0, a.stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_window_fwd(const WindowArgs& a, int dtype) {
  if (dtype == LINATTN_BF16) {
    const TokenArgs keys{a.k, a.v, a.lengths, a.kr};
    const RowsArgs r{a.q, a.o, a.lse, nullptr, a.B, a.H, a.HK, a.H / a.HK, a.n, 0, 1, a.qr, a.sight, a.scale * kLog2e};
    return a.d == 64 ? launch_rows<64, 64, TokenSource<64, 64>>(r, keys, a.stream) : launch_rows<128, 64, TokenSource<128, 64>>(r, keys, a.stream);
  }
  if (dtype == LINATTN_F32) return a.d == 64 ? launch_fwd_f32<64>(a) : launch_fwd_f32<128>(a);
  return a.d == 64 ? fwd_as<64, uint16_t>(a) : fwd_as<128, uint16_t>(a);
}
hipError_t launch_window_bwd(const WindowArgs& a, int dtype) {
  if (dtype == LINATTN_BF16) {
    BwdRows r{};
    r.q = a.q; r.k = a.k; r.v = a.v; r.out = a.out; r.dout = a.dout; r.dq = a.dq; r.dk = a.dk; r.dv = a.dv;
    r.lse = a.lse; r.nl = a.nl; r.nd = a.nd; r.parts = a.parts;
    r.lengths = a.lengths; r.B = a.B; r.H = a.H; r.HK = a.HK; r.G = a.H / a.HK; r.n = a.n;
    r.qr = a.qr; r.kr = a.kr; r.sight = a.sight; r.scale = a.scale; r.scale2 = a.scale * kLog2e;
    return a.d == 64 ? launch_bwd_rows<64>(r, a.stream) : launch_bwd_rows<128>(r, a.stream);
  }
  if (dtype == LINATTN_F32) return a.d == 64 ? launch_bwd_f32<64>(a) : launch_bwd_f32<128>(a);
  return a.d == 64 ? bwd_as<64, uint16_t>(a) : bwd_as<128, uint16_t>(a);
}

}  // namespace attn
}  // namespace linattn
