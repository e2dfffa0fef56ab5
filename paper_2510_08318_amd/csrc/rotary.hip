// linattn_rotary: rows of q and k turned, pair by pair, by the angles of their positions.
//
//   y1 = x1 cos t - x2 sin t,  y2 = x1 sin t + x2 cos t,  t = position base^(-2m / dims)
//
// Bytes bound it: a row is read and written once.  An angle serves all heads of its token, so a thread keeps its channels' sines and cosines and goes through the heads; it has 16 bytes of a
// row (with pairs in halves of the axes 16 of either half, or single channels where the halves are not whole 16 bytes).  2 x 12 x 32760 x 128 bf16, 44 + 42 + 42 channels: 64 us, 6.3 TB/s;
// one token of 64 sequences, 32 + 8 heads: 5 us, of which a launch is 3.
#include "../../include/linattn.h"
#include "rotary.h"
#include "f32_split.h"

namespace linattn {
namespace rotary {
namespace {

// The angle as a fraction of a turn, reduced in 64 bits: in 32, position 10^5 has its angle to 2^-8 only.
__device__ __forceinline__ void sine_of(double turns, float& s, float& c) { sincospif(2.f * (float)(turns - rint(turns)), &s, &c); }

template <typename T, int N>
struct Run {                // N adjacent values of a row
  static constexpr int W = (N * (int)sizeof(T) + 3) / 4;
  uint32_t w[W];
  template <bool STREAM>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W == 4) {
      const uint4 x = STREAM ? ld_nt(reinterpret_cast<const uint4*>(p)) : *reinterpret_cast<const uint4*>(p);
      w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else if constexpr (sizeof(T) == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
    else w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (W == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    else *reinterpret_cast<uint32_t*>(p) = w[0];
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
    else return i % 2 ? f32::hi_f32(w[i / 2]) : f32::lo_f32(w[i / 2]);
  }
  __device__ __forceinline__ void put(const float (&f)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __builtin_bit_cast(uint32_t, f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1 < N ? 2 * i + 1 : 2 * i]);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
  }
};

// A thread's NP pairs of a row: HALVES, NP channels of the first half of an axis and NP of its second; else 2 NP adjacent channels.
template <typename T, int NP, bool HALVES>
struct Pairs {
  static constexpr int N = HALVES ? NP : 2 * NP;
  Run<T, N> a, b;           // b: HALVES only
  template <bool STREAM>
  __device__ __forceinline__ void load(const T* row, int at, int other) {
    a.template load<STREAM>(row + at);
    if constexpr (HALVES) b.template load<STREAM>(row + other);
  }
  __device__ __forceinline__ void store(T* row, int at, int other) const {
    a.store(row + at);
    if constexpr (HALVES) b.store(row + other);
  }
  __device__ __forceinline__ void turn(const float (&s)[NP], const float (&c)[NP], uint32_t kept) {
    float y[N], z[N];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float x1 = HALVES ? a.get(i) : a.get(2 * i), x2 = HALVES ? b.get(i) : a.get(2 * i + 1);
      // (channels of no axis: as they are, also where a neighbour is not finite)
      const float y1 = kept >> i & 1 ? x1 : fmaf(x1, c[i], -x2 * s[i]), y2 = kept >> i & 1 ? x2 : fmaf(x1, s[i], x2 * c[i]);
      if constexpr (HALVES) { y[i] = y1; z[i] = y2; }
      else { y[2 * i] = y1; y[2 * i + 1] = y2; }
    }
    a.put(y);
    if constexpr (HALVES) b.put(z);
  }
  __device__ __forceinline__ void clear() { a.clear(); if constexpr (HALVES) b.clear(); }
};

constexpr int kAhead = 4;      // rows whose loads are in flight together

template <typename T, int D, int NP, bool HALVES, bool STREAM>
__global__ __launch_bounds__(256) void rotary_kernel(Args a, int heads) {
  constexpr int PARTS = D / 2 / NP;
  const int part = threadIdx.x % PARTS;
  const long long token = (long long)blockIdx.x * (256 / PARTS) + threadIdx.x / PARTS, tokens = (long long)a.B * a.n;
  if (token >= tokens) return;
  const int b = tokens >> 32 ? (int)(token / a.n) : (int)((uint32_t)token / (uint32_t)a.n), t = (int)(token - (long long)b * a.n);
  const bool live = t < (a.lengths ? a.lengths[b] : a.n);

  // this thread's channels: pairs p0 .. p0 + NP - 1
  const int p0 = part * NP;
  int at = 2 * p0, other = 0;
  if constexpr (HALVES) {
    // (an axis has whole chunks of pairs, and so have the channels behind the last)
    const int x = at >= a.from[3] ? 3 : at >= a.from[2] ? 2 : at >= a.from[1] ? 1 : 0;
    const int size = x == 3 ? 2 * NP : (x == 2 ? a.from[3] : x == 1 ? a.from[2] : a.from[1]) - (x == 2 ? a.from[2] : x == 1 ? a.from[1] : 0);
    if (x < 3) at = (x == 2 ? a.from[2] : x == 1 ? a.from[1] : 0) + (2 * p0 - (x == 2 ? a.from[2] : x == 1 ? a.from[1] : 0)) / 2;
    other = at + size / 2;
  }
  // the first rows are asked for before the angles are worked out
  const int h0 = blockIdx.y * heads, h1 = h0 + heads < a.H + a.HK ? h0 + heads : a.H + a.HK;
  const size_t q0 = (size_t)b * a.qr.sb + (size_t)t * a.qr.sn, k0 = (size_t)b * a.kr.sb + (size_t)t * a.kr.sn;
  auto from = [&](int h) { return h < a.H ? static_cast<const T*>(a.q) + q0 + (size_t)h * a.qr.sh : static_cast<const T*>(a.k) + k0 + (size_t)(h - a.H) * a.kr.sh; };
  auto to = [&](int h) { return h < a.H ? static_cast<T*>(a.qo) + q0 + (size_t)h * a.qr.sh : static_cast<T*>(a.ko) + k0 + (size_t)(h - a.H) * a.kr.sh; };
  Pairs<T, NP, HALVES> x[kAhead];
  auto ask = [&](int h) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (live && h + i < h1) x[i].template load<STREAM>(from(h + i), at, other);
      else x[i].clear();
    }
  };
  ask(h0);

  double pos[3] = {0., 0., 0.};
  if (a.positions) {
    const int* p = a.positions + (size_t)b * a.item + (size_t)t * a.axes;
    pos[0] = p[0];
    if (a.axes > 1) pos[1] = p[1];
    if (a.axes > 2) pos[2] = p[2];
  } else {
    int i = (int)t;
    if (a.axes > 2) { const int y = i / a.grid2; pos[2] = (double)(i - y * a.grid2) + a.first[2]; i = y; }
    if (a.axes > 1) { const int y = i / a.grid1; pos[1] = (double)(i - y * a.grid1) + a.first[1]; i = y; }
    pos[0] = (double)i + a.first[0];
  }
  float s[NP], c[NP];
  uint32_t kept = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int ch = 2 * (p0 + i);
    if (ch >= a.from[3]) kept |= 1u << i;
    const double angle = (ch >= a.from[2] ? pos[2] : ch >= a.from[1] ? pos[1] : pos[0]) * a.turns[p0 + i];
    sine_of(a.back ? -angle : angle, s[i], c[i]);
  }

  for (int h = h0;;) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (h + i < h1) {
        if (live) x[i].turn(s, c, kept);
        x[i].store(to(h + i), at, other);
      }
    h += kAhead;
    if (h >= h1) break;
    ask(h);
  }
}

template <typename T, int D, int NP, bool HALVES>
hipError_t run(const Args& a, hipStream_t s) {
  constexpr int TOKENS = 256 / (D / 2 / NP);
  const long long blocks = ((long long)a.B * a.n + TOKENS - 1) / TOKENS;
  const int all = a.H + a.HK;
  // Heads of a thread: all of them, or fewer where that fills the chip.
  long long groups = (4 * kCUs + blocks - 1) / blocks;
  groups = groups < all ? groups : all;
  const int heads = (int)((all + groups - 1) / groups);
  const dim3 grid((unsigned)blocks, (all + heads - 1) / heads);
  // Rows that the last-level cache of 256 MB has no room for, with the results, are read past it, which leaves it to the results.  Us, so / through the cache, 2 x 12 heads of bf16 x 128:
  // 32760 tokens (403 MB with the results) 65 / 82, 24000 (295 MB) 51 / 51, 16000 35 / 32, 12000 28 / 25.
  const bool big = 2. * (double)a.B * a.n * all * D * sizeof(T) > 300e6;
  if (big) rotary_kernel<T, D, NP, HALVES, true><<<grid, 256, 0, s>>>(a, heads);
  else rotary_kernel<T, D, NP, HALVES, false><<<grid, 256, 0, s>>>(a, heads);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t run_type(const Args& a, hipStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if (!a.halves) return run<T, D, V / 2, false>(a, s);
  // 16 bytes of either half, where the halves of every axis have whole ones
  return (a.from[1] | a.from[2] | a.from[3]) % (2 * V) == 0 ? run<T, D, V, true>(a, s) : run<T, D, 1, true>(a, s);
}

}  // namespace

hipError_t launch(const Args& a, bool f32, hipStream_t s) {
  if (f32) return a.d == 64 ? run_type<float, 64>(a, s) : run_type<float, 128>(a, s);
  return a.d == 64 ? run_type<uint16_t, 64>(a, s) : run_type<uint16_t, 128>(a, s);
}

}  // namespace rotary
}  // namespace linattn
