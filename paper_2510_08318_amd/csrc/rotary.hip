// linattn_rotary: rows of q and k turned, pair by pair, by the angles of their positions.
//
//   y1 = x1 cos t - x2 sin t,  y2 = x1 sin t + x2 cos t,  t = position base^(-2m / dims)
//
// Bytes bound it: a row is read and written once.  An angle serves all heads of its token, so a thread keeps its channels' sines and cosines and goes through the heads; it has 16 bytes of a
// row, or, with pairs in halves of the axes, 16 of either half.  Where the halves are not whole 16 bytes rows pass through LDS (rotary_staged_kernel).  2 x 12 x 32760 x 128 bf16, adjacent pairs: 77 us
// heads interleaved (5.2 TB/s), 73 else; one token of 64 sequences, 32 + 8 heads: 5 us, of which a launch is 3.
#include "../../include/linattn.h"
#include "rotary.h"
#include "f32_split.h"

namespace linattn {
namespace rotary {
namespace {

// The angle as a fraction of a turn, reduced in 64 bits: in 32, position 10^5 has its angle to 2^-8 only.  The fraction, at most half a turn, is then fp32, off by at most 2^-26 of a turn,
// an angle of 9e-8: the results of fp32 tensors are 4.3e-8 to 5.3e-8 of their 2-norm off, where sines of 64 bits, rounded to 32, give 4.0e-8 to 4.2e-8.  What is left of
// the fraction, put into the sine and cosine as their first derivative, would bring a second rounding of these and with it most of the same back.
__device__ __forceinline__ void sine_of(double turns, float& s, float& c) { sincospif(2.f * (float)(turns - rint(turns)), &s, &c); }

template <typename T>
constexpr int kValues = 16 / (int)sizeof(T);

template <typename T>
struct Run {                // 16 bytes of a row
  static constexpr int N = kValues<T>;
  uint4 w;
  template <bool STREAM>
  __device__ __forceinline__ void load(const T* p) { w = STREAM ? ld_nt(reinterpret_cast<const uint4*>(p)) : *reinterpret_cast<const uint4*>(p); }
  template <bool STREAM>
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (STREAM) st_nt(reinterpret_cast<uint4*>(p), w);
    else *reinterpret_cast<uint4*>(p) = w;
  }
  __device__ __forceinline__ void get(float (&f)[N]) const {
    if constexpr (sizeof(T) == 2) unpack_bf16x8(w, f);
    else f32::unpack_f32x4(w, f);
  }
  __device__ __forceinline__ void put(const float (&f)[N]) {
    if constexpr (sizeof(T) == 2) w = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    else w = make_uint4(__builtin_bit_cast(uint32_t, f[0]), __builtin_bit_cast(uint32_t, f[1]), __builtin_bit_cast(uint32_t, f[2]), __builtin_bit_cast(uint32_t, f[3]));
  }
  __device__ __forceinline__ void clear() { w = make_uint4(0, 0, 0, 0); }
};

// A thread's pairs of a row: HALVES, 16 bytes of the first half of an axis and 16 of its second; else 16 bytes of adjacent channels.
template <typename T, bool HALVES>
struct Pairs {
  static constexpr int N = kValues<T>, NP = HALVES ? N : N / 2;
  Run<T> a, b;              // b: HALVES only
  template <bool STREAM>
  __device__ __forceinline__ void load(const T* row, int at, int other) {
    a.template load<STREAM>(row + at);
    if constexpr (HALVES) b.template load<STREAM>(row + other);
  }
  template <bool STREAM>
  __device__ __forceinline__ void store(T* row, int at, int other) const {
    a.template store<STREAM>(row + at);
    if constexpr (HALVES) b.template store<STREAM>(row + other);
  }
  __device__ __forceinline__ void turn(const float (&s)[NP], const float (&c)[NP], uint32_t kept) {
    float x[N], z[N], y[N], u[N];
    a.get(x);
    if constexpr (HALVES) b.get(z);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float x1 = HALVES ? x[i] : x[2 * i], x2 = HALVES ? z[i] : x[2 * i + 1];
      // (channels of no axis: as they are, also where a neighbour is not finite)
      const float y1 = kept >> i & 1 ? x1 : fmaf(x1, c[i], -x2 * s[i]), y2 = kept >> i & 1 ? x2 : fmaf(x1, s[i], x2 * c[i]);
      if constexpr (HALVES) { y[i] = y1; u[i] = y2; }
      else { y[2 * i] = y1; y[2 * i + 1] = y2; }
    }
    a.put(y);
    if constexpr (HALVES) b.put(u);
  }
  __device__ __forceinline__ void clear() { a.clear(); if constexpr (HALVES) b.clear(); }
};

constexpr int kAhead = 4;      // rows whose loads are in flight together

template <typename T, int D, bool HALVES, bool STREAM>
__global__ __launch_bounds__(256) void rotary_kernel(Args a, int heads) {
  constexpr int NP = Pairs<T, HALVES>::NP, PARTS = D / 2 / NP;
  const int part = threadIdx.x % PARTS;
  const long long token = block_of() * (256 / PARTS) + threadIdx.x / PARTS, tokens = (long long)a.B * a.n;
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
  Pairs<T, HALVES> x[kAhead];
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
        x[i].template store<STREAM>(to(h + i), at, other);
      }
    h += kAhead;
    if (h >= h1) break;
    ask(h);
  }
}

// Pairs in halves that are not whole 16 bytes.  A workgroup works the sines and cosines of some tokens out into LDS, then goes through their rows, 16 bytes a thread, in the order of memory; the
// other channels of the pairs come through LDS too.  2 x 12 x 32760 x 128 bf16, 44 + 42 + 42 channels: 90 us; a pair a thread, 2 bytes an access, 123.
template <typename T, int D, bool INNER, bool STREAM>      // INNER: [B, n, H, d]
__global__ __launch_bounds__(256) void rotary_staged_kernel(Args a, int heads) {
  constexpr int V = kValues<T>, PARTS = D / V, ROWS = 256 / PARTS, TOKENS = 2048 / D;
  __shared__ float2 turns[TOKENS][D / 2];              // cosine and sine
  __shared__ size_t first[TOKENS][2];                  // element of the token's row of head 0 of q, of k
  __shared__ int live[TOKENS];
  __shared__ uint4 staged[256];
  const long long token0 = block_of() * TOKENS, tokens = (long long)a.B * a.n;
  if (token0 >= tokens) return;
  const int count = tokens - token0 < TOKENS ? (int)(tokens - token0) : TOKENS;
  for (int i = threadIdx.x; i < count * (D / 2); i += 256) {
    const int x = i / (D / 2), pair = i % (D / 2), ch = 2 * pair;
    const long long token = token0 + x;
    const int b = tokens >> 32 ? (int)(token / a.n) : (int)((uint32_t)token / (uint32_t)a.n), t = (int)(token - (long long)b * a.n);
    const int axis = ch >= a.from[2] ? 2 : ch >= a.from[1] ? 1 : 0;
    if (ch < a.from[3]) {
      double pos;
      if (a.positions) pos = a.positions[(size_t)b * a.item + (size_t)t * a.axes + axis];
      else {
        int at = t, of[3] = {0, 0, 0};
        if (a.axes > 2) { const int y = at / a.grid2; of[2] = at - y * a.grid2; at = y; }
        if (a.axes > 1) { const int y = at / a.grid1; of[1] = at - y * a.grid1; at = y; }
        of[0] = at;
        pos = axis == 2 ? (double)of[2] + a.first[2] : axis == 1 ? (double)of[1] + a.first[1] : (double)of[0] + a.first[0];
      }
      const double angle = pos * a.turns[pair];
      sine_of(a.back ? -angle : angle, turns[x][pair].y, turns[x][pair].x);
    }
    if (pair == 0) {
      live[x] = t < (a.lengths ? a.lengths[b] : a.n);
      first[x][0] = (size_t)b * a.qr.sb + (size_t)t * a.qr.sn;
      first[x][1] = (size_t)b * a.kr.sb + (size_t)t * a.kr.sn;
    }
  }

  // This thread's channels c .. c + V - 1: channel c + e is one of pair pair[e], with other[e]; sign: of the sine, + for the second of a pair.
  const int c = threadIdx.x % PARTS * V;
  int pair[V], other[V];
  float sign[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int ch = c + e, lo = ch >= a.from[2] ? a.from[2] : ch >= a.from[1] ? a.from[1] : 0;
    const int hi = ch >= a.from[2] ? a.from[3] : ch >= a.from[1] ? a.from[2] : a.from[1], half = (hi - lo) / 2;
    const bool second = ch - lo >= half;
    pair[e] = ch < a.from[3] ? lo / 2 + ch - lo - (second ? half : 0) : 0;
    other[e] = ch < a.from[3] ? ch + (second ? -half : half) : ch;
    sign[e] = second ? 1.f : -1.f;
  }
  __syncthreads();

  const int h0 = blockIdx.y * heads, h1 = h0 + heads < a.H + a.HK ? h0 + heads : a.H + a.HK;
  for (int tensor = 0; tensor < 2; ++tensor) {
    // heads g0 .. g0 + n - 1 of q, of k
    const int g0 = tensor ? (h0 > a.H ? h0 - a.H : 0) : h0, n = tensor ? (h1 > a.H ? h1 - a.H - g0 : 0) : (h1 < a.H ? h1 : a.H) - g0;
    if (n <= 0) continue;
    const T* in = static_cast<const T*>(tensor ? a.k : a.q);
    T* out = static_cast<T*>(tensor ? a.ko : a.qo);
    const size_t sh = tensor ? a.kr.sh : a.qr.sh;
    const int rows = n * count, inner = INNER ? n : count, over = ROWS / inner, left = ROWS % inner;
    int row = threadIdx.x / PARTS, major = row / inner, minor = row % inner;
    while (row - (int)(threadIdx.x / PARTS) < rows) {      // (the same turns for all threads)
      uint4 x[kAhead];
      int tok[kAhead];
      size_t at[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        tok[i] = row < rows ? (INNER ? major : minor) : -1;
        x[i] = make_uint4(0, 0, 0, 0);
        if (tok[i] >= 0) {
          at[i] = first[tok[i]][tensor] + (size_t)(g0 + (INNER ? minor : major)) * sh + c;
          if (live[tok[i]]) x[i] = STREAM ? ld_nt(reinterpret_cast<const uint4*>(in + at[i])) : *reinterpret_cast<const uint4*>(in + at[i]);
        }
        row += ROWS;
        major += over;
        minor += left;
        if (minor >= inner) { minor -= inner; ++major; }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        {
          // a row's threads are of one wavefront, whose LDS accesses go in order
          asm volatile("" ::: "memory");
          staged[threadIdx.x] = x[i];
          asm volatile("" ::: "memory");
        }
        if (tok[i] < 0) continue;
        const float2* turn = turns[tok[i]];
        const T* whole = reinterpret_cast<const T*>(staged + threadIdx.x / PARTS * PARTS);
        Run<T> r{x[i]};
        float f[V], y[V];
        r.get(f);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 cs = turn[pair[e]];
          const float z = f32::ldf(whole, other[e]);
          y[e] = c + e < a.from[3] ? fmaf(f[e], cs.x, sign[e] * z * cs.y) : f[e];
        }
        if (!live[tok[i]])
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] = 0.f;
        r.put(y);
        r.template store<STREAM>(out + at[i]);
      }
    }
  }
}

// Heads of a workgroup: all of them, or fewer where that fills the chip.
inline int heads_of(int all, long long blocks) {
  long long groups = (4 * kCUs + blocks - 1) / blocks;
  groups = groups < all ? groups : all;
  return (int)((all + groups - 1) / groups);
}

template <typename T, int D>
hipError_t run(const Args& a, hipStream_t s) {
  constexpr int V = kValues<T>;
  const bool whole = !a.halves || (a.from[1] | a.from[2] | a.from[3]) % (2 * V) == 0;      // 16 bytes of either half, in every axis
  const int tokens = whole ? 256 / (a.halves ? D / 2 / V : D / V) : 2048 / D, all = a.H + a.HK;
  const long long blocks = ((long long)a.B * a.n + tokens - 1) / tokens;
  const int heads = heads_of(all, blocks);
  const dim3 grid = grid_of(blocks, (all + heads - 1) / heads);
  // Rows that the last-level cache of 256 MB has no room for, with the results, go past it.  Us, so / through the cache, with rows that are not in it, 2 x 12 heads of bf16 x 128: 32760 tokens (403
  // MB with the results) 77 / 82, [B, H, n, d] 73 / 78; 16000 (197 MB) 39 / 43, 35 / 41, where the results are left for what reads them next.
  const bool big = 2. * (double)a.B * a.n * all * D * sizeof(T) > 300e6;
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, s>>>(a, heads);
    return hipGetLastError();
  };
  if (!whole) {
    const bool inner = a.qr.sh < a.qr.sn;
    return inner ? big ? go(rotary_staged_kernel<T, D, true, true>) : go(rotary_staged_kernel<T, D, true, false>)
                 : big ? go(rotary_staged_kernel<T, D, false, true>) : go(rotary_staged_kernel<T, D, false, false>);
  }
  if (a.halves) return go(rotary_kernel<T, D, true, false>);      // (its pieces of rows are shorter than a line: past the cache 110 us, through it 92)
  return big ? go(rotary_kernel<T, D, false, true>) : go(rotary_kernel<T, D, false, false>);
}

}  // namespace

hipError_t launch(const Args& a, bool f32, hipStream_t s) {
  if (f32) return a.d == 64 ? run<float, 64>(a, s) : run<float, 128>(a, s);
  return a.d == 64 ? run<uint16_t, 64>(a, s) : run<uint16_t, 128>(a, s);
}

}  // namespace rotary
}  // namespace linattn
