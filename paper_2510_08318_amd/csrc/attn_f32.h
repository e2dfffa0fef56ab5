// Windowed softmax attention of fp32 tensors on v_mfma_f32_32x32x2_f32, forward and backward.  A workgroup has 32 rows (queries, or keys for dk and dv), on
// the lanes of each of its four wavefronts, which take the tiles of 32 that the rows see in turn and join their results in LDS at the end: a short sequence then
// has four times the wavefronts, and nothing waits for a barrier.  An operand is read from global memory where it is used: a 16-byte load feeds four
// instructions of 64 cycles, so the caches are idle most of the time, and LDS would save nothing.
// Where the blocks of 32 rows are fewer than the compute units, `shares` workgroups have the tiles of one in turn, and write fp32 parts that a second kernel
// sums in their order.  A step of 2 heads x 1024 x 64, window 2 x 256: 13 + 4, 17 + 4 and 21 + 4 us for out, dq, dk and dv (20, 28 and 52 without shares); the instructions
// alone take 4.8 us on all compute units, the blocks that hold first tokens 7.5 us one after the other.
// Contraction over the channels: four k-steps have eight channels, of which lane group g has the four from 4 g on.  Contraction over the tile's rows: k-step r has the rows
// that register r of a score block holds, 8 (r/4) + 4 g + r%4.  Accumulator rows m of block c are channels CB m + c.
#pragma once
#include "attn_rows.h"

namespace linattn {
namespace attn {

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// S[i][lane's row] += rows i of the tile . the lane's row x, whose channels of group g are in registers.  row: of tile row `lane % 32`.
template <int D>
__device__ __forceinline__ void scores_f32(const float* row, int g, const float4 (&x)[D / 8], f32x16& s) {
  pipelined_operands<D / 8, 6>([&](int i) { return *reinterpret_cast<const uint4*>(row + 8 * i + 4 * g); },
                               [&](int i, uint4 v) {
                                 float f[4];
                                 f32::unpack_f32x4(v, f);
                                 s = mfma_f32(f[0], x[i].x, s); s = mfma_f32(f[1], x[i].y, s); s = mfma_f32(f[2], x[i].z, s); s = mfma_f32(f[3], x[i].w, s);
                               });
}
// acc^T[channel][lane's row] += sum over the tile's rows i of rows[i][channel] w[i]: w as a score block, at(i): row i of the tile.
template <int D, typename At>
__device__ __forceinline__ void weighted_f32(At at, int lane, const f32x16& w, f32x16 (&acc)[D / 32]) {
  constexpr int CB = D / 32;
  const int m = lane % 32, g = lane / 32;
  pipelined_operands<16, 4>(
      [&](int r) {
        const float* p = at(8 * (r / 4) + 4 * g + r % 4) + CB * m;
        if constexpr (CB == 4) return *reinterpret_cast<const uint4*>(p);
        else { const uint2 y = *reinterpret_cast<const uint2*>(p); return make_uint4(y.x, y.y, 0, 0); }
      },
      [&](int r, uint4 v) {
        float f[4];
        f32::unpack_f32x4(v, f);
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[c] = mfma_f32(f[c], w[r], acc[c]);
      });
}
// This lane's accumulators -> row `lane % 32` of a [32][D] fp32 block.
template <int D>
__device__ __forceinline__ void put_acc_f32(float* block, int lane, const f32x16 (&acc)[D / 32]) {
  constexpr int CB = D / 32;
  float* to = block + lane % 32 * D;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int ch = CB * (8 * (r / 4) + 4 * (lane / 32) + r % 4);
    if constexpr (CB == 4) *reinterpret_cast<float4*>(to + ch) = make_float4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]);
    else *reinterpret_cast<float2*>(to + ch) = make_float2(acc[0][r], acc[1][r]);
  }
}
template <int D>
__device__ __forceinline__ void load_half_row(const float* row, int g, bool live, float4 (&x)[D / 8]) {
#pragma unroll
  for (int i = 0; i < D / 8; ++i) x[i] = live ? *reinterpret_cast<const float4*>(row + 8 * i + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// p = exp(scale s - lse) = 2^(scale2 s - lse log2(e)): the forward's weights up to the rounding of lse itself, with the product in two parts.  nl: -lse.
__device__ __forceinline__ float weight_f32(float s, float scale2, float nl) {
  constexpr float lo = 1.925963033500011e-8f;          // log2(e) - kLog2e
  const float h = nl * kLog2e, l = fmaf(nl, lo, fmaf(nl, kLog2e, -h));
  return nl == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(s, scale2, h) + l);
}

constexpr int kF32Smem(int D) { return kRowWaves * 32 * (D * 4 + 8); }      // the wavefronts' sums, and pairs of maximum and sum

template <int D>
__global__ __launch_bounds__(256, 2) void window_fwd_f32_kernel(WindowArgs a) {
  constexpr int CB = D / 32, NW = kRowWaves;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const int blocks = (a.n + 31) / 32;
  const PairPlace place = pair_place(blockIdx.x, a.B * a.H, blocks * a.shares);
  const int bh = place.pair, share = place.at % a.shares, block = row_block(a.sight, place.at / a.shares, blocks);
  const int b = bh / a.H, h = bh % a.H, len = clamp_length(a.lengths, b, a.n), t = block * 32 + m;
  const bool live = t < len;
  const float* qbase = static_cast<const float*>(a.q) + head_base(a.qr, bh, a.H);
  const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
  const float *kbase = static_cast<const float*>(a.k) + kv, *vbase = static_cast<const float*>(a.v) + kv;
  const int lo = live ? key_lo(a.sight, t) : 0, hi = live ? key_hi(a.sight, t, len) : 0;
  float4 q[D / 8];
  load_half_row<D>(qbase + (size_t)t * a.qr.sn, g, live, q);
  f32x16 o[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) o[c] = fill16(0.f);
  float mx = -INFINITY, l = 0.f;
  const float scale2 = a.scale * kLog2e;
  const int p1 = (block * 32 + 32 < len ? block * 32 + 32 : len) - 1;
  const KeyTiles<32> tiles(a.sight, block * 32, p1 < block * 32 ? -1 : p1, len);
  const WaveSight sight(a.sight, block * 32, p1 < block * 32 ? -1 : p1, len);
  for (int it = share * NW + w; it < tiles.count; it += NW * a.shares) {
    const int j0 = tiles.start(it), last = tiles.end - 1 - j0;
    f32x16 s[1] = {fill16(0.f)};
    scores_f32<D>(kbase + (size_t)(j0 + (m < last ? m : last)) * a.kr.sn, g, q, s[0]);
    if (!sight.everything(j0, 32)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = j0 + 8 * (r / 4) + 4 * g + r % 4;
        s[0][r] = j < hi && (j >= lo || j < a.sight.sinks) ? s[0][r] : -INFINITY;
      }
    }
    softmax_step<1, CB>(s, scale2, mx, l, o);
    weighted_f32<D>([&](int i) { return vbase + (size_t)(j0 + (i < last ? i : last)) * a.kr.sn; }, lane, s[0], o);
  }
  float* const os = reinterpret_cast<float*>(smem);
  float2* const ml = reinterpret_cast<float2*>(os + NW * 32 * D);
  float x, y;
  pair32(l, x, y);
  put_acc_f32<D>(os + w * 32 * D, lane, o);
  if (g == 0) ml[w * 32 + m] = make_float2(mx, x + y);
  __syncthreads();
  unsigned again = 0;
  for (int i = 0; i < 32 / NW; ++i) {
    const int rr = w * (32 / NW) + i, tt = block * 32 + rr;
    if (tt >= a.n) break;
    float top = -INFINITY, sum = 0.f, acc[D / 64] = {}, test = 0.f;
    if (tt < len) {
      for (int v = 0; v < NW; ++v) top = fmaxf(top, ml[v * 32 + rr].x);
      for (int v = 0; v < NW; ++v) {
        const float2 e = ml[v * 32 + rr];
        const float f = e.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e.x - top);
        sum = fmaf(f, e.y, sum);
        test = fmaf(0.f, e.y, test);
        for (int c = 0; c < D / 64; ++c) {
          const float z = os[(v * 32 + rr) * D + lane + 64 * c];
          acc[c] = fmaf(f, z, acc[c]);
          test = fmaf(0.f, z, test);
        }
      }
      if (a.shares == 1 && __any(test != 0.f)) { again |= 1u << i; continue; }
    }
    if (a.shares > 1) {
      const size_t rows = (size_t)a.B * a.H * a.n, row = (size_t)share * rows + (size_t)bh * a.n + tt;
      for (int c = 0; c < D / 64; ++c) a.parts[row * D + lane + 64 * c] = acc[c];
      if (lane == 0) reinterpret_cast<float2*>(a.parts + (size_t)a.shares * rows * D)[row] = make_float2(top, sum);
      continue;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    float* out = static_cast<float*>(a.o) + head_base(a.qr, bh, a.H) + (size_t)tt * a.qr.sn;
    for (int c = 0; c < D / 64; ++c) out[lane + 64 * c] = acc[c] * inv;
    if (a.lse && lane == 0) a.lse[(size_t)bh * a.n + tt] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
  }
  __syncthreads();
  for (; again; again &= again - 1) {      // rows that are not finite, once more over what they see alone
    const int tt = block * 32 + w * (32 / NW) + __ffs(again) - 1;
    PlainScratch<D>& ps = reinterpret_cast<PlainScratch<D>*>(smem)[w];
    ps.put(ps.a, qbase + (size_t)tt * a.qr.sn, lane);
    const TokenKeys<float> keys{kbase, vbase, a.kr.sn};
    float pm, pl, acc[D / 64];
    plain_row<D>(keys, ps.a, ps.p, tt, len, a.sight, tiles.sink_key(0), tiles.sink_key(tiles.count), tiles.window_key(0), tiles.window_key(tiles.count),
                 scale2, lane, pm, pl, acc);
    const float inv = pl == 0.f ? 0.f : 1.0f / pl;
    float* out = static_cast<float*>(a.o) + head_base(a.qr, bh, a.H) + (size_t)tt * a.qr.sn;
    for (int c = 0; c < D / 64; ++c) out[lane + 64 * c] = acc[c] * inv;
    if (a.lse && lane == 0) a.lse[(size_t)bh * a.n + tt] = pl == 0.f ? -INFINITY : (pm + __builtin_amdgcn_logf(pl)) * kLn2;
  }
}

// The sums of the four wavefronts' [32][D] blocks, row by row: put(row, sums of channels lane, lane + 64); `again` gets those that are not finite, if they are looked for.
template <int D, typename Put>
__device__ __forceinline__ void join_rows_f32(const float* os, int w, int lane, int rows, bool look, unsigned& again, Put put) {
  constexpr int NW = kRowWaves;
  for (int i = 0; i < 32 / NW; ++i) {
    const int rr = w * (32 / NW) + i;
    if (rr >= rows) break;
    float acc[D / 64] = {}, test = 0.f;
    for (int c = 0; c < D / 64; ++c) {
      for (int v = 0; v < NW; ++v) acc[c] += os[(v * 32 + rr) * D + lane + 64 * c];
      test = fmaf(0.f, acc[c], test);
    }
    if (look && __any(test != 0.f)) again |= 1u << i;
    else put(rr, acc);
  }
}

template <int D>
__global__ __launch_bounds__(256, 1) void window_dq_f32_kernel(WindowArgs a) {
  constexpr int CB = D / 32, NW = kRowWaves;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const int blocks = (a.n + 31) / 32;
  const PairPlace place = pair_place(blockIdx.x, a.B * a.H, blocks * a.shares);
  const int bh = place.pair, share = place.at % a.shares, block = row_block(a.sight, place.at / a.shares, blocks);
  const int b = bh / a.H, h = bh % a.H, len = clamp_length(a.lengths, b, a.n), t = block * 32 + m;
  const bool live = t < len;
  const size_t head = head_base(a.qr, bh, a.H), row = head + (size_t)t * a.qr.sn, li = (size_t)bh * a.n + t;
  const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
  const float *kbase = static_cast<const float*>(a.k) + kv, *vbase = static_cast<const float*>(a.v) + kv;
  const int lo = live ? key_lo(a.sight, t) : 0, hi = live ? key_hi(a.sight, t, len) : 0;
  float4 q[D / 8], go[D / 8];
  load_half_row<D>(static_cast<const float*>(a.q) + row, g, live, q);
  load_half_row<D>(static_cast<const float*>(a.dout) + row, g, live, go);
  float delta = 0.f;
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    const float4 y = live ? *reinterpret_cast<const float4*>(static_cast<const float*>(a.out) + row + 8 * i + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f);
    delta = fmaf(go[i].x, y.x, fmaf(go[i].y, y.y, fmaf(go[i].z, y.z, fmaf(go[i].w, y.w, delta))));
  }
  float x, y;
  pair32(delta, x, y);
  delta = x + y;
  const float lse = live ? a.lse[li] : -INFINITY, nl = lse == -INFINITY ? lse : -lse;
  if (t < a.n && w == 0 && g == 0 && share == 0) { a.nl[li] = nl; a.nd[li] = -delta; }
  f32x16 dq[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) dq[c] = fill16(0.f);
  const float scale2 = a.scale * kLog2e;
  const int p1 = (block * 32 + 32 < len ? block * 32 + 32 : len) - 1;
  const KeyTiles<32> tiles(a.sight, block * 32, p1 < block * 32 ? -1 : p1, len);
  const WaveSight sight(a.sight, block * 32, p1 < block * 32 ? -1 : p1, len);
  for (int it = share * NW + w; it < tiles.count; it += NW * a.shares) {
    const int j0 = tiles.start(it), last = tiles.end - 1 - j0, mine = j0 + (m < last ? m : last);
    f32x16 s = fill16(0.f), dp = fill16(-delta);
    scores_f32<D>(kbase + (size_t)mine * a.kr.sn, g, q, s);
    scores_f32<D>(vbase + (size_t)mine * a.kr.sn, g, go, dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] *= weight_f32(s[r], scale2, nl);
    if (!sight.everything(j0, 32)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = j0 + 8 * (r / 4) + 4 * g + r % 4;
        dp[r] = j < hi && (j >= lo || j < a.sight.sinks) ? dp[r] : 0.f;
      }
    }
    weighted_f32<D>([&](int i) { return kbase + (size_t)(j0 + (i < last ? i : last)) * a.kr.sn; }, lane, dp, dq);
  }
  if (!live) {
#pragma unroll
    for (int c = 0; c < CB; ++c) dq[c] = fill16(0.f);
  }
  float* const os = reinterpret_cast<float*>(smem);
  put_acc_f32<D>(os + w * 32 * D, lane, dq);
  __syncthreads();
  unsigned again = 0;
  float* const to = static_cast<float*>(a.dq) + head + (size_t)block * 32 * a.qr.sn;
  float* const part = a.parts + ((size_t)share * a.B * a.H * a.n + (size_t)bh * a.n + block * 32) * D;
  join_rows_f32<D>(os, w, lane, a.n - block * 32, a.shares == 1, again, [&](int rr, const float (&acc)[D / 64]) {
    for (int c = 0; c < D / 64; ++c) {
      if (a.shares > 1) part[(size_t)rr * D + lane + 64 * c] = acc[c];
      else to[(size_t)rr * a.qr.sn + lane + 64 * c] = a.scale * acc[c];
    }
  });
  __syncthreads();
  for (; again; again &= again - 1) {
    const int rr = w * (32 / NW) + __ffs(again) - 1, tt = block * 32 + rr;
    const size_t from = head + (size_t)tt * a.qr.sn;
    PlainScratch<D>& ps = reinterpret_cast<PlainScratch<D>*>(smem)[w];
    ps.put(ps.a, static_cast<const float*>(a.q) + from, lane);
    ps.put(ps.b, static_cast<const float*>(a.dout) + from, lane);
    const TokenKeys<float> keys{kbase, vbase, a.kr.sn};
    float acc[D / 64];
    plain_dq_row<D>(keys, ps.a, ps.b, ps.p, tt, len, a.sight, scale2, __shfl(nl, rr), kLog2e, __shfl(delta, rr), lane, acc);
    for (int c = 0; c < D / 64; ++c) to[(size_t)rr * a.qr.sn + lane + 64 * c] = a.scale * acc[c];
  }
}

template <int D>
__global__ __launch_bounds__(256, 1) void window_dkv_f32_kernel(WindowArgs a) {
  constexpr int CB = D / 32, NW = kRowWaves;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32, G = a.H / a.HK;
  // blocks in turn to the XCDs: those of the first tokens, at the start of each head, have the most to do
  const int x0 = blockIdx.x / (a.B * a.HK), block = x0 / a.shares, share = x0 % a.shares, bk = blockIdx.x % (a.B * a.HK), b = bk / a.HK, hk = bk % a.HK;
  const int len = clamp_length(a.lengths, b, a.n), jb = block * 32, j = jb + m, j1 = (jb + 32 < len ? jb + 32 : len) - 1;
  const bool live = j < len;
  const int lo = live ? query_lo(a.sight, j) : 0, hi = live ? query_hi(a.sight, j, len) : 0;
  const size_t head = head_base(a.kr, bk, a.HK), row = head + (size_t)j * a.kr.sn;
  float4 k[D / 8], v[D / 8];
  load_half_row<D>(static_cast<const float*>(a.k) + row, g, live, k);
  load_half_row<D>(static_cast<const float*>(a.v) + row, g, live, v);
  f32x16 dk[CB], dv[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) { dk[c] = fill16(0.f); dv[c] = fill16(0.f); }
  const float scale2 = a.scale * kLog2e;
  const int q0 = j1 >= jb ? query_lo(a.sight, jb) / 32 : 0, qe = j1 < jb ? 0 : jb < a.sight.sinks ? len : query_hi(a.sight, j1, len);
  const int T = (qe + 31) / 32 > q0 ? (qe + 31) / 32 - q0 : 0;
  const int blo1 = query_lo(a.sight, j1 < 0 ? 0 : j1), bhi0 = j1 < a.sight.sinks ? len : query_hi(a.sight, jb < a.sight.sinks ? a.sight.sinks : jb, len);
  auto rows_of_head = [&](int hd) {
    const size_t base = head_base(a.qr, b * a.H + hk * G + hd, a.H);
    return TokenKeys<float>{static_cast<const float*>(a.q) + base, static_cast<const float*>(a.dout) + base, a.qr.sn};
  };
  for (int e = share * NW + w; e < T * G; e += NW * a.shares) {
    const int hd = e / T, i0 = (q0 + e - hd * T) * 32, last = len - 1 - i0, mine = i0 + (m < last ? m : last);
    const TokenKeys<float> rows = rows_of_head(hd);
    const size_t li = (size_t)(b * a.H + hk * G + hd) * a.n + i0;
    f32x16 s = fill16(0.f), dp;
    float nl[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int i = 8 * (r / 4) + 4 * g + r % 4, at = i < last ? i : last;
      nl[r] = a.nl[li + at]; dp[r] = a.nd[li + at];
    }
    scores_f32<D>(rows.k + (size_t)mine * a.qr.sn, g, k, s);
    scores_f32<D>(rows.v + (size_t)mine * a.qr.sn, g, v, dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = weight_f32(s[r], scale2, nl[r]);
    if (!(i0 >= blo1 && i0 + 32 <= bhi0)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = i0 + 8 * (r / 4) + 4 * g + r % 4;
        const bool on = i >= lo && i < hi;
        s[r] = on ? s[r] : 0.f;
        dp[r] = on ? dp[r] : 0.f;
      }
    }
    weighted_f32<D>([&](int i) { return rows.v + (size_t)(i0 + (i < last ? i : last)) * a.qr.sn; }, lane, s, dv);
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] *= s[r];
    weighted_f32<D>([&](int i) { return rows.k + (size_t)(i0 + (i < last ? i : last)) * a.qr.sn; }, lane, dp, dk);
  }
  if (!live) {
#pragma unroll
    for (int c = 0; c < CB; ++c) { dk[c] = fill16(0.f); dv[c] = fill16(0.f); }
  }
  float* const os = reinterpret_cast<float*>(smem);
  unsigned again = 0;
  float *const tk = static_cast<float*>(a.dk) + head + (size_t)jb * a.kr.sn, *const tv = static_cast<float*>(a.dv) + head + (size_t)jb * a.kr.sn;
  put_acc_f32<D>(os + w * 32 * D, lane, dk);
  __syncthreads();
  float* const part = a.parts + ((size_t)share * a.B * a.HK * a.n + (size_t)bk * a.n + jb) * 2 * D;      // dk, dv of a key side by side
  join_rows_f32<D>(os, w, lane, a.n - jb, a.shares == 1, again, [&](int rr, const float (&acc)[D / 64]) {
    for (int c = 0; c < D / 64; ++c) {
      if (a.shares > 1) part[(size_t)rr * 2 * D + lane + 64 * c] = acc[c];
      else tk[(size_t)rr * a.kr.sn + lane + 64 * c] = a.scale * acc[c];
    }
  });
  __syncthreads();
  put_acc_f32<D>(os + w * 32 * D, lane, dv);
  __syncthreads();
  join_rows_f32<D>(os, w, lane, a.n - jb, a.shares == 1, again, [&](int rr, const float (&acc)[D / 64]) {
    for (int c = 0; c < D / 64; ++c) {
      if (a.shares > 1) part[(size_t)rr * 2 * D + D + lane + 64 * c] = acc[c];
      else tv[(size_t)rr * a.kr.sn + lane + 64 * c] = acc[c];
    }
  });
  __syncthreads();
  for (; again; again &= again - 1) {
    const int rr = w * (32 / NW) + __ffs(again) - 1, jj = jb + rr;
    const size_t from = head + (size_t)jj * a.kr.sn;
    PlainScratch<D>& ps = reinterpret_cast<PlainScratch<D>*>(smem)[w];
    ps.put(ps.a, static_cast<const float*>(a.k) + from, lane);
    ps.put(ps.b, static_cast<const float*>(a.v) + from, lane);
    float sk[D / 64] = {}, sv[D / 64] = {};
    for (int hd = 0; hd < G; ++hd) {
      const size_t li = (size_t)(b * a.H + hk * G + hd) * a.n;
      plain_dkv_row<D>(rows_of_head(hd), ps.a, ps.b, ps.p, ps.s, query_lo(a.sight, jj), query_hi(a.sight, jj, len), scale2, kLog2e, a.nl + li, a.nd + li, lane, sk, sv);
    }
    for (int c = 0; c < D / 64; ++c) {
      tk[(size_t)rr * a.kr.sn + lane + 64 * c] = a.scale * sk[c];
      tv[(size_t)rr * a.kr.sn + lane + 64 * c] = sv[c];
    }
  }
}

// The sums over the shares, a wavefront to a row; rows that are not finite once more over what they see alone.
template <int D>
__global__ __launch_bounds__(256) void window_fwd_sum_f32_kernel(WindowArgs a) {
  __shared__ PlainScratch<D> ws[4];
  const int lane = threadIdx.x % 64, t = blockIdx.x * 4 + threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  if (t >= a.n) return;
  const size_t rows = (size_t)a.B * a.H * a.n, row = (size_t)bh * a.n + t, at = head_base(a.qr, bh, a.H) + (size_t)t * a.qr.sn;
  const float2* ml = reinterpret_cast<const float2*>(a.parts + (size_t)a.shares * rows * D);
  const float2 own = lane < a.shares ? ml[(size_t)lane * rows + row] : make_float2(-INFINITY, 0.f);
  float m = wave_max(own.x);
  const float weight = own.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(own.x - m);
  float l = wave_sum(weight * own.y), acc[D / 64] = {}, test = 0.f * (own.y + l);
  for (int s = 0; s < a.shares; ++s) {
    const float f = __shfl(weight, s);
    for (int c = 0; c < D / 64; ++c) {
      const float x = a.parts[((size_t)s * rows + row) * D + lane + 64 * c];
      acc[c] = fmaf(f, x, acc[c]);
      test = fmaf(0.f, x, test);
    }
  }
  const int len = clamp_length(a.lengths, b, a.n);
  if (t < len && __any(test != 0.f)) {
    PlainScratch<D>& ps = ws[threadIdx.x / 64];
    ps.put(ps.a, static_cast<const float*>(a.q) + at, lane);
    const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
    const TokenKeys<float> keys{static_cast<const float*>(a.k) + kv, static_cast<const float*>(a.v) + kv, a.kr.sn};
    const int lo = key_lo(a.sight, t), hi = key_hi(a.sight, t, len);
    plain_row<D>(keys, ps.a, ps.p, t, len, a.sight, 0, a.sight.sinks < lo ? a.sight.sinks : lo, lo, hi, a.scale * kLog2e, lane, m, l, acc);
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  for (int c = 0; c < D / 64; ++c) static_cast<float*>(a.o)[at + lane + 64 * c] = acc[c] * inv;
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
template <int D>
__global__ __launch_bounds__(256) void window_dq_sum_f32_kernel(WindowArgs a) {
  __shared__ PlainScratch<D> ws[4];
  const int lane = threadIdx.x % 64, t = blockIdx.x * 4 + threadIdx.x / 64, bh = blockIdx.y, b = bh / a.H, h = bh % a.H;
  if (t >= a.n) return;
  const size_t rows = (size_t)a.B * a.H * a.n, row = (size_t)bh * a.n + t, at = head_base(a.qr, bh, a.H) + (size_t)t * a.qr.sn;
  float acc[D / 64] = {}, test = 0.f;
  for (int c = 0; c < D / 64; ++c) {
    for (int s = 0; s < a.shares; ++s) acc[c] += a.parts[((size_t)s * rows + row) * D + lane + 64 * c];
    test = fmaf(0.f, acc[c], test);
  }
  const int len = clamp_length(a.lengths, b, a.n);
  if (t < len && __any(test != 0.f)) {
    PlainScratch<D>& ps = ws[threadIdx.x / 64];
    ps.put(ps.a, static_cast<const float*>(a.q) + at, lane);
    ps.put(ps.b, static_cast<const float*>(a.dout) + at, lane);
    const size_t kv = head_base(a.kr, b * a.HK + h / (a.H / a.HK), a.HK);
    const TokenKeys<float> keys{static_cast<const float*>(a.k) + kv, static_cast<const float*>(a.v) + kv, a.kr.sn};
    plain_dq_row<D>(keys, ps.a, ps.b, ps.p, t, len, a.sight, a.scale * kLog2e, a.nl[row], kLog2e, -a.nd[row], lane, acc);
  }
  for (int c = 0; c < D / 64; ++c) static_cast<float*>(a.dq)[at + lane + 64 * c] = a.scale * acc[c];
}
template <int D>
__global__ __launch_bounds__(256) void window_dkv_sum_f32_kernel(WindowArgs a) {
  __shared__ PlainScratch<D> ws[4];
  const int lane = threadIdx.x % 64, j = blockIdx.x * 4 + threadIdx.x / 64, bk = blockIdx.y, b = bk / a.HK, hk = bk % a.HK, G = a.H / a.HK;
  if (j >= a.n) return;
  const size_t rows = (size_t)a.B * a.HK * a.n, row = (size_t)bk * a.n + j, at = head_base(a.kr, bk, a.HK) + (size_t)j * a.kr.sn;
  float dk[D / 64] = {}, dv[D / 64] = {}, test = 0.f;
  for (int c = 0; c < D / 64; ++c) {
    for (int s = 0; s < a.shares; ++s) {
      const float* from = a.parts + ((size_t)s * rows + row) * 2 * D + lane + 64 * c;
      dk[c] += from[0];
      dv[c] += from[D];
    }
    test = fmaf(0.f, dk[c], fmaf(0.f, dv[c], test));
  }
  const int len = clamp_length(a.lengths, b, a.n);
  if (j < len && __any(test != 0.f)) {
    PlainScratch<D>& ps = ws[threadIdx.x / 64];
    ps.put(ps.a, static_cast<const float*>(a.k) + at, lane);
    ps.put(ps.b, static_cast<const float*>(a.v) + at, lane);
    for (int c = 0; c < D / 64; ++c) dk[c] = dv[c] = 0.f;
    for (int hd = 0; hd < G; ++hd) {
      const int bh = b * a.H + hk * G + hd;
      const size_t base = head_base(a.qr, bh, a.H), li = (size_t)bh * a.n;
      const TokenKeys<float> from{static_cast<const float*>(a.q) + base, static_cast<const float*>(a.dout) + base, a.qr.sn};
      plain_dkv_row<D>(from, ps.a, ps.b, ps.p, ps.s, query_lo(a.sight, j), query_hi(a.sight, j, len), a.scale * kLog2e, kLog2e, a.nl + li, a.nd + li, lane, dk, dv);
    }
  }
  for (int c = 0; c < D / 64; ++c) {
    static_cast<float*>(a.dk)[at + lane + 64 * c] = a.scale * dk[c];
    static_cast<float*>(a.dv)[at + lane + 64 * c] = dv[c];
  }
}

template <int D, typename Main, typename Sum>
hipError_t launch_f32(Main, Sum, WindowArgs a, int heads) {
  constexpr auto main = Main::value;
  constexpr auto sum = Sum::value;
  const long long blocks = (a.n + 31) / 32 * (long long)(a.B * heads);
  a.shares = a.parts ? f32_shares(blocks) : 1;
  if (hipError_t e = set_smem_once<main>(kF32Smem(D)); e != hipSuccess) return e;
  main<<<(unsigned)(blocks * a.shares), 256, kF32Smem(D), a.stream>>>(a);
  if (a.shares > 1) sum<<<dim3((a.n + 3) / 4, a.B * heads), 256, 0, a.stream>>>(a);
  return hipGetLastError();
}
template <int D>
hipError_t launch_fwd_f32(const WindowArgs& a) {
  return launch_f32<D>(KernelTag<&window_fwd_f32_kernel<D>>{}, KernelTag<&window_fwd_sum_f32_kernel<D>>{}, a, a.H);
}
template <int D>
hipError_t launch_bwd_f32(const WindowArgs& a) {
  if (hipError_t e = launch_f32<D>(KernelTag<&window_dq_f32_kernel<D>>{}, KernelTag<&window_dq_sum_f32_kernel<D>>{}, a, a.H); e != hipSuccess) return e;
  return launch_f32<D>(KernelTag<&window_dkv_f32_kernel<D>>{}, KernelTag<&window_dkv_sum_f32_kernel<D>>{}, a, a.HK);
}

}  // namespace attn
}  // namespace linattn
