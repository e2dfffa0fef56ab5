// Attention with the keys, not the rows, dealt to a workgroup's wavefronts: of few rows (a token or some, with the heads of their group) over a paged cache, which is
// bound by reading the cache once, and of short sequences, of which blocks of 128 rows would leave most of the chip empty.  A wavefront has tiles of its own in LDS and no barrier in its loop; the next tile is on its way while one is worked
// on, 32 KB a wavefront and 64 KB in flight for a compute unit.  Codes stay codes in LDS (half the bytes) and become bf16 where the operand is made.
// One token of 32 sequences up to 16384 tokens, 32 / 8 heads of 128: bf16 291 us = 5.2 TB/s, e4m3 159 us = 4.8 (a kernel that only reads, non-temporally, reaches 6.5 to
// 7.2 on different machines, with plain loads 6.1); one of 2000 tokens, e4m3: 10 us, latency.
#pragma once
#include "attn_rows.h"

namespace linattn {
namespace attn {

// A tile of TK rows of a wavefront's own.
template <int D, bool E4M3>
struct KeyTile {
  static constexpr int RB = D * (E4M3 ? 1 : 2), TK = 8192 / RB < 64 ? 8192 / RB : 64, BYTES = TK * RB, N = BYTES / 1024, LPR = RB / 16, KB = TK / 32;
  // where 16-byte chunk c of row r lies in its row: rows that are read together lie in different banks
  __device__ static __forceinline__ int swizzle(int r) {
    if constexpr (!E4M3) return swz<D>(r);
    else return D == 128 ? (r & 7) ^ (r >> 1 & 4) : r >> 2 & 3;
  }
  // this lane's addresses: of its row in a block of 32 (k), of its reads of the transposed rows (v)
  uint32_t krow, vrow;
  __device__ __forceinline__ explicit KeyTile(int lane) {
    const int m = lane % 32, g = lane / 32;
    if constexpr (!E4M3) {
      krow = row_at<D>(lane); vrow = turned_at<D>(lane);
    } else {
      krow = (uint32_t)(m * RB + swizzle(m) * 16 + 8 * g);
      const int x = lane % 16 / 2, r = x < 4 ? 4 * g + x : 4 + 4 * g + x;      // rows 4g .. 4g+3, 8+4g .. 8+4g+3
      vrow = (uint32_t)(r * RB + ((lane / 16 % 2) ^ swizzle(r)) * 16 + lane % 2 * 8);
    }
  }
  __device__ __forceinline__ bf16x8 k(uint32_t tile, int kb, int ks, float scale) const {
    if constexpr (!E4M3) return as_bf16x8(row_chunk<D>(tile + krow, ks, 32 * kb));
    else {
      typedef __attribute__((address_space(3))) const u32x2* P;
      const u32x2 c = *(P)(((tile + krow) ^ (uint32_t)(16 * ks)) + (uint32_t)(32 * kb * RB));
      return as_bf16x8(decode8(make_uint2(c[0], c[1]), scale));
    }
  }
  // channels 32 c .. of the sixteen rows from 16 st on, in the order that a score block's registers have
  __device__ __forceinline__ bf16x8 v(uint32_t tile, int st, int c) const {
    if constexpr (!E4M3) return turned<D>(tile + vrow, c, 16 * st);
    else {
      typedef int i32x2 __attribute__((ext_vector_type(2)));
      typedef __attribute__((address_space(3))) i32x2* P;
      // the swizzle of row r + 16 is that of row r for D = 128; for D = 64 too (16 rows are four groups of four)
      const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((P)(((tile + vrow) ^ (uint32_t)(32 * c)) + (uint32_t)(16 * st * RB)));
      return as_bf16x8(decode8(make_uint2((uint32_t)x[0], (uint32_t)x[1]), 1.0f));
    }
  }
};

// Where the keys come from: look(j0, end) finds the rows of a tile (of keys from `end` on the last one's again), k_row and v_row are where row r of it lies.
template <int D, bool E4M3>
struct KeysOfPool {
  using Args = Pool;
  static constexpr bool kE4M3 = E4M3;
  const Pool& p;
  int b, hk, lane, len, tokens, count;
  PoolRows rows;
  unsigned long long there;
  __device__ __forceinline__ KeysOfPool(const Args& a, int b_, int hk_, int n, int lane_) : p(a), b(b_), hk(hk_), lane(lane_) {
    len = pool_length(p, b);
    tokens = pool_tokens(p, b);
    count = clamp_length(p.counts, b, n);
  }
  template <int TK>
  __device__ __forceinline__ void look(int j0, int end) {
    rows.find<TK>(p, b, hk, j0, end, lane);
    there = rows.there;
  }
  __device__ __forceinline__ size_t offset(int r) const { return (size_t)rows.of(r) * (D * (E4M3 ? 1 : 2)); }
  __device__ __forceinline__ const char* k_row(size_t at) const { return static_cast<const char*>(p.k) + at; }
  __device__ __forceinline__ const char* v_row(size_t at) const { return static_cast<const char*>(p.v) + at; }
  __device__ __forceinline__ PoolKeys<E4M3> keys() const { return {&p, b, hk, D}; }
};
template <int D>
struct KeysOfTokens {
  using Args = TokenArgs;
  static constexpr bool kE4M3 = false;
  const char *k, *v;
  size_t sn;
  int len, tokens, count, j0, last;
  static constexpr unsigned long long there = ~0ull;
  __device__ __forceinline__ KeysOfTokens(const Args& a, int b, int hk, int n, int) : sn(a.kr.sn) {
    count = tokens = len = clamp_length(a.lengths, b, n);
    const size_t at = ((size_t)b * a.kr.sb + (size_t)hk * a.kr.sh) * 2;
    k = static_cast<const char*>(a.k) + at;
    v = static_cast<const char*>(a.v) + at;
  }
  template <int TK>
  __device__ __forceinline__ void look(int j, int end) { j0 = j; last = end - 1; }
  __device__ __forceinline__ size_t offset(int r) const { return (size_t)(j0 + r < last ? j0 + r : last) * sn * 2; }
  __device__ __forceinline__ const char* k_row(size_t at) const { return k + at; }
  __device__ __forceinline__ const char* v_row(size_t at) const { return v + at; }
  __device__ __forceinline__ TokenKeys<uint16_t> keys() const { return {reinterpret_cast<const uint16_t*>(k), reinterpret_cast<const uint16_t*>(v), sn}; }
};

template <int D, int QB, typename From>
__global__ __launch_bounds__(64 * kRowWaves, 1) void attn_keys_kernel(RowsArgs a, typename From::Args from_args) {
  constexpr bool E4M3 = From::kE4M3;
  using T = KeyTile<D, E4M3>;
  constexpr int KS = D / 16, CB = D / 32, TK = T::TK, KB = T::KB, NW = kRowWaves, WAVE = 4 * T::BYTES + 256;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const int split = blockIdx.x % a.splits, row0 = blockIdx.x / a.splits * (32 * QB), b = blockIdx.y / a.HK, hk = blockIdx.y % a.HK, G = a.G;
  From src(from_args, b, hk, a.n, lane);
  const int len = src.len, count = src.count, pos0 = src.tokens - count, t0 = pos0 < 0 ? -pos0 : 0, rows = count * G, all = a.n * G;

  uint4 q[QB][KS];
  int lo[QB], hi[QB];
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    const int r = row0 + 32 * i + m, t = r / G, h = hk * G + (r - t * G);
    const bool live = r < rows && t >= t0;
    lo[i] = live ? key_lo(a.sight, pos0 + t) : 0;
    hi[i] = live ? key_hi(a.sight, pos0 + t, len) : 0;
    const uint16_t* from = static_cast<const uint16_t*>(a.q) + (size_t)b * a.qr.sb + (size_t)h * a.qr.sh + (size_t)t * a.qr.sn + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[i][ks] = live ? *reinterpret_cast<const uint4*>(from + 16 * ks) : make_uint4(0, 0, 0, 0);
  }
  f32x16 o[QB][CB];
  float mx[QB], l[QB];
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    mx[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < CB; ++c) o[i][c] = fill16(0.f);
  }

  const int first = row0 / G > t0 ? row0 / G : t0, end_row = (row0 + 32 * QB < rows ? row0 + 32 * QB : rows) - 1;
  const int p0 = pos0 + first, p1 = end_row >= 0 && end_row / G >= first ? pos0 + end_row / G : -1;
  const KeyTiles<TK> tiles(a.sight, p0, p1, len);
  const WaveSight sight(a.sight, p0, p1, len);
  const int it0 = (int)((long long)tiles.count * split / a.splits), it1 = (int)((long long)tiles.count * (split + 1) / a.splits);
  const uint32_t lds = lds_address(smem) + (uint32_t)(w * WAVE);
  float* const vs = reinterpret_cast<float*>(smem + w * WAVE + 4 * T::BYTES);      // the scales of the tile's v rows
  const T tile(lane);
  unsigned long long there_next = 0;
  uint32_t ek = 0, ev = 0;
  auto look = [&](int i) { src.template look<TK>(tiles.start(i), tiles.end); };
  auto request = [&](int i, uint32_t to) {
    there_next = src.there;
#pragma unroll
    for (int x = 0; x < T::N; ++x) {
      const int r = x * (64 / T::LPR) + lane / T::LPR;
      const size_t from = src.offset(r) + (size_t)(((lane % T::LPR) ^ T::swizzle(r)) * 16);
      load_to_lds(src.k_row(from), to + x * 1024);
      load_to_lds(src.v_row(from), to + T::BYTES + x * 1024);
    }
    if constexpr (E4M3) { ek = src.p.k_exp[src.rows.row]; ev = src.p.v_exp[src.rows.row]; }
  };
  int it = it0 + w;
  if (it < it1) {
    look(it);
    request(it, lds);
    if (it + NW < it1) look(it + NW);
  }
  for (int buf = 0; it < it1; it += NW, buf ^= 1) {
    const uint32_t kt = lds + (uint32_t)buf * 2 * T::BYTES, vt = kt + T::BYTES;
    const unsigned long long there = there_next;
    const float ks_own = E4M3 ? row_scale((uint8_t)ek) : 1.f;      // of key `lane`
    if constexpr (E4M3) vs[lane] = row_scale((uint8_t)ev);
    lds_loads_landed();
    if (it + NW < it1) {
      request(it + NW, lds + (uint32_t)(buf ^ 1) * 2 * T::BYTES);
      if (it + 2 * NW < it1) look(it + 2 * NW);
    }
    if (there == 0) continue;
    const int j0 = tiles.start(it);
    const bool plain = sight.everything(j0, TK) && there == ~0ull;
    f32x16 s[QB][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const float scale = E4M3 ? __shfl(ks_own, 32 * kb + m) : 1.f;
#pragma unroll
      for (int i = 0; i < QB; ++i) s[i][kb] = fill16(0.f);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 kop = tile.k(kt, kb, ks, scale);
#pragma unroll
        for (int i = 0; i < QB; ++i) s[i][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop, as_bf16x8(q[i][ks]), s[i][kb], 0, 0, 0);
      }
    }
    uint4 p[QB][2 * KB];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      if (!plain) {
        asm volatile("");
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int x = 32 * kb + 8 * (r / 4) + 4 * g + r % 4, j = j0 + x;
            const bool on = j < hi[i] && (j >= lo[i] || j < a.sight.sinks) && (there >> x & 1);
            s[i][kb][r] = on ? s[i][kb][r] : -INFINITY;
          }
      }
      softmax_step<KB, CB>(s[i], a.scale2, mx[i], l[i], o[i]);
      if constexpr (E4M3) {
        // The codes of v enter as they are: their scales go to the weights, before those are rounded to bf16.  The scales are powers of two, so that the
        // rounding is the same relative one as of the weights alone.
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const float4 f = *reinterpret_cast<const float4*>(vs + 32 * kb + 2 * r + 4 * g);
            s[i][kb][r] *= f.x; s[i][kb][r + 1] *= f.y; s[i][kb][r + 2] *= f.z; s[i][kb][r + 3] *= f.w;
          }
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) p[i][2 * kb + h2] = pack8(s[i][kb], h2);
    }
#pragma unroll
    for (int st = 0; st < 2 * KB; ++st)
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const bf16x8 vop = tile.v(vt, st, c);
#pragma unroll
        for (int i = 0; i < QB; ++i) o[i][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop, as_bf16x8(p[i][st]), o[i][c], 0, 0, 0);
      }
  }

  // The wavefronts' parts, joined in LDS: [wavefront][row][OS] and the pairs of maximum and sum behind them.  Eight threads have a row.
  __syncthreads();
  constexpr int OS = D + 4;                              // floats from row to row, so that rows begin in different banks
  float* const os = reinterpret_cast<float*>(smem);
  float2* const ml = reinterpret_cast<float2*>(os + NW * 32 * OS);
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    float x, y;
    pair32(l[i], x, y);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<float4*>(os + (w * 32 + m) * OS + 32 * c + 2 * e + 4 * g) =
            make_float4(o[i][c][e], o[i][c][e + 1], o[i][c][e + 2], o[i][c][e + 3]);
    if (g == 0) ml[w * 32 + m] = make_float2(mx[i], x + y);
    __syncthreads();
    const int rr = w * 8 + lane / 8, part = lane % 8, r = row0 + 32 * i + rr, t = r / G, h = hk * G + (r - t * G);
    const bool live = r < rows && t >= t0;
    float top = -INFINITY, sum = 0.f, test = 0.f, f[NW];
    float4 acc[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int v = 0; v < NW; ++v) top = fmaxf(top, ml[v * 32 + rr].x);
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float2 e = ml[v * 32 + rr];
      f[v] = e.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e.x - top);
      sum = fmaf(f[v], e.y, sum);
      test = fmaf(0.f, e.y, test);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const float4 z = *reinterpret_cast<const float4*>(os + (v * 32 + rr) * OS + 32 * c + 4 * part);
        acc[c].x = fmaf(f[v], z.x, acc[c].x); acc[c].y = fmaf(f[v], z.y, acc[c].y);
        acc[c].z = fmaf(f[v], z.z, acc[c].z); acc[c].w = fmaf(f[v], z.w, acc[c].w);
        test = fmaf(0.f, z.x, fmaf(0.f, z.y, fmaf(0.f, z.z, fmaf(0.f, z.w, test))));
      }
    }
    if (!live) {
      top = -INFINITY; sum = 0.f; test = 0.f;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const unsigned long long off = __ballot(test != 0.f);
    if (r < all && !(off >> (lane & 56) & 255)) {
      const size_t at = (size_t)b * a.qr.sb + (size_t)h * a.qr.sh + (size_t)t * a.qr.sn + 4 * part, li = ((size_t)b * a.H + h) * a.n + t;
      if (a.splits > 1) {
        float* to = a.parts + ((size_t)split * a.B * a.H * a.n + li) * D + 4 * part;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) *reinterpret_cast<float4*>(to + 32 * c) = acc[c];
        if (part == 0) put_part(a, D, split, li, top, sum);
      } else {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o) + at + 32 * c) =
              make_uint2(pack_bf16x2(acc[c].x * inv, acc[c].y * inv), pack_bf16x2(acc[c].z * inv, acc[c].w * inv));
        if (a.lse && part == 0) a.lse[li] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
      }
    }
    __syncthreads();
    for (int x8 = 0; x8 < 8; ++x8)
      if (off >> (8 * x8) & 255)
        plain_again<D>(a, src.keys(), tiles, it0, it1, row0 + 32 * i + w * 8 + x8, b, hk, split, a.splits, pos0, len, reinterpret_cast<PlainScratch<D>*>(smem)[w],
                       lane);
    if (QB > 1) __syncthreads();
  }
}

template <int D, typename From>
hipError_t launch_keys(RowsArgs a, const typename From::Args& from, hipStream_t s) {
  using T = KeyTile<D, From::kE4M3>;
  constexpr size_t tiles = kRowWaves * (4 * T::BYTES + 256), join = kRowWaves * 32 * ((D + 4) * 4 + 8), smem = tiles > join ? tiles : join;
  auto go = [&](auto kernel, int rows) -> hipError_t {
    constexpr auto k = decltype(kernel)::value;
    if (hipError_t e = set_smem_once<k>(smem); e != hipSuccess) return e;
    a.blocks = (a.n * a.G + rows - 1) / rows;
    k<<<dim3(a.splits * a.blocks, a.B * a.HK), 64 * kRowWaves, smem, s>>>(a, from);
    return launch_join<D>(a, s);
  };
  // blocks of 64 rows where there are more than 32 and a cache is to be read once
  if constexpr (!std::is_same_v<typename From::Args, TokenArgs>)
    if (a.n * a.G > 32) return go(KernelTag<&attn_keys_kernel<D, 2, From>>{}, 64);
  return go(KernelTag<&attn_keys_kernel<D, 1, From>>{}, 32);
}

}  // namespace attn
}  // namespace linattn
