// Softmax attention of blocks of query rows on the matrix cores (bf16 operands, fp32 scores and sums).
#pragma once
#include "attn_plain.h"
#include "attn_tile.h"

namespace linattn {
namespace attn {

// Rows of a block: the query heads of a key head's group side by side, row = token * G + head, so that a group's keys are read once.
struct RowsArgs {
  const void *q, *k, *v;
  void* o;
  float* lse;
  const int* lengths;
  int B, H, HK, G, n;
  int blocks;               // row blocks of a (batch item, key head)
  Rows qr, kr;
  Sight sight;
  float scale2;             // scale * log2(e)
};

__device__ __forceinline__ f32x16 fill16(float x) {
  f32x16 r;
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = x;
  return r;
}

// Workgroups are dealt to the eight XCDs in turn; neighbouring blocks of rows share keys, so each XCD gets a stretch of neighbours.
__device__ __forceinline__ int xcd_stretch(int i, int count) {
  const int per = (count + kXCDs - 1) / kXCDs, full = count % kXCDs ? count % kXCDs : kXCDs;      // the first `full` XCDs have `per`
  const int x = i % kXCDs, at = i / kXCDs;
  return x < full ? x * per + at : full * per + (x - full) * (per - 1) + at;
}

// The row block of the i-th workgroup of a head.  Where a row's keys grow along the sequence (a limit on one side only) long and short blocks alternate, so
// that any stretch of them has the same work.
__device__ __forceinline__ int row_block(const Sight& s, int i, int blocks) {
  if ((s.left < 0) == (s.right < 0)) return blocks - 1 - i;
  return i % 2 ? i / 2 : blocks - 1 - i / 2;
}

// The tiles of KT keys that the rows of a block see, positions p0 .. p1: those of the first tokens, then those of the window.
template <int KT>
struct KeyTiles {
  int nsink, wtile, count, end;
  __device__ __forceinline__ KeyTiles(const Sight& s, int p0, int p1, int len) {
    end = p1 >= p0 ? key_hi(s, p1, len) : 0;
    const int from = key_lo(s, p0), first = s.sinks < from ? s.sinks : from, last = (end + KT - 1) / KT;
    nsink = (first + KT - 1) / KT;
    wtile = from / KT > nsink ? from / KT : nsink;
    nsink = nsink < last ? nsink : last;
    count = nsink + (last > wtile ? last - wtile : 0);
  }
  __device__ __forceinline__ int start(int i) const { return (i < nsink ? i : wtile + i - nsink) * KT; }
};
// What a wavefront's rows at positions p0 .. p1 see of a tile from key j0 on: nothing, or everything.
struct WaveSight {
  int lo0, lo1, hi0, hi1, sinks;
  bool rows, whole;         // whether it has any; whether all of its rows are tokens
  __device__ __forceinline__ WaveSight(const Sight& s, int p0, int p1, int len, bool all)
      : lo0(key_lo(s, p0)), lo1(key_lo(s, p1)), hi0(key_hi(s, p0, len)), hi1(key_hi(s, p1, len)), sinks(s.sinks), rows(p1 >= p0), whole(all) {}
  __device__ __forceinline__ bool nothing(int j0, int count) const { return !rows || j0 >= hi1 || (j0 + count <= lo0 && j0 >= sinks); }
  __device__ __forceinline__ bool everything(int j0, int count) const { return whole && j0 + count <= hi0 && (j0 >= lo1 || j0 + count <= sinks); }
};

template <int D, int QB, int NW, int KT, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void attn_rows_kernel(RowsArgs a) {
  constexpr int KB = KT / 32, KS = D / 16, CB = D / 32, BM = 32 * QB * NW, TILE = KT * D * 2;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const int id = xcd_stretch(blockIdx.x, gridDim.x), bk = id / a.blocks, block = row_block(a.sight, id % a.blocks, a.blocks);
  const int b = bk / a.HK, hk = bk % a.HK, G = a.G;
  const int len = clamp_length(a.lengths, b, a.n), rows = len * G, all = a.n * G;
  const int row0 = block * BM + w * 32 * QB;

  // this lane's queries
  uint4 q[QB][KS];
  int lo[QB], hi[QB];
  size_t at[QB];
  bool store[QB];
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    const int r = row0 + 32 * i + m, t = r / G, h = hk * G + (r - t * G);
    store[i] = r < all;
    at[i] = (size_t)b * a.qr.sb + (size_t)h * a.qr.sh + (size_t)t * a.qr.sn;
    const bool live = r < rows;
    lo[i] = live ? key_lo(a.sight, t) : 0;
    hi[i] = live ? key_hi(a.sight, t, len) : 0;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      q[i][ks] = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at[i] + 16 * ks + 8 * g) : make_uint4(0, 0, 0, 0);
  }

  f32x16 o[QB][CB];
  float mx[QB], l[QB];
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    mx[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][c][r] = 0.f;
  }

  const int last_row = ((block + 1) * BM < rows ? (block + 1) * BM : rows) - 1, wlast = (row0 + 32 * QB < rows ? row0 + 32 * QB : rows) - 1;
  const KeyTiles<KT> tiles(a.sight, block * BM / G, last_row < block * BM ? -1 : last_row / G, len);
  const WaveSight sight(a.sight, row0 / G, wlast < row0 ? -1 : wlast / G, len, row0 + 32 * QB <= rows);
  const size_t kv = (size_t)b * a.kr.sb + (size_t)hk * a.kr.sh, pitch = a.kr.sn * 2;
  const char *kbase = static_cast<const char*>(a.k) + kv * 2, *vbase = static_cast<const char*>(a.v) + kv * 2;
  const RowTile<D, NW, KT> loader(w, lane);
  const uint32_t lds = lds_address(smem);
  auto request = [&](int i) {
    const int j0 = tiles.start(i);
    const uint32_t to = lds + (uint32_t)(i & 1) * 2 * TILE;
    loader.load(kbase, pitch, j0, tiles.end, to, w);
    loader.load(vbase, pitch, j0, tiles.end, to + TILE, w);
  };
  const uint32_t rows_at = row_at<D>(lane), turned_rows = turned_at<D>(lane);

  if (tiles.count) request(0);
  lds_loads_landed();
  __syncthreads();
  for (int it = 0; it < tiles.count; ++it) {
    if (it + 1 < tiles.count) request(it + 1);
    const int j0 = tiles.start(it);
    const uint32_t kt = lds + (uint32_t)(it & 1) * 2 * TILE, vt = kt + TILE;
    if (!sight.nothing(j0, KT)) {
      const bool plain = sight.everything(j0, KT);
      f32x16 s[QB][KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < QB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[i][kb][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const bf16x8 kop = as_bf16x8(row_chunk<D>(kt + rows_at, ks, 32 * kb));
#pragma unroll
          for (int i = 0; i < QB; ++i) s[i][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop, as_bf16x8(q[i][ks]), s[i][kb], 0, 0, 0);
        }
      uint4 p[QB][2 * KB];
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        if (!plain) {
          asm volatile("");        // a branch: as selects, the mask is computed for every tile
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = j0 + 32 * kb + 8 * (r / 4) + 4 * g + r % 4;
              s[i][kb][r] = j < hi[i] && (j >= lo[i] || j < a.sight.sinks) ? s[i][kb][r] : -INFINITY;
            }
        }
        float top = s[i][0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][kb][r]);
        float x, y;
        pair32(top, x, y);
        top = fmaxf(x, y) * a.scale2;
        // The running maximum moves only where it has grown by more than 8: the probabilities are then at most 2^8, and the sums the same
        // after the division.
        if (__any(top > mx[i] + 8.f)) {
          const float next = fmaxf(mx[i], top), alpha = mx[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx[i] - next);
          mx[i] = next;
          l[i] *= alpha;
#pragma unroll
          for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][c][r] *= alpha;
        }
        const float c0 = mx[i] == -INFINITY ? 0.f : -mx[i];
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[i][kb][r], a.scale2, c0));
            s[i][kb][r] = e;
            sum += e;
          }
        l[i] += sum;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int h2 = 0; h2 < 2; ++h2) {
            const f32x16& e = s[i][kb];
            p[i][2 * kb + h2] = make_uint4(pack_bf16x2(e[8 * h2], e[8 * h2 + 1]), pack_bf16x2(e[8 * h2 + 2], e[8 * h2 + 3]),
                                           pack_bf16x2(e[8 * h2 + 4], e[8 * h2 + 5]), pack_bf16x2(e[8 * h2 + 6], e[8 * h2 + 7]));
          }
      }
#pragma unroll
      for (int st = 0; st < 2 * KB; ++st)
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          const bf16x8 vop = turned<D>(vt + turned_rows, c, 16 * st);
#pragma unroll
          for (int i = 0; i < QB; ++i) o[i][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop, as_bf16x8(p[i][st]), o[i][c], 0, 0, 0);
        }
    }
    lds_loads_landed();
    __syncthreads();
  }

#pragma unroll
  for (int i = 0; i < QB; ++i) {
    float x, y;
    pair32(l[i], x, y);
    const float sum = x + y, inv = sum == 0.f ? 0.f : 1.0f / sum;
    const int r = row0 + 32 * i + m, t = r / G;
    const size_t li = ((size_t)b * a.H + hk * G + (r - t * G)) * a.n + t;
    // A key that is masked has weight 0, and 0 times an infinity or NaN in its value would be NaN: rows that come out not finite are done again
    // key by key.
    if (!sight.whole && hi[i] == 0) {
#pragma unroll
      for (int c = 0; c < CB; ++c) o[i][c] = fill16(0.f);
    }
    float test = 0.f * sum;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) test = fmaf(0.f, o[i][c][e], test);
    uint32_t again = (uint32_t)__ballot(test != 0.f) | (uint32_t)(__ballot(test != 0.f) >> 32);
    if (store[i] && !(again >> m & 1)) {
      uint16_t* out = static_cast<uint16_t*>(a.o) + at[i] + 4 * g;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<uint2*>(out + 32 * c + 2 * e) = make_uint2(pack_bf16x2(o[i][c][e] * inv, o[i][c][e + 1] * inv),
                                                                       pack_bf16x2(o[i][c][e + 2] * inv, o[i][c][e + 3] * inv));
      if (a.lse && g == 0) a.lse[li] = sum == 0.f ? -INFINITY : (mx[i] + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    for (; again; again &= again - 1) {
      const int rr = row0 + 32 * i + __ffs(again) - 1, tt = rr / G, hh = hk * G + (rr - tt * G);
      const size_t from = (size_t)b * a.qr.sb + (size_t)hh * a.qr.sh + (size_t)tt * a.qr.sn;
      PlainScratch<D>& ps = reinterpret_cast<PlainScratch<D>*>(smem)[w];
      ps.put(ps.a, static_cast<const uint16_t*>(a.q) + from, lane);
      const TokenKeys<uint16_t> keys{reinterpret_cast<const uint16_t*>(kbase), reinterpret_cast<const uint16_t*>(vbase), a.kr.sn};
      float pm, pl, acc[D / 64];
      plain_row<D>(keys, ps.a, ps.p, tt, len, a.sight, a.scale2, lane, pm, pl, acc);
      const float pinv = pl == 0.f ? 0.f : 1.0f / pl;
      for (int c = 0; c < D / 64; ++c) store1(static_cast<uint16_t*>(a.o) + from + lane + 64 * c, acc[c] * pinv);
      if (a.lse && lane == 0) a.lse[((size_t)b * a.H + hh) * a.n + tt] = pl == 0.f ? -INFINITY : (pm + __builtin_amdgcn_logf(pl)) * kLn2;
    }
  }
}

template <int D, int QB, int NW, int KT, int OCC>
hipError_t launch_rows(RowsArgs a, hipStream_t s) {
  constexpr int BM = 32 * QB * NW;
  constexpr size_t smem = 4 * KT * D * 2;
  a.blocks = (int)(((long long)a.n * a.G + BM - 1) / BM);
  constexpr auto kernel = &attn_rows_kernel<D, QB, NW, KT, OCC>;
  if (hipError_t e = set_smem_once<kernel>(smem); e != hipSuccess) return e;
  kernel<<<(unsigned)(a.B * a.HK * a.blocks), 64 * NW, smem, s>>>(a);
  return hipGetLastError();
}

}  // namespace attn
}  // namespace linattn
