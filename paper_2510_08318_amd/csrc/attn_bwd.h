// Backward of windowed softmax attention on the matrix cores (bf16 operands, fp32 scores, gradients and sums), without atomics: one kernel owns the
// rows of dq, one those of dk and dv, and each works the probabilities out again from the forward's lse.
#pragma once
#include "attn_rows.h"
#include "mfma16.h"

namespace linattn {
namespace attn {

constexpr int BT = 64;                       // keys, or queries, of a tile

struct BwdRows {
  const void *q, *k, *v, *out, *dout;
  void *dq, *dk, *dv;
  const float* lse;
  float *nl, *nd;           // fp32 [B*H][n], written by the query side: -lse / scale (-inf where nothing is seen), -delta
  float* parts;             // fp32 [part][2][key_block][D]: dk (not yet scaled) and dv of the key blocks that several workgroups share
  const int* lengths;
  int B, H, HK, G, n;
  int blocks;               // row blocks, or key blocks, of a (batch item, key head)
  int sink_blocks;          // key blocks that hold first tokens
  int sink_share, share;    // workgroups to such a block, to another
  Rows qr, kr;
  Sight sight;
  float scale, scale2;
};

// ---- dq -----------------------------------------------------------------------------------
// Queries on the lanes, as in the forward: S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.  12 heads x 32760 x 128, window 2 x 1560 and 1560 first tokens: 1.40 to 1.43 ms,
// 950 to 970 TFLOP/s; the matrix cores are busy 49 % of the cycles, a quarter of a wavefront's time goes to waits.  Width 64, 2 x 12 heads of unlike lengths to 4133, causal,
// window 1024: 75 us; the matrix cores are busy 15 % of the cycles, with 1.35 wavefronts to a SIMD on average over the kernel.
// dS is rounded to bf16, as K is stored (PIECES 1): the error of dq that this and the store leave is 2.35e-3.
// EXACT: delta from a first pass over the keys, sum_j p_ij dp_ij, and not from dout . out.  Where a row sees few keys its output is as large as the
// values, and the rounding of the stored output would be the largest error of dq and dk.  With fp32 arithmetic (PIECES 3) always.
// A key counts as a row's heaviest only with more weight than this.  Error of dq (2-norm over two heads, 1e-3), without the correction / above 1/2 / 1/8 / 1/32: 12 heads x 4133 x 64
// causal 2.75 / 2.59 / 2.50 / 2.49, with scores nine times as large 4.56 / 2.84 / 2.64 / 2.64; window 1024 2.51 / 2.47 / 2.43 / 2.42 and 5.50 / 2.76 / 2.64 / 2.64; 600 x 64, all keys,
// 2.49 / 2.49 / 2.41 / 2.40 and 4.95 / 2.67 / 2.55 / 2.55.  Us of the backward there: 229 / 227 / 229 / 235, 115 / 115 / 116 / 121, 39 / 39 / 41 / 43.
constexpr float kHeavyWeight = 0.125f;

template <int D, bool EXACT, int PIECES>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void window_dq_kernel(BwdRows a) {
  constexpr int NW = 4, KB = BT / 32, KS = D / 16, CB = D / 32, BM = 32 * NW, TILE = BT * D * 2;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const PairPlace where = pair_place(blockIdx.x, a.B * a.HK, a.blocks);
  const int bk = where.pair, block = row_block(a.sight, where.at, a.blocks);
  const int b = bk / a.HK, hk = bk % a.HK, G = a.G;
  const int len = clamp_length(a.lengths, b, a.n), rows = len * G, all = a.n * G;
  const int row0 = block * BM + w * 32;

  // where a lane's row lies (worked out again after the loop, where there are registers for it)
  struct Place {
    int t;
    bool store, live;
    size_t at, li;
  };
  auto place = [&](int lane_) {
    Place p;
    const int r = row0 + lane_ % 32;
    p.t = r / G;
    const int h = hk * G + (r - p.t * G);
    p.store = r < all; p.live = r < rows;
    p.at = (size_t)b * a.qr.sb + (size_t)h * a.qr.sh + (size_t)p.t * a.qr.sn;
    p.li = ((size_t)b * a.H + h) * a.n + p.t;
    return p;
  };
  const Place first = place(lane);
  const bool live = first.live;
  const size_t at = first.at;
  uint4 q[KS], go[KS];
  float delta = 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const size_t c = at + 16 * ks + 8 * g;
    q[ks] = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + c) : make_uint4(0, 0, 0, 0);
    go[ks] = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.dout) + c) : make_uint4(0, 0, 0, 0);
  }
  if (!EXACT) {
    uint4 ov[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      ov[ks] = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.out) + at + 16 * ks + 8 * g) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float x[8], y[8];
      unpack_bf16x8(ov[ks], x);
      unpack_bf16x8(go[ks], y);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(x[e], y[e], delta);
    }
    float x, y;
    pair32(delta, x, y);
    delta = x + y;
  }
  const float lse = live ? a.lse[first.li] : -INFINITY, nl2 = lse == -INFINITY ? lse : -lse * kLog2e;

  const int last_row = ((block + 1) * BM < rows ? (block + 1) * BM : rows) - 1, wlast = (row0 + 32 < rows ? row0 + 32 : rows) - 1;
  const KeyTiles<BT> tiles(a.sight, block * BM / G, last_row < block * BM ? -1 : last_row / G, len);
  const WaveSight sight(a.sight, row0 / G, wlast < row0 ? -1 : wlast / G, len);
  const size_t kv = (size_t)b * a.kr.sb + (size_t)hk * a.kr.sh, pitch = a.kr.sn * 2;
  const char *kbase = static_cast<const char*>(a.k) + kv * 2, *vbase = static_cast<const char*>(a.v) + kv * 2;
  const RowTile<D, NW, BT> loader(w, lane);
  const TileOrder<BT> order(tiles, 0, tiles.count);
  const uint32_t lds = lds_address(smem);
  auto request = [&](int i) {
    const int j0 = tiles.start(order(i));
    const uint32_t to = lds + (uint32_t)(i & 1) * 2 * TILE;
    loader.load(kbase, pitch, j0, tiles.end, to, w);
    loader.load(vbase, pitch, j0, tiles.end, to + TILE, w);
  };

  arrived(q);
  arrived(go);
  f32x16 dq[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) dq[c] = fill16(0.f);

  // one pass over the tiles: use(kb, p, dp, kt) of the probabilities and dP of 32 keys
  auto pass = [&](auto use) {
    if (tiles.count) request(0);
    lds_loads_landed();
    __syncthreads();
    for (int it = 0; it < tiles.count; ++it) {
      if (it + 1 < tiles.count) request(it + 1);
      const int j0 = tiles.start(order(it));
      const uint32_t kt = lds + (uint32_t)(it & 1) * 2 * TILE, vt = kt + TILE;
      if (!sight.nothing(j0, BT)) {
        const bool plain = sight.everything(j0, BT);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          f32x16 s = fill16(0.f), dp = fill16(0.f);
          const uint32_t rows_at = row_at<D>((int)opaque_lane(lane));
          pipelined_operands<2 * KS, 4>([&](int x) { return row_chunk<D>((x % 2 ? vt : kt) + rows_at, x / 2, 32 * kb); },
                                        [&](int x, uint4 op) {
                                          if (x % 2) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(op), as_bf16x8(go[x / 2]), dp, 0, 0, 0);
                                          else s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(op), as_bf16x8(q[x / 2]), s, 0, 0, 0);
                                        });
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, nl2));
          if (!plain) {
            const Place mine = place((int)opaque_lane(lane));      // (opaque: a branch; as selects, the mask is computed for every tile)
            const int lo = mine.live ? key_lo(a.sight, mine.t) : 0, hi = mine.live ? key_hi(a.sight, mine.t, len) : 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = j0 + 32 * kb + 8 * (r / 4) + 4 * g + r % 4;
              const bool on = j < hi && (j >= lo || j < a.sight.sinks);
              s[r] = on ? s[r] : 0.f;
              dp[r] = on ? dp[r] : 0.f;
            }
          }
          use(kb, s, dp, kt, j0);
        }
      }
      lds_loads_landed();
      __syncthreads();
    }
  };
  if (EXACT) {
    pass([&](int, const f32x16& p, const f32x16& dp, uint32_t, int) {
#pragma unroll
      for (int r = 0; r < 16; ++r) delta = fmaf(p[r], dp[r], delta);
    });
    float x, y;
    pair32(delta, x, y);
    delta = x + y;
  }
  // delta from the stored output is off by what its rounding took, which is the sum of the row's dS; the key side gets it corrected.  dq is off by that times the
  // mean key of the row, which is small beside a key unless a few have most of the weight: the heaviest one's part of it is taken out at the end (12
  // heads x 4133 x 64, causal, normalised q and k of scale 0.5 to 1.5: error of dq 2.6e-3, with it 2.4e-3, where rounding dS and dq alone is 2.35e-3).
  float off = 0.f, heavy = kHeavyWeight;
  int at_key = -1;
  pass([&](int kb, const f32x16& p, f32x16& dp, uint32_t kt, int j0) {
    const uint32_t turned_rows = turned_at<D>((int)opaque_lane(lane));
    if (!EXACT) {
      float top = p[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, p[r]);
      if (__any(top > heavy)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (p[r] > heavy) { heavy = p[r]; at_key = j0 + 32 * kb + 8 * (r / 4) + 4 * g + r % 4; }
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dp[r] = p[r] * (dp[r] - delta);
      if (!EXACT) off += dp[r];
    }
    uint4 ds[PIECES == 1 ? 2 : 1][PIECES];
    if constexpr (PIECES == 1) { ds[0][0] = pack8(dp, 0); ds[1][0] = pack8(dp, 1); }
    pipelined_operands<2 * CB, 3>([&](int x) { return __builtin_bit_cast(uint4, turned<D>(kt + turned_rows, x % CB, 16 * (2 * kb + x / CB))); },
                                  [&](int x, uint4 op) {
                                    if (PIECES > 1 && x % CB == 0) weights_operand<PIECES>(dp, x / CB, ds[0]);
                                    dq[x % CB] = mfma_weights<PIECES>(as_bf16x8(op), ds[PIECES == 1 ? x / CB : 0], dq[x % CB]);
                                  });
  });
  if (!EXACT) {
    float x, y;
    pair32(off, x, y);
    off = x + y;
    delta += off;
    if (__any(at_key >= 0)) {
      float h0, h1, k0, k1;
      pair32(heavy, h0, h1);
      pair32(__builtin_bit_cast(float, at_key), k0, k1);
      heavy = fmaxf(h0, h1);
      at_key = __builtin_bit_cast(int, h1 > h0 ? k1 : k0);
      if (at_key >= 0) {
        const uint16_t* kr = reinterpret_cast<const uint16_t*>(kbase + (size_t)at_key * pitch) + 4 * g;
        const float f = -off * heavy;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const uint2 y4 = *reinterpret_cast<const uint2*>(kr + 32 * c + 2 * r);
            dq[c][r] = fmaf(f, f32::lo_f32(y4.x), dq[c][r]); dq[c][r + 1] = fmaf(f, f32::hi_f32(y4.x), dq[c][r + 1]);
            dq[c][r + 2] = fmaf(f, f32::lo_f32(y4.y), dq[c][r + 2]); dq[c][r + 3] = fmaf(f, f32::hi_f32(y4.y), dq[c][r + 3]);
          }
      }
    }
  }
  const Place here = place((int)opaque_lane(lane));
  const float nl = nl2 == -INFINITY ? nl2 : nl2 / a.scale2;
  if (here.store && g == 0) {
    a.nl[here.li] = nl;
    a.nd[here.li] = -delta;
  }

  // Masked keys have dS = 0, which an infinity or NaN in k would make NaN: rows that come out not finite are done again key by key.
  if (!here.live) {
#pragma unroll
    for (int c = 0; c < CB; ++c) dq[c] = fill16(0.f);
  }
  float test = 0.f;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) test = fmaf(0.f, dq[c][r], test);
  uint32_t again = (uint32_t)__ballot(test != 0.f) | (uint32_t)(__ballot(test != 0.f) >> 32);
  if (here.store && !(again >> m & 1)) {
    uint16_t* to = static_cast<uint16_t*>(a.dq) + here.at + 4 * g;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<uint2*>(to + 32 * c + 2 * r) = make_uint2(pack_bf16x2(dq[c][r] * a.scale, dq[c][r + 1] * a.scale),
                                                                    pack_bf16x2(dq[c][r + 2] * a.scale, dq[c][r + 3] * a.scale));
  }
  for (; again; again &= again - 1) {
    const int x = __ffs(again) - 1, rr = row0 + x, tt = rr / G, hh = hk * G + (rr - tt * G);
    const size_t from = (size_t)b * a.qr.sb + (size_t)hh * a.qr.sh + (size_t)tt * a.qr.sn;
    PlainScratch<D>& ps = reinterpret_cast<PlainScratch<D>*>(smem)[w];
    ps.put(ps.a, static_cast<const uint16_t*>(a.q) + from, lane);
    ps.put(ps.b, static_cast<const uint16_t*>(a.dout) + from, lane);
    const TokenKeys<uint16_t> keys{reinterpret_cast<const uint16_t*>(kbase), reinterpret_cast<const uint16_t*>(vbase), a.kr.sn};
    float acc[D / 64];
    plain_dq_row<D>(keys, ps.a, ps.b, ps.p, tt, len, a.sight, a.scale2, __shfl(nl, x), a.scale2, __shfl(delta, x), lane, acc);
    for (int c = 0; c < D / 64; ++c) store1(static_cast<uint16_t*>(a.dq) + from + lane + 64 * c, a.scale * acc[c]);
  }
}

// ---- dk, dv -------------------------------------------------------------------------------

// A workgroup's key block and its share of it.
struct KeyShare {
  int bk, block, part, parts, slot;      // slot: of its partial sums, -1 where it is the only one
};
__device__ __forceinline__ KeyShare key_share(const BwdRows& a, int id) {
  // the blocks of the first tokens come first, as their workgroups may have the most to do, and in turn to the XCDs
  KeyShare r;
  const int heads = a.B * a.HK, sink_wgs = heads * a.sink_blocks * a.sink_share, ns = a.sink_blocks > 0 ? a.sink_blocks : 1;
  const int rest = a.blocks - a.sink_blocks > 0 ? a.blocks - a.sink_blocks : 1;
  if (id < sink_wgs) {
    const int x = id / a.sink_share;
    r.part = id % a.sink_share; r.parts = a.sink_share; r.block = x % ns; r.bk = x / ns;
    r.slot = a.sink_share > 1 ? id : -1;
  } else {
    const PairPlace place = pair_place(id - sink_wgs, heads, rest * a.share);
    r.part = place.at % a.share; r.parts = a.share; r.block = a.sink_blocks + place.at / a.share; r.bk = place.pair;
    r.slot = a.share > 1 ? (a.sink_share > 1 ? sink_wgs : 0) + (place.pair * rest + place.at / a.share) * a.share + r.part : -1;
  }
  return r;
}

// Keys on the lanes: S = Q K^T, dP = dO V^T with queries on the accumulator rows, started from -lse / scale and -delta, so that p = exp2(scale2 S)
// and dS = p dP; dV^T += dO^T P, dK^T += Q^T dS with P and dS as they lie (rounded to bf16, as Q and dO are stored: PIECES 1).  12 heads x 32760 x 128, window 2 x 1560 and
// 1560 first tokens: 2.0 ms, 900 TFLOP/s; the
// matrix cores are busy 45 % of the cycles, a third of a wavefront's time goes to waits (every operand is read from LDS, 40 KB for the four products of 32 x 32).
// Width 128: eight wavefronts, k in LDS.  With k and v in registers beside the 128 of the sums, a lane needs more than the 256 that two wavefronts to a SIMD
// leave it.
template <int D, int PIECES>
__global__ __launch_bounds__(2 * key_block(D), 2) void window_dkv_kernel(BwdRows a) {
  constexpr int BK = key_block(D), NW = BK / 32, KS = D / 16, CB = D / 32, TILE = BT * D * 2, BUF = 2 * TILE + 2 * BT * 4;
  constexpr bool KLDS = D == 128;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const KeyShare ks_ = key_share(a, blockIdx.x);
  const int b = ks_.bk / a.HK, hk = ks_.bk % a.HK, G = a.G;
  const int len = clamp_length(a.lengths, b, a.n);
  const int jb0 = ks_.block * BK, jb1 = (jb0 + BK < len ? jb0 + BK : len) - 1;      // the block's keys
  const int j = jb0 + 32 * w + m;
  const bool live = j < len;
  const int lo = live ? query_lo(a.sight, j) : 0, hi = live ? query_hi(a.sight, j, len) : 0;
  const size_t at = (size_t)b * a.kr.sb + (size_t)hk * a.kr.sh + (size_t)j * a.kr.sn;
  uint4 k[KLDS ? 1 : KS], v[KS];
  const uint32_t kat = lds_address(smem) + 2 * BUF + w * 32 * D * 2;      // k: the wavefront's own rows, no barrier
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const size_t c = at + 16 * ks + 8 * g;
    uint4& kr = k[KLDS ? 0 : ks];
    kr = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.k) + c) : make_uint4(0, 0, 0, 0);
    v[ks] = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.v) + c) : make_uint4(0, 0, 0, 0);
    if (KLDS) *reinterpret_cast<uint4*>(smem + 2 * BUF + (32 * w + m) * (D * 2) + (((2 * ks + g) ^ swz<D>(m)) * 16)) = kr;
  }
  f32x16 dk[CB], dv[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) { dk[c] = fill16(0.f); dv[c] = fill16(0.f); }

  // the query tiles of the block, head after head of the group, and this workgroup's share of them
  const int q0 = jb1 >= jb0 ? query_lo(a.sight, jb0) / BT : 0;
  const int qe = jb1 < jb0 ? 0 : jb0 < a.sight.sinks ? len : query_hi(a.sight, jb1, len);
  const int T = (qe + BT - 1) / BT > q0 ? (qe + BT - 1) / BT - q0 : 0;
  const int per = (T * G + ks_.parts - 1) / ks_.parts, e0 = ks_.part * per, e1 = e0 + per < T * G ? e0 + per : T * G;
  // the first query of the e-th tile; a whole block's tiles in an order that neighbouring blocks share (TileOrder)
  const int turn = ks_.parts == 1 && T > 0 ? q0 % T : 0;
  auto first_query = [&](int e) {
    const int x = e % T - turn;
    return (q0 + (x < 0 ? x + T : x)) * BT;
  };
  // what the wavefront's keys are seen by
  const int jw0 = jb0 + 32 * w, jw1 = (jw0 + 32 < len ? jw0 + 32 : len) - 1;
  const bool any = jw1 >= jw0;
  const int wlo0 = query_lo(a.sight, jw0), wlo1 = query_lo(a.sight, jw1 < 0 ? 0 : jw1);
  const int whi1 = jw0 < a.sight.sinks ? len : query_hi(a.sight, jw1 < 0 ? 0 : jw1, len);
  const int whi0 = jw1 < a.sight.sinks ? len : query_hi(a.sight, jw0 < a.sight.sinks ? a.sight.sinks : jw0, len);

  const size_t pitch = a.qr.sn * 2;
  const RowTile<D, NW, BT> loader(w, lane);
  const uint32_t lds = lds_address(smem);
  auto request = [&](int e) {
    const int hd = e / T, i0 = first_query(e), h = hk * G + hd;
    const size_t base = ((size_t)b * a.qr.sb + (size_t)h * a.qr.sh) * 2, li = ((size_t)b * a.H + h) * a.n;
    const uint32_t to = lds + (uint32_t)(e & 1) * BUF;
    loader.load(static_cast<const char*>(a.q) + base, pitch, i0, len, to, w);
    loader.load(static_cast<const char*>(a.dout) + base, pitch, i0, len, to + TILE, w);
    if (w < 2) {
      const int i = i0 + lane < len ? i0 + lane : len - 1;
      const float* from = (w == 0 ? a.nl : a.nd) + li + i;
      load_word_to_lds(from, to + 2 * TILE + w * BT * 4);
    }
  };

  arrived(k);
  arrived(v);
  if (e0 < e1) request(e0);
  lds_loads_landed();
  __syncthreads();
  for (int e = e0; e < e1; ++e) {
    if (e + 1 < e1) request(e + 1);
    const int i0 = first_query(e);
    const uint32_t qt = lds + (uint32_t)(e & 1) * BUF, gt = qt + TILE;
    const float* nl = reinterpret_cast<const float*>(smem + (e & 1) * BUF + 2 * TILE);
    if (any && i0 < whi1 && i0 + BT > wlo0) {
      const bool plain = i0 >= wlo1 && i0 + BT <= whi0;
#pragma unroll
      for (int qb = 0; qb < BT / 32; ++qb) {
        f32x16 s, dp;
        uint4 held;
        const int lz = (int)opaque_lane(lane);        // (addresses are worked out here, and k operands read again, not held)
        const uint32_t ra = row_at<D>(lz), ta = turned_at<D>(lz);
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const float4 x = *reinterpret_cast<const float4*>(nl + 32 * qb + 2 * r + 4 * g), y = *reinterpret_cast<const float4*>(nl + BT + 32 * qb + 2 * r + 4 * g);
          s[r] = x.x; s[r + 1] = x.y; s[r + 2] = x.z; s[r + 3] = x.w;
          dp[r] = y.x; dp[r + 1] = y.y; dp[r + 2] = y.z; dp[r + 3] = y.w;
        }
        if constexpr (KLDS)      // q, k, dout of a k-step in turn
          pipelined_operands<2 * KS, 3>([&](int x) { return row_chunk<D>((x % 2 ? kat : qt + 32 * qb * D * 2) + ra, x / 2, 0); },
                                        [&](int x, uint4 op) {
                                          if (x % 2) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(held), as_bf16x8(op), s, 0, 0, 0);
                                          else held = op;
                                        });
        else
          pipelined_operands<KS, 4>([&](int x) { return row_chunk<D>(qt + ra, x, 32 * qb); },
                                    [&](int x, uint4 op) { s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(op), as_bf16x8(k[x]), s, 0, 0, 0); });
        pipelined_operands<KS, 4>([&](int x) { return row_chunk<D>(gt + ra, x, 32 * qb); },
                                  [&](int x, uint4 op) { dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(op), as_bf16x8(v[x]), dp, 0, 0, 0); });
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * a.scale2);
        if (!plain) {
          asm volatile("");
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int i = i0 + 32 * qb + 8 * (r / 4) + 4 * g + r % 4;
            const bool on = i >= lo && i < hi;
            s[r] = on ? s[r] : 0.f;
            dp[r] = on ? dp[r] : 0.f;
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] *= s[r];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          uint4 x[PIECES];
          if constexpr (PIECES == 1) {
            const uint4 p[1] = {pack8(s, st)};
            x[0] = pack8(dp, st);
            pipelined_operands<2 * CB, 3>([&](int i) { return __builtin_bit_cast(uint4, turned<D>((i % 2 ? qt : gt) + ta, i / 2, 16 * (2 * qb + st))); },
                                          [&](int i, uint4 op) {
                                            if (i % 2) dk[i / 2] = mfma_weights<1>(as_bf16x8(op), x, dk[i / 2]);
                                            else dv[i / 2] = mfma_weights<1>(as_bf16x8(op), p, dv[i / 2]);
                                          });
          } else {
            weights_operand<PIECES>(s, st, x);
#pragma unroll
            for (int c = 0; c < CB; ++c) dv[c] = mfma_weights<PIECES>(turned<D>(gt + ta, c, 16 * (2 * qb + st)), x, dv[c]);
            weights_operand<PIECES>(dp, st, x);
#pragma unroll
            for (int c = 0; c < CB; ++c) dk[c] = mfma_weights<PIECES>(turned<D>(qt + ta, c, 16 * (2 * qb + st)), x, dk[c]);
          }
        }
      }
    }
    lds_loads_landed();
    __syncthreads();
  }

  // as for dq: masked queries have P = dS = 0
  if (!live) {
#pragma unroll
    for (int c = 0; c < CB; ++c) { dk[c] = fill16(0.f); dv[c] = fill16(0.f); }
  }
  float test = 0.f;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) test = fmaf(0.f, dk[c][r], fmaf(0.f, dv[c][r], test));
  uint32_t again = (uint32_t)__ballot(test != 0.f) | (uint32_t)(__ballot(test != 0.f) >> 32);
  float* const part = a.parts + (ks_.slot < 0 ? 0 : (size_t)ks_.slot * 2 * BK * D);
  if (!(again >> m & 1)) {
    if (ks_.slot >= 0) {
      float* to = part + (size_t)(32 * w + m) * D + 4 * g;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          *reinterpret_cast<float4*>(to + 32 * c + 2 * r) = make_float4(dk[c][r], dk[c][r + 1], dk[c][r + 2], dk[c][r + 3]);
          *reinterpret_cast<float4*>(to + BK * D + 32 * c + 2 * r) = make_float4(dv[c][r], dv[c][r + 1], dv[c][r + 2], dv[c][r + 3]);
        }
    } else if (j < a.n) {
      uint16_t *tk = static_cast<uint16_t*>(a.dk) + at + 4 * g, *tv = static_cast<uint16_t*>(a.dv) + at + 4 * g;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          *reinterpret_cast<uint2*>(tk + 32 * c + 2 * r) = make_uint2(pack_bf16x2(dk[c][r] * a.scale, dk[c][r + 1] * a.scale),
                                                                      pack_bf16x2(dk[c][r + 2] * a.scale, dk[c][r + 3] * a.scale));
          *reinterpret_cast<uint2*>(tv + 32 * c + 2 * r) = make_uint2(pack_bf16x2(dv[c][r], dv[c][r + 1]), pack_bf16x2(dv[c][r + 2], dv[c][r + 3]));
        }
    }
  }
  for (; again; again &= again - 1) {
    const int x = 32 * w + __ffs(again) - 1, jj = jb0 + x;
    const size_t from = (size_t)b * a.kr.sb + (size_t)hk * a.kr.sh + (size_t)jj * a.kr.sn;
    PlainScratch<D>& ps = reinterpret_cast<PlainScratch<D>*>(smem)[w];
    ps.put(ps.a, static_cast<const uint16_t*>(a.k) + from, lane);
    ps.put(ps.b, static_cast<const uint16_t*>(a.v) + from, lane);
    const int jlo = query_lo(a.sight, jj), jhi = query_hi(a.sight, jj, len);
    float sk[D / 64] = {}, sv[D / 64] = {};
    for (int e = e0; e < e1; ++e) {
      const int hd = e / T, i0 = first_query(e), h = hk * G + hd;
      const size_t base = (size_t)b * a.qr.sb + (size_t)h * a.qr.sh, li = ((size_t)b * a.H + h) * a.n;
      const TokenKeys<uint16_t> rows{static_cast<const uint16_t*>(a.q) + base, static_cast<const uint16_t*>(a.dout) + base, a.qr.sn};
      plain_dkv_row<D>(rows, ps.a, ps.b, ps.p, ps.s, i0 > jlo ? i0 : jlo, i0 + BT < jhi ? i0 + BT : jhi, a.scale2, a.scale2, a.nl + li, a.nd + li, lane, sk, sv);
    }
    for (int c = 0; c < D / 64; ++c) {
      if (ks_.slot >= 0) {
        part[(size_t)x * D + lane + 64 * c] = sk[c];
        part[(size_t)(BK + x) * D + lane + 64 * c] = sv[c];
      } else {
        store1(static_cast<uint16_t*>(a.dk) + from + lane + 64 * c, a.scale * sk[c]);
        store1(static_cast<uint16_t*>(a.dv) + from + lane + 64 * c, sv[c]);
      }
    }
  }
}

// Sums of the parts of the shared key blocks, in their order.  A thread has four channels of a row of dk or dv.
template <int D>
__global__ __launch_bounds__(256) void window_dkv_sum_kernel(BwdRows a, int shared_sinks, int shared_rest) {
  constexpr int BK = key_block(D);
  const int heads = a.B * a.HK, items = 2 * BK * D / 4;
  int x = blockIdx.x / (items / 256);                       // the shared block
  const int i = blockIdx.x % (items / 256) * 256 + threadIdx.x;
  int slot, parts, bk, block;
  if (x < heads * shared_sinks) {
    parts = a.sink_share; slot = x * parts; block = x % shared_sinks; bk = x / shared_sinks;
  } else {
    x -= heads * shared_sinks;
    parts = a.share; slot = heads * shared_sinks * a.sink_share + x * parts; block = a.sink_blocks + x % shared_rest; bk = x / shared_rest;
  }
  const float* from = a.parts + (size_t)slot * 2 * BK * D + 4 * i;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < parts; ++p) {
    const float4 y = *reinterpret_cast<const float4*>(from + (size_t)p * 2 * BK * D);
    s.x += y.x; s.y += y.y; s.z += y.z; s.w += y.w;
  }
  const int of = i / (BK * D / 4), row = i % (BK * D / 4) / (D / 4), c = i % (D / 4) * 4, j = block * BK + row;
  if (j >= a.n) return;
  const float f = of == 0 ? a.scale : 1.f;
  uint16_t* to = static_cast<uint16_t*>(of == 0 ? a.dk : a.dv) + (size_t)(bk / a.HK) * a.kr.sb + (size_t)(bk % a.HK) * a.kr.sh + (size_t)j * a.kr.sn + c;
  *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x * f, s.y * f), pack_bf16x2(s.z * f, s.w * f));
}

template <int D, int PIECES>
hipError_t launch_bwd_rows(BwdRows a, hipStream_t s) {
  constexpr size_t q_smem = 4 * BT * D * 2, k_smem = 2 * (2 * BT * D * 2 + 2 * BT * 4) + (D == 128 ? key_block(D) * D * 2 : 0);
  a.blocks = (int)(((long long)a.n * a.G + 127) / 128);
  const int reach = a.sight.left < 0 || a.sight.right < 0 ? a.n : a.sight.left + a.sight.right + 1;
  const bool exact = PIECES > 1 || (long long)reach + a.sight.sinks <= kFewKeys;
  const unsigned grid = (unsigned)(a.B * a.HK * a.blocks);
  if (exact) {
    constexpr auto kernel = &window_dq_kernel<D, true, PIECES>;
    if (hipError_t e = set_smem_once<kernel>(q_smem); e != hipSuccess) return e;
    kernel<<<grid, 256, q_smem, s>>>(a);
  } else if constexpr (PIECES == 1) {
    constexpr auto kernel = &window_dq_kernel<D, false, 1>;
    if (hipError_t e = set_smem_once<kernel>(q_smem); e != hipSuccess) return e;
    kernel<<<grid, 256, q_smem, s>>>(a);
  }
  const KeySplit split = key_split(a.B * a.HK, a.G, a.n, D, a.sight);
  a.blocks = split.blocks; a.sink_blocks = split.sink_blocks; a.sink_share = split.sink_share; a.share = split.share;
  constexpr auto kernel = &window_dkv_kernel<D, PIECES>;
  if (hipError_t e = set_smem_once<kernel>(k_smem); e != hipSuccess) return e;
  kernel<<<(unsigned)split.workgroups, 2 * key_block(D), k_smem, s>>>(a);
  if (split.parts) {
    const int ss = split.sink_share > 1 ? split.sink_blocks : 0, sr = split.share > 1 ? split.blocks - split.sink_blocks : 0;
    window_dkv_sum_kernel<D><<<(unsigned)(a.B * a.HK * (ss + sr) * (2 * key_block(D) * D / 4 / 256)), 256, 0, s>>>(a, ss, sr);
  }
  return hipGetLastError();
}

}  // namespace attn
}  // namespace linattn
