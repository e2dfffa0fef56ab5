// Softmax attention of blocks of query rows on the matrix cores (bf16 operands, fp32 scores and sums).
#pragma once
#include "attn_plain.h"
#include "attn_tile.h"

namespace linattn {
namespace attn {

// Rows of a block: the query heads of a key head's group side by side, row = token * G + head, so that a group's keys are read once.
struct RowsArgs {
  const void* q;
  void* o;
  float* lse;               // nullable
  float* parts;             // with several splits: see parts_of
  int B, H, HK, G, n;
  int blocks;               // row blocks of a (batch item, key head)
  int splits;               // parts that the keys of a block are dealt to
  Rows qr;
  Sight sight;
  float scale2;             // scale * log2(e)
  // of a pool's keys `splits` is the most that a sequence gets, and each has about part_keys of its keys at least (0: all get `splits`)
  int part_keys, reach;
  const int* lengths;
};
// Splits of a sequence of len tokens, in the kernel and in the join.
__device__ __forceinline__ int splits_of(const RowsArgs& a, int len) {
  if (a.part_keys == 0) return a.splits;
  const int s = ((len < a.reach ? len : a.reach) + a.part_keys / 2) / a.part_keys;
  return s < 1 ? 1 : s < a.splits ? s : a.splits;
}
// Results over a part of the keys: o not divided by its sum, fp32 [splits][B*H*n][D], and then [splits][B*H*n] pairs of the largest score (base 2) and
// the sum.
__device__ __forceinline__ void put_part(const RowsArgs& a, int D, int split, size_t row, float m, float l) {
  const size_t rows = (size_t)a.B * a.H * a.n;
  reinterpret_cast<float2*>(a.parts + (size_t)a.splits * rows * D)[(size_t)split * rows + row] = make_float2(m, l);
}

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

// Workgroup id of pairs * per -> its (batch item, key head) pair and its place among the pair's `per` workgroups.  A pair's workgroups, which read the same
// keys, go to one XCD, neighbouring pairs (of one item, or of sequences of unlike lengths) to different ones; the pairs that are left over are cut into stretches.
struct PairPlace {
  int pair, at;
};
__device__ __forceinline__ PairPlace pair_place(int id, int pairs, int per) {
  const int each = pairs / kXCDs * per, x = id % kXCDs, i = id / kXCDs;
  if (i < each) return {x + kXCDs * (i / per), i % per};
  const int rest = xcd_stretch(id - kXCDs * each, (pairs % kXCDs) * per);
  return {pairs / kXCDs * kXCDs + rest / per, rest % per};
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
  // where tile i starts among the keys of the first tokens, among those of the window
  __device__ __forceinline__ int sink_key(int i) const { return (i < nsink ? i : nsink) * KT; }
  __device__ __forceinline__ int window_key(int i) const { return (wtile + (i > nsink ? i - nsink : 0)) * KT; }
};
// The order in which a workgroup takes tiles it0 .. it1 - 1: those of the first tokens, then those of the window from the one on whose number is a multiple of
// how many they are, and the ones before it last.  Neighbouring blocks, whose windows overlap but for a tile or two, then read the same tile at the same time.  Each
// from its own first tile on, the 64 workgroups of an XCD were spread over more keys than its L2 holds: 12 heads x 32760 x 128, window 2 x 3120 and 1560 first tokens,
// forward 1564 us, so 1528; training step, window 2 x 1560, 4.42 ms, so 4.18.
template <int KT>
struct TileOrder {
  int w0, count, turn;
  __device__ __forceinline__ TileOrder(const KeyTiles<KT>& t, int it0, int it1) {
    w0 = it0 > t.nsink ? it0 : t.nsink;
    count = it1 - w0;
    turn = count > 0 ? (t.wtile + w0 - t.nsink) % count : 0;
  }
  __device__ __forceinline__ int operator()(int i) const {
    if (i < w0) return i;
    const int x = i - turn;
    return x < w0 ? x + count : x;
  }
};

// What a wavefront's rows at positions p0 .. p1 see of a tile from key j0 on: nothing, or everything.  (Lanes without a token are not looked at: what they
// come to is dropped.)
struct WaveSight {
  int lo0, lo1, hi0, hi1, sinks;
  bool rows;                // whether it has any
  __device__ __forceinline__ WaveSight(const Sight& s, int p0, int p1, int len)
      : lo0(key_lo(s, p0)), lo1(key_lo(s, p1)), hi0(key_hi(s, p0, len)), hi1(key_hi(s, p1, len)), sinks(s.sinks), rows(p1 >= p0) {}
  __device__ __forceinline__ bool nothing(int j0, int count) const { return !rows || j0 >= hi1 || (j0 + count <= lo0 && j0 >= sinks); }
  __device__ __forceinline__ bool everything(int j0, int count) const { return j0 + count <= hi0 && (j0 >= lo1 || j0 + count <= sinks); }
};

__device__ __forceinline__ uint4 pack8(const f32x16& e, int h) {
  return make_uint4(pack_bf16x2(e[8 * h], e[8 * h + 1]), pack_bf16x2(e[8 * h + 2], e[8 * h + 3]), pack_bf16x2(e[8 * h + 4], e[8 * h + 5]),
                    pack_bf16x2(e[8 * h + 6], e[8 * h + 7]));
}

// The operand of weights e[8h .. 8h+7]: PIECES of 1 rounds them to bf16, as the values that they multiply are stored (an error of the result like that of its store,
// 1.66e-3 in 2-norm each; sums of weights are taken before), 3 hands them on whole, as the exact sum of three bf16 numbers (LINATTN_BF16_F32MATH: the other
// operand of their product is bf16, so three products give it in fp32).
template <int PIECES>
__device__ __forceinline__ void weights_operand(const f32x16& e, int h, uint4 (&p)[PIECES]) {
  if constexpr (PIECES == 1) p[0] = pack8(e, h);
  else {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = e[8 * h + i];
    f32::split8(f, p);
  }
}
// acc += a p, the smallest piece first
template <int PIECES>
__device__ __forceinline__ f32x16 mfma_weights(bf16x8 a, const uint4 (&p)[PIECES], f32x16 acc) {
#pragma unroll
  for (int i = PIECES - 1; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, as_bf16x8(p[i]), acc, 0, 0, 0);
  return acc;
}

// Scores of a query's keys (half of them in each lane of a pair) -> weights 2^(scale2 s - mx), with the running maximum mx, the sum l of the lane's weights, and o
// brought to it.  The maximum moves only where it has grown by more than 8: the weights are then at most 2^8, and the result the same after
// the division.
template <int KB, int CB>
__device__ __forceinline__ void softmax_step(f32x16 (&s)[KB], float scale2, float& mx, float& l, f32x16 (&o)[CB]) {
  float top = s[0][0];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
  float x, y;
  pair32(top, x, y);
  top = fmaxf(x, y) * scale2;
  if (__any(top > mx + 8.f)) {
    const float next = fmaxf(mx, top), alpha = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - next);
    mx = next;
    l *= alpha;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[c][r] *= alpha;
  }
  const float c0 = mx == -INFINITY ? 0.f : -mx;
  float sum = 0.f;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], scale2, c0));
      sum += s[kb][r];
    }
  l += sum;
}

// Row r of a block once more, key by key, over the keys of tiles it0 .. it1 - 1.
template <int D, typename Keys, typename Tiles>
__device__ void plain_again(const RowsArgs& a, const Keys& keys, const Tiles& tiles, int it0, int it1, int r, int b, int hk, int split, int splits, int pos0,
                            int len, PlainScratch<D>& ps, int lane) {
  const int t = r / a.G, h = hk * a.G + (r - t * a.G);
  const size_t at = (size_t)b * a.qr.sb + (size_t)h * a.qr.sh + (size_t)t * a.qr.sn, li = ((size_t)b * a.H + h) * a.n + t;
  ps.put(ps.a, static_cast<const uint16_t*>(a.q) + at, lane);
  float m, l, acc[D / 64];
  plain_row<D>(keys, ps.a, ps.p, pos0 + t, len, a.sight, tiles.sink_key(it0), tiles.sink_key(it1), tiles.window_key(it0), tiles.window_key(it1), a.scale2,
               lane, m, l, acc);
  if (splits > 1) {
    for (int c = 0; c < D / 64; ++c) a.parts[((size_t)split * a.B * a.H * a.n + li) * D + lane + 64 * c] = acc[c];
    if (lane == 0) put_part(a, D, split, li, m, l);
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  for (int c = 0; c < D / 64; ++c) store1(static_cast<uint16_t*>(a.o) + at + lane + 64 * c, acc[c] * inv);
  if (a.lse && lane == 0) a.lse[li] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Queries on the lanes: S^T = K Q^T gives a lane its query's scores against 32 of a tile's 64 keys (the lane 32 further has the others), the softmax of a row is in
// the lane, and its weights lie as the right operand of O^T += V^T P^T wants them; V^T comes from transposing LDS reads.  A wavefront has 32 rows and a workgroup four
// of them, so that two workgroups fit a compute unit: with 64 rows a wavefront LDS is read half as much, but one wavefront to a SIMD leaves nothing to hide its reads
// (2214 us in place of 1607 at 12 heads x 32760 x 128, window 2 x 3120, 1560 first tokens; 32 keys to a tile 1666, eight wavefronts to a workgroup 1619).
// There, as built: 1.41 to 1.56 ms on different machines, 940 to 1040 TFLOP/s of the 1310 to 1350 that a large matrix product reaches.  The matrix cores are busy 49 % of the
// cycles, a third of a wavefront's time goes to waits for LDS and for the tile's barrier, and the power limit takes the clock to 1.9 GHz; without its LDS reads and loads
// the kernel reaches 1230, without the softmax 1070.
// Two tiles in LDS and one barrier a tile.  (With a second barrier, between the scores and the product with v, a buffer can be asked for half a tile earlier; but then
// the exponentials no longer overlap with that product: 12 heads x 32760 x 128, window 2 x 3120, 1562 us in place of 1507, on one machine.)
template <int D, int KT, typename Source, int PIECES>
__global__ __launch_bounds__(64 * kRowWaves, 2) void attn_rows_kernel(RowsArgs a, typename Source::Args from) {
  constexpr int NW = kRowWaves, KB = KT / 32, KS = D / 16, CB = D / 32, BM = 32 * NW, TILE = KT * D * 2;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  // (first parts first: where a sequence has only one, the workgroups that leave at once come behind those that have work)
  const int pairs = a.B * a.HK, split = (int)blockIdx.x / (pairs * a.blocks);
  const PairPlace place = pair_place((int)blockIdx.x - split * pairs * a.blocks, pairs, a.blocks);
  const int bk = place.pair, block = row_block(a.sight, place.at, a.blocks);
  const int b = bk / a.HK, hk = bk % a.HK, G = a.G;
  Source src(from, b, hk, a.n, w, lane);
  // token t has position pos0 + t; tokens t0 .. count - 1 have rows
  const int splits = Source::kPaged ? splits_of(a, src.len) : 1;
  if (split >= splits) return;
  const int len = src.len, pos0 = src.tokens - src.count, t0 = pos0 < 0 ? -pos0 : 0, rows = src.count * G, all = a.n * G;
  const int row0 = block * BM + w * 32;

  // this lane's query
  const int r = row0 + m, t = r / G, h = hk * G + (r - t * G);
  const size_t at = (size_t)b * a.qr.sb + (size_t)h * a.qr.sh + (size_t)t * a.qr.sn;
  const bool store = r < all, live = r < rows && t >= t0;
  const int lo = live ? key_lo(a.sight, pos0 + t) : 0, hi = live ? key_hi(a.sight, pos0 + t, len) : 0;
  uint4 q[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    q[ks] = live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at + 16 * ks + 8 * g) : make_uint4(0, 0, 0, 0);
  f32x16 o[CB];
  float mx = -INFINITY, l = 0.f;
#pragma unroll
  for (int c = 0; c < CB; ++c) o[c] = fill16(0.f);

  auto from_row = [&](int x) { return pos0 + (x / G > t0 ? x / G : t0); };      // the first position from row x on
  auto to_row = [&](int x) { x = (x < rows ? x : rows) - 1; return x >= 0 && x / G >= t0 ? pos0 + x / G : -1; };      // the last before row x
  const int bp0 = from_row(block * BM), bp1 = to_row((block + 1) * BM), wp0 = from_row(row0), wp1 = to_row(row0 + 32);
  const KeyTiles<KT> tiles(a.sight, bp0, bp1 < bp0 ? -1 : bp1, len);
  const WaveSight sight(a.sight, wp0, wp1 < wp0 ? -1 : wp1, len);
  const int it0 = (int)((long long)tiles.count * split / splits), it1 = (int)((long long)tiles.count * (split + 1) / splits);
  const TileOrder<KT> order(tiles, it0, it1);
  const uint32_t lds = lds_address(smem);
  auto ktile = [&](int i) { return lds + (uint32_t)((i - it0) & 1) * 2 * TILE; };
  auto look = [&](int i) { src.look(tiles.start(order(i)), tiles.end); };
  const uint32_t rows_at = row_at<D>(lane), turned_rows = turned_at<D>(lane);

  arrived(q);
  auto ask = [&](int i) { src.ask_k(ktile(i)); src.ask_v(ktile(i) + TILE); };
  auto put = [&](int i) { src.put_k(ktile(i)); src.put_v(ktile(i) + TILE); };
  unsigned long long there = ~0ull;      // the keys that the tile has
  if (it0 < it1) {
    look(it0);
    there = src.there;
    ask(it0);
    put(it0);
    if (it0 + 1 < it1) look(it0 + 1);
  }
  src.landed();
  __syncthreads();
  for (int it = it0; it < it1; ++it) {
    const unsigned long long there_next = src.there;
    if (it + 1 < it1) {
      ask(it + 1);
      if (it + 2 < it1) look(it + 2);
    }
    const int j0 = tiles.start(order(it));
    if (!sight.nothing(j0, KT) && (!Source::kPaged || there != 0)) {
      const uint32_t kt = ktile(it), vt = kt + TILE;
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = fill16(0.f);
      pipelined_operands<KS * KB, 6>([&](int x) { return row_chunk<D>(kt + rows_at, x / KB, 32 * (x % KB)); },
                                     [&](int x, uint4 kop) {
                                       s[x % KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kop), as_bf16x8(q[x / KB]), s[x % KB], 0, 0, 0);
                                     });
      if (!(sight.everything(j0, KT) && there == ~0ull)) {
        asm volatile("");        // a branch: as selects, the mask is computed for every tile
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int j = j0 + 32 * kb + 8 * (e / 4) + 4 * g + e % 4;
            bool on = j < hi && (j >= lo || j < a.sight.sinks);
            if (Source::kPaged) on = on && (there >> (j - j0) & 1);
            s[kb][e] = on ? s[kb][e] : -INFINITY;
          }
      }
      softmax_step<KB, CB>(s, a.scale2, mx, l, o);
      if constexpr (Source::kPaged) {      // (short of registers the compiler would read an operand, wait, multiply, and so on)
        uint4 x[2 * KB][1];
#pragma unroll
        for (int st = 0; st < 2 * KB; ++st) weights_operand<1>(s[st / 2], st % 2, x[st]);
        pipelined_operands<2 * KB * CB, 3>([&](int i) { return __builtin_bit_cast(uint4, turned<D>(vt + turned_rows, i % CB, 16 * (i / CB))); },
                                           [&](int i, uint4 op) { o[i % CB] = mfma_weights<1>(as_bf16x8(op), x[i / CB], o[i % CB]); });
      } else {
#pragma unroll
        for (int st = 0; st < 2 * KB; ++st) {
          uint4 x[PIECES];
          weights_operand<PIECES>(s[st / 2], st % 2, x);
#pragma unroll
          for (int c = 0; c < CB; ++c) o[c] = mfma_weights<PIECES>(turned<D>(vt + turned_rows, c, 16 * st), x, o[c]);
        }
      }
    }
    if (it + 1 < it1) put(it + 1);
    there = there_next;
    src.landed();
    __syncthreads();
  }

  // A key that is masked has weight 0, and 0 times an infinity or NaN in its value would be NaN: rows that come out not finite are done again
  // key by key.
  float x, y;
  pair32(l, x, y);
  const float sum = live ? x + y : 0.f, inv = sum == 0.f ? 0.f : 1.0f / sum;
  if (!live) {
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = fill16(0.f);
  }
  const size_t li = ((size_t)b * a.H + h) * a.n + t;
  float test = 0.f * sum;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) test = fmaf(0.f, o[c][e], test);
  uint32_t again = (uint32_t)__ballot(test != 0.f) | (uint32_t)(__ballot(test != 0.f) >> 32);
  if (store && !(again >> m & 1)) {
    if (splits > 1) {
      float* part = a.parts + ((size_t)split * a.B * a.H * a.n + li) * D + 4 * g;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(part + 32 * c + 2 * e) = make_float4(o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]);
      if (g == 0) put_part(a, D, split, li, mx, sum);
    } else {
      uint16_t* out = static_cast<uint16_t*>(a.o) + at + 4 * g;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<uint2*>(out + 32 * c + 2 * e) = make_uint2(pack_bf16x2(o[c][e] * inv, o[c][e + 1] * inv), pack_bf16x2(o[c][e + 2] * inv, o[c][e + 3] * inv));
      if (a.lse && g == 0) a.lse[li] = sum == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
  for (; again; again &= again - 1)
    plain_again<D>(a, src.keys(), tiles, it0, it1, row0 + __ffs(again) - 1, b, hk, split, splits, pos0, len, reinterpret_cast<PlainScratch<D>*>(smem)[w],
                   lane);
}

// The sum over the splits.  A wavefront to a row.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(RowsArgs a) {
  const int lane = threadIdx.x % 64, t = blockIdx.x * 4 + threadIdx.x / 64, bh = blockIdx.y;
  const int splits = splits_of(a, a.part_keys ? clamp_length(a.lengths, bh / a.H, a.reach) : 0);
  if (t >= a.n || (splits == 1 && a.part_keys)) return;      // (one part: the kernel has stored the result)
  const size_t rows = (size_t)a.B * a.H * a.n, row = (size_t)bh * a.n + t;
  const float2* ml = reinterpret_cast<const float2*>(a.parts + (size_t)a.splits * rows * D);
  // a lane to a split, at most 64 of them
  const float2 own = lane < splits ? ml[(size_t)lane * rows + row] : make_float2(-INFINITY, 0.f);
  const float top = wave_max(own.x);
  const float weight = own.x == -INFINITY ? (own.y == 0.f ? 0.f : own.y) : __builtin_amdgcn_exp2f(own.x - top);      // (a sum without a maximum is NaN)
  const float sum = wave_sum(weight * own.y), inv = sum == 0.f ? 0.f : 1.0f / sum;
  float acc[D / 64] = {};
  for (int s0 = 0; s0 < splits; s0 += 8) {      // eight parts in flight
    float x[8][D / 64];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) x[i][c] = s0 + i < splits ? a.parts[((size_t)(s0 + i) * rows + row) * D + lane + 64 * c] : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = __shfl(weight, s0 + i);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) acc[c] = f == 0.f ? acc[c] : fmaf(f, x[i][c], acc[c]);
    }
  }
  uint16_t* out = static_cast<uint16_t*>(a.o) + (size_t)(bh / a.H) * a.qr.sb + (size_t)(bh % a.H) * a.qr.sh + (size_t)t * a.qr.sn;
  for (int c = 0; c < D / 64; ++c) store1(out + lane + 64 * c, acc[c] * inv);
  if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int D>
hipError_t launch_join(const RowsArgs& a, hipStream_t s) {
  if (a.splits > 1) attn_join_kernel<D><<<dim3((a.n + 3) / 4, a.B * a.H), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int D, int KT, typename Source, int PIECES = 1>
hipError_t launch_rows(RowsArgs a, const typename Source::Args& from, hipStream_t s) {
  constexpr int BM = 32 * kRowWaves;
  constexpr size_t smem = 4 * KT * D * 2;
  a.blocks = (int)(((long long)a.n * a.G + BM - 1) / BM);
  constexpr auto kernel = &attn_rows_kernel<D, KT, Source, PIECES>;
  if (hipError_t e = set_smem_once<kernel>(smem); e != hipSuccess) return e;
  kernel<<<(unsigned)(a.B * a.HK * a.blocks * a.splits), 64 * kRowWaves, smem, s>>>(a, from);
  return launch_join<D>(a, s);
}

}  // namespace attn
}  // namespace linattn
