// Softmax attention with a sliding window and first tokens that stay visible, over token tensors (linattn_window_*) and over a
// paged cache (linattn_cache_*): what the host dispatch and the kernels agree on.
#pragma once
#include "kernels.h"

namespace linattn {
namespace attn {

// Which keys the query at position p sees of a sequence of `len` tokens: j < len, j <= p + right (right >= 0), and j >= p - left
// (left >= 0) or j < sinks.  As ranges: the first tokens [0, first) and the window [lo, hi), first <= lo.
// left, right: -1 (no limit) or below kMostTokens, positions and lengths up to it, so that sums and differences fit 32 bits.
constexpr int kMostTokens = 1 << 30;
struct Sight {
  int left, right, sinks;
};
__host__ __device__ inline int key_lo(const Sight& s, int p) { return s.left < 0 || p < s.left ? 0 : p - s.left; }
__host__ __device__ inline int key_hi(const Sight& s, int p, int len) { return s.right < 0 || p >= len - s.right ? len : p + s.right + 1; }
__host__ __device__ inline bool sees(const Sight& s, int p, int j, int len) {
  return j < len && (s.right < 0 || j - s.right <= p) && (s.left < 0 || j >= p - s.left || j < s.sinks);
}
// The queries that see key j: [query_lo, query_hi).
__host__ __device__ inline int query_lo(const Sight& s, int j) { return s.right < 0 || j < s.right ? 0 : j - s.right; }
__host__ __device__ inline int query_hi(const Sight& s, int j, int len) {
  return s.left < 0 || j < s.sinks || j + s.left >= len ? len : j + s.left + 1;
}

__host__ __device__ inline int clamp_length(const int* lengths, int b, int n) {
  if (!lengths) return n;
  const int x = lengths[b];
  return x < 0 ? 0 : x < n ? x : n;
}

// Rows that see at most this many keys take delta from a pass over them (window_dq_kernel EXACT), others from the stored output with the heaviest key's part of
// the correction.  Error of dq (2-norm over two heads, 1e-3) and us of the backward, that way / this, 12 heads x 4133 x 64, causal windows: of 64 keys 2.42 37.0 / 2.37 40.7, of 128
// 2.46 42.1 / 2.40 48, of 256 2.41 49.9 / 2.36 60, of 512 2.46 84 / 2.39 96, of 1024 2.43 116 / 2.39 138 (2.64 / 2.43 with scores nine times as large), all keys 2.50 229 / 2.39
// 283; rounding dS and dq alone is 2.35.  The second pass is a fixed share of the time, and what it saves grows with the weight of a row's few keys.
constexpr int kFewKeys = 256;

// How the key side of the bf16 backward is dealt: blocks of key_block(d) keys, the ones that hold first tokens, which all later queries see, to sink_share
// workgroups each, the others to `share`; the parts of a block that has several are summed afterwards.
constexpr int kQueryTile = 64;
constexpr int key_block(int d) { return d == 128 ? 256 : 128; }
struct KeySplit {
  int blocks, sink_blocks, sink_share, share;
  long long workgroups, parts;      // parts: of the blocks that have several workgroups
};
inline KeySplit key_split(int heads, int G, int n, int d, const Sight& s) {
  KeySplit r{};
  const int kKeyBlock = key_block(d), slots = kCUs * 256 / kKeyBlock;      // resident workgroups
  r.blocks = (n + kKeyBlock - 1) / kKeyBlock;
  r.sink_blocks = s.left < 0 ? 0 : (int)(((long long)(s.sinks < n ? s.sinks : n) + kKeyBlock - 1) / kKeyBlock);
  const long long all = (n + kQueryTile - 1) / kQueryTile;
  long long window = s.left < 0 || s.right < 0 ? all : ((long long)s.left + s.right + kKeyBlock) / kQueryTile + 1;
  if (window > all) window = all;
  // tiles of a block of each kind, of the whole call
  const long long sink_tiles = all * G, tiles = window * G;
  const long long total = heads * (r.sink_blocks * sink_tiles + (r.blocks - r.sink_blocks) * tiles);
  // A workgroup's share: two thirds of what an even deal to the resident ones would give, at least 8 tiles.
  long long most = total * 2 / (3 * slots);
  if (most < 8) most = 8;
  auto shares = [&](long long t) { const long long x = (t + most - 1) / most; return (int)(x < 1 ? 1 : x < 64 ? x : 64); };
  r.sink_share = shares(sink_tiles);
  r.share = shares(tiles);
  r.workgroups = (long long)heads * ((long long)r.sink_blocks * r.sink_share + (long long)(r.blocks - r.sink_blocks) * r.share);
  r.parts = (long long)heads * ((r.sink_share > 1 ? (long long)r.sink_blocks * r.sink_share : 0) +
                                (r.share > 1 ? (long long)(r.blocks - r.sink_blocks) * r.share : 0));
  return r;
}

// One call of linattn_window_fwd / linattn_window_bwd.
struct WindowArgs {
  const void *q, *k, *v, *out, *dout;
  void *o, *dq, *dk, *dv;
  float* lse;               // written by the forward, read by the backward
  float *nl, *nd;           // workspace of the backward: fp32 [B*H][n] each, -lse / scale (fp32 tensors: -lse; -inf where nothing is seen) and -delta
  float* parts;             // and the sums' parts: bf16 tensors fp32 [part][2][key block][d] (key_split); fp32 tensors [share][row][d], with pairs of maximum and
                            // sum behind them (forward), [share][key][2][d]; null: no shares
  int shares;               // fp32 tensors: workgroups to a block of 32 rows
  const int* lengths;       // nullable
  int B, H, HK, n, d;
  Rows qr, kr;              // rows of q, out, dout, dq and of k, v, dk, dv
  Sight sight;
  float scale;
  hipStream_t stream;
};

// The pool of a paged cache and who owns which page.  Rows are [pages][HK][page][d].
struct Pool {
  void *k, *v;
  uint8_t *k_exp, *v_exp;   // e4m3: biased exponent of a row's scale, [pages][HK][page]
  const int* table;         // [B][width]
  const int* lengths;       // [B]
  const int* counts;        // [B], nullable
  int B, HK, d, page, pages, width;
  uint32_t magic, shift;    // of page_of
};
// Division by a page size that only the call knows: m = ceil(2^(31 + s) / page), s = ceil(log2(page)), gives the quotient of every j
// below 2^31 as (j * m) >> (31 + s), and m is below 2^32.
inline void set_divisor(Pool* p) {
  uint32_t s = 0;
  while ((1u << s) < (uint32_t)p->page) ++s;
  p->shift = s;
  p->magic = (uint32_t)((((uint64_t)1 << (31 + s)) + p->page - 1) / p->page);
}
__host__ __device__ inline int page_of(const Pool& p, int j) { return (int)(((uint64_t)(uint32_t)j * p.magic) >> (31 + p.shift)); }
// Row of key j of sequence b in the pool, in rows of one head: -1 where the table names no page of the pool.  j >= 0.
__device__ __forceinline__ long long pool_row(const Pool& p, int b, int h, int j) {
  const int i = page_of(p, j);
  const int at = i < p.width ? p.table[(size_t)b * p.width + i] : -1;
  if ((unsigned)at >= (unsigned)p.pages) return -1;
  return ((long long)at * p.HK + h) * p.page + (j - i * p.page);
}
// Tokens of sequence b that the table has places for, and, which positions go by, all that it counts.
__device__ __forceinline__ int pool_length(const Pool& p, int b) { return clamp_length(p.lengths, b, p.width * p.page); }
__device__ __forceinline__ int pool_tokens(const Pool& p, int b) { return clamp_length(p.lengths, b, kMostTokens); }

// One call of linattn_cache_attn.
struct CacheArgs {
  Pool pool;
  const void* q;
  void* o;
  float* lse;               // nullable
  float* work;
  int H, n;
  Rows qr;
  Sight sight;
  float scale;
  hipStream_t stream;
};

// Workgroups to a block of 32 rows of fp32 tensors: as many as there are compute units for.
inline int f32_shares(long long blocks) { return blocks * 2 > kCUs ? 1 : blocks * 8 <= kCUs ? 8 : (int)(kCUs / blocks); }

// Whether a forward call goes to the kernel that deals keys, not rows, to a workgroup's wavefronts: where its blocks of 32 rows are no more than the compute units
// and see some keys.  Us, blocks of 128 rows / of 32, window to both sides: 4 heads x 1000 x 64, 128 13.8 / 9.1; 2 heads x 4000 x 128, causal 76 / 48; but 16 heads x
// 1000 x 64 (512 blocks), 256 16.6 / 20.6, 4 x 60 x 64 5.4 / 6.2.
inline bool few_blocks(long long pairs, long long rows, int n, const Sight& s) {
  const long long reach = s.left < 0 || s.right < 0 ? n : (long long)s.left + s.right + s.sinks;
  return pairs * ((rows + 31) / 32) <= kCUs && (reach < n ? reach : n) >= 128;
}

// Whether a chunk's rows of a key head (its group's heads side by side) go to the kernel that deals keys, not rows, to a workgroup's wavefronts.
inline bool few_rows(int H, int HK, int n) { return (long long)n * (H / HK) <= 64; }
// The keys that a row of a chunk sees at most, together with the rest of the chunk's.
inline long long reach_of(const CacheArgs& a) {
  const long long all = (long long)a.pool.page * a.pool.width;
  if (a.sight.left < 0) return all;
  const long long r = (long long)a.sight.left + a.n + (a.sight.right < 0 ? a.n : a.sight.right) + a.sight.sinks + 64;
  return r < all ? r : all;
}
// Parts that the keys of a row are dealt to, for chunks whose keys number `reach` at most: as many workgroups as fill the chip, with enough tiles each.  Blocks of rows that
// nearly fill it, or two or three times, are cut as well where parts stay long: the last round is then full, and sums over some 8192 keys (`keys`; each sequence gets
// parts by its own length, see splits_of) are worth writing and reading.  12 heads x 4680 rows over 32760 x 128, e4m3, 444 blocks in 512 places, us: 1300, in four parts 1200
// (a sequence of 16384 in a table of 32768 592 / 603, of 8000, one part, 293 / 302: the empty workgroups and the join); 8 heads x 4680 over 32760 x 64 709 / 506; 512 rows over
// 32760, 20000, 9000 and 3000, 32/8 heads x 128, 852 / 727.  Shorter parts do not pay: 512 rows over a window of 4096, 152, in four parts 187.
constexpr int kMostSplits = 64, kLongPart = 8192;
struct KeyParts {
  int splits, keys;
};
inline KeyParts cache_splits(int B, int H, int HK, int n, int d, bool e4m3, long long reach) {
  const bool few = few_rows(H, HK, n);
  const long long blocks = (long long)B * HK * (few ? 1 : ((long long)n * (H / HK) + 127) / 128);
  const int tile = few ? (e4m3 || d == 64 ? 64 : 32) * 4 : 64 * 8;
  long long s = 2 * kCUs / blocks, most = (reach + tile - 1) / tile;
  int keys = 0;
  if (!few && s <= 1 && reach >= 2 * kLongPart) {
    s = 8 * kCUs / blocks;
    keys = kLongPart;
    most = (reach + keys / 2) / keys;
  }
  s = s < most ? s : most;
  return {s < 1 ? 1 : s < kMostSplits ? (int)s : kMostSplits, keys};
}

hipError_t launch_window_fwd(const WindowArgs& a, int dtype);
hipError_t launch_window_bwd(const WindowArgs& a, int dtype);
hipError_t launch_cache_write(const Pool& p, bool e4m3, const void* k, const void* v, int n, const Rows& r, hipStream_t s);
hipError_t launch_cache_read(const Pool& p, bool e4m3, void* k, void* v, int n, const Rows& r, hipStream_t s);
hipError_t launch_cache_attn(const CacheArgs& a, bool e4m3);

}  // namespace attn
}  // namespace linattn
