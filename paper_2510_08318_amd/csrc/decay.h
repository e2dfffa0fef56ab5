// Causal linear attention with a decay for each head (linattn_decay_*): what the host dispatch and the kernels agree on.
//
//   S_t = lambda S_{t-1} + k_t v_t^T        o_t = scale q_t S_t
//   D_t = lambda D_{t+1} + scale q_t dout_t^T, lambda D_n := dS_out
//   dq_t = scale S_t dout_t     dk_t = D_t v_t     dv_t = D_t^T k_t     dS_in = lambda D_0
//
// All four are one pass with other tensors in its roles.  For token rows a, b, c in the pass's order and a state X,
//
//   o_i = out_scale a_i (lambda^i X + in_scale sum_{j <= i} lambda^{i-j} b_j^T c_j)
//
//   out: (q, k, v), X = lambda S_in;  dq: (dout, v, k), X = lambda S_in^T;  from the last token back, dv: (k, q, dout), X = dS_out, and dk: (v, dout, q),
//   X = dS_out^T.  A pass that is `turned` reads its state transposed.
#pragma once
#include "kernels.h"

namespace linattn {
namespace decay {

constexpr int kMostTokens = 1 << 30;

// A token tensor in a role: its head of query head h is h / group.
struct Role {
  const void* p;
  Rows r;
  int group;
};
struct Pass {
  Role a, b, c;
  void* o;                  // rows of query heads, in the tensors' type, or (part) in fp32 [B, H, n, d]
  Rows orow;
  int part;
  const float* in;          // state, nullable: zeros
  float* out;               // nullable; not of a turned pass
  int turned, back;         // back: from the last token to the first
  float in_scale, out_scale;
};
struct Common {
  const float* log_decay;   // [H]
  const int* lengths;       // [B], nullable
  const int* slots;         // [B], nullable: row of an item in the state tensors
  int states, B, H, group, n;      // group: query heads to a key head
};

// A head's decay as the kernels use it: what is above 0, or NaN, counts as 0, and -inf as a number whose product with a distance of 0 is 0.  (Products with far distances may be -inf; exp
// gives 0 for them.)
__device__ __forceinline__ float log_decay_of(const Common& c, int h) { return fmaxf(fminf(c.log_decay[h], 0.f), -1e30f); }
__host__ __device__ inline int length_of(const Common& c, int b) {
  if (!c.lengths) return c.n;
  const int x = c.lengths[b];
  return x < 0 ? 0 : x < c.n ? x : c.n;
}
// Workgroup id -> its segment of a pass of a query head.  The workgroups that read the same rows at the same time, of the passes and of the query heads of a group, follow each other on one XCD
// (ids go to the XCDs in turn).  A pass that goes back has its segments in the other order, over the same tokens where the sequence fills them.
struct Place {
  int pass, b, h, seg;
};
__device__ __forceinline__ Place place_of(const Common& c, int id, int segs, int passes) {
  const int members = passes * c.group, heads = c.H / c.group, units = c.B * heads * segs, even = units / kXCDs * kXCDs;
  const bool mapped = id < even * members;
  const int i = mapped ? id / kXCDs : id - even * members;
  const int unit = mapped ? i / members * kXCDs + id % kXCDs : even + i / members, member = i % members, bk = unit / segs;
  return {member % passes, bk / heads, bk % heads * c.group + member / passes, unit % segs};
}
// Row of item b, head h in the state tensors; -1 where its slot is none.
__device__ __forceinline__ long long state_row(const Common& c, int b, int h) {
  const int s = c.slots ? c.slots[b] : b;
  return (unsigned)s < (unsigned)c.states ? (long long)s * c.H + h : -1;
}

// One call of linattn_decay_fwd / linattn_decay_bwd.
struct Args {
  const void *q, *k, *v, *dout;
  void *o, *dq, *dk, *dv;
  const float *state, *dstate;
  float *state_out, *dstate_in;
  Common c;
  int HK, d, dtype;
  Rows qr, kr;
  float scale;
  float* work;
  hipStream_t stream;
};

// How a call's tokens are cut: chunks of a kernel's own size, segments of several of them, each a workgroup's.  Where there are several segments, a first kernel takes every
// segment's own sum of b_j^T c_j, a second the states between them from it.
constexpr int kChunk = 64, kChunkF32 = 32;
struct Plan {
  int segs, tokens;         // tokens of a segment
};
// The number of segments by what each choice should take.  A chunk of a workgroup takes `rows` us in the rows kernel and `sums` in the kernel of the sums where the chip is empty, and
// longer by `more` for each workgroup to a compute unit (of `resident`, beyond which it is another round); a state is written, read and written, and read.  Us of kernels, fewer
// segments / as chosen / more: 12 x 32760 x 128, 21 / 40 / 64, 195 / 172 / 200; 12 x 4680, with its state, 13 / 25 / 37, 56.4 / 52.1 / 51.9; 40 x 75600, 6 / 12 / 19, 1176 / 998 / 1099;
// prompts, 4 x 32 x 2048, 2 / 4 / 8, 127 / 107 / 132; step of 12 x 32760 x 128, 21 both ways / 40 forward and 14 backward / 40 both ways, 614 / 580 / 623; step of 2 x 12 x 4133 x 64, 10 both
// ways / 22 and 10 / 33 both ways, 114 / 108 / 123; fp32, 12 x 32760 x 128, 21 / 41 / 64, 630 / 551 / 590; 24 x 4133 x 64, 21 / 33 / 64, 94 / 71 / 83; step of 2 x 1024 x 64, 16 / 32, 53 / 41.
struct ChunkTimes {
  float rows, sums, more;
  int resident, chunk;
};
inline ChunkTimes chunk_times(bool f32, bool whole, int d) {      // of fp32 tensors; of bf16 tensors in fp32 arithmetic
  if (f32) return d == 128 ? ChunkTimes{6.5f, 4.f, 2.f, 2, kChunkF32} : ChunkTimes{4.4f, 3.f, 0.8f, 4, kChunkF32};
  if (whole) return d == 128 ? ChunkTimes{5.f, 1.6f, 1.5f, 1, kChunk} : ChunkTimes{3.f, 1.1f, 0.6f, 2, kChunk};
  return d == 128 ? ChunkTimes{3.1f, 1.4f, 1.5f, 2, kChunk} : ChunkTimes{2.f, 1.f, 0.6f, 3, kChunk};
}
inline Plan plan_of(int B, int H, int n, const ChunkTimes& t, int d, int row_passes, int sum_passes) {
  const int chunk = t.chunk;
  const int chunks = (n + chunk - 1) / chunk;
  const float heads = (float)B * (float)H;
  auto kernel = [&](float groups, float per, float one) {
    const float units = groups * (1.f / kCUs), full = (float)t.resident, rounds = units <= full ? 1.f : (float)(int)(units / full + 0.999f);
    return 4.f + rounds * per * (one + t.more * (units < full ? units : full));
  };
  Plan best{1, chunks * chunk};
  float least = 0;
  // (the next choice is the least number of segments that makes them shorter)
  for (int per = chunks, segs = 1;; per = (chunks - 1) / ((chunks - 1) / (per - 1) + 1) + 1) {
    segs = (chunks + per - 1) / per;
    if (segs > 256) break;
    float cost = kernel(heads * row_passes * segs, (float)per, t.rows);
    if (segs > 1) cost += kernel(heads * sum_passes * segs, (float)per, t.sums) + 4.f + heads * sum_passes * segs * (float)(d * d) * (16.f / 5.5e6f);
    if (segs == 1 || cost < least) { least = cost; best = Plan{segs, per * chunk}; }
    if (per == 1) break;
  }
  return best;
}

size_t work_bytes(int dtype, int B, int H, int HK, int n, int d, bool backward);
hipError_t launch_fwd(const Args& a);
hipError_t launch_bwd(const Args& a);

}  // namespace decay
}  // namespace linattn
