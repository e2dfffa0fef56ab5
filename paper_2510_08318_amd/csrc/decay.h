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

// A head's decay as the kernels use it: what is above 0, or NaN, counts as 0, and -inf as a number whose products with distances stay finite.
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
// The number of segments by a count of what each choice costs, in chunks of a workgroup of the rows kernel: as many rounds of resident workgroups as the call makes, and
// with several segments the sums, which read two tensors of three, and two launches more.
inline Plan plan_of(int B, int H, int n, int d, int chunk, int row_passes, int sum_passes) {
  const long long chunks = (n + chunk - 1) / chunk, heads = (long long)B * H, slots = kCUs * (chunk == kChunkF32 && d == 128 ? 1 : 2);
  Plan best{1, (int)chunks * chunk};
  double least = 0;
  for (long long want = 1; want <= chunks && want <= 256; ++want) {
    const long long per = (chunks + want - 1) / want, segs = (chunks + per - 1) / per;
    if (segs != want) continue;
    const long long rounds = (heads * row_passes * segs + slots - 1) / slots, sums = (heads * sum_passes * segs + slots - 1) / slots;
    double cost = (double)rounds * (double)(per + 1);
    if (segs > 1) cost += (double)sums * (0.6 * (double)per + 1) + 5 + 0.1 * (double)segs;
    if (want == 1 || cost < least) { least = cost; best = Plan{(int)segs, (int)per * chunk}; }
  }
  return best;
}

size_t work_bytes(int dtype, int B, int H, int HK, int n, int d, bool backward);
hipError_t launch_fwd(const Args& a);
hipError_t launch_bwd(const Args& a);

}  // namespace decay
}  // namespace linattn
