// The passes of decay.h for fp32 tensors, on v_mfma_f32_32x32x2_f32.  Chunks of kChunkF32 tokens; a wavefront has 32 columns of the state.
//   lane l = (m, g), m = l % 32, g = l / 32.  A: A[m][g], B: B[g][m], D: rows 8 (r / 4) + 4 g + r % 4 of column m
// so register r of an accumulator is, as it lies, the operand of a step over rows 8 (r / 4) + r % 4 and that + 4.
// 12 x 32760 x 128 takes 557 us: these instructions alone 290, the bytes 137, and the rest is waits of a chunk between its barriers (loads, the scores' sum through LDS) that the other
// workgroups of the compute unit do not fill.  A step of 2 x 1024 x 64 41 (rows 8, sums 6, states between 6, twice).  (bf16 tensors in fp32 arithmetic are on the bf16 instructions, three
// pieces to an fp32 number, in 250; of fp32 tensors both factors of a product would be three, six products to one.)
#pragma once
#include "decay_rows.h"

namespace linattn {
namespace decay {

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// Rows of a token tensor into an fp32 LDS tile [32][D], its 16-byte pieces swizzled by row, through registers: ask requests, put writes.  Rows from `end` on are row end - 1 again.
template <int D>
struct TileF32 {
  static constexpr int NT = 2 * D, V = 4, N = kChunkF32 * D / V / NT, WORDS = kChunkF32 * D;
  const float* base;
  size_t pitch;
  uint4 x[N];
  __device__ __forceinline__ void of(const Role& r, int b, int h) {
    base = static_cast<const float*>(r.p) + (size_t)b * r.r.sb + (size_t)(h / r.group) * r.r.sh;
    pitch = r.r.sn;
  }
  __device__ __forceinline__ void ask(int i0, int end, int len, bool back) {
#pragma unroll
    for (int y = 0; y < N; ++y) {
      const int item = y * NT + threadIdx.x, row = item / (D / V), i = i0 + row < end ? i0 + row : end - 1;
      x[y] = *reinterpret_cast<const uint4*>(base + (size_t)token_at(i, len, back) * pitch + item % (D / V) * V);
    }
  }
  static __device__ __forceinline__ int word(int row, int c) { return row * D + (((c / 4) ^ (row % (D / 4))) * 4) + c % 4; }
  __device__ __forceinline__ void put(float* tile) const {
#pragma unroll
    for (int y = 0; y < N; ++y) {
      const int item = y * NT + threadIdx.x, row = item / (D / V), c = item % (D / V) * V;
      *reinterpret_cast<uint4*>(tile + word(row, c)) = x[y];
    }
  }
};

__device__ __forceinline__ int row_of_reg(int r, int g) { return 8 * (r / 4) + 4 * g + r % 4; }

// LDS addresses that the compiler need not keep (it held one in a register for each read: half a wavefront's registers).  In a tile that starts at a multiple of a row's bytes, element
// (row_of_reg(r, g), 32 f + m) is at down_at(lane, r % 4) + down(f, r), that of a column block f that is no constant at (down_at ^ 128 f ^ down_block(r)) + down_row(r), and elements
// (m, 32 f + 8 q + 4 g) .. + 3 at across_at(lane) ^ across(f, q).
template <int D>
__device__ __forceinline__ uint32_t down_at(int lane, int y) {
  const int m = lane % 32, g = lane / 32;
  return (uint32_t)(4 * g * D * 4 + (((m / 4) ^ (4 * g) ^ y) << 4) + m % 4 * 4);
}
template <int D>
__device__ __forceinline__ constexpr uint32_t down_row(int r) { return (uint32_t)((8 * (r / 4) + r % 4) * D * 4); }
template <int D>
__device__ __forceinline__ constexpr uint32_t down_block(int r) { return (uint32_t)((r / 4 % (D / 32)) << 7); }
template <int D>
__device__ __forceinline__ constexpr uint32_t down(int f, int r) { return down_row<D>(r) + ((uint32_t)(f << 7) ^ down_block<D>(r)); }
template <int D>
__device__ __forceinline__ uint32_t across_at(int lane) { return (uint32_t)(lane % 32 * D * 4 + (((lane / 32) ^ (lane % 32 % (D / 4))) << 4)); }
__device__ __forceinline__ constexpr uint32_t across(int f, int q) { return (uint32_t)((8 * f + 2 * q) << 4); }
__device__ __forceinline__ float number_at(uint32_t at) { return *(__attribute__((address_space(3))) const float*)at; }
__device__ __forceinline__ f32x4 numbers_at(uint32_t at) { return *(__attribute__((address_space(3))) const f32x4*)at; }

// A segment's own sum, as decay_sum_kernel.
template <int D>
__global__ __launch_bounds__(2 * D) void decay_sum_f32_kernel(SumArgs a) {
  using Tile_ = TileF32<D>;
  constexpr int FB = D / 32, WORDS = Tile_::WORDS;
  extern __shared__ __align__(1024) float tiles[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const Place at = place_of(a.c, blockIdx.x, a.plan.segs, a.passes);
  const SumPass& p = a.pass[at.pass];
  const int pass = at.pass, b = at.b, h = at.h, bh = b * a.c.H + h, seg = p.back ? a.plan.segs - 1 - at.seg : at.seg;
  const int len = length_of(a.c, b), i0 = seg * a.plan.tokens, i1 = min(len, i0 + a.plan.tokens);
  if (i0 >= i1) return;
  const float decay = log_decay_of(a.c, h);
  Tile_ rows, columns;
  rows.of(p.b, b, h);
  columns.of(p.c, b, h);
  f32x16 sum[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) sum[f] = zero16();
  auto ask = [&](int i) { rows.ask(i, i1, len, p.back); columns.ask(i, i1, len, p.back); };
  auto put = [&](int buffer) { rows.put(tiles + buffer * 2 * WORDS); columns.put(tiles + buffer * 2 * WORDS + WORDS); };
  ask(i0);
  float rel[16];            // weights of a whole chunk's tokens, relative to its last
#pragma unroll
  for (int r = 0; r < 16; ++r) rel[r] = expf(decay * (float)(kChunkF32 - 1 - row_of_reg(r, g)));
  put(0);
  const uint32_t lds = lds_address(tiles);
  for (int i = i0, buffer = 0; i < i1; i += kChunkF32, buffer ^= 1) {
    __syncthreads();
    const bool more = i + kChunkF32 < i1, whole = i + kChunkF32 <= i1;
    if (more) ask(i + kChunkF32);
    uint32_t b_at[4], c_at[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      b_at[y] = lds + buffer * 2 * WORDS * 4 + down_at<D>(lane, y);
      c_at[y] = b_at[y] + WORDS * 4 + 128 * w;
      hide(b_at[y]);
      hide(c_at[y]);
    }
    const float after = whole ? expf(decay * (float)(i1 - i - kChunkF32)) : 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float c = number_at((c_at[r % 4] ^ down_block<D>(r)) + down_row<D>(r));
      if (whole) c *= rel[r] * after;
      else {
        const int j = i + row_of_reg(r, g);
        c = j < i1 ? c * expf(decay * (float)(i1 - 1 - j)) : 0.f;
      }
#pragma unroll
      for (int f = 0; f < FB; ++f) sum[f] = mfma_f32(number_at(b_at[r % 4] + down<D>(f, r)), c, sum[f]);
    }
    if (more) put(buffer ^ 1);
  }
  float* out = a.sums + (((size_t)pass * a.c.B * a.c.H + bh) * a.plan.segs + seg) * D * D;
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int r = 0; r < 16; ++r) out[(32 * f + row_of_reg(r, g)) * D + 32 * w + m] = sum[f][r];
}

// Rows of a segment, as decay_rows_kernel: every wavefront takes 32 channels of the scores a_i . b_j of all pairs, and their sum through LDS gives it all of them, where the product with c_j
// wants them.  Tiles once, the next chunk's in registers on the way, and weights from a table in LDS, so that two workgroups fit a compute unit at d 128 and four at 64, and fill each
// other's waits: 12 x 32760 x 128 419 us with one, 386 with two.  (A workgroup of d 64 has two wavefronts; two such workgroups on a compute unit may share two of its four SIMDs: 2 x 12 x 4133
// x 64 60 us with as many segments as that fills, 42 with half as many again.)  At d 128 one vector register is spilled.
template <int D>
__global__ __launch_bounds__(2 * D, 2) void decay_rows_f32_kernel(RowArgs a) {
  using Tile_ = TileF32<D>;
  constexpr int NW = D / 32, FB = D / 32, WORDS = Tile_::WORDS;
  extern __shared__ __align__(1024) float tiles[];
  float4* const parts = reinterpret_cast<float4*>(tiles + 3 * WORDS);      // [wavefront][4][64]: four registers
  float* const table = reinterpret_cast<float*>(parts + NW * 256);           // [65]: lambda^(i - 32), with in_scale; 0 for what comes later
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const Place at = place_of(a.c, blockIdx.x, a.plan.segs, a.passes);
  const RowPass& rp = a.pass[at.pass];
  const Pass& p = rp.p;
  const int b = at.b, h = at.h, bh = b * a.c.H + h, seg = p.back ? a.plan.segs - 1 - at.seg : at.seg;
  const int len = length_of(a.c, b), i0 = seg * a.plan.tokens, all = min(a.c.n, i0 + a.plan.tokens), i1 = min(len, all);
  const Results<float> out(p, b, h);
  zero_rows<D, 2 * D>(out, max(i0, i1), all);
  float* const state_out = a.plan.segs == 1 ? state_out_of<D>(a, rp, b, h) : nullptr;      // (with several segments the scan writes it)
  if (i0 >= i1) {
    if (state_out) copy_state<D, 2 * D>(a, rp, b, h, state_out);
    return;
  }

  Tile_ ta, tb, tc;
  ta.of(p.a, b, h);
  tb.of(p.b, b, h);
  tc.of(p.c, b, h);
  auto ask = [&](int i) { ta.ask(i, i1, len, p.back); tb.ask(i, i1, len, p.back); tc.ask(i, i1, len, p.back); };
  auto put = [&] {
    ta.put(tiles);
    tb.put(tiles + WORDS);
    tc.put(tiles + 2 * WORDS);
  };
  ask(i0);
  put();
  const float decay = log_decay_of(a.c, h);
  f32x16 x[FB];
  load_state<D>(a, rp, bh, seg, decay, [&](auto get) {
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[f][r] = get(32 * f + row_of_reg(r, g), 32 * w + m);
  });
  if (w == 0) {
    table[lane] = lane < kChunkF32 ? 0.f : expf(decay * (float)(lane - kChunkF32)) * p.in_scale;
    if (lane == 0) table[2 * kChunkF32] = expf(decay * (float)kChunkF32) * p.in_scale;
  }
  const float mine = expf(decay * (float)m);
  float hi, lo;
  power_of(decay, kChunkF32, hi, lo);
  // weights of tokens row_of_reg(r, g) in row m, and in the state behind the chunk: from here 4 (LAST - row_of_reg(r, 0)) on
  constexpr int LAST = 27;
  const uint32_t lds = lds_address(tiles);
  uint32_t diag_at = lds_address(table) + 4 * (uint32_t)(kChunkF32 + m - 4 * g - LAST), keep_at = lds_address(table) + 4 * (uint32_t)(2 * kChunkF32 - 4 * g - LAST);

  for (int i = i0; i < i1; i += kChunkF32) {
    __syncthreads();
    const bool more = i + kChunkF32 < i1;
    if (more) ask(i + kChunkF32);
    const float* const lc = tiles + 2 * WORDS;
    uint32_t a_at = lds + across_at<D>(lane), b_at[4], c_at[4];
    hide(a_at);
    hide(diag_at);
    hide(keep_at);
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      b_at[y] = lds + WORDS * 4 + down_at<D>(lane, y);
      c_at[y] = b_at[y] + WORDS * 4 + 128 * w;
      hide(b_at[y]);
      hide(c_at[y]);
    }

    f32x16 s = zero16();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t at = a_at ^ across(w, q);
      const f32x4 kb = numbers_at(at + WORDS * 4), qa = numbers_at(at);
      s = mfma_f32(kb.x, qa.x, s); s = mfma_f32(kb.y, qa.y, s); s = mfma_f32(kb.z, qa.z, s); s = mfma_f32(kb.w, qa.w, s);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) parts[(w * 4 + q) * 64 + lane] = make_float4(s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]);

    f32x16 o;
    auto before = [&] {
      o = zero16();
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 qa = numbers_at(a_at ^ across(f, q));
          o = mfma_f32(x[f][4 * q], qa.x, o); o = mfma_f32(x[f][4 * q + 1], qa.y, o);
          o = mfma_f32(x[f][4 * q + 2], qa.z, o); o = mfma_f32(x[f][4 * q + 3], qa.w, o);
        }
#pragma unroll
      for (int r = 0; r < 16; ++r) o[r] *= mine;
    };
    before();
    float c[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = number_at((c_at[r % 4] ^ down_block<D>(r)) + down_row<D>(r));
    __syncthreads();
    auto score = [&](int q, int from) {
      float4 t = parts[q * 64 + from];
#pragma unroll
      for (int y = 1; y < NW; ++y) {
        const float4 u = parts[(y * 4 + q) * 64 + from];
        t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
      }
      return t;
    };
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 t = score(q, lane);
      const float e[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int r = 4 * q + y;
        o = mfma_f32(c[r], row_of_reg(r, g) <= m ? e[y] * number_at(diag_at + 4 * (LAST - row_of_reg(r, 0))) : 0.f, o);
      }
    }

    // rows that are not finite once more, over what they see (see decay_rows_kernel)
    float odd = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = fmaf(o[r], 0.f, odd);
    if (__any(odd != 0.f)) {
      before();
      for (int j = 0; j <= m; ++j) {
        const float4 t = score(j / 8, 32 * (j / 4 % 2) + m);
        const float wt = (j % 4 == 0 ? t.x : j % 4 == 1 ? t.y : j % 4 == 2 ? t.z : t.w) * (expf(decay * (float)(m - j)) * p.in_scale);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[r] = fmaf(wt, lc[Tile_::word(j, 32 * w + row_of_reg(r, g))], o[r]);
      }
    }
    if (i + m < i1) {
      const int token = token_at(i + m, len, p.back);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int ch = 32 * w + 4 * g + 8 * q;
        const float4 v = make_float4(o[4 * q] * p.out_scale, o[4 * q + 1] * p.out_scale, o[4 * q + 2] * p.out_scale, o[4 * q + 3] * p.out_scale);
        *reinterpret_cast<float4*>(out.row(token, ch)) = v;      // (parts have the same type)
      }
    }
    if (more || state_out) {
      // the last chunk's tokens: see decay_rows_kernel
      const int last = i1 - i - (p.back ? 0 : 1);
      float fade = hi, fade_lo = lo;
      if (!more) power_of(decay, last, fade, fade_lo);
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[f][r] = fmaf(x[f][r], fade, x[f][r] * fade_lo);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = row_of_reg(r, g);
        const float cw = more ? c[r] * number_at(keep_at + 4 * (LAST - row_of_reg(r, 0))) : i + j < i1 ? c[r] * (expf(decay * (float)(last - j)) * p.in_scale) : 0.f;
#pragma unroll
        for (int f = 0; f < FB; ++f) x[f] = mfma_f32(number_at(b_at[r % 4] + down<D>(f, r)), cw, x[f]);
      }
      if (more) {
        __syncthreads();
        put();
      }
    }
  }
  if (state_out) {
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) state_out[(32 * f + row_of_reg(r, g)) * D + 32 * w + m] = x[f][r];
  }
}

template <int D>
constexpr int rows_f32_lds() { return 3 * kChunkF32 * D * 4 + D / 32 * 4096 + 320; }
template <int D>
constexpr int sum_f32_lds() { return 4 * kChunkF32 * D * 4; }

}  // namespace decay
}  // namespace linattn
