// The passes of decay.h on the matrix cores, bf16 operands and fp32 sums: chunks of kChunk tokens, inside of which a row's pairs are taken one by one, while what lies
// before comes through the state.  Bytes bound the whole: a forward call reads q, k and v, writes out, and reads k and v once more for the segments' sums (from the last-level cache, where
// they fit it).  Per token and head the products are 6 d^2 + 144 d multiply-adds (a X, the update, the segment's sum and the weights' products in two pieces; scores), which keep the matrix cores
// for 37 us of 12 x 32760 x 128, where the bytes are 69; the rest is the way of a chunk from memory through the matrix cores and back, which two workgroups on a compute unit overlap in part.
#pragma once
#include "attn_tile.h"
#include "decay.h"
#include "f32_split.h"

namespace linattn {
namespace decay {

using attn::lds_loads_landed;
using attn::row_at;
using attn::turned;

// attn::load_to_lds; STREAM: of data that will not be in the caches when it is read again.
#define LINATTN_LDS_LOAD(LOAD) "s_mov_b32 m0, %0\n\ts_nop 0\n\t" LOAD
template <bool STREAM>
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
  if constexpr (STREAM) asm volatile(LINATTN_LDS_LOAD("global_load_lds_dwordx4 %1, %2 nt") ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
  else attn::load_to_lds(base, offset, lds);
}
template <bool STREAM>
__device__ __forceinline__ void load_to_lds(const void* at, uint32_t lds) {
  if constexpr (STREAM) asm volatile(LINATTN_LDS_LOAD("global_load_lds_dwordx4 %1, off nt") ::"s"(lds), "v"(at) : "memory", "m0");
  else attn::load_to_lds(at, lds);
}
#undef LINATTN_LDS_LOAD

// The token at place i of a pass's order; places behind the last token are padding.
__device__ __forceinline__ int token_at(int i, int len, bool back) { return back && i < len ? len - 1 - i : i; }

// Rows i0 .. i0 + 63 of the pass's order into an LDS tile [64][D], chunks of 16 bytes swizzled by row, by four wavefronts; rows from `end` on are row end - 1 again.  Where a chunk is
// whole, a lane's offset from its first token in memory is the same for every chunk, and its loads differ by a multiple of the pitch (from the base, a scalar) and in the swizzle.
template <int D, bool STREAM>
struct Tile {
  static constexpr int ROWS = 512 / D, N = kChunk / ROWS / 4, BYTES = kChunk * D * 2;
  const char* base;
  size_t pitch;
  uint32_t offset;
  __device__ __forceinline__ void of(const Role& r, int b, int h, bool back, int w, int lane) {
    base = static_cast<const char*>(r.p) + ((size_t)b * r.r.sb + (size_t)(h / r.group) * r.r.sh) * 2;
    pitch = r.r.sn * 2;
    const int row = w * N * ROWS + lane / (D / 8);
    offset = (uint32_t)(back ? kChunk - 1 - row : row) * (uint32_t)pitch + (uint32_t)(((lane % (D / 8)) ^ swz<D>(row)) * 16);
  }
  __device__ __forceinline__ void load(int i0, int end, int len, bool back, uint32_t lds, int w, int lane) const {
    if (i0 + kChunk <= end) {
      const uint64_t first = reinterpret_cast<uint64_t>(base) + (size_t)(back ? len - i0 - kChunk : i0) * pitch, step = back ? -(uint64_t)(ROWS * pitch) : (uint64_t)(ROWS * pitch);
      // (The value is the same in all lanes, but the compiler may work it out in vector registers.  A scalar that a vector instruction wrote may be an address five wait states later, which
      // the compiler does not look after in assembly.)
      uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(first >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)first);
      asm volatile("s_nop 4" : "+s"(at));
      const char* from = reinterpret_cast<const char*>(at);
#pragma unroll
      for (int x = 0; x < N; ++x, from += step) load_to_lds<STREAM>(from, offset ^ (uint32_t)(swz<D>(ROWS * x) * 16), lds + (uint32_t)((w * N + x) * 1024));
      return;
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int row = (w * N + x) * ROWS + lane / (D / 8), i = i0 + row < end ? i0 + row : end - 1;
      const char* at = base + (size_t)token_at(i, len, back) * pitch + (((lane % (D / 8)) ^ swz<D>(row)) * 16);
      load_to_lds<STREAM>(at, lds + (uint32_t)((w * N + x) * 1024));
    }
  }
};

// Accumulators of a 32 x 32 block have rows 8a + 4g + b in the lanes of group g (registers 4a + b).  With bits 2 and 3 of a column's number exchanged where it becomes an
// operand's row, those are columns 16 (a / 2) + 8 g + 4 (a % 2) + b: eight adjacent ones to eight registers, so that operands of other tensors are whole 16-byte
// pieces of their rows, and so are a lane's results.  column_of: the column that operand row m stands for.  turned_columns: the transposing read's address (turned_at) with the
// columns in that order; in each group of 16 lanes, lane s gives the address of columns 4 (s % 4) .. + 3, and receives column s.
__device__ __forceinline__ int column_of(int m) { return (m & 19) | ((m & 4) << 1) | ((m & 8) >> 1); }
template <int D>
__device__ __forceinline__ uint32_t turned_columns(int lane) {
  return (uint32_t)tr_lane<D, 4>((unsigned)((lane & ~3) | ((lane & 1) << 1) | ((lane & 2) >> 1)));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
__device__ __forceinline__ bf16x8 pack8(const f32x16& e, int h) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(e[8 * h + 2 * i], e[8 * h + 2 * i + 1]);
  return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// An operand at an LDS address.  (As a vector: a struct of four words is taken apart by the compiler and read in two halves or four quarters.)
__device__ __forceinline__ bf16x8 operand_at(uint32_t at) {
  typedef __attribute__((address_space(3))) const bf16x8* P;
  return *(P)at;
}
// A value that the compiler cannot see through here: of an LDS address and a constant, the sum is then made in the instruction, and not kept (or made again and again) in a register
// of its own.
__device__ __forceinline__ void hide(uint32_t& x) { asm volatile("" : "+v"(x)); }
// An operand by the transposing reads from the addresses of its first 8 and its other 8 rows
__device__ __forceinline__ bf16x8 turned_at2(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(bf16x8, read_tr(lo, hi)); }

// Row of a k-step's element e in lane group g, as the transposing reads give them.
__device__ __forceinline__ constexpr int row_of(int e, int g) { return 8 * (e / 4) + 4 * g + e % 4; }

// Eight numbers, by pairs, as the sum of PIECES bf16 numbers each (three hold fp32 whole).
template <int PIECES, typename Two>
__device__ __forceinline__ void split(Two two, bf16x8 (&p)[PIECES]) {
  u32x4 out[PIECES];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    two(i, a, b);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      out[j][i] = pack_bf16x2(a, b);
      a -= f32::lo_f32(out[j][i]); b -= f32::hi_f32(out[j][i]);
    }
  }
#pragma unroll
  for (int j = 0; j < PIECES; ++j) p[j] = __builtin_bit_cast(bf16x8, out[j]);
}
// Rows times their weights.
template <int PIECES>
__device__ __forceinline__ void weigh(bf16x8 x, const float* w, bf16x8 (&p)[PIECES]) {
  const u32x4 in = __builtin_bit_cast(u32x4, x);
  split([&](int i, float& a, float& b) { a = f32::lo_f32(in[i]) * w[2 * i]; b = f32::hi_f32(in[i]) * w[2 * i + 1]; }, p);
}
// Registers 8 h .. 8 h + 7 of an accumulator.
template <int PIECES>
__device__ __forceinline__ void split8(const f32x16& e, int h, bf16x8 (&p)[PIECES]) {
  split([&](int i, float& a, float& b) { a = e[8 * h + 2 * i]; b = e[8 * h + 2 * i + 1]; }, p);
}
// acc += a p, the smallest piece first
template <int PIECES>
__device__ __forceinline__ f32x16 mfma_pieces(bf16x8 a, const bf16x8 (&p)[PIECES], f32x16 acc) {
#pragma unroll
  for (int j = PIECES - 1; j >= 0; --j) acc = mfma(a, p[j], acc);
  return acc;
}

// ---- a segment's own sum --------------------------------------------------------------------------------------------

struct SumPass {
  Role b, c;
  int back;
};
struct SumArgs {
  SumPass pass[2];
  int passes;
  Common c;
  Plan plan;
  float* sums;              // [pass][B * H][segment][D][D]
};

// sum_j lambda^(end - 1 - j) b_j^T c_j over a segment's tokens, end: the first behind them.  The rows c_j enter with their weights, whole, as three bf16 pieces (PIECES 3), where a
// state is handed out, as two where rows alone are made from it (their state enters them as two); b_j is bf16 as it is, so that the sum is one of exact products in fp32.
// Four wavefronts share a state's 32 x 32 blocks; the next chunk's rows load while this one's are multiplied.  12 x 32760 x 128 56 us with k and v from memory (201 MB, 3.6 TB/s, the matrix
// cores busy for 16 % of it, no LDS conflicts); deeper loads, of four chunks of 32 tokens, took as long.
template <int D, int PIECES, bool STREAM>
__global__ __launch_bounds__(256, 2) void decay_sum_kernel(SumArgs a) {
  constexpr int CB = D / 32, BLOCKS = CB * CB / 4, KS = kChunk / 16, TILE = Tile<D, false>::BYTES;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const Place at = place_of(a.c, blockIdx.x, a.plan.segs, a.passes);
  const SumPass& p = a.pass[at.pass];
  const int pass = at.pass, b = at.b, h = at.h, bh = b * a.c.H + h, seg = p.back ? a.plan.segs - 1 - at.seg : at.seg;
  const int len = __builtin_amdgcn_readfirstlane(length_of(a.c, b)), i0 = seg * a.plan.tokens, i1 = min(len, i0 + a.plan.tokens);
  if (i0 >= i1) return;
  const float decay = log_decay_of(a.c, h);
  Tile<D, STREAM> rows, columns;
  rows.of(p.b, b, h, p.back, w, lane);
  columns.of(p.c, b, h, p.back, w, lane);
  const uint32_t lds = lds_address(smem), from = turned_columns<D>(lane);
  const int cb = w % CB, fb0 = w / CB * BLOCKS;
  f32x16 sum[BLOCKS];
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) sum[i] = zero16();
  float rel[KS][8];         // of a whole chunk's tokens, relative to its last
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int e = 0; e < 8; ++e) rel[ks][e] = expf(decay * (float)(kChunk - 1 - 16 * ks - row_of(e, g)));

  auto ask = [&](int i, int buffer) {
    rows.load(i, i1, len, p.back, lds + buffer * 2 * TILE, w, lane);
    columns.load(i, i1, len, p.back, lds + buffer * 2 * TILE + TILE, w, lane);
  };
  ask(i0, 0);
  for (int i = i0, buffer = 0; i < i1; i += kChunk, buffer ^= 1) {
    lds_loads_landed();
    __syncthreads();
    if (i + kChunk < i1) ask(i + kChunk, buffer ^ 1);
    const uint32_t tile = lds + buffer * 2 * TILE;
    const bool whole = i + kChunk <= i1;
    const float after = whole ? expf(decay * (float)(i1 - i - kChunk)) : 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float wt[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) wt[e] = rel[ks][e] * after;
      bf16x8 x = turned<D>(from + tile + TILE, cb, 16 * ks);
      if (!whole) {
        u32x4 v = __builtin_bit_cast(u32x4, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = i + 16 * ks + row_of(e, g);
          wt[e] = j < i1 ? expf(decay * (float)(i1 - 1 - j)) : 0.f;
          if (j >= i1) v[e / 2] &= e % 2 ? 0xffffu : 0xffff0000u;
        }
        x = __builtin_bit_cast(bf16x8, v);
      }
      bf16x8 c[PIECES];
      weigh<PIECES>(x, wt, c);
#pragma unroll
      for (int y = 0; y < BLOCKS; ++y) {
        sum[y] = mfma_pieces(turned<D>(from + tile, fb0 + y, 16 * ks), c, sum[y]);
      }
    }
  }
  float* out = a.sums + (((size_t)pass * a.c.B * a.c.H + bh) * a.plan.segs + seg) * D * D;
#pragma unroll
  for (int y = 0; y < BLOCKS; ++y)
#pragma unroll
    for (int r = 0; r < 16; ++r) out[(32 * (fb0 + y) + 16 * (r / 8) + 8 * g + r % 8) * D + 32 * cb + column_of(m)] = sum[y][r];
}

// ---- the states in front of the segments ------------------------------------------------------------------------------

struct ScanPass {
  const float* in;          // nullable
  float* out;               // nullable
  int back;
  float in_scale;
  int by_item;              // states by item, not by slot
};
struct ScanArgs {
  ScanPass pass[2];
  int passes;
  Common c;
  Plan plan;
  float* sums;              // replaced by the states
  int size;                 // D * D
};

// lambda^r as a sum of two fp32 numbers: rounded to one, products along a sequence would be off by a multiple of its error.
__device__ __forceinline__ void power_of(float decay, int r, float& hi, float& lo) {
  const double x = exp((double)decay * (double)r);
  hi = (float)x;
  lo = (float)(x - (double)hi);
}

// Two elements of a head's state a thread, segment after segment: X in front of segment s (as decay.h has it: out's and dq's times lambda) takes the place of its
// sum, X' = lambda^tokens X + lambda sum.  A chain of segments, each a read and a write: at 40 segments of 12 heads 14 us (31 MB each way), at the largest call, 40 heads of 12, the same.
__global__ __launch_bounds__(256) void decay_scan_kernel(ScanArgs a) {
  const int pass = blockIdx.z, bh = blockIdx.y, b = bh / a.c.H, h = bh % a.c.H, e = (blockIdx.x * 256 + threadIdx.x) * 2;
  const ScanPass& p = a.pass[pass];
  Common com = a.c;
  if (p.by_item) { com.slots = nullptr; com.states = com.B; }
  const int len = length_of(com, b), step = a.plan.tokens, live = (len + step - 1) / step;
  const long long row = state_row(com, b, h);
  const float decay = log_decay_of(com, h), lambda = expf(decay);
  f32x2 x = {0.f, 0.f};
  if (p.in && row >= 0) x = *reinterpret_cast<const f32x2*>(p.in + row * a.size + e);
  if (!p.back && len > 0) x *= lambda;
  f32x2* at = reinterpret_cast<f32x2*>(a.sums + ((size_t)pass * a.c.B * a.c.H + bh) * a.plan.segs * a.size + e);
  const size_t next = a.size / 2;
  const float first = p.in_scale * lambda;
  float hi, lo, last_hi, last_lo;
  power_of(decay, step, hi, lo);
  // behind the last token: forward S_n = lambda^(tokens - 1) X + sum, back lambda^tokens X + lambda sum
  const int tokens = len - (live - 1) * step;
  power_of(decay, p.back ? tokens : tokens - 1, last_hi, last_lo);
  constexpr int AHEAD = 8;
  for (int s0 = 0; s0 < live; s0 += AHEAD) {
    f32x2 sum[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) sum[i] = s0 + i < live ? at[(s0 + i) * next] : f32x2{0.f, 0.f};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (s0 + i >= live) break;
      at[(s0 + i) * next] = x;
      const bool last = s0 + i == live - 1;
      const float f = last && !p.back ? p.in_scale : first, m = last ? last_hi : hi, l = last ? last_lo : lo;
      for (int y = 0; y < 2; ++y) x[y] = fmaf(x[y], m, fmaf(x[y], l, f * sum[i][y]));
    }
  }
  if (p.out && row >= 0) *reinterpret_cast<f32x2*>(p.out + row * a.size + e) = x;
}

// ---- rows -----------------------------------------------------------------------------------------------------------

struct RowPass {
  Pass p;
  const float* states;      // [B * H][segment][D][D], or null: p.in is in front of the one segment
  int by_item;
};
struct RowArgs {
  RowPass pass[3];
  int passes;
  Common c;
  Plan plan;
};

// A head's results, in the tensors' type or as fp32 parts.
template <typename T>
struct Results {
  void* base;
  size_t pitch;
  bool part;
  __device__ __forceinline__ Results(const Pass& p, int b, int h) : pitch(p.orow.sn), part(p.part) {
    const size_t at = (size_t)b * p.orow.sb + (size_t)h * p.orow.sh;
    base = part ? (void*)(static_cast<float*>(p.o) + at) : (void*)(static_cast<T*>(p.o) + at);
  }
  __device__ __forceinline__ float* part_row(int token, int c) const { return static_cast<float*>(base) + (size_t)token * pitch + c; }
  __device__ __forceinline__ T* row(int token, int c) const { return static_cast<T*>(base) + (size_t)token * pitch + c; }
};

// Rows from..to-1 of a head's results: zeros, for padding.
template <int D, int NT, typename T>
__device__ __forceinline__ void zero_rows(const Results<T>& out, int from, int to) {
  for (int i = from + threadIdx.x / (D / 8); i < to; i += NT / (D / 8)) {
    const int c = threadIdx.x % (D / 8) * 8;
    uint4* z = reinterpret_cast<uint4*>(out.part ? (void*)out.part_row(i, c) : (void*)out.row(i, c));
    z[0] = make_uint4(0, 0, 0, 0);
    if (sizeof(T) == 4 || out.part) z[1] = make_uint4(0, 0, 0, 0);
  }
}

// The state X in front of a segment: take(get), get(row, column).
template <int D, typename Take>
__device__ __forceinline__ void load_state(const RowArgs& a, const RowPass& rp, int bh, int seg, float decay, Take take) {
  const float* from = rp.states ? rp.states + ((size_t)bh * a.plan.segs + seg) * D * D : nullptr;
  float factor = 1.f;
  if (!from && rp.p.in) {
    Common com = a.c;
    if (rp.by_item) { com.slots = nullptr; com.states = com.B; }
    const long long row = state_row(com, bh / com.H, bh % com.H);
    if (row >= 0) from = rp.p.in + row * D * D;
    if (!rp.p.back) factor = expf(decay);
  }
  if (!from) take([](int, int) { return 0.f; });
  else if (rp.p.turned) take([&](int row, int column) { return from[column * D + row] * factor; });
  else take([&](int row, int column) { return from[row * D + column] * factor; });
}

constexpr int kPieces = 2, kAhead = 6;      // kPieces: bf16 numbers to a factor of products that make rows; kAhead: operands that are requested ahead of their products

// Where a pass's state goes, null where nowhere; of a sequence without tokens it is the state that it came with.
template <int D>
__device__ __forceinline__ float* state_out_of(const RowArgs& a, const RowPass& rp, int b, int h) {
  if (!rp.p.out) return nullptr;
  Common com = a.c;
  if (rp.by_item) { com.slots = nullptr; com.states = com.B; }
  const long long row = state_row(com, b, h);
  return row >= 0 ? rp.p.out + row * D * D : nullptr;
}
template <int D, int NT>
__device__ __forceinline__ void copy_state(const RowArgs& a, const RowPass& rp, int b, int h, float* to) {
  const float* from = rp.p.in ? rp.p.in + (to - rp.p.out) : nullptr;      // (the same row of the tensor)
  for (int i = threadIdx.x * 4; i < D * D; i += NT * 4)
    *reinterpret_cast<float4*>(to + i) = from ? *reinterpret_cast<const float4*>(from + i) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// WHOLE, fp32 arithmetic on bf16 tensors: weights, states and weighted rows enter as three pieces each, so that every product is that of fp32 numbers (a_i . b_j is one of bf16 as it is).
// STATE, of a call with one segment: the state behind the last token is handed out, so the rows c_j enter it whole, as three pieces, and lambda^chunk is a sum of two numbers.  (Else it
// is one number, and what came k chunks of a segment before is off by at most k 2^-24, as much as a factor's two pieces at 256 chunks.)
// Rows of a segment, chunk by chunk.  A wavefront has 32 columns of the state X in its accumulators, where they are the left operand of a_i X as they lie.  X, the weights P and
// the weighted rows c_j that go into the state are the sum of two bf16 numbers each, 2^-16 of a factor next to the 2^-8 of a result's own store, so that a result is as good as the store
// (1.66e-3 of its 2-norm; with X and P rounded to one bf16 number 2.35e-3, and a forward call 148 us at 12 x 32760 x 128 where it takes 156).  The chunk's weights P, on the lanes as
// S^T = B A^T gives them, are made by three of the wavefronts and go round through LDS.
// 64 tokens and not 32: half as many products with X, for pairs that cost as much as they save; a wavefront has 84 products a chunk at d 128.  Two workgroups on a compute unit (76 KB of LDS
// each, 242 to 256 registers a lane) and not one with all its tiles twice, which took 7 % longer at 40 x 75600 x 128 with X and P as one number.  12 x 32760 x 128, a mean of 20 calls in a
// row from a standing start, 103 us (the shortest 91: 435 MB at 4.8 TB/s), and without its loads and stores 84; the matrix cores are busy for 29 % of it, vector instructions for 37 %, a
// wavefront waits for 35 %.  40 x 75600 x 128 726 to 737 us, 511 without.
// At d 128 135 to 154 scalars wait in lanes of vector registers, 15 to 22 at d 64; two vector registers are spilled at d 128 with STATE.
template <int D, bool STATE, bool WHOLE>
__global__ __launch_bounds__(256, WHOLE ? 1 : 2) void decay_rows_kernel(RowArgs a) {
  constexpr int CB = D / 32, FB = D / 32, KS = D / 16, JS = kChunk / 16, IW = 4 / CB, IB = 2 / IW, TILE = Tile<D, false>::BYTES, ONE = WHOLE ? 3 : kPieces, PIECES = WHOLE || STATE ? 3 : kPieces;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 32, g = lane / 32;
  const Place at = place_of(a.c, blockIdx.x, a.plan.segs, a.passes);
  const RowPass& rp = a.pass[at.pass];
  const Pass& p = rp.p;
  const int b = at.b, h = at.h, bh = b * a.c.H + h, seg = p.back ? a.plan.segs - 1 - at.seg : at.seg;
  const int len = __builtin_amdgcn_readfirstlane(length_of(a.c, b)), i0 = seg * a.plan.tokens, all = min(a.c.n, i0 + a.plan.tokens), i1 = min(len, all);
  const Results<uint16_t> out(p, b, h);
  zero_rows<D, 256>(out, max(i0, i1), all);
  float* const state_out = STATE ? state_out_of<D>(a, rp, b, h) : nullptr;
  if (i0 >= i1) {
    if (STATE && state_out) copy_state<D, 256>(a, rp, b, h, state_out);
    return;
  }

  Tile<D, true> ta;         // (read once; b and c again by the neighbours of this workgroup, or just now by the sums' kernel)
  Tile<D, false> tb, tc;
  ta.of(p.a, b, h, p.back, w, lane);
  tb.of(p.b, b, h, p.back, w, lane);
  tc.of(p.c, b, h, p.back, w, lane);
  // in LDS: a chunk's a, its c, two of b; its pairs' weights; the weights that tokens have in the state behind a chunk
  const uint32_t lds = lds_address(smem), la = lds, lc = lds + TILE, weights = lds + 4 * TILE, kept = weights + ONE * 6 * 1024;
  auto b_tile = [&](int buffer) { return lds + (uint32_t)(2 + buffer) * TILE; };
  auto ask_ac = [&](int i) {
    ta.load(i, i1, len, p.back, la, w, lane);
    tc.load(i, i1, len, p.back, lc, w, lane);
  };
  tb.load(i0, i1, len, p.back, b_tile(0), w, lane);
  ask_ac(i0);

  const int cb = w % CB, ib0 = w / CB * IB, column = 32 * cb + column_of(m);
  const float decay = log_decay_of(a.c, h);
  f32x16 x[FB];
  load_state<D>(a, rp, bh, seg, decay, [&](auto get) {
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[f][r] = get(32 * f + 16 * (r / 8) + 8 * g + r % 8, column);
  });
  // weights: of a pair in the wavefront's block; of a token in the state behind the chunk; of the state in a row, and over a chunk
  float pairs[16], mine[IB];
  const float pair_scale = p.in_scale * p.out_scale;      // (one of them is 1)
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int gap = m - row_of(r % 8, g) - 16 * (r / 8) + (w == 1 ? 32 : 0);
    pairs[r] = gap >= 0 ? expf(decay * (float)gap) * pair_scale : 0.f;
  }
  auto keep_weights = [&](int from, int tokens) {      // lambda^(from - j) of token j, [k-step][g][8], by a wavefront
    const int j = 16 * (lane / 16) + row_of(lane % 8, lane / 8 % 2);
    *(__attribute__((address_space(3))) float*)(kept + 4 * (uint32_t)lane) = j < tokens ? expf(decay * (float)(from - j)) * p.in_scale : 0.f;
  };
  if (w == 3 && (!STATE || i0 + kChunk < i1)) keep_weights(kChunk, kChunk);
#pragma unroll
  for (int i = 0; i < IB; ++i) mine[i] = expf(decay * (float)(32 * (ib0 + i) + m)) * p.out_scale;
  float over, over_lo;
  power_of(decay, kChunk, over, over_lo);

  // Addresses in the tile of a, and so, with constants that fit an instruction, in the others: 16-byte pieces 2 ks + g of row m; first and second 8 rows of a block's columns, transposed.
  uint32_t rows_at[KS], columns_at[FB][2], c_at[2], weights_at = weights + 16 * (uint32_t)lane, kept_at = kept + 32 * (uint32_t)g;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) rows_at[ks] = la + (row_at<D>(lane) ^ (uint32_t)(32 * ks));
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int f = 0; f < FB; ++f) columns_at[f][x] = la + (turned_columns<D>(lane) ^ (uint32_t)(64 * f + 32 * x));
    c_at[x] = lc + (turned_columns<D>(lane) ^ (uint32_t)(64 * cb + 32 * x));
  }
  const uint32_t pair_rows = (uint32_t)((w > 0) * 32 * D * 2), pair_tokens = (uint32_t)((w == 2) * 32 * D * 2);
  auto chunk = [&](int i, auto buffer_) {
    constexpr int buffer = decltype(buffer_)::value;
    constexpr uint32_t lb = (uint32_t)(2 + buffer) * TILE;      // from la
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) hide(rows_at[ks]);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int f = 0; f < FB; ++f) hide(columns_at[f][x]);
      hide(c_at[x]);
    }
    hide(weights_at);
    hide(kept_at);
    lds_loads_landed();
    __syncthreads();
    const bool more = i + kChunk < i1;
    if (more) tb.load(i + kChunk, i1, len, p.back, b_tile(buffer ^ 1), w, lane);

    // The rows of a chunk go before the state behind it: the other workgroup of the compute unit is in another phase, and its products fill the waits of this one's (40 x 75600
    // x 128 754 us with one priority, 726 so; raised for the state instead 734).
    __builtin_amdgcn_s_setprio(1);
    // weights of block w: (0, 0), (1, 0), (1, 1) of rows and tokens
    if (w < 3) {
      f32x16 s = zero16();
      bf16x8 op[2 * KS];
      auto get = [&](int i) { op[i] = operand_at((rows_at[i / 2] + (i % 2 ? pair_rows : pair_tokens)) + (i % 2 ? 0 : lb)); };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) get(i);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        for (int i = 2 * ks + kAhead; i < 2 * ks + kAhead + 2 && i < 2 * KS; ++i) get(i);
        __builtin_amdgcn_sched_barrier(0);
        s = mfma(op[2 * ks], op[2 * ks + 1], s);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = w == 1 || row_of(r % 8, g) + 16 * (r / 8) <= m ? s[r] * pairs[r] : 0.f;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        bf16x8 piece[ONE];
        split8(s, hh, piece);
#pragma unroll
        for (int j = 0; j < ONE; ++j) *(__attribute__((address_space(3))) bf16x8*)(weights_at + (uint32_t)((6 * j + 2 * w + hh) * 1024)) = piece[j];
      }
    }

    // Behind the last token (see decay_scan_kernel) weights go by the chunk's tokens; those that are not there have none.
    if (STATE && w == 3 && !more) keep_weights(i1 - i - (p.back ? 0 : 1), i1 - i);

    // a_i X, and what lies before the chunk fades
    f32x16 o[IB];
    {
#pragma unroll
      for (int y = 0; y < IB; ++y) o[y] = zero16();
      bf16x8 op[KS * IB], xs[ONE];
      auto get = [&](int i) { op[i] = operand_at(rows_at[i / IB] + (uint32_t)((ib0 + i % IB) * 32 * D * 2)); };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) get(i);
#pragma unroll
      for (int i = 0; i < KS * IB; ++i) {
        if (i + kAhead < KS * IB) get(i + kAhead);
        __builtin_amdgcn_sched_barrier(0);
        if (i % IB == 0) split8(x[i / IB / 2], i / IB % 2, xs);
#pragma unroll
        for (int j = ONE - 1; j >= 0; --j) o[i % IB] = mfma(xs[j], op[i], o[i % IB]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int y = 0; y < IB; ++y)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[y][r] *= mine[y];
    }
    bf16x8 c[JS];
#pragma unroll
    for (int ks = 0; ks < JS; ++ks) c[ks] = turned_at2(c_at[0] + (uint32_t)(16 * ks * D * 2), c_at[1] + (uint32_t)((16 * ks + 8) * D * 2));
    // A weight of 0 does not keep an infinity or NaN of a later token out of a product: where there is one, the chunk's pairs one by one, over what a row sees.
    float odd = 0.f;
#pragma unroll
    for (int ks = 0; ks < JS; ++ks) {
      const u32x4 words = __builtin_bit_cast(u32x4, c[ks]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = words[e];      // (the bit cast of a vector's element takes the first one's)
        odd = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0u), odd, false);
      }
    }
    const bool one_by_one = __any(odd != 0.f);
    __syncthreads();
    if (more) ask_ac(i + kChunk);

    if (!one_by_one) {
      auto pairs_of = [&](f32x16& acc, int blk, int block) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          bf16x8 piece[ONE];
#pragma unroll
          for (int j = 0; j < ONE; ++j) piece[j] = operand_at(weights_at + (uint32_t)((6 * j + 2 * blk + hh) * 1024));
          acc = mfma_pieces(c[2 * block + hh], piece, acc);
        }
      };
#pragma unroll
      for (int y = 0; y < IB; ++y) {
        pairs_of(o[y], ib0 + y, 0);
        if (ib0 + y) pairs_of(o[y], 2, 1);
      }
    } else {
#pragma unroll
      for (int y = 0; y < IB; ++y)
        for (int j = 0; j <= 32 * (ib0 + y) + m; ++j) {
          const int jj = j % 16, src = 32 * ((jj / 4) % 2) + m, elem = jj / 8 * 4 + jj % 4;
          const int blk = ib0 + y == 0 ? 0 : j < 32 ? 1 : 2;
          const uint32_t pw = weights + (uint32_t)((2 * blk + j % 32 / 16) * 1024 + 16 * src + 2 * elem);
          float wt = 0.f;
#pragma unroll
          for (int piece = ONE - 1; piece >= 0; --piece)
            wt += __builtin_bit_cast(float, (uint32_t)*(__attribute__((address_space(3))) const uint16_t*)(pw + (uint32_t)(piece * 6 * 1024)) << 16);
          const uint16_t* from = reinterpret_cast<const uint16_t*>(tc.base + (size_t)token_at(min(i + j, i1 - 1), len, p.back) * tc.pitch) + 32 * cb + 8 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) o[y][r] = fmaf(wt, f32::ldf(from, 16 * (r / 8) + r % 8), o[y][r]);
        }
    }
    __builtin_amdgcn_s_setprio(0);
    // A lane has channels 8 g .. + 7 and 16 + 8 g .. + 7 of the wavefront's 32 of row m.  Exchanged with the lane 16 further, an instruction has 64 bytes of 16 rows, not 32 of
    // 32: 16 x 32 heads x 1024 x 128 136 us, and 132 to 135 so; a step of 12 x 32760 x 128 405 and 400.  (Past the cache, 40 x 75600 x 128, 846 and 734, where it takes 726 so.)
#pragma unroll
    for (int y = 0; y < IB; ++y) {
      const int from = i + 32 * (ib0 + y);
      if (!out.part) {
        u32x4 first = __builtin_bit_cast(u32x4, pack8(o[y], 0)), second = __builtin_bit_cast(u32x4, pack8(o[y], 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const auto r = __builtin_amdgcn_permlane16_swap(first[e], second[e], false, false);
          first[e] = r[0]; second[e] = r[1];
        }
        const int ch = 32 * cb + 8 * g + (m & 16), place = from + m % 16;
        if (place < i1) *reinterpret_cast<u32x4*>(out.row(token_at(place, len, p.back), ch)) = first;
        if (place + 16 < i1) *reinterpret_cast<u32x4*>(out.row(token_at(place + 16, len, p.back), ch)) = second;
      } else if (from + m < i1) {
        float* to = out.part_row(token_at(from + m, len, p.back), 32 * cb + 8 * g);
#pragma unroll
        for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(to + 16 * (r / 8) + r % 8) = f32x4{o[y][r], o[y][r + 1], o[y][r + 2], o[y][r + 3]};
      }
    }

    if (more || (STATE && state_out)) {
      float fade = over, fade_lo = over_lo;
      if (STATE && !more) power_of(decay, i1 - i - (p.back ? 0 : 1), fade, fade_lo);
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[f][r] = WHOLE || STATE ? fmaf(x[f][r], fade, x[f][r] * fade_lo) : x[f][r] * fade;
#pragma unroll
      for (int ks = 0; ks < JS; ++ks) {
        bf16x8 cw[PIECES];
        float keep[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const f32x4 four = *(__attribute__((address_space(3))) const f32x4*)(kept_at + (uint32_t)(64 * ks + 16 * half));
#pragma unroll
          for (int e = 0; e < 4; ++e) keep[4 * half + e] = four[e];
        }
        weigh<PIECES>(c[ks], keep, cw);
#pragma unroll
        for (int f = 0; f < FB; ++f) {
          x[f] = mfma_pieces(turned_at2(columns_at[f][0] + lb + (uint32_t)(16 * ks * D * 2), columns_at[f][1] + lb + (uint32_t)((16 * ks + 8) * D * 2)), cw, x[f]);
        }
      }
    }
  };
  for (int i = i0; i < i1; i += 2 * kChunk) {
    chunk(i, std::integral_constant<int, 0>{});
    if (i + kChunk < i1) chunk(i + kChunk, std::integral_constant<int, 1>{});
  }
  if (STATE && state_out && (IB == 2 || ib0 == 0)) {
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) state_out[(32 * f + 16 * (r / 8) + 8 * g + r % 8) * D + column] = x[f][r];
  }
}

template <int D, bool WHOLE>
constexpr int rows_lds() { return 4 * Tile<D, false>::BYTES + (WHOLE ? 3 : kPieces) * 6 * 1024 + kChunk * 4; }
template <int D>
constexpr int sum_lds() { return 4 * Tile<D, false>::BYTES; }

}  // namespace decay
}  // namespace linattn
