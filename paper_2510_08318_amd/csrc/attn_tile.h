// Tiles of keys and values in LDS for the bf16 attention kernels: rows of D bf16, 16-byte chunks XOR-swizzled by row (swz), and how they are filled.
#pragma once
#include "attn_pool.h"

namespace linattn {
namespace attn {

// 16 (or 4) bytes a lane from global memory straight to LDS, at `lds` + 16 (4) lane (lds uniform).  As assembly, because the compiler, which cannot tell the
// buffer that is being filled from the one that is being read, waits for the builtin's loads before every LDS read.  What it would do for the builtin is therefore done
// here: m0, which holds the LDS address, has to be written one wait state before the load that uses it (the hardware does not hold the load back).  The caller waits:
// lds_loads_landed() before the barrier that hands the tile over.
#define LINATTN_LDS_LOAD(LOAD) "s_mov_b32 m0, %0\n\ts_nop 0\n\t" LOAD
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile(LINATTN_LDS_LOAD("global_load_lds_dwordx4 %1, %2") ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(const void* at, uint32_t lds) {
  asm volatile(LINATTN_LDS_LOAD("global_load_lds_dwordx4 %1, off") ::"s"(lds), "v"(at) : "memory", "m0");
}
__device__ __forceinline__ void load_word_to_lds(const void* at, uint32_t lds) {
  asm volatile(LINATTN_LDS_LOAD("global_load_lds_dword %1, off") ::"s"(lds), "v"(at) : "memory", "m0");
}
#undef LINATTN_LDS_LOAD
__device__ __forceinline__ void lds_loads_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Operands that a kernel loads before its loop.  The compiler has to see them arrive there: it would otherwise wait for them at their first use, in every turn of the
// loop, and with them for the tile that has just been asked for (forward, 12 heads x 32760 x 128, window 2 x 3120: 1528 us, so, and with the operands of the scores read
// ahead, 1507).
template <int N>
__device__ __forceinline__ void arrived(uint4 (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i].x), "+v"(x[i].y), "+v"(x[i].z), "+v"(x[i].w));
}

// Rows j0 .. j0+KT-1 of a token tensor, by NW wavefronts: each instruction brings 1024 bytes, 512 / D rows.  Rows from `end` on are row end - 1 again (what is
// computed with them is masked).
template <int D, int NW, int KT>
struct RowTile {
  static constexpr int ROWS = 512 / D, N = KT / ROWS / NW;      // rows an instruction, instructions a wavefront
  static_assert(N * ROWS * NW == KT, "whole instructions");
  uint32_t chunk[N], row[N];
  __device__ __forceinline__ RowTile(int w, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      row[i] = (uint32_t)((w * N + i) * ROWS + lane / (D / 8));
      chunk[i] = (uint32_t)(((lane % (D / 8)) ^ swz<D>((int)row[i])) * 16);
    }
  }
  // base: the head's row 0; pitch: bytes from row to row
  __device__ __forceinline__ void load(const void* base, size_t pitch, int j0, int end, uint32_t lds, int w) const {
    const char* from = static_cast<const char*>(base) + (size_t)j0 * pitch;
    const uint32_t last = (uint32_t)(end - 1 - j0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t r = row[i] < last ? row[i] : last;
      load_to_lds(from, r * (uint32_t)pitch + chunk[i], lds + (uint32_t)((w * N + i) * 1024));
    }
  }
};

// Where a lane reads of a tile, as LDS addresses: row_at, the 16-byte chunks 2 ks + g of row m (lane = 32 g + m), and turned_at, the transposing reads of
// columns 32 c .. 32 c + 31 in the row order that a score block's registers have (tr_offset_g4).  k-steps and column blocks enter by exclusive-or, as tiles lie
// at multiples of 256 bytes, and rows by addition: two registers hold all addresses of a tile.
template <int D>
__device__ __forceinline__ uint32_t row_at(int lane) {
  return (uint32_t)(lane % 32 * (D * 2) + (((lane / 32) ^ swz<D>(lane % 32)) * 16));
}
template <int D>
__device__ __forceinline__ uint4 row_chunk(uint32_t at, int ks, int row0) {
  typedef __attribute__((address_space(3))) const u32x4* P;
  return __builtin_bit_cast(uint4, *(P)((at ^ (uint32_t)(32 * ks)) + (uint32_t)(row0 * D * 2)));
}
template <int D>
__device__ __forceinline__ uint32_t turned_at(int lane) { return (uint32_t)tr_lane<D, 4>((unsigned)lane); }
template <int D>
__device__ __forceinline__ bf16x8 turned(uint32_t at, int c, int row0) {
  const uint32_t x = at ^ (uint32_t)(64 * c), off = (uint32_t)(row0 * D * 2);
  return __builtin_bit_cast(bf16x8, read_tr(x + off, (x ^ 32u) + off + 8 * D * 2));
}

constexpr int kRowWaves = 4;                 // wavefronts that fill a tile together

// Where a workgroup's keys come from.  look(j0, end): the tile of KT keys from j0 on (there is memory behind every key below end, of later ones the last is taken again) is
// what the next ask_k and ask_v are for, which request its k or its v; put_k and put_v, before the next of them, bring what came through registers to LDS; landed() waits
// for what goes there directly.  there: the keys of the tile that exist.  len: the sequence's keys; tokens: its tokens, of which the last `count` are the chunk's (more
// than len where a sequence has outgrown its table).
struct TokenArgs {
  const void *k, *v;
  const int* lengths;
  Rows kr;
};
template <int D, int KT>
struct TokenSource {
  using Args = TokenArgs;
  static constexpr bool kPaged = false;
  const char *k, *v;
  size_t sn;
  int w, len, tokens, count, b, hk;
  RowTile<D, kRowWaves, KT> rows;
  __device__ __forceinline__ TokenSource(const Args& a, int b_, int hk_, int n, int w_, int lane) : sn(a.kr.sn), w(w_), b(b_), hk(hk_), rows(w_, lane) {
    len = clamp_length(a.lengths, b, n);
    tokens = count = len;
    const size_t at = ((size_t)b * a.kr.sb + (size_t)hk * a.kr.sh) * 2;
    k = static_cast<const char*>(a.k) + at;
    v = static_cast<const char*>(a.v) + at;
  }
  int j0, end;
  static constexpr unsigned long long there = ~0ull;
  __device__ __forceinline__ void look(int j0_, int end_) { j0 = j0_; end = end_; }
  __device__ __forceinline__ void ask_k(uint32_t lds) { rows.load(k, sn * 2, j0, end, lds, w); }
  __device__ __forceinline__ void ask_v(uint32_t lds) { rows.load(v, sn * 2, j0, end, lds, w); }
  __device__ __forceinline__ void put_k(uint32_t) {}
  __device__ __forceinline__ void put_v(uint32_t) {}
  __device__ __forceinline__ void landed() { lds_loads_landed(); }
  __device__ __forceinline__ TokenKeys<uint16_t> keys() const { return {reinterpret_cast<const uint16_t*>(k), reinterpret_cast<const uint16_t*>(v), sn}; }
};

// From the pool of a paged cache.  bf16 rows go straight to LDS; codes come through registers, where they become bf16.
template <int D, int KT, bool E4M3>
struct PoolSource {
  using Args = Pool;
  static constexpr bool kPaged = true;
  static constexpr int NW = kRowWaves, LPR = D / (E4M3 ? 16 : 8), N = KT * LPR / (64 * NW);      // lanes to a row, instructions a wavefront
  static_assert(N >= 1, "whole instructions");
  const Pool& p;
  int w, lane, len, tokens, count, b, hk;
  PoolRows at;
  unsigned long long there;
  uint4 ck[E4M3 ? N : 1], cv[E4M3 ? N : 1];
  uint32_t ek, ev;
  __device__ __forceinline__ PoolSource(const Args& a, int b_, int hk_, int n, int w_, int lane_) : p(a), w(w_), lane(lane_), b(b_), hk(hk_) {
    len = pool_length(p, b);
    tokens = pool_tokens(p, b);
    count = clamp_length(p.counts, b, n);
  }
  __device__ __forceinline__ int row(int i) const { return (w * N + i) * (64 / LPR) + lane / LPR; }
  __device__ __forceinline__ void look(int j0, int end) {
    at.find<KT>(p, b, hk, j0, end, lane);
    there = at.there;
  }
  __device__ __forceinline__ void ask(const void* pool, const uint8_t* exps, uint32_t lds, uint4* codes, uint32_t& e) {
    if constexpr (E4M3) e = exps[at.row];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i);
      const long long from = at.of(r) * D;
      if constexpr (E4M3) codes[i] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(pool) + from + 16 * (lane % LPR));
      else load_to_lds(static_cast<const char*>(pool) + (size_t)from * 2 + (size_t)(((lane % LPR) ^ swz<D>(r)) * 16), lds + (uint32_t)((w * N + i) * 1024));
    }
  }
  __device__ __forceinline__ void put(uint32_t lds, const uint4* codes, uint32_t e) {
    if constexpr (E4M3) {
      typedef __attribute__((address_space(3))) u32x4* P;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = row(i), c = 2 * (lane % LPR);
        const float s = row_scale((uint8_t)__shfl((int)e, r));
        const uint32_t to = lds + (uint32_t)(r * (D * 2)), c0 = (uint32_t)((c ^ swz<D>(r)) * 16);
        *(P)(to + c0) = __builtin_bit_cast(u32x4, decode8(make_uint2(codes[i].x, codes[i].y), s));
        *(P)(to + (c0 ^ 16u)) = __builtin_bit_cast(u32x4, decode8(make_uint2(codes[i].z, codes[i].w), s));
      }
    }
  }
  __device__ __forceinline__ void ask_k(uint32_t lds) { ask(p.k, p.k_exp, lds, ck, ek); }
  __device__ __forceinline__ void ask_v(uint32_t lds) { ask(p.v, p.v_exp, lds, cv, ev); }
  __device__ __forceinline__ void put_k(uint32_t lds) { put(lds, ck, ek); }
  __device__ __forceinline__ void put_v(uint32_t lds) { put(lds, cv, ev); }
  __device__ __forceinline__ void landed() { if constexpr (!E4M3) lds_loads_landed(); }
  __device__ __forceinline__ PoolKeys<E4M3> keys() const { return {&p, b, hk, D}; }
};

}  // namespace attn
}  // namespace linattn
