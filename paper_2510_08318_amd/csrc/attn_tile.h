// Tiles of keys and values in LDS for the bf16 attention kernels: rows of D bf16, 16-byte chunks XOR-swizzled by row (swz), and how they are filled.
#pragma once
#include "attn.h"
#include "mfma_common.h"

namespace linattn {
namespace attn {

// 16 bytes a lane from global memory straight to LDS, at `lds` + 16 lane (lds uniform).  As assembly, because the compiler, which cannot tell the
// buffer that is being filled from the one that is being read, waits for the builtin's loads before every LDS read.  The caller waits:
// lds_loads_landed() before the barrier that hands the tile over.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(const void* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory");
}
__device__ __forceinline__ void lds_loads_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

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

}  // namespace attn
}  // namespace linattn
