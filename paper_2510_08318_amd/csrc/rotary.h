// Rotary positions (linattn_rotary): what the host dispatch and the kernels agree on.
#pragma once
#include "kernels.h"

namespace linattn {
namespace rotary {

struct Args {
  const void *q, *k;        // k: nullable
  void *qo, *ko;
  Rows qr, kr;
  int B, H, HK, n, d;       // HK 0 without k
  int from[4];              // first channel of each axis; the channels from[3] .. d-1, and axes that are not there, have none
  int halves, back;
  int grid1, grid2;         // tokens along the second and third axis
  int first[3], axes;
  const int* positions;     // nullable
  size_t item;              // positions from item to item of the batch
  const int* lengths;       // nullable
  double turns[64];         // of pair p, in the order of the axes: turns for each position, base^(-2m / dims) / (2 pi)
};

// Workgroups of the tokens, `blocks` in all, in grid.x and grid.z (the last of z has ones behind the end), the groups of heads in grid.y.  A launch holds fewer than 2^32 threads in grid.x,
// 2^24 workgroups; 2^27 tokens of fp32 x 128, 64 GB with one head, are as many.  The most blocks, 2^35 tokens in eights, are 2^12 in grid.z.
constexpr unsigned kGridX = 1u << 20;
inline dim3 grid_of(long long blocks, int groups) {
  const unsigned x = blocks < kGridX ? (unsigned)blocks : kGridX;
  return dim3(x, (unsigned)groups, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ long long block_of() { return (long long)blockIdx.z * gridDim.x + blockIdx.x; }

hipError_t launch(const Args& a, bool f32, hipStream_t s);

}  // namespace rotary
}  // namespace linattn
