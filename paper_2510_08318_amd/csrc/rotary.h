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

hipError_t launch(const Args& a, bool f32, hipStream_t s);

}  // namespace rotary
}  // namespace linattn
