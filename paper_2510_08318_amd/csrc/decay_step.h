// The recurrence of decay.h token by token, in fp32: the state's elements stay in registers.  For few tokens, where a call reads and writes its states
// and little else: 64 sequences of 32 states of 128 x 128 (270 MB) take 57 us at one token, 4.7 TB/s, the rate of a copy; 12 states of 64 x 64 3.8, of which a launch is 3.
// The backward's turned passes read a state by columns, 64 bytes of a row to a thread: dq or dk of 64 x 32 states (134 MB read) 82 us at one token, where dv, which reads and writes as many,
// takes 55; at 8 tokens 106 and 78.
#pragma once
#include "decay.h"
#include "f32_plain.h"

namespace linattn {
namespace decay {

// N adjacent values, 4 bytes at least
template <int N, typename T>
__device__ __forceinline__ void load_run(const T* p, float (&f)[N]) {
  constexpr int BYTES = N * (int)sizeof(T);
  uint32_t w[BYTES / 4];
  if constexpr (BYTES >= 16) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const uint4 x = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
  } else if constexpr (BYTES == 8) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  } else w[0] = *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
  for (int i = 0; i < BYTES / 4; ++i) {
    if constexpr (sizeof(T) == 4) f[i] = __builtin_bit_cast(float, w[i]);
    else { f[2 * i] = f32::lo_f32(w[i]); f[2 * i + 1] = f32::hi_f32(w[i]); }
  }
}

// A workgroup has COLS columns of a state: a thread four of them, in ROWS rows.  The rows' products are summed over the lanes that share columns, then over the
// four wavefronts through LDS.
template <typename T, int D, int COLS>
__global__ __launch_bounds__(256) void decay_step_kernel(Pass p, Common com) {
  constexpr int CG = COLS / 4, RG = 256 / CG, ROWS = D / RG;
  __shared__ __align__(16) float red[2][4][COLS];
  const int tid = threadIdx.x, lane = tid % 64, w = tid / 64, cg = tid % CG, f0 = tid / CG * ROWS;
  const int h = blockIdx.x / (D / COLS), c0 = blockIdx.x % (D / COLS) * COLS, b = blockIdx.y;
  const int len = length_of(com, b);
  const long long at = state_row(com, b, h);
  const float lambda = expf(log_decay_of(com, h));
  const T* pa = static_cast<const T*>(p.a.p) + (size_t)b * p.a.r.sb + (size_t)(h / p.a.group) * p.a.r.sh + f0;
  const T* pb = static_cast<const T*>(p.b.p) + (size_t)b * p.b.r.sb + (size_t)(h / p.b.group) * p.b.r.sh + f0;
  const T* pc = static_cast<const T*>(p.c.p) + (size_t)b * p.c.r.sb + (size_t)(h / p.c.group) * p.c.r.sh + c0 + 4 * cg;
  const size_t po = (size_t)b * p.orow.sb + (size_t)h * p.orow.sh + c0;
  auto put = [&](int t, float v) {
    const size_t i = po + (size_t)t * p.orow.sn + tid;
    if (p.part) static_cast<float*>(p.o)[i] = v;
    else f32::stf(static_cast<T*>(p.o), i, v);
  };

  float s[ROWS][4];
  if (p.in && at >= 0) {
    const float* in = p.in + at * D * D;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (p.turned) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = in[(c0 + 4 * cg + e) * D + f0 + i];
      } else {
        const float4 x = *reinterpret_cast<const float4*>(in + (f0 + i) * D + c0 + 4 * cg);
        s[i][0] = x.x; s[i][1] = x.y; s[i][2] = x.z; s[i][3] = x.w;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = 0.f;
  }

  for (int i = 0; i < len; ++i) {
    const int t = p.back ? len - 1 - i : i;
    float fa[ROWS], fb[ROWS], fc[4], o[4] = {0.f, 0.f, 0.f, 0.f};
    load_run<ROWS>(pa + (size_t)t * p.a.r.sn, fa);
    load_run<ROWS>(pb + (size_t)t * p.b.r.sn, fb);
    load_run<4>(pc + (size_t)t * p.c.r.sn, fc);
    const float decay = p.back && i == 0 ? 1.f : lambda;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[r][e] = fmaf(s[r][e], decay, p.in_scale * fb[r] * fc[e]);
        o[e] = fmaf(fa[r], s[r][e], o[e]);
      }
#pragma unroll
    for (int x = CG; x < 64; x *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x);
    if (lane < CG) *reinterpret_cast<float4*>(&red[i % 2][w][4 * cg]) = make_float4(o[0], o[1], o[2], o[3]);
    __syncthreads();
    if (tid < COLS) put(t, p.out_scale * ((red[i % 2][0][tid] + red[i % 2][1][tid]) + (red[i % 2][2][tid] + red[i % 2][3][tid])));
  }
  for (int t = len; t < com.n; ++t)
    if (tid < COLS) put(t, 0.f);

  if (p.out && at >= 0) {
    const float last = p.back && len > 0 ? lambda : 1.f;
    float* out = p.out + at * D * D;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      *reinterpret_cast<float4*>(out + (f0 + i) * D + c0 + 4 * cg) = make_float4(s[i][0] * last, s[i][1] * last, s[i][2] * last, s[i][3] * last);
  }
}

// Whole states, whose reads and writes are the longest runs, where that gives every compute unit two; else 32 columns to a workgroup.
template <typename T, int D>
hipError_t launch_step(const Pass& p, const Common& c, hipStream_t s) {
  if ((long long)c.B * c.H >= 2 * kCUs) decay_step_kernel<T, D, D><<<dim3(c.H, c.B), 256, 0, s>>>(p, c);
  else decay_step_kernel<T, D, 32><<<dim3(c.H * (D / 32), c.B), 256, 0, s>>>(p, c);
  return hipGetLastError();
}

}  // namespace decay
}  // namespace linattn
