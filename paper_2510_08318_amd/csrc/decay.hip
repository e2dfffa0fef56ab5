// linattn_decay_fwd, linattn_decay_bwd: launches.
#include "../../include/linattn.h"
#include "decay_f32.h"
#include "decay_step.h"

namespace linattn {
namespace decay {
namespace {

// fp32 parts of dv and dk (blockIdx.z) of the query heads of a group -> their sums, in order, in the tensors' type: an order of its own, where adding
// to one sum from all heads' workgroups would have none.  Four channels a thread; 2 x 12 query heads to 2 x 4 x 4133 x 64 10.5 us (59 MB, 5.6 TB/s).
template <typename T, int D>
__global__ __launch_bounds__(256) void sum_heads_kernel(const float* parts, T* dv, T* dk, Rows r, int HK, int G, int n) {
  const long long i = (long long)blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4);
  const int c = threadIdx.x % (D / 4) * 4, b = blockIdx.y;
  if (i >= (long long)HK * n) return;
  const int h = (int)(i / n), t = (int)(i % n);
  const size_t head = (size_t)n * D;
  const float* from = parts + ((size_t)(blockIdx.z * gridDim.y + b) * HK + h) * G * head + (size_t)t * D + c;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int g = 0; g < G; ++g, from += head) {
    const float4 x = *reinterpret_cast<const float4*>(from);
    sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
  }
  T* at = (blockIdx.z ? dk : dv) + (size_t)b * r.sb + (size_t)h * r.sh + (size_t)t * r.sn + c;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
  else *reinterpret_cast<float4*>(at) = sum;
}

template <typename T, int D>
hipError_t sum_heads(const float* parts, const Args& a) {
  const int rows = 256 / (D / 4);
  sum_heads_kernel<T, D><<<dim3((unsigned)(((long long)a.HK * a.c.n + rows - 1) / rows), a.c.B, 2), 256, 0, a.stream>>>(parts, static_cast<T*>(a.dv), static_cast<T*>(a.dk), a.kr, a.HK, a.c.H / a.HK,
                                                                                                                    a.c.n);
  return hipGetLastError();
}

// The three passes of the backward, and where those of shared key heads put their parts: fp32 [dv, dk][B, H, n, d].
template <int D>
void backward_passes(const Args& a, float* parts, Pass& dq, Pass& dv, Pass& dk) {
  const int G = a.c.group;
  const Role q{a.q, a.qr, 1}, k{a.k, a.kr, G}, v{a.v, a.kr, G}, dout{a.dout, a.qr, 1};
  dq = Pass{dout, v, k, a.dq, a.qr, 0, a.state, nullptr, 1, 0, 1.f, a.scale};
  dv = Pass{k, q, dout, a.dv, a.kr, 0, a.dstate, a.dstate_in, 0, 1, a.scale, 1.f};
  dk = Pass{v, dout, q, a.dk, a.kr, 0, a.dstate, nullptr, 1, 1, a.scale, 1.f};
  if (G == 1) return;
  const size_t all = (size_t)a.c.B * a.c.H * a.c.n * D;
  dv.o = parts;
  dk.o = parts + all;
  dv.part = dk.part = 1;
  dv.orow = dk.orow = Rows{(size_t)a.c.H * a.c.n * D, (size_t)a.c.n * D, (size_t)D};
}

// Tokens up to which the recurrence is taken token by token.  Us of kernels, so / in chunks: bf16, 4 x 32 states of 128 x 128, 8 tokens 12.3 / 14.1, 16 18.7 / 14.4; 32 x 32 states, 8
// tokens 45.2 / 43.7, 16 65 / 45; fp32, 4 x 32 states, 8 12.2 / 16.8, 12 15.3 / 16.1, 16 18.1 / 17.1, 24 24.7 / 16.9; bf16 in fp32 arithmetic as fp32, with chunks that take longer.
constexpr int step_tokens(int dtype) { return dtype == LINATTN_BF16 ? 8 : dtype == LINATTN_F32 ? 12 : 16; }

struct Layout {
  Plan plan;
  size_t states, parts;     // of the workspace, in floats: all states; dv and dk of all query heads
};
Layout layout_of(int dtype, int B, int H, int HK, int n, int d, bool backward) {
  Layout r{};
  if (n > step_tokens(dtype)) {
    r.plan = plan_of(B, H, n, chunk_times(dtype == LINATTN_F32, dtype == LINATTN_BF16_F32MATH, d), d, backward ? 3 : 1, backward ? 2 : 1);
    if (r.plan.segs > 1) r.states = (size_t)r.plan.segs * (backward ? 2 : 1) * B * H * d * d;
  }
  if (backward && H != HK) r.parts = 2 * (size_t)B * H * n * d;
  return r;
}

template <auto KERNEL, typename A>
hipError_t launch(const A& args, const Common& c, const Plan& plan, int passes, int threads, size_t smem, hipStream_t s) {
  if (hipError_t e = set_smem_once<KERNEL>(smem); e != hipSuccess) return e;
  KERNEL<<<(unsigned)(c.B * c.H * plan.segs * passes), threads, smem, s>>>(args);
  return hipGetLastError();
}
// T: the tensors' type; F32: fp32 arithmetic
template <typename T, int D, bool F32>
hipError_t launch_rows(const RowArgs& r, hipStream_t s) {
  if constexpr (sizeof(T) == 4) return launch<&decay_rows_f32_kernel<D>>(r, r.c, r.plan, r.passes, 2 * D, rows_f32_lds<D>(), s);
  else {
    bool state = false;
    for (int i = 0; i < r.passes; ++i) state |= r.pass[i].p.out != nullptr && r.plan.segs == 1;
    return state ? launch<&decay_rows_kernel<D, true, F32>>(r, r.c, r.plan, r.passes, 256, rows_lds<D, F32>(), s)
                 : launch<&decay_rows_kernel<D, false, F32>>(r, r.c, r.plan, r.passes, 256, rows_lds<D, F32>(), s);
  }
}
template <typename T, int D, bool F32>
hipError_t launch_states(const SumArgs& sums, const ScanArgs& scan, hipStream_t s) {
  bool whole = F32;         // the sums have to be those of fp32
  for (int i = 0; i < scan.passes; ++i) whole |= scan.pass[i].out != nullptr;
  hipError_t e;
  if constexpr (sizeof(T) == 4) e = launch<&decay_sum_f32_kernel<D>>(sums, sums.c, sums.plan, sums.passes, 2 * D, sum_f32_lds<D>(), s);
  else {
    auto go = [&](auto pieces, auto stream) { return launch<&decay_sum_kernel<D, decltype(pieces)::value, decltype(stream)::value>>(sums, sums.c, sums.plan, sums.passes, 256, sum_lds<D>(), s); };
    // What it reads is read again by the rows kernel, from the last-level cache of 256 MB as far as it has room.  Us of both, loads that stay there / that do not: 12 x 32760 x 128 (201 MB)
    // 157 to 164 / 158 to 162, a step of 30 x 17550 x 64 (135 MB forward) 365 / 372, 40 x 75600 x 128 (1550 MB) 1009 / 983.
    const bool big = (double)sums.c.B * sums.c.n * D * 4. * (sums.passes * (sums.c.H / sums.pass[0].b.group + sums.c.H / sums.pass[0].c.group) / 2) > 256e6;
    using std::integral_constant;
    if (whole) e = big ? go(integral_constant<int, 3>{}, std::true_type{}) : go(integral_constant<int, 3>{}, std::false_type{});
    else e = big ? go(integral_constant<int, kPieces>{}, std::true_type{}) : go(integral_constant<int, kPieces>{}, std::false_type{});
  }
  if (e != hipSuccess) return e;
  decay_scan_kernel<<<dim3(D * D / 512, scan.c.B * scan.c.H, scan.passes), 256, 0, s>>>(scan);
  return hipGetLastError();
}

template <typename T, int D, bool F32>
hipError_t chunked_fwd(const Args& a) {
  const int G = a.c.group;
  const Plan plan = layout_of(a.dtype, a.c.B, a.c.H, a.HK, a.c.n, D, false).plan;
  const Role q{a.q, a.qr, 1}, k{a.k, a.kr, G}, v{a.v, a.kr, G};
  const bool states = plan.segs > 1;
  if (states) {
    const SumArgs sums{{{k, v, 0}}, 1, a.c, plan, a.work};
    const ScanArgs scan{{{a.state, a.state_out, 0, 1.f, 0}}, 1, a.c, plan, a.work, D * D};
    if (hipError_t e = launch_states<T, D, F32>(sums, scan, a.stream); e != hipSuccess) return e;
  }
  const RowArgs rows{{{Pass{q, k, v, a.o, a.qr, 0, a.state, a.state_out, 0, 0, 1.f, a.scale}, states ? a.work : nullptr, 0}}, 1, a.c, plan};
  return launch_rows<T, D, F32>(rows, a.stream);
}

template <typename T, int D, bool F32>
hipError_t chunked_bwd(const Args& a) {
  const int G = a.c.group;
  const Role q{a.q, a.qr, 1}, k{a.k, a.kr, G}, v{a.v, a.kr, G}, dout{a.dout, a.qr, 1};
  const Layout lay = layout_of(a.dtype, a.c.B, a.c.H, a.HK, a.c.n, D, true);
  const Plan& plan = lay.plan;
  const bool states = plan.segs > 1;
  const size_t one = lay.states / 2;
  float *s = states ? a.work : nullptr, *d = states ? a.work + one : nullptr;
  if (states) {
    const SumArgs sums{{{k, v, 0}, {q, dout, 1}}, 2, a.c, plan, a.work};
    const ScanArgs scan{{{a.state, nullptr, 0, 1.f, 0}, {a.dstate, a.dstate_in, 1, a.scale, 1}}, 2, a.c, plan, a.work, D * D};
    if (hipError_t e = launch_states<T, D, F32>(sums, scan, a.stream); e != hipSuccess) return e;
  }
  float* const parts = a.work + lay.states;
  RowArgs rows{{{{}, s, 0}, {{}, d, 1}, {{}, d, 1}}, 3, a.c, plan};
  backward_passes<D>(a, parts, rows.pass[0].p, rows.pass[1].p, rows.pass[2].p);
  if (hipError_t e = launch_rows<T, D, F32>(rows, a.stream); e != hipSuccess || G == 1) return e;
  return sum_heads<T, D>(parts, a);
}

template <typename T, int D, bool F32>
hipError_t fwd(const Args& a) {
  if (a.c.n > step_tokens(a.dtype)) return chunked_fwd<T, D, F32>(a);
  const int G = a.c.group;
  return launch_step<T, D>(Pass{{a.q, a.qr, 1}, {a.k, a.kr, G}, {a.v, a.kr, G}, a.o, a.qr, 0, a.state, a.state_out, 0, 0, 1.f, a.scale}, a.c, a.stream);
}

template <typename T, int D, bool F32>
hipError_t bwd(const Args& a) {
  if (a.c.n > step_tokens(a.dtype)) return chunked_bwd<T, D, F32>(a);
  Common of_items = a.c;      // dS_out and dS_in are by item
  of_items.slots = nullptr;
  of_items.states = a.c.B;
  Pass dq, dv, dk;
  backward_passes<D>(a, a.work, dq, dv, dk);
  hipError_t e = launch_step<T, D>(dq, a.c, a.stream);
  if (e == hipSuccess) e = launch_step<T, D>(dv, of_items, a.stream);
  if (e == hipSuccess) e = launch_step<T, D>(dk, of_items, a.stream);
  return e != hipSuccess || a.c.group == 1 ? e : sum_heads<T, D>(a.work, a);
}

}  // namespace

size_t work_bytes(int dtype, int B, int H, int HK, int n, int d, bool backward) {
  const Layout r = layout_of(dtype, B, H, HK, n, d, backward);
  return ((r.states + r.parts) * sizeof(float) + 255) & ~(size_t)255;
}

hipError_t launch_fwd(const Args& a) {
  if (a.dtype == LINATTN_F32) return a.d == 64 ? fwd<float, 64, true>(a) : fwd<float, 128, true>(a);
  if (a.dtype == LINATTN_BF16_F32MATH) return a.d == 64 ? fwd<uint16_t, 64, true>(a) : fwd<uint16_t, 128, true>(a);
  return a.d == 64 ? fwd<uint16_t, 64, false>(a) : fwd<uint16_t, 128, false>(a);
}
hipError_t launch_bwd(const Args& a) {
  if (a.dtype == LINATTN_F32) return a.d == 64 ? bwd<float, 64, true>(a) : bwd<float, 128, true>(a);
  if (a.dtype == LINATTN_BF16_F32MATH) return a.d == 64 ? bwd<uint16_t, 64, true>(a) : bwd<uint16_t, 128, true>(a);
  return a.d == 64 ? bwd<uint16_t, 64, false>(a) : bwd<uint16_t, 128, false>(a);
}

}  // namespace decay
}  // namespace linattn
