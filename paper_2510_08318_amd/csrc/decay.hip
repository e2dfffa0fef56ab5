// linattn_decay_fwd, linattn_decay_bwd: launches.
#include "../../include/linattn.h"
#include "decay_step.h"

namespace linattn {
namespace decay {
namespace {

// fp32 parts of dk (or dv) of the query heads of a group -> their sum, in order, in the tensor's type.  Four channels a thread.
template <typename T, int D>
__global__ __launch_bounds__(256) void sum_heads_kernel(const float* parts, T* to, Rows r, int HK, int G, int n) {
  const long long i = (long long)blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4);
  const int c = threadIdx.x % (D / 4) * 4, b = blockIdx.y;
  if (i >= (long long)HK * n) return;
  const int h = (int)(i / n), t = (int)(i % n);
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int g = 0; g < G; ++g) {
    const float4 x = *reinterpret_cast<const float4*>(parts + (((size_t)b * HK * G + (size_t)h * G + g) * n + t) * D + c);
    sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
  }
  T* at = to + (size_t)b * r.sb + (size_t)h * r.sh + (size_t)t * r.sn + c;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
  else *reinterpret_cast<float4*>(at) = sum;
}

template <typename T, int D>
hipError_t fwd(const Args& a) {
  const int G = a.c.H / a.HK;
  Pass p{{a.q, a.qr, 1}, {a.k, a.kr, G}, {a.v, a.kr, G}, a.o, a.qr, a.state, a.state_out, 0, 0, 1.f, a.scale};
  return launch_step<T, T, D>(p, a.c, a.stream);
}

template <typename T, int D>
hipError_t bwd(const Args& a) {
  const int G = a.c.H / a.HK;
  const Role q{a.q, a.qr, 1}, k{a.k, a.kr, G}, v{a.v, a.kr, G}, dout{a.dout, a.qr, 1};
  Common of_items = a.c;      // dS_out and dS_in are by item
  of_items.slots = nullptr;
  of_items.states = a.c.B;
  hipError_t e = launch_step<T, T, D>(Pass{dout, v, k, a.dq, a.qr, a.state, nullptr, 1, 0, 1.f, a.scale}, a.c, a.stream);
  if (e != hipSuccess) return e;
  Pass dv{k, q, dout, a.dv, a.kr, a.dstate, a.dstate_in, 0, 1, a.scale, 1.f}, dk{v, dout, q, a.dk, a.kr, a.dstate, nullptr, 1, 1, a.scale, 1.f};
  if (G == 1) {
    e = launch_step<T, T, D>(dv, of_items, a.stream);
    return e != hipSuccess ? e : launch_step<T, T, D>(dk, of_items, a.stream);
  }
  const Rows parts{(size_t)a.c.H * a.c.n * D, (size_t)a.c.n * D, (size_t)D};
  for (Pass* p : {&dv, &dk}) {
    T* to = static_cast<T*>(p->o);
    p->o = a.work;
    p->orow = parts;
    e = launch_step<T, float, D>(*p, of_items, a.stream);
    if (e != hipSuccess) return e;
    const int rows = 256 / (D / 4);
    sum_heads_kernel<T, D><<<dim3((unsigned)(((long long)a.HK * a.c.n + rows - 1) / rows), a.c.B), 256, 0, a.stream>>>(a.work, to, a.kr, a.HK, G, a.c.n);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return e;
}

}  // namespace

size_t work_bytes(int, int B, int H, int HK, int n, int d, bool backward) {
  return backward && H != HK ? ((size_t)B * H * n * d * sizeof(float) + 255) & ~(size_t)255 : 0;
}

hipError_t launch_fwd(const Args& a) {
  if (a.dtype == LINATTN_F32) return a.d == 64 ? fwd<float, 64>(a) : fwd<float, 128>(a);
  return a.d == 64 ? fwd<uint16_t, 64>(a) : fwd<uint16_t, 128>(a);
}
hipError_t launch_bwd(const Args& a) {
  if (a.dtype == LINATTN_F32) return a.d == 64 ? bwd<float, 64>(a) : bwd<float, 128>(a);
  return a.d == 64 ? bwd<uint16_t, 64>(a) : bwd<uint16_t, 128>(a);
}

}  // namespace decay
}  // namespace linattn
