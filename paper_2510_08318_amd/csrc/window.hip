// Softmax attention with a sliding window and first tokens: linattn_window_fwd, linattn_window_bwd.
#include "../../include/linattn.h"
#include "attn_bwd.h"
#include "attn_keys.h"
#include "attn_f32.h"

namespace linattn {
namespace attn {

template <int D, int PIECES>
static hipError_t fwd_as(const WindowArgs& a) {
  const TokenArgs keys{a.k, a.v, a.lengths, a.kr};
  const RowsArgs r{a.q, a.o, a.lse, nullptr, a.B, a.H, a.HK, a.H / a.HK, a.n, 0, 1, a.qr, a.sight, a.scale * kLog2e};
  if (PIECES == 1 && few_blocks((long long)a.B * a.HK, (long long)a.n * r.G, a.n, a.sight)) return launch_keys<D, KeysOfTokens<D>>(r, keys, a.stream);
  return launch_rows<D, 64, TokenSource<D, 64>, PIECES>(r, keys, a.stream);
}
template <int D, int PIECES>
static hipError_t bwd_as(const WindowArgs& a) {
  BwdRows r{};
  r.q = a.q; r.k = a.k; r.v = a.v; r.out = a.out; r.dout = a.dout; r.dq = a.dq; r.dk = a.dk; r.dv = a.dv;
  r.lse = a.lse; r.nl = a.nl; r.nd = a.nd; r.parts = a.parts;
  r.lengths = a.lengths; r.B = a.B; r.H = a.H; r.HK = a.HK; r.G = a.H / a.HK; r.n = a.n;
  r.qr = a.qr; r.kr = a.kr; r.sight = a.sight; r.scale = a.scale; r.scale2 = a.scale * kLog2e;
  return launch_bwd_rows<D, PIECES>(r, a.stream);
}

hipError_t launch_window_fwd(const WindowArgs& a, int dtype) {
  if (dtype == LINATTN_F32) return a.d == 64 ? launch_fwd_f32<64>(a) : launch_fwd_f32<128>(a);
  if (dtype == LINATTN_BF16_F32MATH) return a.d == 64 ? fwd_as<64, 3>(a) : fwd_as<128, 3>(a);
  return a.d == 64 ? fwd_as<64, 1>(a) : fwd_as<128, 1>(a);
}
hipError_t launch_window_bwd(const WindowArgs& a, int dtype) {
  if (dtype == LINATTN_F32) return a.d == 64 ? launch_bwd_f32<64>(a) : launch_bwd_f32<128>(a);
  if (dtype == LINATTN_BF16_F32MATH) return a.d == 64 ? bwd_as<64, 3>(a) : bwd_as<128, 3>(a);
  return a.d == 64 ? bwd_as<64, 1>(a) : bwd_as<128, 1>(a);
}

}  // namespace attn
}  // namespace linattn
