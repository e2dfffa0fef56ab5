// Host side of linattn_rotary and linattn_decay_*: argument checks (all of them before the first HIP call) and dispatch.
#include "../../include/linattn.h"
#include "checks.h"
#include "decay.h"
#include "rotary.h"

#include <cmath>

using namespace linattn;
using namespace linattn::checks;

namespace {

int check_tokens(int dtype, int B, int H, int HK, int n, int d, int layout) {
  if (dtype != LINATTN_BF16 && dtype != LINATTN_F32 && dtype != LINATTN_BF16_F32MATH) return LINATTN_E_DTYPE;
  if (B <= 0 || H <= 0 || HK <= 0 || n <= 0 || (d != 64 && d != 128)) return LINATTN_E_SHAPE;
  if (layout != LINATTN_LAYOUT_BHND && layout != LINATTN_LAYOUT_BNHD) return LINATTN_E_SHAPE;
  if ((long long)B * H > 65535 || (long long)B * HK > 65535 || n > decay::kMostTokens || (long long)B * (H > HK ? H : HK) * n > 1LL << 35) return LINATTN_E_SHAPE;
  return LINATTN_OK;
}
size_t tensor_bytes(int dtype, int B, int heads, int n, int d) { return (size_t)B * heads * n * d * (dtype == LINATTN_F32 ? 4 : 2); }

struct DecaySizes {
  size_t q, k, state, item_state;      // bytes of a tensor of H heads, of HK heads, of the state tensors, of one state for each item
};
int check_decay(const linattn_decay_desc* w, decay::Args* a, DecaySizes* z) {
  if (!w) return LINATTN_E_NULL;
  if (int st = check_tokens(w->dtype, w->B, w->H, w->HK, w->n, w->d, w->layout)) return st;
  if (w->H % w->HK) return LINATTN_E_SHAPE;
  if (w->slots && (w->states <= 0 || (long long)w->states * w->H > 1LL << 30)) return LINATTN_E_SHAPE;
  if (!(w->scale == 0.f || (w->scale >= 0x1p-100f && w->scale <= 0x1p100f))) return LINATTN_E_VALUE;
  if (!w->log_decay) return LINATTN_E_NULL;
  if (misaligned(w->log_decay, 4) || misaligned(w->lengths, 4) || misaligned(w->slots, 4)) return LINATTN_E_ALIGN;
  *a = decay::Args{};
  a->c = decay::Common{w->log_decay, w->lengths, w->slots, w->slots ? w->states : w->B, w->B, w->H, w->H / w->HK, w->n};
  a->HK = w->HK; a->d = w->d; a->dtype = w->dtype;
  a->qr = token_rows(w->H, w->n, w->d, w->layout == LINATTN_LAYOUT_BHND);
  a->kr = token_rows(w->HK, w->n, w->d, w->layout == LINATTN_LAYOUT_BHND);
  a->scale = w->scale == 0.f ? 1.0f / std::sqrt((float)w->d) : w->scale;
  z->q = tensor_bytes(w->dtype, w->B, w->H, w->n, w->d);
  z->k = tensor_bytes(w->dtype, w->B, w->HK, w->n, w->d);
  const size_t one = (size_t)w->H * w->d * w->d * sizeof(float);
  z->state = one * a->c.states;
  z->item_state = one * w->B;
  return LINATTN_OK;
}
// The workspace, where one is needed; `need` bytes of it.
int check_work(const linattn_decay_desc* w, size_t need) {
  if (need && (!w->workspace || w->workspace_bytes < need)) return LINATTN_E_WORKSPACE;
  return misaligned(w->workspace, 256) ? LINATTN_E_ALIGN : LINATTN_OK;
}

}  // namespace

extern "C" {

int linattn_rotary(const linattn_rotary_desc* w, const void* q, const void* k, void* q_out, void* k_out, void* stream) {
  if (!w) return LINATTN_E_NULL;
  if (int st = check_tokens(w->dtype, w->B, w->H, k ? w->HK : 1, w->n, w->d, w->layout)) return st;
  if (w->axes < 1 || w->axes > 3) return LINATTN_E_SHAPE;
  rotary::Args a{};
  int used = 0;
  const double base = w->base == 0. ? 10000. : w->base;
  if (!(base >= 1. && base <= 0x1p60) || (w->pairs != LINATTN_PAIRS_ADJACENT && w->pairs != LINATTN_PAIRS_HALVES)) return LINATTN_E_VALUE;
  for (int i = 0; i < 3; ++i) {
    a.from[i] = used;
    if (i >= w->axes) continue;
    const int size = w->dims[i];
    if (size <= 0 || size % 2 || size > w->d - used) return LINATTN_E_SHAPE;
    if (!w->positions && i > 0 && w->grid[i] <= 0) return LINATTN_E_SHAPE;
    a.first[i] = w->first[i];
    for (int m = 0; m < size / 2; ++m) a.turns[used / 2 + m] = std::pow(base, -2. * m / size) / (2. * M_PI);
    used += size;
  }
  a.from[3] = used;
  if (w->positions && w->position_items != 1 && w->position_items != w->B) return LINATTN_E_SHAPE;
  if (!q || !q_out || (k == nullptr) != (k_out == nullptr)) return LINATTN_E_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(q_out) || misaligned(k_out) || misaligned(w->positions, 4) || misaligned(w->lengths, 4)) return LINATTN_E_ALIGN;
  a.B = w->B; a.H = w->H; a.HK = k ? w->HK : 0; a.n = w->n; a.d = w->d; a.axes = w->axes;
  const size_t qb = tensor_bytes(w->dtype, a.B, a.H, a.n, a.d), kb = tensor_bytes(w->dtype, a.B, a.HK, a.n, a.d);
  const Region outs[2] = {{q_out, qb}, {k_out, kb}};
  const Region ins[4] = {{q == q_out ? nullptr : q, qb}, {k == k_out ? nullptr : k, kb},
                         {w->positions, (size_t)(w->position_items > 0 ? w->position_items : 0) * a.n * a.axes * sizeof(int)}, {w->lengths, (size_t)a.B * sizeof(int)}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  a.q = q; a.k = k; a.qo = q_out; a.ko = k_out;
  a.qr = token_rows(a.H, a.n, a.d, w->layout == LINATTN_LAYOUT_BHND);
  a.kr = token_rows(a.HK, a.n, a.d, w->layout == LINATTN_LAYOUT_BHND);
  a.halves = w->pairs == LINATTN_PAIRS_HALVES;
  a.back = w->inverse != 0;
  a.grid1 = w->grid[1]; a.grid2 = w->grid[2];
  a.positions = w->positions;
  a.item = w->position_items == 1 ? 0 : (size_t)a.n * a.axes;
  a.lengths = w->lengths;
  return rotary::launch(a, w->dtype == LINATTN_F32, static_cast<hipStream_t>(stream)) == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

size_t linattn_decay_workspace_bytes(const linattn_decay_desc* w, int backward) {
  decay::Args a;
  DecaySizes z;
  return check_decay(w, &a, &z) == LINATTN_OK ? decay::work_bytes(w->dtype, w->B, w->H, w->HK, w->n, w->d, backward != 0) : 0;
}

int linattn_decay_fwd(const linattn_decay_desc* w, const void* q, const void* k, const void* v, const float* state_in, void* out, float* state_out,
                      void* stream) {
  decay::Args a;
  DecaySizes z;
  if (int st = check_decay(w, &a, &z)) return st;
  if (!q || !k || !v || !out) return LINATTN_E_NULL;
  for (const void* p : {q, k, v, (const void*)out, (const void*)state_in, (const void*)state_out})
    if (misaligned(p)) return LINATTN_E_ALIGN;
  const size_t need = decay::work_bytes(w->dtype, w->B, w->H, w->HK, w->n, w->d, false);
  if (int st = check_work(w, need)) return st;
  const Region outs[3] = {{out, z.q}, {state_out, z.state}, {need ? w->workspace : nullptr, need}};
  const Region ins[7] = {{q, z.q}, {k, z.k}, {v, z.k}, {state_in == state_out ? nullptr : state_in, z.state}, {w->log_decay, (size_t)w->H * sizeof(float)},
                         {w->lengths, (size_t)w->B * sizeof(int)}, {w->slots, (size_t)w->B * sizeof(int)}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  a.q = q; a.k = k; a.v = v; a.o = out; a.state = state_in; a.state_out = state_out;
  a.work = need ? static_cast<float*>(w->workspace) : nullptr;
  a.stream = static_cast<hipStream_t>(stream);
  return decay::launch_fwd(a) == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

int linattn_decay_bwd(const linattn_decay_desc* w, const void* q, const void* k, const void* v, const float* state_in, const void* dout,
                      const float* dstate_out, void* dq, void* dk, void* dv, float* dstate_in, void* stream) {
  decay::Args a;
  DecaySizes z;
  if (int st = check_decay(w, &a, &z)) return st;
  if (!q || !k || !v || !dout || !dq || !dk || !dv) return LINATTN_E_NULL;
  for (const void* p : {q, k, v, dout, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)state_in, (const void*)dstate_out, (const void*)dstate_in})
    if (misaligned(p)) return LINATTN_E_ALIGN;
  const size_t need = decay::work_bytes(w->dtype, w->B, w->H, w->HK, w->n, w->d, true);
  if (int st = check_work(w, need)) return st;
  const Region outs[5] = {{dq, z.q}, {dk, z.k}, {dv, z.k}, {dstate_in, z.item_state}, {need ? w->workspace : nullptr, need}};
  const Region ins[9] = {{q, z.q}, {k, z.k}, {v, z.k}, {state_in, z.state}, {dout, z.q}, {dstate_out, z.item_state},
                         {w->log_decay, (size_t)w->H * sizeof(float)}, {w->lengths, (size_t)w->B * sizeof(int)}, {w->slots, (size_t)w->B * sizeof(int)}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  a.q = q; a.k = k; a.v = v; a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
  a.state = state_in; a.dstate = dstate_out; a.dstate_in = dstate_in;
  a.work = need ? static_cast<float*>(w->workspace) : nullptr;
  a.stream = static_cast<hipStream_t>(stream);
  return decay::launch_bwd(a) == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

}  // extern "C"
