// Host side of linattn_window_* and linattn_cache_*: argument checks (all of them before the first HIP call) and dispatch.
#include "../../include/linattn.h"
#include "attn.h"
#include "checks.h"

#include <cmath>

namespace linattn {
namespace attn {
namespace {

using namespace checks;

Rows rows_of(int H, int n, int d, int layout) { return token_rows(H, n, d, layout == LINATTN_LAYOUT_BHND); }

int check_sight(const linattn_sight& s, int d, Sight* sight, float* scale) {
  // (the backward starts its scores from -lse / scale)
  if (s.sinks < 0 || !(s.scale == 0.f || (s.scale >= 0x1p-100f && s.scale <= 0x1p100f))) return LINATTN_E_VALUE;
  sight->left = s.left < 0 || s.left >= kMostTokens ? -1 : s.left;
  sight->right = s.right < 0 || s.right >= kMostTokens ? -1 : s.right;
  sight->sinks = s.sinks < kMostTokens ? s.sinks : kMostTokens;
  *scale = s.scale == 0.f ? 1.0f / std::sqrt((float)d) : s.scale;
  return LINATTN_OK;
}

int check_heads(int B, int H, int HK, int n, int d, int layout) {
  if (B <= 0 || H <= 0 || HK <= 0 || n <= 0 || H % HK) return LINATTN_E_SHAPE;
  if (d != 64 && d != 128) return LINATTN_E_SHAPE;
  if (layout != LINATTN_LAYOUT_BHND && layout != LINATTN_LAYOUT_BNHD) return LINATTN_E_SHAPE;
  if ((long long)B * H > 65535 || (long long)n * (H / HK) > kMostTokens || (long long)B * H * n > 1LL << 35) return LINATTN_E_SHAPE;
  return LINATTN_OK;
}

struct WindowSizes {
  size_t q, k, lse, parts, work;      // bytes of a tensor of H heads, of HK heads, of lse; where the parts start in the workspace, its size
};
int check_window(const linattn_window_desc* w, WindowArgs* a, WindowSizes* z) {
  if (!w) return LINATTN_E_NULL;
  if (w->dtype != LINATTN_BF16 && w->dtype != LINATTN_F32 && w->dtype != LINATTN_BF16_F32MATH) return LINATTN_E_DTYPE;
  if (int st = check_heads(w->B, w->H, w->HK, w->n, w->d, w->layout)) return st;
  *a = WindowArgs{};
  if (int st = check_sight(w->sight, w->d, &a->sight, &a->scale)) return st;
  if (misaligned(w->lengths, 4)) return LINATTN_E_ALIGN;
  a->lengths = w->lengths;
  a->B = w->B; a->H = w->H; a->HK = w->HK; a->n = w->n; a->d = w->d;
  a->qr = rows_of(w->H, w->n, w->d, w->layout);
  a->kr = rows_of(w->HK, w->n, w->d, w->layout);
  const size_t esz = w->dtype == LINATTN_F32 ? 4 : 2;
  z->q = (size_t)w->B * w->H * w->n * w->d * esz;
  z->k = (size_t)w->B * w->HK * w->n * w->d * esz;
  z->lse = (size_t)w->B * w->H * w->n * sizeof(float);
  z->parts = (2 * z->lse + 255) & ~(size_t)255;
  z->work = z->parts;
  if (w->dtype == LINATTN_F32) {
    const long long blocks = (w->n + 31) / 32;
    const size_t q = (size_t)f32_shares(blocks * w->B * w->H) * w->B * w->H * (w->d + 2), k = (size_t)f32_shares(blocks * w->B * w->HK) * w->B * w->HK * 2 * w->d;
    if (f32_shares(blocks * w->B * w->HK) > 1) z->work += (((q > k ? q : k) * w->n * sizeof(float)) + 255) & ~(size_t)255;
  } else z->work += (size_t)key_split(w->B * w->HK, w->H / w->HK, w->n, w->d, a->sight).parts * 2 * key_block(w->d) * w->d * sizeof(float);
  return LINATTN_OK;
}

struct CacheSizes {
  size_t pool, exps;           // bytes of the k (or v) rows, of their exponents
};
int check_cache(const linattn_cache_desc* c, int n, Pool* p, CacheSizes* z) {
  if (!c) return LINATTN_E_NULL;
  if (c->type != LINATTN_CACHE_BF16 && c->type != LINATTN_CACHE_E4M3) return LINATTN_E_DTYPE;
  if (int st = check_heads(c->B, c->H, c->H, n, c->d, c->layout)) return st;
  if (c->page <= 0 || c->pages <= 0 || c->width <= 0 || (long long)c->page * c->width > kMostTokens) return LINATTN_E_SHAPE;
  if (!c->k || !c->v || !c->table || !c->lengths) return LINATTN_E_NULL;
  const bool e4m3 = c->type == LINATTN_CACHE_E4M3;
  if (e4m3 && (!c->k_exp || !c->v_exp)) return LINATTN_E_NULL;
  if (misaligned(c->k) || misaligned(c->v) || misaligned(c->table, 4) || misaligned(c->lengths, 4) || misaligned(c->counts, 4)) return LINATTN_E_ALIGN;
  const size_t rows = (size_t)c->pages * c->H;
  if (rows > ((size_t)1 << 40) / c->page) return LINATTN_E_SHAPE;
  z->exps = e4m3 ? rows * c->page : 0;
  z->pool = rows * c->page * c->d * (e4m3 ? 1 : 2);
  *p = Pool{c->k, c->v, c->k_exp, c->v_exp, c->table, c->lengths, c->counts, c->B, c->H, c->d, c->page, c->pages, c->width, 0, 0};
  set_divisor(p);
  const Region outs[4] = {{c->k, z->pool}, {c->v, z->pool}, {e4m3 ? c->k_exp : nullptr, z->exps}, {e4m3 ? c->v_exp : nullptr, z->exps}};
  const Region none[1] = {{nullptr, 0}};
  return any_overlap(outs, none) ? LINATTN_E_ALIAS : LINATTN_OK;
}

size_t attn_work_bytes(const linattn_cache_desc* c, int H, int n) {
  const int splits = cache_splits(c->B, H, c->H, n, c->d, c->type == LINATTN_CACHE_E4M3, (long long)c->page * c->width).splits;
  return splits > 1 ? ((size_t)splits * c->B * H * n * (c->d + 2) * sizeof(float) + 255) & ~(size_t)255 : 0;
}

}  // namespace
}  // namespace attn
}  // namespace linattn

using namespace linattn;
using namespace linattn::attn;
using namespace linattn::checks;

extern "C" {

size_t linattn_window_workspace_bytes(const linattn_window_desc* w) {
  WindowArgs a;
  WindowSizes z;
  return check_window(w, &a, &z) == LINATTN_OK ? z.work : 0;
}

int linattn_window_fwd(const linattn_window_desc* w, const void* q, const void* k, const void* v, void* out, float* lse, void* stream) {
  WindowArgs a;
  WindowSizes z;
  if (int st = check_window(w, &a, &z)) return st;
  if (!q || !k || !v || !out) return LINATTN_E_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(lse, 4)) return LINATTN_E_ALIGN;
  const Region outs[2] = {{out, z.q}, {lse, z.lse}}, ins[3] = {{q, z.q}, {k, z.k}, {v, z.k}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  if (w->workspace) {
    if (misaligned(w->workspace, 256)) return LINATTN_E_ALIGN;
    if (w->workspace_bytes < z.work) return LINATTN_E_WORKSPACE;
    const Region work[1] = {{w->workspace, z.work}}, tensors[5] = {{q, z.q}, {k, z.k}, {v, z.k}, {out, z.q}, {lse, z.lse}};
    if (any_overlap(work, tensors)) return LINATTN_E_ALIAS;
    a.parts = z.work > z.parts ? reinterpret_cast<float*>(static_cast<char*>(w->workspace) + z.parts) : nullptr;
  }
  a.q = q; a.k = k; a.v = v; a.o = out; a.lse = lse;
  a.stream = static_cast<hipStream_t>(stream);
  return launch_window_fwd(a, w->dtype) == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

int linattn_window_bwd(const linattn_window_desc* w, const void* q, const void* k, const void* v, const void* out, const float* lse,
                       const void* dout, void* dq, void* dk, void* dv, void* stream) {
  WindowArgs a;
  WindowSizes z;
  if (int st = check_window(w, &a, &z)) return st;
  if (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv) return LINATTN_E_NULL;
  for (const void* p : {q, k, v, out, dout, (const void*)dq, (const void*)dk, (const void*)dv})
    if (misaligned(p)) return LINATTN_E_ALIGN;
  if (misaligned(lse, 4)) return LINATTN_E_ALIGN;
  if (!w->workspace || w->workspace_bytes < z.work) return LINATTN_E_WORKSPACE;
  if (misaligned(w->workspace, 256)) return LINATTN_E_ALIGN;
  const Region outs[4] = {{dq, z.q}, {dk, z.k}, {dv, z.k}, {w->workspace, z.work}};
  const Region ins[6] = {{q, z.q}, {k, z.k}, {v, z.k}, {out, z.q}, {dout, z.q}, {lse, z.lse}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  a.q = q; a.k = k; a.v = v; a.out = out; a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
  a.lse = const_cast<float*>(lse);
  a.nl = static_cast<float*>(w->workspace);
  a.nd = a.nl + (size_t)w->B * w->H * w->n;
  a.parts = z.work > z.parts ? reinterpret_cast<float*>(static_cast<char*>(w->workspace) + z.parts) : nullptr;
  a.stream = static_cast<hipStream_t>(stream);
  return launch_window_bwd(a, w->dtype) == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

int linattn_cache_write(const linattn_cache_desc* c, const void* k, const void* v, int n, void* stream) {
  Pool p;
  CacheSizes z;
  if (int st = check_cache(c, n, &p, &z)) return st;
  if (!k || !v) return LINATTN_E_NULL;
  if (misaligned(k) || misaligned(v)) return LINATTN_E_ALIGN;
  const size_t bytes = (size_t)c->B * c->H * n * c->d * 2;
  for (const void* in : {k, v})
    for (const Region& r : {Region{c->k, z.pool}, Region{c->v, z.pool}, Region{c->k_exp, z.exps}, Region{c->v_exp, z.exps}})
      if (overlaps(in, bytes, r.p, r.bytes)) return LINATTN_E_ALIAS;
  const hipError_t e = launch_cache_write(p, c->type == LINATTN_CACHE_E4M3, k, v, n, rows_of(c->H, n, c->d, c->layout), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

int linattn_cache_read(const linattn_cache_desc* c, void* k, void* v, int n, void* stream) {
  Pool p;
  CacheSizes z;
  if (int st = check_cache(c, n, &p, &z)) return st;
  if (!k || !v) return LINATTN_E_NULL;
  if (misaligned(k) || misaligned(v)) return LINATTN_E_ALIGN;
  const size_t bytes = (size_t)c->B * c->H * n * c->d * 2;
  const Region outs[2] = {{k, bytes}, {v, bytes}};
  const Region ins[4] = {{c->k, z.pool}, {c->v, z.pool}, {c->k_exp, z.exps}, {c->v_exp, z.exps}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  const hipError_t e = launch_cache_read(p, c->type == LINATTN_CACHE_E4M3, k, v, n, rows_of(c->H, n, c->d, c->layout), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

size_t linattn_cache_workspace_bytes(const linattn_cache_desc* c, int H, int n) {
  Pool p;
  CacheSizes z;
  if (check_cache(c, n, &p, &z) || check_heads(c->B, H, c->H, n, c->d, c->layout)) return 0;
  return attn_work_bytes(c, H, n);
}

int linattn_cache_attn(const linattn_cache_desc* c, const linattn_sight* sight, const void* q, void* out, float* lse, int H, int n,
                       void* workspace, size_t workspace_bytes, void* stream) {
  CacheArgs a{};
  CacheSizes z;
  if (!sight) return LINATTN_E_NULL;
  if (int st = check_cache(c, n, &a.pool, &z)) return st;
  if (int st = check_heads(c->B, H, c->H, n, c->d, c->layout)) return st;
  if (int st = check_sight(*sight, c->d, &a.sight, &a.scale)) return st;
  if (!q || !out) return LINATTN_E_NULL;
  if (misaligned(q) || misaligned(out) || misaligned(lse, 4)) return LINATTN_E_ALIGN;
  const size_t need = attn_work_bytes(c, H, n);
  if (need && (!workspace || workspace_bytes < need)) return LINATTN_E_WORKSPACE;
  if (misaligned(workspace, 256)) return LINATTN_E_ALIGN;
  const size_t bytes = (size_t)c->B * H * n * c->d * 2;
  const Region outs[3] = {{out, bytes}, {lse, (size_t)c->B * H * n * sizeof(float)}, {need ? workspace : nullptr, need}};
  const Region ins[5] = {{q, bytes}, {c->k, z.pool}, {c->v, z.pool}, {c->k_exp, z.exps}, {c->v_exp, z.exps}};
  if (any_overlap(outs, ins)) return LINATTN_E_ALIAS;
  a.q = q; a.o = out; a.lse = lse; a.work = static_cast<float*>(workspace);
  a.H = H; a.n = n; a.qr = rows_of(H, n, c->d, c->layout);
  a.stream = static_cast<hipStream_t>(stream);
  return launch_cache_attn(a, c->type == LINATTN_CACHE_E4M3) == hipSuccess ? LINATTN_OK : LINATTN_E_HIP;
}

}  // extern "C"
