"""PyTorch as plumbing: device buffers and the current stream for the C-ABI calls.

Nothing of the operator is computed here; `Layer` owns the buffers a converted attention layer
needs (W~_q, W~_k, state, workspace), registers them as a phi descriptor and forwards to
linattn_fwd / linattn_bwd.  `window_attention`, `window_attention_backward` and `PagedCache` do the same for the softmax branch.
"""
from __future__ import annotations

import functools

import numpy as np
import torch

from . import binding as B_


# The handle without the Stream object that torch.cuda.current_stream() makes for it, 2.8 us of a forward call of 13.5 (the handle alone 0.2).  The
# function is torch's own and not documented: without it, the Stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _current_stream() -> int:
    """Handle of the current device's current stream."""
    return _raw_stream(torch.cuda.current_device())


def to_device(stored: np.ndarray, device="cuda") -> torch.Tensor:
    """Stored numpy tensor (float32, or uint16 bf16 bit patterns) -> device tensor of that dtype."""
    if stored.dtype == np.uint16:
        return torch.from_numpy(stored.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(stored, dtype=np.float32)).to(device)


def to_host_f64(t: torch.Tensor) -> np.ndarray:
    """Device tensor -> fp64 numpy (exact widening)."""
    return t.detach().to("cpu").to(torch.float64).numpy()


class ReluLayer:
    """Buffers + descriptor of one linear-attention layer with the weight-free map phi(x) = max(x, 0)
    (the "ReLU" row of the paper's ablation of kernel functions)."""

    def __init__(self, H: int, d: int, B: int, n: int, dtype: torch.dtype, *, layout: str = "bhnd", device="cuda",
                 f32_math: bool = False):
        assert layout in ("bhnd", "bnhd") and dtype in (torch.bfloat16, torch.float32)
        self.layout, self.H, self.d, self.B, self.n, self.tdtype = layout, H, d, B, n, dtype
        self.dtype = (B_.BF16_F32MATH if f32_math else B_.BF16) if dtype == torch.bfloat16 else B_.F32
        self.state = torch.empty((B, H, d + 1, d), dtype=torch.float32, device=device)
        self.workspace_bytes = B_.linattn_workspace_bytes(B, H, n, d, B_.PHI_RELU, self.dtype)
        if self.workspace_bytes == 0:
            raise ValueError("unsupported shape")
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
        assert self.workspace.data_ptr() % 256 == 0
        self.phi_id = B_.linattn_phi_create(B_.PHI_RELU, self.dtype, H, d, None, None, None, None, self.state,
                                            self.workspace, self.workspace_bytes,
                                            B_.LAYOUT_BNHD if layout == "bnhd" else B_.LAYOUT_BHND)

    def close(self):
        if self.phi_id is not None:
            B_.linattn_phi_destroy(self.phi_id)
            self.phi_id = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, *ts):
        shape = (self.B, self.n, self.H, self.d) if self.layout == "bnhd" else (self.B, self.H, self.n, self.d)
        for t in ts:
            assert t.is_cuda and t.is_contiguous() and t.dtype == self.tdtype and tuple(t.shape) == shape

    def forward(self, q, k, v, out=None):
        self._check(q, k, v)
        out = torch.empty_like(q) if out is None else out
        B_.linattn_fwd(q, k, v, out, self.B, self.H, self.n, self.d, self.phi_id, _current_stream())
        return out

    def backward(self, q, k, v, dout, dq=None, dk=None, dv=None):
        self._check(q, k, v, dout)
        dq = torch.empty_like(q) if dq is None else dq
        dk = torch.empty_like(q) if dk is None else dk
        dv = torch.empty_like(q) if dv is None else dv
        B_.linattn_bwd(q, k, v, dout, dq, dk, dv, self.B, self.H, self.n, self.d, self.phi_id, _current_stream())
        return dq, dk, dv


class Layer:
    """Buffers + descriptor of one linear-attention layer (Eq. 3 with the map of Eq. 5)."""

    def __init__(self, wq: torch.Tensor, wk: torch.Tensor, B: int, n: int, *, keep_state: bool = True,
                 want_wgrads: bool = False, layout: str = "bhnd", f32_math: bool = False, centred: bool = False):
        """layout "bhnd": q, k, v, out are [B, H, n, d]; "bnhd": [B, n, H, d] (heads interleaved per token).
        want_wgrads: False, True (both dW~_q and dW~_k), or "q" / "k" for one of them.
        f32_math (bf16 tensors only): fp32 arithmetic on the bf16 tensors (LINATTN_BF16_F32MATH).
        centred (bf16 matrix-core path only): LINATTN_FLAG_CENTRED."""
        assert layout in ("bhnd", "bnhd")
        self.layout = layout
        assert wq.is_cuda and wk.is_cuda and wq.dtype == wk.dtype and wq.shape == wk.shape
        self.H, self.d, half = wq.shape
        assert half * 2 == self.d
        self.dtype = (B_.BF16_F32MATH if f32_math else B_.BF16) if wq.dtype == torch.bfloat16 else B_.F32
        assert wq.dtype in (torch.bfloat16, torch.float32)
        self.wq, self.wk = wq.contiguous(), wk.contiguous()
        self.B, self.n = B, n
        dev = wq.device
        self.state = torch.empty((B, self.H, self.d + 1, self.d), dtype=torch.float32, device=dev) if keep_state else None
        assert want_wgrads in (False, True, "q", "k")
        self.dwq = torch.empty((self.H, self.d, half), dtype=torch.float32, device=dev) if want_wgrads in (True, "q") else None
        self.dwk = torch.empty((self.H, self.d, half), dtype=torch.float32, device=dev) if want_wgrads in (True, "k") else None
        size_fn = B_.linattn_workspace_bytes_wgrads if want_wgrads else B_.linattn_workspace_bytes
        self.workspace_bytes = size_fn(B, self.H, n, self.d, B_.PHI_HEDGEHOG, self.dtype)
        if self.workspace_bytes == 0:
            raise ValueError("unsupported shape")
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=dev)
        assert self.workspace.data_ptr() % 256 == 0
        self.phi_id = B_.linattn_phi_create(B_.PHI_HEDGEHOG, self.dtype, self.H, self.d, self.wq, self.wk,
                                            self.dwq, self.dwk, self.state, self.workspace, self.workspace_bytes,
                                            B_.LAYOUT_BNHD if layout == "bnhd" else B_.LAYOUT_BHND,
                                            flags=B_.FLAG_CENTRED if centred else 0)

    def set_blend(self, s=None, r=None, dr=None):
        """Mixed attention (Eq. 6): s = softmax-branch output (dtype and layout of out), r = device fp32[1],
        dr = optional device fp32[1] receiving dL/dr in backward.  All None switches it off."""
        if s is not None:
            assert s.is_cuda and s.is_contiguous() and s.dtype == self.wq.dtype
            assert r.is_cuda and r.dtype == torch.float32 and r.numel() == 1
            assert dr is None or (dr.is_cuda and dr.dtype == torch.float32 and dr.numel() == 1)
        self._blend = (s, r, dr)          # keep the buffers alive
        B_.linattn_phi_set_blend(self.phi_id, s, r, dr)

    def close(self):
        if self.phi_id is not None:
            B_.linattn_phi_destroy(self.phi_id)
            self.phi_id = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _dims(self, t):
        if self.layout == "bnhd":
            Bq, n, H, d = t.shape
        else:
            Bq, H, n, d = t.shape
        assert (Bq, H, n, d) == (self.B, self.H, self.n, self.d)
        return Bq, H, n, d

    def forward(self, q, k, v, out=None):
        Bq, H, n, d = self._dims(q)
        for t in (q, k, v):
            assert t.is_cuda and t.is_contiguous() and t.dtype == self.wq.dtype and t.shape == q.shape
        if out is None:
            out = torch.empty_like(q)
        B_.linattn_fwd(q, k, v, out, Bq, H, n, d, self.phi_id, _current_stream())
        return out

    def backward(self, q, k, v, dout, dq=None, dk=None, dv=None):
        Bq, H, n, d = self._dims(q)
        for t in (q, k, v, dout):
            assert t.is_cuda and t.is_contiguous() and t.dtype == self.wq.dtype and t.shape == q.shape
        dq = torch.empty_like(q) if dq is None else dq
        dk = torch.empty_like(q) if dk is None else dk
        dv = torch.empty_like(q) if dv is None else dv
        B_.linattn_bwd(q, k, v, dout, dq, dk, dv, Bq, H, n, d, self.phi_id, _current_stream())
        return dq, dk, dv


# ---- softmax attention: a sliding window with first tokens that stay visible, and a paged cache ---------------------------
# Scratch memory comes from torch's allocator call by call, so that calls on several streams, or captured into several graphs, share none.


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


@functools.lru_cache(maxsize=None)
def _one_device() -> bool:
    return torch.cuda.device_count() == 1


def _on_device_of(fn):
    """Runs `fn` with the device of its first argument (a cache, or the tensor q) current: the library launches on the current device."""
    @functools.wraps(fn)
    def call(*args, **kw):
        first = args[0] if args else kw.get("q")
        index = first.index if isinstance(first, PagedCache) else first.get_device() if isinstance(first, torch.Tensor) else -1
        _need(index >= 0, "q: a tensor on the GPU")
        if _one_device() or index == torch.cuda.current_device():
            return fn(*args, **kw)
        with torch.cuda.device(index):
            return fn(*args, **kw)
    return call


def _check_tokens(name, t, shape, dtype, index):
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {tuple(shape)} on GPU {index}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")


def _check_ints(name, t, shape, index):
    if t is not None:
        _check_tokens(name, t, shape, torch.int32, index)


def _token_dims(t, layout):
    """(B, heads, n, d) of a token tensor."""
    _need(layout in ("bhnd", "bnhd"), "layout is 'bhnd' or 'bnhd'")
    _need(t.dim() == 4, "expected four dimensions")
    B, x, y, d = t.shape
    return (B, y, x, d) if layout == "bnhd" else (B, x, y, d)


def _token_shape(B, heads, n, d, layout):
    return (B, n, heads, d) if layout == "bnhd" else (B, heads, n, d)


def _window_desc(q, k, v, left, right, sinks, scale, layout, lengths, f32_math):
    B, H, n, d = _token_dims(q, layout)
    HK = _token_dims(k, layout)[1]
    _need(q.dtype in (torch.bfloat16, torch.float32), "bf16 or fp32 tensors")
    index, shape = q.get_device(), _token_shape(B, HK, n, d, layout)
    _check_tokens("q", q, q.shape, q.dtype, index)
    _check_tokens("k", k, shape, q.dtype, index)
    _check_tokens("v", v, shape, q.dtype, index)
    _check_ints("lengths", lengths, (B,), index)
    dtype = (B_.BF16_F32MATH if f32_math else B_.BF16) if q.dtype == torch.bfloat16 else B_.F32
    return B_.WindowDesc(dtype, B, H, HK, n, d, B_.LAYOUT_BNHD if layout == "bnhd" else B_.LAYOUT_BHND,
                         B_.Sight(left, right, sinks, scale), B_._ptr(lengths), None, 0)


def _workspace(desc, q):
    size = B_.linattn_window_workspace_bytes(desc)
    work = q.new_empty(size, dtype=torch.uint8)
    desc.workspace, desc.workspace_bytes = B_._ptr(work), size
    return work


def _lse(q, lse, shape):
    if lse is None:
        return q.new_empty(shape, dtype=torch.float32)
    _check_tokens("lse", lse, shape, torch.float32, q.get_device())
    return lse


@_on_device_of
def window_attention(q, k, v, *, left=-1, right=-1, sinks=0, scale=0.0, layout="bhnd", lengths=None, f32_math=False, out=None, lse=None):
    """Softmax attention in which token i sees tokens i - left .. i + right and the first `sinks` tokens (up to i + right); a negative
    limit is none, right=0 is causal.  q [B, H, n, d] ("bhnd") or [B, n, H, d] ("bnhd"); k, v with H or a divisor of H heads.
    lengths: int32 [B], the tokens of each item; the rest is padding.  scale: 0 for 1/sqrt(d).  f32_math: fp32 arithmetic on bf16 tensors.
    Returns (out, lse); lse is fp32 [B, H, n].  Nothing is recorded for autograd, also where inputs require a gradient: window_attention_backward
    gives it, and a torch.autograd.Function around the two has it recorded."""
    desc = _window_desc(q, k, v, left, right, sinks, scale, layout, lengths, f32_math)
    index = q.get_device()
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_tokens("out", out, q.shape, q.dtype, index)
    lse = _lse(q, lse, (desc.B, desc.H, desc.n))
    work = _workspace(desc, q) if desc.dtype == B_.F32 else None      # (a name holds it until the call has been queued)
    B_.linattn_window_fwd(desc, q, k, v, out, lse, _raw_stream(index))
    return out, lse


@_on_device_of
def window_attention_backward(q, k, v, out, lse, dout, *, left=-1, right=-1, sinks=0, scale=0.0, layout="bhnd", lengths=None,
                              f32_math=False, dq=None, dk=None, dv=None):
    """Gradients (dq, dk, dv) of window_attention (same keyword arguments) for the upstream gradient dout, from its out and lse.  Nothing is recorded for
    autograd."""
    desc = _window_desc(q, k, v, left, right, sinks, scale, layout, lengths, f32_math)
    index = q.get_device()
    dq, dk, dv = [torch.empty_like(t) if g is None else g for g, t in ((dq, q), (dk, k), (dv, v))]
    for name, t, like in (("out", out, q), ("dout", dout, q), ("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        _check_tokens(name, t, like.shape, q.dtype, index)
    _check_tokens("lse", lse, (desc.B, desc.H, desc.n), torch.float32, index)
    work = _workspace(desc, q)      # (a name holds it until the call has been queued)
    B_.linattn_window_bwd(desc, q, k, v, out, lse, dout, dq, dk, dv, _raw_stream(index))
    return dq, dk, dv


def _cache_tensor(name):
    """Attribute of a PagedCache for one of its tensors."""
    return property(lambda self: self._tensors[name], lambda self, t: self._take({**self._tensors, name: t}))


class PagedCache:
    """Keys and values of B sequences in pages of a pool (see linattn_cache_desc).  k, v: [pages, H, page, d], bfloat16 or float8_e4m3fn; k_exp,
    v_exp (float8 only): uint8 [pages, H, page]; table: int32 [B, width]; lengths: int32 [B].  The caller owns the tensors and writes table
    and lengths: a chunk's tokens are counted in lengths before it is written or attended to.  A tensor may be replaced by assigning to its attribute; the new one
    is checked beside the others as here.  (A captured graph goes on using those of its capture.)"""

    def __init__(self, k, v, table, lengths, k_exp=None, v_exp=None):
        self._take(dict(k=k, v=v, table=table, lengths=lengths, k_exp=k_exp, v_exp=v_exp))

    def _take(self, tensors):
        """Check the tensors and make them the cache's: their addresses go into the description that calls hand over."""
        k, v, table, lengths, k_exp, v_exp = [tensors[name] for name in ("k", "v", "table", "lengths", "k_exp", "v_exp")]
        for name in ("k", "v", "table", "lengths"):
            _need(isinstance(tensors[name], torch.Tensor), f"{name}: a tensor")
        _need(k.dim() == 4 and k.dtype in (torch.bfloat16, torch.float8_e4m3fn), "k: a bf16 or float8_e4m3fn tensor [pages, H, page, d]")
        _need(table.dim() == 2, "table: [B, width]")
        index = k.get_device()
        _need(index >= 0, "tensors must be on the GPU")
        quantised = k.dtype == torch.float8_e4m3fn
        for name, t in (("k", k), ("v", v)):
            _check_tokens(name, t, k.shape, k.dtype, index)
        _check_ints("table", table, table.shape, index)
        _check_ints("lengths", lengths, table.shape[:1], index)
        _need((k_exp is not None and v_exp is not None) == quantised, "k_exp and v_exp go with float8 rows")
        for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
            if t is not None:
                _check_tokens(name, t, k.shape[:3], torch.uint8, index)
        self._tensors, self.index = tensors, index
        self.pages, self.H, self.page, self.d = k.shape
        self.B, self.width = table.shape
        self._desc = B_.CacheDesc(B_.CACHE_E4M3 if quantised else B_.CACHE_BF16, self.B, self.H, self.d, self.page, self.pages, self.width,
                                  0, *[B_._ptr(t) for t in (k, v, k_exp, v_exp, table, lengths)], None)

    k, v, table, lengths, k_exp, v_exp = [_cache_tensor(name) for name in ("k", "v", "table", "lengths", "k_exp", "v_exp")]

    @classmethod
    def empty(cls, pages, page, H, d, B, width, *, quantised=False, device="cuda"):
        """A pool of `pages` pages of `page` tokens, tables that name no page, lengths zero."""
        rows = [torch.empty((pages, H, page, d), dtype=torch.float8_e4m3fn if quantised else torch.bfloat16, device=device) for _ in range(2)]
        exps = [torch.empty((pages, H, page), dtype=torch.uint8, device=device) if quantised else None for _ in range(2)]
        return cls(*rows, torch.full((B, width), -1, dtype=torch.int32, device=device), torch.zeros(B, dtype=torch.int32, device=device), *exps)

    def _describe(self, layout, counts):
        _check_ints("counts", counts, (self.B,), self.index)
        desc = B_.CacheDesc.from_buffer_copy(self._desc)
        desc.layout, desc.counts = B_.LAYOUT_BNHD if layout == "bnhd" else B_.LAYOUT_BHND, B_._ptr(counts)
        return desc

    @_on_device_of
    def write(self, k, v, *, counts=None, layout="bnhd"):
        """Put a chunk's rows into the cache.  k, v: bf16 [B, n, H, d] or [B, H, n, d]; counts: int32 [B], the new tokens of each sequence
        (None: n), at its positions lengths - counts, ...; tokens past the table are dropped.  Nothing is recorded for autograd."""
        n = _token_dims(k, layout)[2]
        shape = _token_shape(self.B, self.H, n, self.d, layout)
        _check_tokens("k", k, shape, torch.bfloat16, self.index)
        _check_tokens("v", v, shape, torch.bfloat16, self.index)
        B_.linattn_cache_write(self._describe(layout, counts), k, v, n, _raw_stream(self.index))

    @_on_device_of
    def read(self, n, *, layout="bnhd", k=None, v=None):
        """The first n tokens of every sequence as bf16 tensors (k, v); zeros behind a sequence's end."""
        _need(layout in ("bhnd", "bnhd"), "layout is 'bhnd' or 'bnhd'")
        shape = _token_shape(self.B, self.H, n, self.d, layout)
        k, v = [torch.empty(shape, dtype=torch.bfloat16, device=self.k.device) if t is None else t for t in (k, v)]
        for name, t in (("k", k), ("v", v)):
            _check_tokens(name, t, shape, torch.bfloat16, self.index)
        B_.linattn_cache_read(self._describe(layout, None), k, v, n, _raw_stream(self.index))
        return k, v

    @_on_device_of
    def attend(self, q, *, counts=None, left=-1, right=0, sinks=0, scale=0.0, layout="bnhd", out=None, lse=None):
        """Attention of a chunk over the cache, which holds the chunk's own keys already (write).  q: bf16 [B, n, H, d] or [B, H, n, d] with a
        multiple of the cache's heads; left, right, sinks, scale as in window_attention, by position in the sequence.
        Returns (out, lse); lse is fp32 [B, H, n].  Nothing is recorded for autograd, and there is no backward pass."""
        B, H, n, d = _token_dims(q, layout)
        _check_tokens("q", q, _token_shape(self.B, H, n, self.d, layout), torch.bfloat16, self.index)
        if out is None:
            out = torch.empty_like(q)
        else:
            _check_tokens("out", out, q.shape, q.dtype, self.index)
        lse = _lse(q, lse, (B, H, n))
        desc = self._describe(layout, counts)
        size = B_.linattn_cache_workspace_bytes(desc, H, n)
        work = q.new_empty(size, dtype=torch.uint8) if size else None
        B_.linattn_cache_attn(desc, B_.Sight(left, right, sinks, scale), q, out, lse, H, n, work, size, _raw_stream(self.index))
        return out, lse
