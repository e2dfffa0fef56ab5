/*
 * linattn.h -- C ABI of the MI355X (gfx950) linear-attention library.
 *
 * The operator is the non-causal linear attention that LinVideo puts in place of
 * softmax attention in a video diffusion transformer (paper Sec. 3):
 *
 *   Eq. 3:  o_i = phi(q_i) S / (phi(q_i) . z),   S = sum_j phi(k_j)^T v_j,  z = sum_j phi(k_j)
 *   Eq. 5:  phi(x) = softmax(x W~) (+) softmax(-x W~),  W~ in R^{d x d/2}, one W~ for q, one for k
 *
 * evaluated independently for every (batch, head) pair over all n tokens (no mask, no
 * scaling of q.k, no epsilon: every entry of phi is positive so the denominator is too).
 *
 * Conventions shared by every entry point
 *   - q, k, v, out, dout, dq, dk, dv: DEVICE pointers, 16-byte aligned, d innermost and
 *     contiguous, all eight in the descriptor's layout: [B, H, n, d] (LINATTN_LAYOUT_BHND, the
 *     default) or [B, n, H, d] (LINATTN_LAYOUT_BNHD: heads interleaved per token, the form in
 *     which a transformer block's projection q = x W_q (Sec. 3) leaves them, so no transpose
 *     copy is needed around the operator).  d in {64, 128}, n >= 1 arbitrary, B, H >= 1,
 *     64-bit indexing inside.
 *   - element type of those tensors and of W~ is the descriptor's dtype: bf16 (LINATTN_BF16 and
 *     LINATTN_BF16_F32MATH) or fp32 (LINATTN_F32).  All accumulation is fp32.  The fp32 mode never
 *     rounds to bf16 (it splits fp32 values exactly into bf16 pieces).
 *   - all pointers are borrowed: the caller keeps them alive until the stream work is done.
 *   - calls only enqueue work on `stream` (a hipStream_t passed as void*, NULL = default
 *     stream).  They never synchronise and never allocate.
 *   - every argument error is detected on the host before any HIP call and returned as a
 *     negative status; nothing is enqueued in that case.
 *   - results are bitwise reproducible run to run (no floating-point atomics).
 *   - out must not alias q, k or v; dq, dk, dv must not alias any input.
 *   - calls that share a descriptor share its workspace: do not overlap them on
 *     different streams.
 *
 * Numeric domain of the bf16 mode (the fp32 mode computes in fp32 throughout)
 *   - q, k enter the projection of Eq. 5 as stored; phi, v, dout and the states S, dS enter the
 *     matrix cores as fp16 (11-bit significand) with fp32 accumulation.  phi, the states, dout and
 *     every gradient operand are rescaled by exact powers of two first (per token, per 16-token
 *     block, per head, or per workgroup following the running maximum), so their magnitude does
 *     not matter: any finite bf16 dout is in the domain whose quotient |dout_i| / (phi(q_i) . z) stays
 *     below the largest fp32 (with a larger one dk, dv and dW~ of its head may come out infinite or NaN, never finite
 *     and wrong), and any finite q, k with |x W~| below 2^26 (the
 *     exponent of the softmax, u log2 e minus its maximum, is rounded once at that magnitude; the
 *     fp32-arithmetic modes take the difference first and have no such limit).
 *   - An entry of dout that is an infinity or NaN makes dq of its token, dv of its channel, and dk and dW~
 *     of its head not finite; dq of the other tokens and dv of the other channels do not depend on it.
 *   - v is widened to fp16 unscaled: |v| must be below 65504 (fp16's largest finite value).  Larger
 *     entries become infinite inside the kernels and the call returns LINATTN_OK with Inf/NaN in
 *     out, state and the gradients; the library does not scan for them.  Entries with
 *     0 < |v| < 2^-14 lose their low bits (absolute error below 2^-25).
 *   - Accuracy: out, dq, dk, dv, dW~ agree with exact arithmetic on the stored inputs to 1e-2 of
 *     max(|value|, RMS of the tensor over its (b,h) slice).  Known exception (11-bit operands):
 *     dL/dphi(k_j) = v_j dS^T + dz inherits an absolute error of about 2e-4 |v_j| |dS| from the
 *     fp16 operands behind dS, so the dk row of a key whose v_j is far larger than the other
 *     tokens' carries |v_j| / rms|v| times the error of an ordinary row.  For the rows at 20x
 *     magnitude of the Wan-14B-shaped test recipe (0.1 % of the tokens) this reads up to 1e-1 of the
 *     slice RMS, and dW~_k, which weights those rows by |k_j| once more, up to 2e-2; all other rows of
 *     dk, and dq, dv, dW~_q everywhere, meet 1e-2.  (A common offset of v, however large, is not an
 *     exception: the backward's operand images are built with the head's mean value row taken out.)  Second exception: where phi is within a few per
 *     cent of uniform (the spread of x W~ over the features far below 1), dq, dk and dW~ are
 *     differences of nearly equal rows of S and dS and come out up to 0.2 off; out and dv keep 1e-2.
 *     LINATTN_FLAG_CENTRED removes this exception (not the first) at a cost of 2-4 %.
 *   - LINATTN_BF16_F32MATH reads and writes the same bf16 tensors but does all arithmetic in fp32
 *     (the kernels of the fp32 mode, no fp16 operands): none of the limits above applies, |v| may be
 *     any finite bf16 value, and the only rounding that matters is the bf16 store of the results.  A
 *     training step costs about twice LINATTN_BF16, a forward call 1.6x (Wan-1.3B 480p shape).
 *   - fp32 arithmetic (this mode and LINATTN_F32) runs on the matrix cores as sums of exact products of bf16
 *     pieces with fp32 accumulation.  Operands below 2^-110 lose the bits below 2^-133.  What the pieces cannot
 *     carry (finite values above 3.3895e38, which round to Inf as bf16, infinities and NaN) comes out as plain fp32 FMA
 *     gives it: the workgroups that meet such a value run their share once more that way, at about the time per
 *     token of a scalar kernel (10 to 30 times the usual).
 */
#ifndef LINATTN_H
#define LINATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define LINATTN_OK            0
#define LINATTN_E_NULL       -1   /* a required pointer is NULL */
#define LINATTN_E_SHAPE      -2   /* B, H, n <= 0, unsupported d, shape differs from the descriptor, or too large */
#define LINATTN_E_DTYPE      -3   /* unknown dtype */
#define LINATTN_E_ALIGN      -4   /* a tensor pointer is not 16-byte aligned */
#define LINATTN_E_PHI        -5   /* unknown phi_id / unsupported kind / table full */
#define LINATTN_E_WORKSPACE  -6   /* workspace missing or smaller than linattn_workspace_bytes() */
#define LINATTN_E_HIP        -7   /* a HIP launch reported an error */
#define LINATTN_E_STATE      -8   /* linattn_bwd without a state buffer, or a state buffer too small for this B */
#define LINATTN_E_ALIAS      -9   /* an output aliases an input */
#define LINATTN_E_VALUE     -10   /* a number is outside its range (linattn_sight) */

/* feature-map kinds */
#define LINATTN_PHI_HEDGEHOG  1   /* Eq. 5 */
#define LINATTN_PHI_RELU      2   /* phi(x) = max(x, 0) on the d channels, no weights: the "ReLU" row of the
                                     paper's ablation of kernel functions (appendix "Ablation for Kernel
                                     Function").  The paper gives the name only; this library's reading:
                                     o_i = phi(q_i) S / (phi(q_i) . z + 1e-6), because a row of q or k can be
                                     all non-positive (such a query gets o_i = 0); the derivative of max(x, 0)
                                     at 0 is 0.  Descriptor: wq, wk, dwq, dwk and the three blend pointers
                                     must be NULL (E_PHI otherwise); state rows are the d channels of k. */

/* dtypes */
#define LINATTN_BF16  1          /* bf16 tensors, matrix-core kernels (bf16 / fp16 operands, fp32 accumulation) */
#define LINATTN_F32   2          /* fp32 tensors, fp32 arithmetic */
#define LINATTN_BF16_F32MATH 3   /* bf16 tensors, fp32 arithmetic (see "Numeric domain" above) */

/* descriptor flags */
#define LINATTN_FLAG_CENTRED 1u  /* LINATTN_BF16 with the map of Eq. 5: every fp16 operand that carries phi or a state is
                                    rounded after its mean has been taken out -- phi - 2/d in the two sums over tokens
                                    (state pass: S, z; query-side backward: dS, dz), with (2/d) x the column sums of v
                                    resp. of dout/den added back in fp32; operand images of S - z vbar^T (vbar the
                                    head's mean value row) and of dS, dz minus their means over each half's features,
                                    which the softmax Jacobian drops (dv gets the constant row back).  Exact in real
                                    arithmetic; the roundings then act on the deviation of phi from the uniform map, so
                                    the regime where phi is within a few per cent of uniform meets the 1e-2 contract
                                    for all five gradients.  Costs about 3 % of the forward (8 % of its state pass) and
                                    4 % of the backward.  A layer uses one setting for its forward and backward calls. */

/* memory layouts of q, k, v, out, dout, dq, dk, dv */
#define LINATTN_LAYOUT_BHND  0   /* element (b,h,t,c) at ((b*H + h)*n + t)*d + c */
#define LINATTN_LAYOUT_BNHD  1   /* element (b,h,t,c) at ((b*n + t)*H + h)*d + c */

/*
 * Description of a feature map plus the buffers a layer owns.  Eq. 3 takes q, k, v only;
 * Eq. 5 adds the two learnable matrices, which live here so that linattn_fwd keeps the
 * paper's argument list.  The struct is copied by linattn_phi_create.
 */
typedef struct linattn_phi_desc {
  int kind;               /* LINATTN_PHI_HEDGEHOG or LINATTN_PHI_RELU */
  int dtype;              /* LINATTN_BF16, LINATTN_F32 or LINATTN_BF16_F32MATH: type of q,k,v,out,dout,dq,dk,dv,wq,wk */
  int H, d;               /* wq, wk: device, [H, d, d/2] contiguous, one map per head (Eq. 5) */
  const void *wq, *wk;
  void *dwq, *dwk;        /* optional device fp32 [H, d, d/2]: linattn_bwd OVERWRITES them with the
                             gradient summed over batch and tokens; NULL = not computed */
  void *state;            /* optional device fp32 [B, H, d+1, d]: rows 0..d-1 = S with rows indexed by
                             the feature of phi in the order of Eq. 5 (softmax(+) half first),
                             row d = z.  linattn_fwd writes it when non-NULL; linattn_bwd reads it.
                             Its size is state_bytes (last field). */
  void *workspace;        /* device scratch, 256-byte aligned, >= linattn_workspace_bytes(...) */
  size_t workspace_bytes;
  int layout;             /* LINATTN_LAYOUT_BHND (0) or LINATTN_LAYOUT_BNHD; the state, dW~ and the
                             workspace do not depend on it */
  /* Mixed attention of the selective-transfer stage (Sec. 4.1, Eq. 6), active when blend_in and
   * blend_r are both non-NULL (set only one: E_NULL):
   *     out = r' * blend_in + (1 - r') * (Eq. 3),   r' = clip(*blend_r, 0, 1)  (footnote to Eq. 6)
   * blend_in is the softmax-attention output of the same layer, computed by the caller: device,
   * dtype and layout of out, must not overlap out.  blend_r: device, one fp32, read by the
   * kernels (no host copy).  linattn_bwd then treats dout as the gradient of the blended output:
   * dq, dk, dv, dW~ receive (1 - r') times the gradients of Eq. 3, and blend_dr (optional, device,
   * one fp32) is OVERWRITTEN with dL/dr = sum(dout * (blend_in - o)) for 0 <= r <= 1 and 0 outside
   * (the closed ends let r move from its initial value 1).  The gradient with respect to blend_in
   * is r' * dout, an elementwise product left to the caller. */
  const void *blend_in;
  const float *blend_r;
  float *blend_dr;
  size_t state_bytes;     /* bytes behind `state` (ignored when state is NULL).  A call with batch size B
                             touches B * H * (d+1) * d * 4 of them: linattn_phi_create returns E_STATE if
                             not even B = 1 fits, linattn_fwd / linattn_bwd return E_STATE for a B that
                             does not fit. */
  unsigned flags;         /* 0, or LINATTN_FLAG_CENTRED (Eq. 5 map with LINATTN_BF16 only: E_PHI otherwise) */
} linattn_phi_desc;

/* Register a descriptor; *phi_id_out receives a handle >= 16.  Host-only, no HIP call.
 * Errors: E_NULL (desc, out, wq, wk), E_PHI (kind, table full, flags that do not fit kind or dtype), E_DTYPE, E_SHAPE (H, d, layout),
 * E_ALIGN, E_STATE (state given with state_bytes < H * (d+1) * d * 4). */
int linattn_phi_create(const linattn_phi_desc* desc, int* phi_id_out);

/* Forget a handle.  E_PHI if it is not live.  Buffers stay the caller's. */
int linattn_phi_destroy(int phi_id);

/* Replace the three mixed-attention pointers of a live handle (blend_in changes every step).
 * All NULL switches the blend off.  Host-only.  Errors: E_PHI, E_NULL (exactly one of blend_in,
 * blend_r given, or blend_dr without them), E_ALIGN (blend_in not 16-byte aligned). */
int linattn_phi_set_blend(int phi_id, const void* blend_in, const float* blend_r, float* blend_dr);

/* Scratch bytes linattn_fwd, and linattn_bwd without weight gradients (dwq == dwk == NULL), need
 * for this problem (pure function of its arguments, no HIP call).  Returns 0 for an invalid
 * argument. */
size_t linattn_workspace_bytes(int B, int H, int n, int d, int kind, int dtype);

/* Scratch bytes linattn_bwd needs when the descriptor asks for dwq or dwk (W~ is learnable, Eq. 5):
 * the above plus the partial sums of dW~ (one [d][d/2] fp32 block per workgroup of the two main kernels) and, in
 * the fp32-arithmetic modes only, two fp32 buffers [B,H,n,d/2] for dL/du (the bf16 kernels accumulate dW~ where
 * du is made).  For LINATTN_PHI_RELU (no weights) it equals linattn_workspace_bytes. */
size_t linattn_workspace_bytes_wgrads(int B, int H, int n, int d, int kind, int dtype);

/*
 * Forward, Eq. 3 with the descriptor's phi (Eq. 5, or the ReLU map).  Three stages on `stream`: phi(K) fused with a split-n
 * partial state, a fixed-order reduction of the partials (in the third stage's kernel where a bf16 call is short), phi(Q) S /
 * (phi(Q) . z) with the store of out.  Writes out [B,H,n,d] and, if the descriptor has one, state.
 * Errors: E_PHI, E_NULL, E_SHAPE (also H or d different from the descriptor), E_ALIGN,
 * E_WORKSPACE, E_STATE (state buffer smaller than this B needs), E_ALIAS, E_HIP.
 */
int linattn_fwd(const void* q, const void* k, const void* v, void* out,
                int B, int H, int n, int d, int phi_id, void* stream);

/*
 * linattn_fwd for callers that cannot allocate device memory or size a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same
 * kernels and bit-identical results, but the split-n partials (and the state, when the descriptor
 * has no state buffer) live in a static device array of LINATTN_NOALLOC_SCRATCH_BYTES that is part
 * of the library's code object on each GPU; the descriptor's workspace is ignored and may be NULL.
 * The call allocates nothing and frees nothing.
 *   - Limit: the forward scratch of the problem (what linattn_workspace_bytes counts up to the
 *     state region: partials of at most 256 workgroups plus B*H states) must fit the array;
 *     E_WORKSPACE otherwise.  All five task configurations fit (config 4 needs 31.7 MB).
 *   - Every call on one GPU shares that GPU's array: calls that overlap in time on one GPU (two
 *     streams, two threads) race.  Nothing needs clearing between calls: a call overwrites every
 *     scratch word before reading it.
 *   - The first call on a device looks the array's address up (hipGetSymbolAddress); make that
 *     call outside stream capture.
 * Errors: as linattn_fwd; E_HIP also if the array's address cannot be found.
 */
#define LINATTN_NOALLOC_SCRATCH_BYTES (32u << 20)
int linattn_fwd_noalloc(const void* q, const void* k, const void* v, void* out,
                        int B, int H, int n, int d, int phi_id, void* stream);

/*
 * Backward of linattn_fwd for L with dL/dout = dout: writes dq, dk, dv [B,H,n,d] and, if the
 * descriptor has them, dwq and dwk (Eq. 5 only; the ReLU map has no weights).  Needs the state a
 * forward call with the same q-independent inputs (k, v, wk) left in the descriptor's state buffer.
 * Errors: as linattn_fwd, plus E_STATE.
 */
int linattn_bwd(const void* q, const void* k, const void* v, const void* dout,
                void* dq, void* dk, void* dv,
                int B, int H, int n, int d, int phi_id, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Softmax attention: the softmax branch of a layer (its output is what linattn_phi_set_blend takes as blend_in, its upstream
 * gradient is r' * dout), and the same attention for a chunk of new tokens over a paged cache, for generation piece by piece.
 *
 *   s_ij = scale q_i . k_j,   lse_i = log(sum_j exp(s_ij)),   o_i = sum_j exp(s_ij - lse_i) v_j
 *
 * with the sums over the keys that query i sees.  H query heads share HK key heads in groups of H / HK neighbours: query
 * head h reads key head h / (H / HK).  Which keys a query sees goes by positions; the query at position p sees key j of a
 * sequence of len tokens if
 *
 *   j < len,   and right < 0 or j <= p + right,   and left < 0 or j >= p - left or j < sinks
 *
 * (a window of left tokens before and right tokens after it, and the first `sinks` tokens as far as they are not
 * beyond the window's right end; right = 0 is causal, a negative number is no limit).  A row that sees nothing has out = 0 and lse = -inf.
 * The conventions at the top of this file hold.  Numbers in device memory (lengths, counts, tables) cannot be checked on the host: the
 * kernels take negative lengths and counts for 0, lengths of token tensors and counts beyond n for n, and keys that the table has no page of the pool
 * for as not there.
 *
 * Numeric domain: scores, their softmax, and all sums are fp32.  LINATTN_BF16: the probabilities, and in the backward their gradients, enter the
 * matrix cores as bf16 (the stored type of the values they multiply, so that neither has a range of its own); with the store of the
 * result that is two roundings of at most 2^-8 relative each (1.7e-3 rms each; the backward takes the row sums dout . out without the rounding of the stored
 * out).  The attention over a cache is that form; over LINATTN_CACHE_E4M3 the probabilities may take the scale of their row of v before they are rounded.
 * LINATTN_F32 and LINATTN_BF16_F32MATH: fp32 arithmetic.  The results of a row depend on the keys that it sees and on nothing else: an infinity
 * or NaN in a token that it does not see, or in the padding, does not reach it (a row whose result is not finite is computed once more key by key, at 10 to 30 times
 * the usual time).  A row's sum of |v| times 2^8 has to stay below fp32's largest value; magnitudes below 2^-100 may count as zero. */
typedef struct linattn_sight {
  int left, right, sinks;
  float scale;            /* 2^-100 to 2^100; 0: 1 / sqrt(d), as in Sec. 3 of the paper (Eq. 6 writes 1 / d for its softmax term) */
} linattn_sight;

/* q, out, dout, dq: H heads; k, v, dk, dv: HK heads; all of n tokens, in `layout`.  Token i of a batch item has position i. */
typedef struct linattn_window_desc {
  int dtype;              /* LINATTN_BF16, LINATTN_F32 or LINATTN_BF16_F32MATH: type of q, k, v, out, dout, dq, dk, dv */
  int B, H, HK, n, d;     /* H a multiple of HK, d 64 or 128 */
  int layout;             /* LINATTN_LAYOUT_BHND or LINATTN_LAYOUT_BNHD */
  linattn_sight sight;
  const int* lengths;     /* optional device [B]: tokens of each item, the others are padding.  Padding is not read; its rows of out, dq, dk, dv are
                             zeros, of lse -inf.  NULL: n each. */
  void* workspace;        /* device scratch, 256-byte aligned, not shared by calls that overlap in time.  The backward needs it; the forward of short
                             sequences in LINATTN_F32 is faster with it, and takes NULL */
  size_t workspace_bytes;
} linattn_window_desc;

/* Scratch bytes of a workspace for linattn_window_bwd, or for linattn_window_fwd if that gets one.  Pure function of the descriptor's numbers; 0 for an invalid one. */
size_t linattn_window_workspace_bytes(const linattn_window_desc* desc);

/* Forward.  lse: optional device fp32 [B, H, n], what the backward needs and what joins results over parts of the keys.
 * Errors: E_NULL, E_DTYPE, E_SHAPE, E_VALUE, E_ALIGN, E_WORKSPACE (one that is too small), E_ALIAS, E_HIP. */
int linattn_window_fwd(const linattn_window_desc* desc, const void* q, const void* k, const void* v, void* out, float* lse, void* stream);

/* Backward for L with dL/dout = dout, from the forward's out and lse; writes dq, dk, dv (dk and dv summed over the query heads of a group).
 * Errors: as above, E_WORKSPACE also without one. */
int linattn_window_bwd(const linattn_window_desc* desc, const void* q, const void* k, const void* v, const void* out, const float* lse,
                       const void* dout, void* dq, void* dk, void* dv, void* stream);

/* How a cache holds rows of k and v */
#define LINATTN_CACHE_BF16 1
#define LINATTN_CACHE_E4M3 2    /* d codes of 8 bits (e4m3, the variant without infinities) and the exponent e of a scale 2^e, per token, head and
                                   tensor: e = the least integer with max|x| 2^-e <= 448, at least -117; stored as the byte e + 127.  The codes round to
                                   nearest even.  Scaled codes are bf16 numbers (none is 2^128: entries
                                   that would round to it are held as 240 2^120), so reading back rounds no further.  Infinities become NaN; the maximum is
                                   taken over the finite entries. */

/*
 * A paged cache of B sequences: position j of sequence b is row j % page of page table[b * width + j / page] of the pool.  Rows of a
 * page's head lie together: the pools are [pages, H, page, d], the exponents [pages, H, page].
 * A chunk of n tokens per sequence (k, v of a write; q, out of an attention) is bf16 [B, H, n, d] or [B, n, H, d]; its token t has position
 * lengths[b] - counts[b] + t, and tokens from counts[b] on, or with a negative position, are padding: not read, not written
 * to the cache, their rows of out are zeros and of lse -inf.  lengths counts the chunk, before the write as after.  A sequence may have outgrown
 * its table: its tokens keep their positions (lengths up to 2^30), those from page * width on have no keys.
 */
typedef struct linattn_cache_desc {
  int type;               /* LINATTN_CACHE_BF16 or LINATTN_CACHE_E4M3 */
  int B, H, d;            /* H: heads of k and v; d 64 or 128 */
  int page, pages;        /* tokens to a page (any number), pages of the pool */
  int width;              /* table entries of a sequence; page * width <= 2^30 */
  int layout;             /* of the token tensors, not of the pool */
  void *k, *v;            /* device, 16-byte aligned */
  unsigned char *k_exp, *v_exp;      /* device; LINATTN_CACHE_E4M3 only */
  const int* table;       /* device [B, width]; entries outside 0 .. pages-1 stand for no page */
  const int* lengths;     /* device [B] */
  const int* counts;      /* optional device [B]: new tokens of each sequence.  NULL: n */
} linattn_cache_desc;

/* Put the k and v rows of a chunk into the cache; nothing else in the pool changes.  No two tokens of a call may have the same place.  A token
 * whose position is page * width or more, or whose table entry names no page, is dropped.
 * Errors: E_NULL, E_DTYPE, E_SHAPE, E_ALIGN, E_ALIAS, E_HIP. */
int linattn_cache_write(const linattn_cache_desc* desc, const void* k, const void* v, int n, void* stream);

/* The first n tokens of every sequence as bf16 [B, H, n, d] or [B, n, H, d]; rows behind a sequence's end, or without a page, are zeros.
 * counts is not looked at.  Errors: as above. */
int linattn_cache_read(const linattn_cache_desc* desc, void* k, void* v, int n, void* stream);

/* Scratch bytes linattn_cache_attn needs for chunks of n tokens of H query heads: pure function of the descriptor's numbers.  0 for an invalid
 * argument. */
size_t linattn_cache_workspace_bytes(const linattn_cache_desc* desc, int H, int n);

/* Attention of a chunk of n tokens, H query heads, over the cache (which already holds the chunk's own keys).  n = 1 is the step of
 * generation token by token.  lse: optional device fp32 [B, H, n].  workspace: 256-byte aligned, not shared by calls that overlap in time.
 * Errors: as above, E_VALUE, E_WORKSPACE. */
int linattn_cache_attn(const linattn_cache_desc* desc, const linattn_sight* sight, const void* q, void* out, float* lse, int H, int n,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Static description of a status code. */
const char* linattn_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* LINATTN_H */
