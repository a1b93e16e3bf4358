/*
 * moe.h -- C ABI of the MI355X (gfx950) MoE expert-layer library.
 *
 * One FFN-group GPU's share of a Mixture-of-Experts layer: top-k gating, the shuffle of
 * tokens from micro-batch order into expert order, the SwiGLU expert FFNs as grouped
 * GEMMs (forward and backward), and the gate-weighted reduction back to token order.
 *
 * Notation (the paper's symbol table in brackets): T tokens [b*s], d hidden size [H],
 * E experts, k top-k, f expert hidden size [D_e].  This GPU holds the contiguous expert
 * slice [e_lo, e_lo+e_cnt) (expert parallelism, background section on distributed
 * training).  R = number of (token, slot) pairs routed to a local expert.
 *
 * Conventions for every entry point
 *   - All pointers are DEVICE pointers unless marked "host".  All matrices are row-major
 *     and densely packed.  Integer scalars are host values.
 *   - dtype is MOE_F32 (float) or MOE_BF16 (bfloat16 storage, fp32 accumulation,
 *     round-to-nearest-even stores).  It is the type of x/xp/h/o/y and of the weights.
 *   - The caller owns every buffer.  The library allocates no device memory, keeps no
 *     pointer past the call and never synchronises with the host: each call only enqueues
 *     kernels on `stream` (a hipStream_t; NULL = the default stream).  Row counts stay on
 *     the device (offsets[e_cnt] = R), so a whole layer can be enqueued without a sync.
 *   - Return value: MOE_OK or an error code.  Arguments are validated on the host before
 *     anything is launched; on error nothing has been enqueued.  No exception or abort
 *     crosses this boundary.  Inputs must be finite (NaN/Inf logits: unspecified
 *     selection, but no out-of-bounds access).
 *   - T == 0 is legal and a no-op (plan outputs are still written: all offsets zero).
 */
#ifndef MOE_MI355X_H
#define MOE_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void* moe_stream_t; /* hipStream_t */

enum { MOE_OK = 0, MOE_EINVAL = 1, MOE_EUNSUPPORTED = 2, MOE_EWORKSPACE = 3, MOE_EHIP = 4 };
enum { MOE_F32 = 0, MOE_BF16 = 1 };
enum { MOE_GATE_SOFTMAX_RENORM = 0, MOE_GATE_SIGMOID_RENORM = 1, MOE_GATE_SOFTMAX = 2 };
enum { MOE_WS_DISPATCH = 0, MOE_WS_EXPERT_FWD = 1, MOE_WS_EXPERT_BWD = 2, MOE_WS_ROUTER = 3,
       MOE_WS_BLOCK_NORM = 4, MOE_WS_MX4_EXPERT_FWD = 5 };

/* Limits checked by the entry points (MOE_EUNSUPPORTED beyond them). */
#define MOE_MAX_EXPERTS 1024 /* E */
#define MOE_MAX_LOCAL 1024   /* e_cnt */
#define MOE_MAX_TOPK 64      /* k */
#define MOE_MAX_NORM_D 16384 /* d of moe_block_norm_fwd and _bwd */

/*
 * moe_route -- top-k gating (MoE background section: a gate network selects the top-k
 * experts with the highest probability scores).
 *
 *   logits  [T,E] float     router outputs (the router GEMM itself is the caller's)
 *   topk_idx[T,k] int32     out: global expert ids; slot j = j-th best.  Ranking is on the
 *                           raw fp32 logits, descending; equal logits (+0 == -0) -> the
 *                           lower expert id first.
 *   topk_w  [T,k] float     out: gate weights.  SOFTMAX_RENORM: softmax over all E,
 *                           renormalised over the k selected; SIGMOID_RENORM: logistic
 *                           scores renormalised over the k selected; SOFTMAX: softmax over
 *                           all E, not renormalised.
 *   counts  [e_cnt] int32   out: number of slots routed to each local expert.
 * Errors: EINVAL for NULL pointers, T<0, E<=0, k<=0, k>E, slice outside [0,E), unknown
 * gate_mode; EUNSUPPORTED beyond the limits above.
 */
int moe_route(const float* logits, int T, int E, int k, int gate_mode, int e_lo, int e_cnt,
              int32_t* topk_idx, float* topk_w, int32_t* counts, moe_stream_t stream);

/*
 * moe_dispatch -- shuffle tokens from micro-batch order to expert order (introduction:
 * tokens are dispatched from the micro-batch ranking to the expert ranking; the paper's
 * resource-allocation section counts 2*S*k*H bytes of bf16 per direction for it).
 *
 * Plan (reuse_plan == 0): from topk_idx build
 *   offsets [e_cnt+1] int32  out: exclusive prefix sum of the local counts; offsets[e_cnt]=R
 *   perm    [cap]     int32  out: perm[r] = flat slot s = t*k + j held by row r; rows are
 *                            sorted by (local expert, s) -- a stable counting sort, so the
 *                            result is unique and reproducible.  Entries [R,cap) untouched.
 *   inv     [T,k]     int32  out: row of slot (t,j), or -1 if its expert is not local; not in
 *                            topk_idx's place, which is read until the plan is done.
 * With reuse_plan == 1 the three arrays are inputs (as written by an earlier call) and
 * topk_idx may be NULL.
 * Row move: xp[inv[t,j], :] = x[t, :] * (row_scale ? row_scale[t,j] : 1) for every local
 * slot.  Rows [R,cap) of xp are left untouched.  The scaled form is the backward of
 * moe_combine with respect to its input (d_o = gate * dy); the product is formed in fp32
 * and rounded once.
 *
 *   x        [T,d] dtype     tokens (or dy)
 *   row_scale[T,k] float     NULL or per-slot factor
 *   xp       [cap,d] dtype   out
 *   cap                      rows available in xp/perm.  cap >= R is the caller's duty
 *                            (T*min(k,e_cnt) always suffices).  If R > cap, rows >= cap are
 *                            dropped (their inv is -1), offsets are clamped to cap and the
 *                            int32 status word at the start of ws is set to 1 (else 0).
 *   ws, ws_bytes             device scratch of at least
 *                            moe_workspace_bytes(MOE_WS_DISPATCH, ...) bytes, 256-byte
 *                            aligned; only used when reuse_plan == 0.
 * Errors: EINVAL (NULL, negative sizes, k>MOE_MAX_TOPK, bad slice, unknown dtype),
 * EUNSUPPORTED (bf16 with d % 8 != 0, fp32 with d % 4 != 0), EWORKSPACE.
 */
int moe_dispatch(const void* x, int dtype, int T, int d, int k, const int32_t* topk_idx,
                 const float* row_scale, int e_lo, int e_cnt, int32_t* offsets, int32_t* perm,
                 int32_t* inv, int reuse_plan, void* xp, int cap, void* ws, size_t ws_bytes,
                 moe_stream_t stream);

/*
 * moe_dispatch_static -- moe_dispatch (plan + row move, reuse_plan == 0) for callers that cannot
 * allocate device memory or pass a workspace: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  The plan's scratch (its per-chunk histogram table and the
 * expert bases) lives in a MOE_STATIC_PLAN_BYTES array inside the library's code object; each GPU
 * that runs the library holds its own copy until the process ends.  The call allocates nothing
 * and frees nothing.  Outputs are bit-identical to moe_dispatch's.
 *   arguments as moe_dispatch, without reuse_plan / ws / ws_bytes, plus
 *   status   int32 (device) out, may be NULL: 1 if R > cap (rows dropped as in moe_dispatch), else 0.
 * Limit: the plan tables must fit the array, 256 + 4 (ceil(T k / 512) e_cnt + e_cnt + 1) <=
 * MOE_STATIC_PLAN_BYTES (at e_cnt = 32 that is T k <= 16.7 million slots); beyond it the call
 * returns MOE_EWORKSPACE and enqueues nothing.  Other errors as moe_dispatch.
 * The array is shared by every call on a GPU and keeps the last call's contents (each call
 * overwrites what it reads, nothing needs clearing): calls that overlap on one GPU, on different
 * streams or from different threads, race; serialise them.  The first call on a device looks up
 * the array's device address (no allocation); make it before a graph capture starts.
 */
#define MOE_STATIC_PLAN_BYTES (4 << 20)
int moe_dispatch_static(const void* x, int dtype, int T, int d, int k, const int32_t* topk_idx,
                        const float* row_scale, int e_lo, int e_cnt, int32_t* offsets, int32_t* perm,
                        int32_t* inv, void* xp, int cap, int32_t* status, moe_stream_t stream);

/*
 * moe_expert_fwd -- the expert FFNs as grouped GEMMs over expert-contiguous rows
 * (resource-allocation section: after gating, GroupGEMMs over the k*S routed tokens).
 * For each local expert e and its rows [offsets[e], offsets[e+1]):
 *     h1 = xp W1[e];  h3 = xp W3[e];  a = silu(h1) * h3;  o = a W2[e]
 * with silu(z) = z / (1 + exp(-z)).
 *
 *   xp [cap,d]; w1,w3 [e_cnt,d,f]; w2 [e_cnt,f,d] (local slice: index 0 = expert e_lo)
 *   h1,h3 [cap,f]  out, saved for the backward pass; both NULL = forward only
 *   a  [cap,f]     out, may be NULL: the activation silu(h1) * h3 as the down projection consumed it
 *                  (rounded to dtype).  A caller that keeps it and hands it to moe_expert_bwd saves that
 *                  call one [cap,f] store; with NULL it goes to ws and the backward recomputes it.
 *   o  [cap,d]     out.  Rows >= R of every output are left untouched.
 *   ws             device scratch (holds a [cap,f] and the tile-scheduler counters),
 *                  moe_workspace_bytes(MOE_WS_EXPERT_FWD, ...) bytes, 256-byte aligned
 * bf16 requires d % 64 == 0 and f % 64 == 0; fp32 requires d % 4 == 0 and f % 4 == 0
 * (EUNSUPPORTED otherwise).  offsets must be non-decreasing with offsets[e_cnt] <= cap.
 * A row's results depend on that row and its expert's weights alone, bit for bit: not on cap (which picks the kernel),
 * nor on the rows beside it.
 * fp32: operands enter with all 24 bits and sums are fp32; a product of two operands may be off by 2^-24 of it before it is
 * added (in the root mean square 2^-27.4).  Infinities, NaN, numbers beyond 2^96 and sums beyond 2^64 behave as in fp32, but a
 * 64x64 tile that holds one takes twice its time.
 */
int moe_expert_fwd(const void* xp, int dtype, int cap, int d, int f, int e_cnt,
                   const int32_t* offsets, const void* w1, const void* w3, const void* w2,
                   void* h1, void* h3, void* a, void* o, void* ws, size_t ws_bytes, moe_stream_t stream);

/*
 * moe_expert_bwd -- backward of moe_expert_fwd (AF-Pipe section: FFN workers run backward
 * passes and send hidden-state gradients back).  Per expert e, on its rows:
 *     dA  = d_o W2[e]^T                      dW2[e] = a^T d_o
 *     dH1 = dA * h3 * silu'(h1)              dH3    = dA * silu(h1)
 *     dW1[e] = xp^T dH1                      dW3[e] = xp^T dH3
 *     dxp = dH1 W1[e]^T + dH3 W3[e]^T
 * with silu'(z) = s(z) (1 + z (1 - s(z))), s the logistic function.
 *
 *   xp,h1,h3 as saved by the forward; d_o [cap,d] gradient w.r.t. o
 *   a [cap,f]     the forward's activation output, or NULL.  With NULL it is recomputed from the saved
 *                 (rounded) h1, h3 into ws, which differs from the forward's value by one rounding of
 *                 h1 and h3; with the forward's copy dW2 is the gradient of exactly what the forward
 *                 multiplied by W2, and the call stores one [cap,f] matrix less.
 *   dxp [cap,d] out; dw1,dw3 [e_cnt,d,f], dw2 [e_cnt,f,d] out (dtype = weight dtype)
 *   accumulate    0: dw* are overwritten (an expert without rows gets zeros);
 *                 1: the new gradient is added to the existing contents.
 *   ws            device scratch (a, dH1, dH3 [cap,f], the tile-scheduler counters and, for bf16,
 *                 fp32 partial tiles for the weight gradients of experts with far more rows than
 *                 the others, which are accumulated in pieces -- at most 512 MB),
 *                 moe_workspace_bytes(MOE_WS_EXPERT_BWD, ...) bytes, 256-byte aligned.
 * Results are bit-reproducible from run to run (every sum has a fixed order).
 * Same shape restrictions as the forward, and the same fp32 products; the weight gradients of an expert with one row are
 * correctly rounded products.
 */
int moe_expert_bwd(const void* xp, const void* h1, const void* h3, const void* a, const void* d_o, int dtype,
                   int cap, int d, int f, int e_cnt, const int32_t* offsets, const void* w1,
                   const void* w3, const void* w2, void* dxp, void* dw1, void* dw3, void* dw2,
                   int accumulate, void* ws, size_t ws_bytes, moe_stream_t stream);

/*
 * moe_combine -- gate-weighted reduction back to token order (MoE background section:
 * the outputs of the active experts are reduced by a weighted sum).
 *     y[t,:] = sum over j with inv[t,j] >= 0, ascending j, of topk_w[t,j] * o[inv[t,j], :]
 * accumulated in fp32 and rounded once; tokens without a local slot get zeros.  With
 * topk_w == NULL every weight is 1 (the backward of the unscaled dispatch: dx from dxp).
 *   o [rows,d] dtype; inv [T,k]; topk_w [T,k] float or NULL; y [T,d] dtype out.
 * Every inv entry must be -1 or a valid row of o.
 */
int moe_combine(const void* o, int dtype, int T, int d, int k, const int32_t* inv,
                const float* topk_w, void* y, moe_stream_t stream);

/* Scratch bytes needed by the call named by `which` (MOE_WS_*) at these sizes; 0 on
 * invalid arguments is never returned for valid ones (at least 256).  For MOE_WS_ROUTER
 * (moe_router_fwd and moe_router_bwd share one size) pass E in the e_cnt argument. */
size_t moe_workspace_bytes(int which, int dtype, int T, int k, int d, int f, int e_cnt, int cap);

/*
 * The trainable gate (MoE background section: the gate network that scores the experts is
 * trainable).  logits = x Wr, and the loss reaches Wr and x a second time through the gate
 * weights that multiply the expert outputs.  Expert selection is held fixed in the backward
 * pass (it is piecewise constant in the logits).  Order of the calls in a training step:
 *   forward : moe_router_fwd -> moe_route -> moe_dispatch -> moe_expert_fwd -> moe_combine
 *   backward: moe_combine_bwd (replaces the scaled moe_dispatch) -> moe_expert_bwd ->
 *             moe_combine(dxp, no gate) -> moe_gate_bwd -> moe_router_bwd (adds into dx)
 *
 * moe_router_fwd -- logits [T,E] float = x [T,d] Wr [d,E], fp32 accumulation.
 *   x and wr have type `dtype`; bf16 requires d % 8 == 0.  ws: moe_workspace_bytes(MOE_WS_ROUTER).
 *   A token's logits are the same bit for bit in every batch, except for bf16 with E % 64 == 0 and
 *   d % 64 == 0, where the order of the sums follows T.
 */
int moe_router_fwd(const void* x, const void* wr, int dtype, int T, int d, int E, float* logits,
                   void* ws, size_t ws_bytes, moe_stream_t stream);

/*
 * moe_combine_bwd -- backward of moe_combine with respect to both of its inputs, in one pass
 * over dy:
 *     d_o[inv[t,j], :] = topk_w[t,j] * dy[t, :]                    (as the scaled moe_dispatch)
 *     dgate[t,j]       = < dy[t, :], o[inv[t,j], :] >               (0 where inv[t,j] == -1)
 *   dy [T,d], o [rows,d], d_o [rows,d] of type dtype; inv [T,k]; topk_w, dgate [T,k] float.
 * The dot product is accumulated in fp32 in a fixed order (reproducible run to run).  With a
 * local expert slice dgate holds this GPU's slots only; moe_gate_bwd is linear in dgate, so
 * partial results add across GPUs.
 */
int moe_combine_bwd(const void* dy, const void* o, int dtype, int T, int d, int k, const int32_t* inv,
                    const float* topk_w, void* d_o, float* dgate, moe_stream_t stream);

/*
 * moe_gate_bwd -- gradient with respect to the logits through the gate weights, selection fixed.
 * With g the gate weights of the k selected experts and c = sum_j g_j dgate_j:
 *   SOFTMAX_RENORM : dlogit_j = g_j (dgate_j - c)                 on the selected experts, else 0
 *   SIGMOID_RENORM : dlogit_j = (dgate_j - c) s_j (1 - s_j) / S   (s logistic scores, S their sum
 *                                                                  over the selection), else 0
 *   SOFTMAX        : dlogit_e = p_e ([e selected] dgate_e - c)    for all E (p softmax over all E)
 *   logits [T,E] float, topk_idx [T,k], dgate [T,k] float -> dlogits [T,E] float (every entry written).
 */
int moe_gate_bwd(const float* logits, const int32_t* topk_idx, const float* dgate, int T, int E, int k,
                 int gate_mode, float* dlogits, moe_stream_t stream);

/*
 * moe_router_bwd -- backward of moe_router_fwd:
 *     dwr [d,E] (+)= x^T dlogits          dx [T,d] (+)= dlogits Wr^T
 *   dwr, dx of type dtype; dlogits [T,E] float.  dwr_accumulate / dx_accumulate: 0 overwrite,
 *   1 add to the existing contents (dx_accumulate = 1 adds the router term to the gradient that
 *   the expert path left in dx).  Either output may be NULL to skip it.
 *   bf16 with d % 64 == 0 and E % 64 == 0: dlogits is rounded to bf16 for the matrix cores.  Other
 *   shapes keep all 24 bits of dlogits, as fp32 or as three bf16 terms on the matrix cores; only the
 *   weight gradient of up to 42 experts may lose bits of dlogits below 2^-109.  All sums are fp32; those
 *   over T are formed in ranges of tokens that depend on the sizes alone and are added in ascending
 *   order, so results are bit-reproducible from run to run.  ws: moe_workspace_bytes(MOE_WS_ROUTER).
 */
int moe_router_bwd(const void* x, const void* wr, const float* dlogits, int dtype, int T, int d, int E,
                   void* dwr, int dwr_accumulate, void* dx, int dx_accumulate, void* ws, size_t ws_bytes,
                   moe_stream_t stream);

/*
 * The norms between two blocks (the layer sits between a norm in front of it and a residual sum behind it; a block may have a norm of its
 * output as well).  One pass takes the residual stream over a block's output y to the next block's input:
 *     u  = (post_norm ? y * r_post : y) * w_post          r_post[t] = (mean_c y[t,c]^2 + eps)^-1/2
 *     h' = alpha * h + beta * gate[t] * u
 *     n  = h' * r_pre * w_pre                             r_pre[t]  = (mean_c h'[t,c]^2 + eps)^-1/2
 *
 * moe_block_norm_fwd
 *   y      [T,d] dtype      the block's output; NULL: there is none yet, h' = h (alpha, beta, gate, w_post and post_norm do not enter), for
 *                           the norm in front of a model's first block
 *   gate   [T] float        NULL: 1
 *   w_post [d] dtype        NULL: 1.  With post_norm == 0 it is a scale per channel.
 *   h      [T,d] res_dtype  the residual stream; res_dtype is dtype or MOE_F32
 *   w_pre  [d] dtype        NULL: n is not formed (behind the last block)
 *   h_out  [T,d] res_dtype  out: h', may be h itself; NULL: not stored.  NULL where y is.
 *   n      [T,d] dtype      out, NULL exactly where w_pre is; may be y itself
 *   r_post, r_pre [T] float out, what the backward needs; NULL: not stored
 * Sums are fp32.  n is formed from h' before its rounding to res_dtype: it is rounded once.
 *
 * moe_block_norm_bwd -- the gradient, at the saved y, h' (h_out; h where y is NULL), r_post and r_pre:
 *     gh = dh_out + r_pre (w_pre dn) - h' r_pre^3 mean_c(w_pre dn h')        dh = alpha gh
 *     du = beta gate[t] gh                                                   dgate[t] = beta sum_c gh u
 *     dy = post_norm ? r_post (w_post du) - y r_post^3 mean_c(w_post du y) : w_post du
 *     dw_pre (+)= sum_t dn h' r_pre          dw_post (+)= sum_t du (post_norm ? y r_post : y)
 *   dh_out [T,d] res_dtype  gradient of h' from further on; NULL: none.  dn [T,d] dtype: NULL exactly where w_pre is.  Not both NULL.
 *   dh [T,d] res_dtype out, may be dh_out itself; dy [T,d] dtype out, may be y or dn itself, NULL exactly where y is; dgate [T] float
 *   out; dw_post, dw_pre [d] dtype out, added to their contents with accumulate == 1.  dh, dgate, dw_post and dw_pre: NULL: not formed.
 *   r_post is read where post_norm is set, r_pre where w_pre is given.
 *   ws: moe_workspace_bytes(MOE_WS_BLOCK_NORM, dtype, T, 0, d, 0, 0, 0) bytes, 256-byte aligned.
 * The column sums are fp32, formed over rows that T, d and dtype decide and added in a fixed order: results are bit-reproducible.
 * Errors of both: EINVAL (NULL, negative sizes, unknown types, res_dtype neither dtype nor MOE_F32, eps not a positive number, outputs without their inputs),
 * EUNSUPPORTED (bf16 with d % 8 != 0, fp32 with d % 4 != 0, d > MOE_MAX_NORM_D, T > 2^31 - 2^16), EWORKSPACE.
 */
int moe_block_norm_fwd(const void* y, const float* gate, const void* w_post, int post_norm, const void* h, const void* w_pre,
                       int dtype, int res_dtype, int T, int d, float alpha, float beta, float eps, void* h_out, void* n,
                       float* r_post, float* r_pre, moe_stream_t stream);
int moe_block_norm_bwd(const void* y, const float* gate, const void* w_post, int post_norm, const void* h_out, const void* w_pre,
                       const float* r_post, const float* r_pre, const void* dh_out, const void* dn, int dtype, int res_dtype,
                       int T, int d, float alpha, float beta, void* dh, void* dy, float* dgate, void* dw_post, void* dw_pre,
                       int accumulate, void* ws, size_t ws_bytes, moe_stream_t stream);

/*
 * Microscaled 4-bit numbers (the OCP MX format of e2m1 elements with one e8m0 scale per 32): an element is 0, 1/2, 1, 3/2, 2, 3, 4, 6 or the
 * negative of one, times a power of two that 32 elements along the contraction share.
 *
 * Layout.  n rows of K elements, K the contraction (weights: n output columns, K inputs), are kept in the order of the matrix instruction:
 *   data    uint8 [ceil(n/16)][ceil(K/128)][4][16][16]    element (i, k): tile i/16, k/128; chunk k%128/32; row i%16; byte k%32/2, the even
 *                                                         element in its low half.  Codes 0..7 are 0, 1/2, .. 6 in order; bit 3 is the sign.
 *   scales  uint8 [ceil(n/16)][ceil(K/512)][4][16][4]     scale of the chunk of (i, k): i/16, k/512; k%128/32; i%16; k%512/128.  The power
 *                                                         of two plus 127; 255 is NaN.
 * Rows past n and elements past K are zeros in both.  A batch of matrices is one after the other.
 *
 * moe_mx4_quantize -- per 32 elements the scale is 2^(floor(log2 max|x|) - 2), not below 2^-127; elements are x / scale rounded to nearest even,
 *   saturating at 6.  A chunk with an infinity or NaN gets scale 255 and codes 0.
 *   along_rows == 0: x [batch][n][K], contraction contiguous (tokens); rows = n, cols = K
 *   along_rows == 1: x [batch][K][n] (weights as the layer keeps them, W1[d][f], W2[f][d]); rows = K, cols = n
 * moe_mx4_dequantize -- out [batch][n][K] of type dtype, exact.
 * Errors: EINVAL (NULL, negative sizes, unknown dtype, pointers not 16-byte aligned), EUNSUPPORTED (K % 32 != 0; along_rows: bf16 with n % 8 != 0,
 * fp32 with n % 4 != 0; 2^31 tiles of 16 x 512 or more, n or K within 511 of 2^31).
 */
int moe_mx4_quantize(const void* x, int dtype, int batch, int rows, int cols, int along_rows, uint8_t* data, uint8_t* scales,
                     moe_stream_t stream);
int moe_mx4_dequantize(const uint8_t* data, const uint8_t* scales, int batch, int n, int K, void* out, int dtype, moe_stream_t stream);

/*
 * moe_mx4_expert_fwd -- the experts' forward for serving, with weights and activations in microscaled 4 bits:
 *     xq = MX4(xp);  a = MX4(silu(xq W1[e]) * (xq W3[e]));  o = a W2[e]
 *   xp [cap,d], o [cap,d] of type dtype, MOE_BF16 (MOE_F32: EUNSUPPORTED); rows as in moe_expert_fwd, rows >= R of o are left untouched
 *   w1, w3  data of e_cnt matrices with n = f, K = d (moe_mx4_quantize of [e_cnt][d][f] along rows); s1, s3 their scales
 *   w2      n = d, K = f; s2.  Elements past K have to be zeros, as the quantisation leaves them.
 *   ws      moe_workspace_bytes(MOE_WS_MX4_EXPERT_FWD, dtype, 0, 0, d, f, e_cnt, cap) bytes, 256-byte aligned
 * Products of 4-bit numbers are exact and their sums fp32; the activation is rounded to 4 bits from fp32.  d % 32 == 0 and f % 32 == 0 (EUNSUPPORTED
 * otherwise, and for d or f beyond 2^20 or 2^30 tiles of 16 rows by 32 columns).  A row that holds an infinity or NaN spoils its own outputs only.
 * A row's results depend on that row, its expert's weights and whether its expert has up to 32 rows or more, bit for bit: not on cap, nor on the rows
 * beside it and of other experts.
 */
int moe_mx4_expert_fwd(const void* xp, int dtype, int cap, int d, int f, int e_cnt, const int32_t* offsets, const uint8_t* w1,
                       const uint8_t* s1, const uint8_t* w3, const uint8_t* s3, const uint8_t* w2, const uint8_t* s2, void* o, void* ws,
                       size_t ws_bytes, moe_stream_t stream);

/*
 * Optional per-kernel timing, for benchmarks (measurement of the grouped GEMMs against the
 * MFMA roofline and of the row movers against HBM bandwidth).  Apart from per-device caches of
 * constants (CU count, the kernels' LDS opt-in attribute, the address of the built-in plan scratch)
 * this is the library's only process-wide state, and it is off by default.  While enabled, every kernel launch of the
 * entry points above except the fp32 expert GEMMs is bracketed by a pair of hipEvents recorded on the call's stream
 * (a few microseconds of host work per launch; no synchronisation).  The launches of one plan count as one.
 *   moe_profile_enable(on)   on != 0: create the event pool (first time) and start recording
 *                            from an empty log; on == 0: stop recording.
 *   moe_profile_read(kernel, &total_ms, &launches)
 *                            synchronises on the recorded events of that kernel (MOE_K_*)
 *                            and returns the summed elapsed time and the launch count.
 *   moe_profile_stats(kernel, &min_ms, &median_ms)
 *                            the shortest and the median launch of that kernel in the log
 *                            (0 if it holds none); synchronises like moe_profile_read.
 * The pool holds MOE_PROFILE_MAX_EVENTS launches; later launches are not recorded.
 * Not thread-safe: enable, run and read from one host thread.
 */
enum { MOE_K_ROUTE = 0,
       /* a dispatch of up to 2048 slots may make its plan in the launch that moves the rows: it is
        * booked as MOE_K_DISPATCH, and MOE_K_PLAN has no launch */
       MOE_K_PLAN = 1, MOE_K_DISPATCH = 2, MOE_K_COMBINE = 3, MOE_K_UP = 4,
       MOE_K_DOWN = 5, MOE_K_DA = 6, MOE_K_DX = 7, MOE_K_WG = 8, MOE_K_WGD = 9, MOE_K_ROUTER_FWD = 10,
       MOE_K_COMBINE_BWD = 11, MOE_K_GATE_BWD = 12, MOE_K_ROUTER_DW = 13, MOE_K_ROUTER_DX = 14,
       MOE_K_WGRAD_REDUCE = 15,   /* sum of the fp32 partial tiles of weight gradients cut along the rows */
       /* bf16 backward: GEMMs that do not depend on each other may share a launch (the second fills
        * the first one's tail): dA with dW2 when moe_expert_bwd is given the forward's a, dX with
        * dW1|dW3, each when the capacity bound gives a workgroup at most a dozen tiles of the first.
        * A shared launch is booked here and not under the single ids. */
       MOE_K_DA_WG = 16, MOE_K_DX_WGD = 17,
       MOE_K_NORM_FWD = 18, MOE_K_NORM_BWD = 19, MOE_K_NORM_SUMS = 20,      /* column sums of dw_post, dw_pre */
       MOE_K_MX4_QUANTIZE = 21, MOE_K_MX4_DEQUANTIZE = 22,
       MOE_K_MX4_ROWS = 23, MOE_K_MX4_UP = 24, MOE_K_MX4_DOWN = 25,
       MOE_K_COUNT = 26 };
#define MOE_PROFILE_MAX_EVENTS 8192
int moe_profile_enable(int on);
int moe_profile_read(int kernel, double* total_ms /* host */, int* launches /* host */);
int moe_profile_stats(int kernel, double* min_ms /* host */, double* median_ms /* host */);

/*
 * Measured ceilings, for benchmarks only (not part of the expert-layer path): the rates this
 * chip sustains under its own clock and power management, to be timed by the caller with
 * events on `stream`.
 *   moe_probe_mfma_bf16  enqueues an MFMA-only loop (32x32x16 bf16, 4 wavefronts per CU,
 *                        16 independent accumulators, no memory traffic), `iters` rounds of 16
 *                        MFMAs per wavefront; operands constant or pseudo-random (the latter
 *                        is the realistic case: switching activity lowers the sustained clock).
 *                        sink: device scratch of >= 256*4 bytes per CU; *flop (host) receives
 *                        the FLOP count of the launch.
 *   moe_probe_mfma_fed_bf16  the same loop with random operands re-read from LDS before every 16 MFMAs, at
 *                        the rate the grouped GEMM's tiling needs (8 fragments of 16 bytes per lane):
 *                        feed = 1 with 16-byte reads, feed = 2 with pairs of 8-byte transposing reads.  It
 *                        prices the operand feed under the package power limit.
 *   moe_probe_copy       enqueues a plain device copy of `bytes` (multiple of 16) bytes.
 *   moe_probe_stream     streaming kernels with the row movers' access width, for their ceilings: over
 *                        `bytes` (multiple of 16) of src, writes = -1 reads only (sink: >= 4 bytes of device
 *                        memory, never written in practice), 0 fills dst, n = 1..3 reads each 16-byte vector
 *                        once and writes it n times (dst must hold n * bytes).
 */
int moe_probe_mfma_bf16(float* sink, size_t sink_bytes, int iters, int random_operands, double* flop /* host */,
                        moe_stream_t stream);
int moe_probe_mfma_fed_bf16(float* sink, size_t sink_bytes, int iters, int feed, double* flop /* host */,
                            moe_stream_t stream);
int moe_probe_copy(const void* src, void* dst, size_t bytes, moe_stream_t stream);
int moe_probe_stream(const void* src, void* dst, size_t bytes, int writes, void* sink, moe_stream_t stream);

/* Static, human-readable text for an error code. */
const char* moe_error_string(int code);

#ifdef __cplusplus
}
#endif
#endif /* MOE_MI355X_H */
