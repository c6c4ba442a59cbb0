/*
 * frameft.h -- C ABI of the FrameFT adapter hot path on MI355X (gfx950).
 *
 * FrameFT fine-tunes a frozen weight W0 (m x n, m = d_out, n = d_in) as
 *     W' = W0 + s * P_out C P_in^T,          s = alpha / sqrt(m n)
 * (paper Sec. 3.1, update equation; Algorithm 1).  P_in (n x k rho_n) and
 * P_out (m x k rho_m) are real Parseval tight fusion frames generated by
 * Spectral Tetris, root-of-unity modulation and realification (Sec. 3.2 and
 * the appendix "Fusion Frames Construction: an example"); C is a sparse fp32
 * coefficient matrix whose support is shared across layers (Sec. 3.3).
 *
 * The library computes, for a batch of T tokens stored one per row:
 *   forward   Y  = beta * Y  + s * P_out C P_in^T x            (per token x)
 *   backward  dX = beta * dX + s * P_in C^T P_out^T g          (per token g)
 *             dC = s * (P_out^T G^T X P_in) on the support of C
 *                  (Appendix A: grad f(C) = P_m^T grad f(W) P_n)
 *   merge     W  = beta * W  + s * P_out C P_in^T            (Algorithm 1, steps 5-6)
 * W0 x itself is the caller's GEMM; the library computes the adapter branch.
 *
 * Conventions shared by every call
 *   - Frame column (coefficient) index, "canonical": i*rho + 2r + s for
 *     subspace i (0..k-1), Spectral Tetris row r (0..rho/2-1) and real part
 *     s (0: image of [Re; Im], 1: image of [-Im; Re]); i.e. P = [P_1..P_k].
 *     Real coordinate 2j / 2j+1 is the real / imaginary part of complex
 *     coordinate j.  Rows of C index P_out columns, columns of C index P_in
 *     columns.
 *   - Activations are row-major, one token per row: element (t, i) of X is
 *     at X[t*ldx + i].  W is row-major m x n (nn.Linear.weight layout).
 *   - Tensors are caller-owned device memory; `stream` is a hipStream_t
 *     (NULL = default stream).  Hot-path calls are asynchronous on `stream`,
 *     never allocate, never synchronise, and write nothing when they return
 *     an error.  Calls that share a plan must be ordered on one stream: they
 *     share the plan's workspace.
 *   - bf16 activations: 16-byte aligned base pointers and leading dimensions
 *     that are multiples of 8 elements; fp32: multiples of 4 (plans with a
 *     lift, below: element alignment and any leading dimension).  Arithmetic
 *     accumulates in fp32; bf16 results are rounded to nearest even.
 *   - Supported frames on the GPU: every tight (k, rho, d) with 2k a multiple
 *     of 8 and at most 4096 (k a power of 4 times at most 64 beyond 512 wide),
 *     and also 2k a multiple of 4 up to 128 when k rho != d.  With k rho = d
 *     the frame is block diagonal with square 2k x 2k blocks.  Any other tight
 *     frame -- redundant (k rho > d, C of size k rho_m x k rho_n) or with a
 *     non-integer d / rho -- is P = L^T Pv: Pv the block frame of dimension
 *     k rho and L a sparse lift that places each Spectral Tetris row at the
 *     positions j mod k of its block (modulation sees j only mod k).  Calls on
 *     plans with such a frame lift their inputs into fp32 staging rows of
 *     width k rho (plan workspace), run the kernels there in fp32 and lift the
 *     results back; batched calls and plan groups do not take them
 *     (FF_EUNSUPPORTED).
 */
#ifndef FRAMEFT_H
#define FRAMEFT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum ff_status {
    FF_OK = 0,
    FF_EINVAL = 1,        /* bad argument: null pointer, size, alignment, index out of range */
    FF_ENOTFF = 2,        /* (k, rho, d) does not give a tight fusion frame */
    FF_EUNSUPPORTED = 3,  /* valid request that the GPU path does not implement */
    FF_ENOMEM = 4,        /* device or host allocation failed (ff_framegen, ff_plan_create only) */
    FF_EDEVICE = 5        /* no usable device, or a HIP call / kernel launch failed */
} ff_status;

typedef enum ff_dtype { FF_F32 = 0, FF_BF16 = 1 } ff_dtype;

typedef struct ff_frame ff_frame;  /* immutable; shareable by every layer of that width (Sec. 3.4, "Memory Overhead") */
typedef struct ff_plan ff_plan;    /* (frame_in, frame_out, support) + device index tables and workspace */

/* Name of a status code.  Never NULL. */
const char* ff_status_string(int status);
/* Detail message of the last failing call on this thread ("" if none). */
const char* ff_last_error(void);
/* ABI version, currently 1. */
int ff_abi_version(void);

/*
 * ff_tff_host -- host construction of the real (k, rho, d) tight fusion frame
 * (Sec. 3.2 construction), any tight case including redundant ones (k rho > d).
 * Writes columns col0 .. col0+ncols-1 (canonical order) of the d x (k rho)
 * matrix P in fp64, row-major d x ncols, into the host buffer `out`.
 * Errors: FF_EINVAL (odd or non-positive sizes, column range outside
 * [0, k rho), out == NULL), FF_ENOTFF (construction not tight).  Needs no GPU.
 */
ff_status ff_tff_host(int64_t d, int64_t k, int64_t rho, int64_t col0, int64_t ncols, double* out);

/*
 * ff_framegen -- generate the frame TFF(k, rho, d) (Algorithm 1, step 2) and
 * place its device form on the current HIP device.  *out receives a new frame
 * (release with ff_frame_destroy).  Errors: FF_EINVAL, FF_ENOTFF,
 * FF_EUNSUPPORTED (a block width 2k outside the supported set above),
 * FF_ENOMEM, FF_EDEVICE.  On error *out is set to NULL.
 */
ff_status ff_framegen(int64_t d, int64_t k, int64_t rho, ff_frame** out);

/*
 * ff_frame_export -- copy back the frame as the kernels use it (fp32 block,
 * read from the device) and expand columns col0 .. col0+ncols-1 of P into
 * the host buffer `out`, fp64 row-major d x ncols.  Synchronises the device.
 */
ff_status ff_frame_export(const ff_frame* f, int64_t col0, int64_t ncols, double* out);

/* Frame geometry: d, k, rho; any pointer may be NULL. */
ff_status ff_frame_info(const ff_frame* f, int64_t* d, int64_t* k, int64_t* rho);

/* Release a frame.  Plans made from it keep it alive until they are destroyed. */
void ff_frame_destroy(ff_frame* f);

/*
 * ff_plan_create -- prepare the coefficient support G of Algorithm 1 (shared
 * by every layer that uses these frames, Sec. 3.3) for repeated calls.
 *   f_in, f_out : frames of the input (n) and output (m) spaces.
 *   nnz         : number of support entries, 0 <= nnz <= (k rho_m)(k rho_n).
 *   rows, cols  : host arrays of nnz canonical indices, rows[e] in [0, k rho_m),
 *                 cols[e] in [0, k rho_n), pairwise distinct ("user order").
 * Coefficient layout.  Algorithm 1 places the coefficient vector into C through
 * G ("rearrange") without fixing the order of the vector; the plan fixes it and
 * may pad it.  Every c_vals and dC array of later calls is a plan-layout array
 * of L = ff_plan_query(FF_Q_COEF_SLOTS) >= nnz fp32 slots: slot j holds the
 * coefficient of support entry user_index[j] as reported by ff_plan_order, or
 * nothing when user_index[j] == -1 (padding).  Padding slots of c_vals must
 * hold zero (as in ELLPACK-style padded formats: the kernels multiply them in);
 * overwriting backward calls set the padding slots of dC to zero and
 * accumulating calls leave them unchanged, so gradient steps keep them zero.  Keep the trainable coefficients in
 * plan layout; convert with c_plan[j] = c_user[user_index[j]] (j not padding)
 * and dC_user[user_index[j]] = dC_plan[j].  The layout follows the kernels'
 * entry streams, so that coefficient reads need no index.
 *   max_tokens  : largest T any later call will pass.
 *   max_batch   : largest `count` of later batched calls (>= 1).
 * Allocates all device workspace here (FF_Q_WORKSPACE_BYTES), whichever activation
 * type the calls will have.  It belongs to one call at a time, and each plan
 * holds its own: plans whose bf16 calls pass a side's coefficients through memory
 * (all but those with FF_Q_FAST128 and those of frames with k rho != d) take 2
 * bytes for every coefficient of the wider side (of both with frames in several
 * radix-4 stages) and token of the longest call of max_batch adapters, up to 128
 * MiB, beside the partial sums of dC.  An MLP projection 4096 <-> 11008 with
 * 50,000 entries and 4096 tokens holds 104 MiB, a 28672 -> 8192 one with 200,000
 * and 8192 tokens 211 MiB: let layers of one shape share a plan (max_batch, or
 * calls one after the other) where their supports agree, and ask for no more
 * tokens than are used where they do not.
 * Errors: FF_EINVAL (range, duplicate entry, null pointer), FF_ENOMEM,
 * FF_EDEVICE.  On error *out is NULL.
 */
ff_status ff_plan_create(const ff_frame* f_in, const ff_frame* f_out, int64_t nnz,
                         const int32_t* rows, const int32_t* cols, int64_t max_tokens,
                         int64_t max_batch, ff_plan** out);

void ff_plan_destroy(ff_plan* p);

/*
 * ff_plan_order -- the plan's coefficient layout: user_index (host array of L =
 * ff_plan_query(FF_Q_COEF_SLOTS) int64) receives, for every slot j, the user
 * index e of the support entry stored there (rows[e], cols[e]), or -1 for a
 * padding slot.  Each e in 0..nnz-1 appears exactly once.
 */
ff_status ff_plan_order(const ff_plan* p, int64_t* user_index);

typedef enum ff_plan_query_key {
    FF_Q_TOKENS_PER_TILE_F32 = 0,   /* tokens per workgroup tile, fp32 activations */
    FF_Q_TOKENS_PER_TILE_BF16 = 1,  /* tokens per workgroup tile, bf16 activations */
    FF_Q_WORKSPACE_BYTES = 2,       /* device workspace held by the plan */
    FF_Q_NNZ = 3,
    FF_Q_FAST128 = 4,               /* 1 if bf16 calls use the fused kernels for 128-wide frame blocks */
    FF_Q_COEF_SLOTS = 5,            /* L: length of every c_vals / dC array (nnz plus padding) */
    FF_Q_SAVED_FLOATS = 6,          /* length of a c_saved array (0: the plan needs none) */
    FF_Q_BWD_TILE_TOKENS = 7,       /* tokens per workgroup tile of the fused 128-wide backward
                                       (16 or 8; 0 without that path) */
    FF_Q_RADIX_IN = 8,              /* 4 if the input frame's block is applied in factored form
                                       (radix-4 stage plus a DFT of size k/4), 1 if densely */
    FF_Q_RADIX_OUT = 9,             /* the same for the output frame */
    FF_Q_GEN_CHUNKS = 10,           /* input-side chunks of a generic-kernel tile (1: the whole
                                       input side at once; more when the support is dense) */
    FF_Q_GEN_TILE_TOKENS_F32 = 11,  /* most tokens per generic-kernel tile with those chunks, fp32 */
    FF_Q_GEN_TILE_TOKENS_BF16 = 12, /* the same, bf16 activations */
    FF_Q_GEN_TOKEN_GROUPS = 13      /* 1 if bf16 forwards on the generic kernels keep four tokens
                                       of a coefficient together in their tiles (frames whose blocks
                                       are applied directly, up to 128 wide, or in one radix-4
                                       stage); their tiles are then a multiple of four tokens */
} ff_plan_query_key;
ff_status ff_plan_query(const ff_plan* p, int key, int64_t* value);

/*
 * ff_adapter_fwd -- Y = beta * Y + scale * P_out C P_in^T x for the T token rows
 * of X (Sec. 3.1 update equation applied to an input).
 *   act      : FF_F32 or FF_BF16, dtype of X and Y.
 *   X        : device, T x n, leading dimension ldx >= n.
 *   c_vals   : device, L fp32 coefficient slots in plan layout (ff_plan_order),
 *              16-byte aligned.
 *   scale    : s = alpha / sqrt(m n), passed by the caller.
 *   beta     : 0 overwrites Y (Y is not read), otherwise Y is read and scaled.
 *   Y        : device, T x m, leading dimension ldy >= m.
 * T = 0 is a no-op.  Errors: FF_EINVAL (T > max_tokens, bad pointers,
 * dimensions or alignment), FF_EDEVICE (launch failure).
 */
ff_status ff_adapter_fwd(const ff_plan* p, int64_t T, int act, const void* X, int64_t ldx,
                         const float* c_vals, float scale, float beta, void* Y, int64_t ldy,
                         void* stream);

/*
 * ff_adapter_bwd -- backward of ff_adapter_fwd for upstream gradient G (T x m):
 *   dX = beta_dx * dX + scale * P_in C^T P_out^T g       (skipped if dX == NULL)
 *   dC = [dC +] scale * sum_t u_t[rows[e]] z_t[cols[e]],  u = P_out^T g, z = P_in^T x
 *        (Appendix A, grad f(C) = P_m^T grad f(W) P_n; skipped if dC == NULL;
 *        added to the existing dC when accumulate_dc != 0, else overwritten)
 * X may be NULL when dC == NULL.  dC is fp32, L slots in plan layout
 * (padding slots zeroed, or unchanged when accumulating), and is reduced
 * deterministically (same inputs give bitwise-equal dC).  c_vals is in plan
 * layout.
 */
ff_status ff_adapter_bwd(const ff_plan* p, int64_t T, int act, const void* X, int64_t ldx,
                         const void* G, int64_t ldg, const float* c_vals, float scale,
                         float beta_dx, void* dX, int64_t lddx, int accumulate_dc, float* dC,
                         void* stream);

/*
 * ff_adapter_bwd_noalloc -- ff_adapter_bwd for callers that cannot allocate
 * device memory or use a plan's workspace (code under HIP graph capture, tight
 * serving loops, harnesses that forbid allocation).  Arguments, results
 * (bitwise those of ff_adapter_bwd) and errors are those of ff_adapter_bwd;
 * the backward's scratch (the coefficients in its own order, the dC partial
 * sums and, where the coefficients of a side pass through memory, those of some
 * tokens at a time) lives instead in a 96 MiB array that the library's code object
 * holds on every device it runs on, until the process ends.  Nothing is allocated
 * and no memset node is issued: the scratch is cleared by a fill kernel where
 * it must start at zero.
 *   Limit: a call needing more than 32 MiB of coefficients and partial sums
 *   (a row of them per tile, at most one per compute unit on the generic
 *   kernels) returns FF_EINVAL and writes nothing (the q_proj layer, 4096 x 4096
 *   with 10,000 coefficients, needs about 13 MB at 4096 bf16 tokens); split the
 *   tokens over several calls with accumulate_dc = 1.
 *   All calls on one device share that array: calls that overlap in time on
 *   one device (different streams, threads or processes' streams without an
 *   ordering between them) race and give undefined results.
 */
ff_status ff_adapter_bwd_noalloc(const ff_plan* p, int64_t T, int act, const void* X, int64_t ldx,
                                 const void* G, int64_t ldg, const float* c_vals, float scale,
                                 float beta_dx, void* dX, int64_t lddx, int accumulate_dc, float* dC,
                                 void* stream);

/*
 * ff_adapter_fwd_save / ff_adapter_bwd_saved -- the forward and backward of a
 * training step that uses the same coefficients in both.  The forward also
 * writes c_saved: the coefficients in the backward's own slot order, which the
 * backward otherwise rebuilds from c_vals with a reordering pass of its own.
 *   c_saved : device, ff_plan_query(FF_Q_SAVED_FLOATS) fp32, 16-byte aligned,
 *             owned by the caller; one per adapter, since a plan is shared by
 *             many layers.  Its contents are opaque.
 * ff_adapter_bwd_saved takes the c_saved written by ff_adapter_fwd_save with
 * the same c_vals, which must not change in between; otherwise the arguments,
 * results and errors are those of ff_adapter_fwd / ff_adapter_bwd.  The saved
 * copy is used by bf16 calls on plans that report FF_Q_FAST128; elsewhere
 * FF_Q_SAVED_FLOATS is 0, c_saved may be NULL and the calls are the plain ones.
 */
ff_status ff_adapter_fwd_save(const ff_plan* p, int64_t T, int act, const void* X, int64_t ldx,
                              const float* c_vals, float scale, float beta, void* Y, int64_t ldy,
                              float* c_saved, void* stream);
ff_status ff_adapter_bwd_saved(const ff_plan* p, int64_t T, int act, const void* X, int64_t ldx,
                               const void* G, int64_t ldg, const float* c_vals, const float* c_saved,
                               float scale, float beta_dx, void* dX, int64_t lddx, int accumulate_dc,
                               float* dC, void* stream);

/*
 * ff_merge_delta -- W = beta * W + scale * P_out C P_in^T (Algorithm 1, steps
 * 5-6; with scale < 0 it un-merges: the adapter hot-swap of Sec. 3.4, "Storage efficiency").  W: device,
 * m x n row-major with leading dimension ldw >= n, dtype w_dtype.  beta = 0
 * writes the dense delta dW without reading W.
 */
ff_status ff_merge_delta(const ff_plan* p, const float* c_vals, float scale, int w_dtype,
                         float beta, void* W, int64_t ldw, void* stream);

/*
 * Plan groups -- adapters that share one frame pair but each have their own
 * support of C, run together: per-layer random masks (Sec. 4.6, the sparsity
 * pattern ablation compares one mask shared across layers with a mask per
 * layer) and multi-tenant serving, where one backbone carries many users'
 * adapters that are hot-swapped or applied per request (Sec. 3.4, "Storage
 * efficiency").
 *   ff_plan_group_create : plans[i] (host array of `count` distinct plans)
 *       serves adapter i.  All plans must use the same two frame objects and
 *       the same kernel path (FF_Q_FAST128 and the generic tile geometry
 *       agree whenever the supports have similar sizes; FF_Q_BWD_TILE_TOKENS
 *       may differ); otherwise FF_EUNSUPPORTED.  The plans must outlive the group,
 *       and a plan in a group must not be used by another call concurrently
 *       (group calls use the plan's own workspace).  Allocates a small device
 *       table.  Errors: FF_EINVAL, FF_EUNSUPPORTED, FF_ENOMEM, FF_EDEVICE.
 *   ff_adapter_fwd_group / ff_adapter_bwd_group : ff_adapter_fwd_batched /
 *       ff_adapter_bwd_batched with adapter i running plans[i]: c_vals[i] and
 *       dC[i] are in plans[i]'s layout.  T (<= every plan's max_tokens) sizes
 *       the launch; `tokens`, if not NULL, is a DEVICE array of `count` int32
 *       token counts (each clamped to [0, T]) so that requests of different
 *       lengths share a launch: adapter i then reads and writes only its first
 *       tokens[i] rows (dC sums over those rows; 0 rows give dC = 0).
 *   Results per adapter equal those of the single calls on its own plan: bit for
 *   bit on plans that report FF_Q_FAST128, and
 *   elsewhere up to the rounding of the activation type, since the kernels that
 *   take a bf16 call depend on its number of tokens there.
 */
typedef struct ff_plan_group ff_plan_group;
ff_status ff_plan_group_create(int64_t count, const ff_plan* const* plans, ff_plan_group** out);
void ff_plan_group_destroy(ff_plan_group* g);
ff_status ff_adapter_fwd_group(const ff_plan_group* g, int64_t T, const int32_t* tokens, int act,
                               const void* const* X, int64_t ldx, const float* const* c_vals, float scale,
                               float beta, void* const* Y, int64_t ldy, void* stream);
ff_status ff_adapter_bwd_group(const ff_plan_group* g, int64_t T, const int32_t* tokens, int act,
                               const void* const* X, int64_t ldx, const void* const* G, int64_t ldg,
                               const float* const* c_vals, float scale, float beta_dx, void* const* dX,
                               int64_t lddx, int accumulate_dc, float* const* dC, void* stream);

/*
 * ff_coef_to_plan / ff_coef_to_user -- move a coefficient vector between the
 * caller's support order (entry e at (rows[e], cols[e]) as passed to
 * ff_plan_create) and the plan layout of every c_vals / dC argument; this is
 * the "rearrange" of Algorithm 1, step 4, run on the device so that a training
 * loop can keep C and dC in its own order without host round trips.
 *   ff_coef_to_plan : c_plan[j] = c_user[user_index[j]], and 0 in padding slots
 *                     (user_index as reported by ff_plan_order).
 *                     c_user: device, nnz fp32, 4-byte aligned.
 *                     c_plan: device, ff_plan_query(FF_Q_COEF_SLOTS) fp32, 16-byte aligned.
 *   ff_coef_to_user : c_user[e] = c_plan[slot of e], or c_user[e] += that value
 *                     when accumulate != 0 (gradient accumulation in user order).
 * Both run asynchronously on `stream`, allocate nothing, and need the two
 * arrays not to overlap.  Errors: FF_EINVAL (NULL, misaligned or overlapping
 * arrays, wrong device), FF_EDEVICE (launch failure).
 */
ff_status ff_coef_to_plan(const ff_plan* p, const float* c_user, float* c_plan, void* stream);
ff_status ff_coef_to_user(const ff_plan* p, const float* c_plan, float* c_user, int accumulate, void* stream);

/*
 * Batched forms for many adapters that share frames and support but own their
 * activations and coefficient values (one layer stack).  X, Y, G, dX, c_vals
 * and dC are DEVICE arrays of `count` device pointers (1 <= count <=
 * max_batch); every other argument is shared.  Semantics per adapter are those
 * of the single calls, including the alignment of each pointer (the pointed-to
 * arrays cannot be checked from the host: misaligned pointers are undefined
 * behaviour).  dX / dC arrays may be NULL to skip that output.
 */
ff_status ff_adapter_fwd_batched(const ff_plan* p, int64_t count, int64_t T, int act,
                                 const void* const* X, int64_t ldx, const float* const* c_vals,
                                 float scale, float beta, void* const* Y, int64_t ldy,
                                 void* stream);
ff_status ff_adapter_bwd_batched(const ff_plan* p, int64_t count, int64_t T, int act,
                                 const void* const* X, int64_t ldx, const void* const* G,
                                 int64_t ldg, const float* const* c_vals, float scale,
                                 float beta_dx, void* const* dX, int64_t lddx, int accumulate_dc,
                                 float* const* dC, void* stream);

/*
 * ff_adamw_step -- one AdamW step on a coefficient vector (the optimizer the
 * paper trains C with, Appendix G): decoupled weight decay, then the
 * bias-corrected Adam step, at step number `step` (1 for the first):
 *     c <- c (1 - lr weight_decay)
 *     m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2
 *     c <- c - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * c, m, v (updated in place) and g are device fp32 arrays of n elements,
 * 4-byte aligned (16-byte aligned ones move in 16-byte accesses); any common
 * layout works, so plan-layout arrays (c_vals, dC) can be stepped directly:
 * their padding slots hold zeros and stay zero.  m and v start at zero.
 * Asynchronous on `stream`; allocates nothing.  Errors: FF_EINVAL (NULL or
 * misaligned array, step < 1, betas outside [0, 1), eps <= 0, negative or
 * non-finite lr / weight_decay), FF_EDEVICE.
 */
ff_status ff_adamw_step(int64_t n, float* c, const float* g, float* m, float* v, float lr, float beta1,
                        float beta2, float eps, float weight_decay, int64_t step, void* stream);
/* The same for `count` equally long vectors (one layer stack) in one launch: c, g, m,
 * v are DEVICE arrays of `count` device pointers, each 16-byte aligned. */
ff_status ff_adamw_step_batched(int64_t count, int64_t n, float* const* c, const float* const* g,
                                float* const* m, float* const* v, float lr, float beta1, float beta2,
                                float eps, float weight_decay, int64_t step, void* stream);
/*
 * ff_adamw_set -- the same step for tensors of any lengths at once (adapters with supports of their own, norm vectors, whole
 * weights), with gradients in fp32 or bf16, a decay for each tensor, and the moments in fp32 or in 8 bits.
 *   ff_adamw_set_create : a set of `count` tensors (at most 2^20); every array is a HOST array of `count` entries, read in the call.
 *     n            : lengths, 0 <= n[i] <= 2^40.
 *     c            : device, fp32 parameters, n[i] each, 4-byte aligned.
 *     copy         : device, bf16 copies of the parameters that a step writes (rounded to nearest), 2-byte aligned; the array or
 *                    entries of it may be NULL.
 *     m, v         : device, moments: n[i] fp32, 4-byte aligned (FF_STATES_F32), or n[i] bytes (FF_STATES_8BIT).
 *     m_exp, v_exp : device, ceil(n[i] / 256) bytes each (FF_STATES_8BIT; else NULL).
 *     All zeros are the states of a first step, of either kind.  The memory stays the caller's and must outlive the set; no two of
 *     these arrays may overlap.
 *     weight_decay : host, per tensor, or NULL for zeros.
 *     Allocates a table on the current device (64 bytes a tensor, 8 for 4096 elements) and copies it there; on error *out is NULL.
 *   ff_adamw_set_step : one step of every tensor whose gradient is not NULL.
 *     g : HOST array of `count` device pointers, gradients of type g_dtype, element aligned, outside of what the set writes; read in
 *         the call, so that a captured step keeps the addresses of its capture.
 *     The hyperparameters are those of ff_adamw_step; gradients are multiplied by grad_scale.  lr_dev, grad_scale_dev (fp32)
 *     and step_dev (int64) are NULL or one device value each, read when the call runs: factors of lr and grad_scale, and an
 *     addend of step (the sum must be at least 1), for captured steps that are replayed.
 *   ff_adamw_set_read : the values of 8-bit moments in bf16, which holds them exactly (but for 2^128, to which a moment just
 *     below it may be rounded, and which reads as infinity): m[i], v[i] (HOST arrays of device
 *     pointers, NULL to skip one) receive n[i] values and zeros up to the next multiple of 256.
 * 8-bit moments: each block of 256 elements of a tensor has a unit 2^(m_exp - 120); the code a (of v: the byte; of m: its low 7
 * bits, bit 7 the sign) stands for a units below 16 and (8 + a mod 8) 2^(a div 8 - 1) from there on.  A step takes the block's
 * exponent as small as its largest new moment (in fp32) allows, at least 0, and rounds each moment up or down at random, with
 * probabilities in proportion, where a random fraction carries it over the next code: (h + 1/2) / 65536 with h the low (m) or high
 * (v) half of word i mod 4 of Philox 4x32-10 with counter (i / 4 (64 bits), low 32 bits of step, number of the tensor) and key seed.
 * A v > 0 has a code of at least 1; where a moment is not finite in fp32, both of the element become 0.  The parameters are stepped with the
 * moments before their rounding; moments and their place between codes are computed in fp64.
 * fp32 moments are made in fp64 and rounded to nearest once a step: a change below half a unit in a moment's last place, as the decay of v
 * alone is for beta2 above 1 - 2^-25, leaves it as it is.
 * Calls on one set must be ordered, and a graph that holds one must not be replayed after the set's destruction (its table is freed).
 * Steps and reads are asynchronous on `stream` and allocate nothing; equal inputs give equal bits.
 * Errors: FF_EINVAL, FF_ENOMEM, FF_EDEVICE; after FF_EDEVICE some tensors may have been stepped.
 */
enum { FF_STATES_F32 = 0, FF_STATES_8BIT = 1 };
typedef struct ff_adamw_set ff_adamw_set;
typedef struct ff_adamw_hyper {
    double lr, beta1, beta2, eps, grad_scale;
    int64_t step;
    uint64_t seed;
    const float* lr_dev;
    const float* grad_scale_dev;
    const int64_t* step_dev;
} ff_adamw_hyper;
ff_status ff_adamw_set_create(int64_t count, const int64_t* n, int states, int g_dtype, float* const* c, void* const* copy,
                              void* const* m, void* const* v, uint8_t* const* m_exp, uint8_t* const* v_exp,
                              const double* weight_decay, ff_adamw_set** out);
void ff_adamw_set_destroy(ff_adamw_set* s);
ff_status ff_adamw_set_step(const ff_adamw_set* s, const void* const* g, const ff_adamw_hyper* h, void* stream);
ff_status ff_adamw_set_read(const ff_adamw_set* s, void* const* m, void* const* v, void* stream);
/* Learning rate of optimizer step `step` (0 for the first) under the linear schedule
 * with warmup of Appendix G: base_lr * step / warmup during the warmup, then falling
 * linearly to 0 at step `total`.  Host function. */
double ff_lr_linear_warmup(int64_t step, int64_t warmup, int64_t total, double base_lr);

/*
 * Operators around the adapter in a training step: layer norm, the join of two blocks, dropout, the gated feed-forward and the
 * loss of the head.  They need no
 * frame and no plan.  Activations are T rows of n elements of type `act` as above, row t at X + t ldx.  The calls are
 * asynchronous on `stream`, allocate nothing, synchronise nothing and may be captured into a graph.  A call that returns
 * FF_EINVAL has written nothing; after FF_EDEVICE (a launch failed) calls that launch several kernels (the backwards and the
 * loss) may have written some of their outputs.  Equal inputs give equal bits.  A workspace belongs to
 * the call until it has run: calls that overlap in time need one each.  Outputs must not overlap inputs or the
 * workspace except where it is said.
 */

/*
 * ff_layernorm_fwd -- y = weight (x - mean) rstd + bias for each row x, rstd = 1 / sqrt(var + eps) with the row's
 * variance over n (not n - 1).  Sums are in fp32, the variance from the centred row.
 *   X, Y         : device, element alignment, any leading dimension >= n.  Y may be X.
 *   weight, bias : device, n elements of type w_dtype; NULL for ones / zeros.
 *   mean, rstd   : device, T fp32 each, for the backward; NULL where not wanted.
 * T = 0 is a no-op.
 */
ff_status ff_layernorm_fwd(int64_t T, int64_t n, int act, const void* X, int64_t ldx, int w_dtype, const void* weight,
                           const void* bias, float eps, void* Y, int64_t ldy, float* mean, float* rstd, void* stream);
/*
 * ff_layernorm_bwd -- with h = (x - mean) rstd, g a row of G and a = weight g:
 *   dX      = beta_dx dX + rstd (a - mean(a) - h mean(a h))     (skipped if dX == NULL; beta_dx = 0 does not read it)
 *   dweight = [dweight +] sum_t g h,   dbias = [dbias +] sum_t g  (fp32, n each; either may be NULL; added to what is
 *             there when accumulate_dw != 0)
 *   mean, rstd : as ff_layernorm_fwd wrote them.
 *   workspace  : device, 16-byte aligned, at least ff_layernorm_workspace bytes; may be NULL without dweight and dbias.
 * With T = 0 dweight and dbias become zero (or stay, accumulating).
 */
ff_status ff_layernorm_workspace(int64_t T, int64_t n, int64_t* bytes);
ff_status ff_layernorm_bwd(int64_t T, int64_t n, int act, const void* X, int64_t ldx, const void* G, int64_t ldg,
                           int w_dtype, const void* weight, const float* mean, const float* rstd, float beta_dx, void* dX,
                           int64_t lddx, int accumulate_dw, float* dweight, float* dbias, void* workspace,
                           int64_t workspace_bytes, void* stream);

/*
 * ff_resnorm_* -- what stands between two blocks: the residual stream r takes a block's output b, through a norm after the block,
 * a gate and the scales of both, and the next block's norm reads the result, in one pass:
 *   p = post(b),   x = res_scale r + block_scale gate p,   y = norm(x)
 *   post, norm : FF_NORM_NONE, FF_NORM_RMS (v / sqrt(mean v^2 + eps)) or FF_NORM_LAYER (as ff_layernorm_fwd), each times its
 *                weight plus its bias (post_weight, post_bias; weight, bias: device, n elements of type w_dtype, NULL for ones /
 *                zeros; those of a norm that is not there are not looked at).
 *   gate       : device, `groups` rows of n elements of type gate_dtype, leading dimension ldgate (not looked at with one row);
 *                row i holds for the rows i T / groups to (i + 1) T / groups - 1, groups divides T.  NULL: ones (groups is not
 *                looked at).
 * ff_resnorm_fwd : R, B -> X (x; may be R) and Y (y; NULL without a norm).  stats: device, 16-byte aligned, T x 4 fp32 for the
 *   backward (mean and 1 / deviation of b, then of x; the mean of an RMS norm is 0, and both of a norm that is not there);
 *   NULL where not wanted.  y is that of x before its rounding.  T = 0 is a no-op.
 * ff_resnorm_bwd : from R and B as the forward read them (x is made again), the gradient dX of x from what else reads the stream
 *   (NULL: zero) and dY of y (not looked at without a norm), with D = dX + the norm's gradient of x:
 *     dR = res_scale D,   dB = gradient of p = block_scale gate D through post   (NULL to skip one; each may be any of R, B, dX,
 *                         dY with its leading dimension, but not both the same)
 *     dgate        = [dgate +] block_scale sum over a gate row's rows of D p     (fp32, groups x n, contiguous)
 *     dpost_weight, dpost_bias, dweight, dbias = [... +] the norms' vectors' gradients   (fp32, n each)
 *   Any of the five may be NULL; they are added to what is there when accumulate != 0.  With T = 0 they become zero (or stay).
 *   No two may share memory (a vector that two norms share takes the sum of two results).
 *   workspace : device, 256-byte aligned, at least ff_resnorm_workspace bytes for the same T, n and groups (1 without a gate).
 * X, Y, R, B, dX, dY, dR, dB: element alignment, any leading dimension >= n.  Sums and statistics are fp32.
 */
enum { FF_NORM_NONE = 0, FF_NORM_RMS = 1, FF_NORM_LAYER = 2 };
typedef struct ff_resnorm {
    int64_t T, n;
    int act, w_dtype, gate_dtype;
    int post, norm;
    const void* post_weight;
    const void* post_bias;
    const void* weight;
    const void* bias;
    const void* gate;
    int64_t ldgate, groups;
    float res_scale, block_scale, post_eps, eps;
} ff_resnorm;
ff_status ff_resnorm_fwd(const ff_resnorm* d, const void* R, int64_t ldr, const void* B, int64_t ldb, void* X, int64_t ldx,
                         void* Y, int64_t ldy, float* stats, void* stream);
ff_status ff_resnorm_workspace(int64_t T, int64_t n, int64_t groups, int64_t* bytes);
ff_status ff_resnorm_bwd(const ff_resnorm* d, const void* R, int64_t ldr, const void* B, int64_t ldb, const void* dX,
                         int64_t lddx, const void* dY, int64_t lddy, const float* stats, void* dR, int64_t lddr, void* dB,
                         int64_t lddb, int accumulate, float* dgate, float* dpost_weight, float* dpost_bias, float* dweight,
                         float* dbias, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * ff_dropout -- y = [r +] m x / (1 - p') for each element, m in {0, 1} from a counter-based generator: a function of
 * (seed, offset, row, column, n) alone, so that the mask is never stored and the backward pass is this call on the
 * gradient with the same seed and offset (R then the gradient of another path, or NULL).
 *   p          : share of elements to drop, 0 <= p <= 1.  p' = D / 65536 with D = p 65536 rounded to nearest (at most
 *                65535 for p < 1); kept elements are scaled by 65536 / (65536 - D).  p = 1 drops all.
 *   seed       : key of the generator, any 64 bits.   offset : number of the draw (another for every layer and step).
 *   offset_dev : device, one uint64 added to offset when the call runs, or NULL: a captured step whose graph is
 *                replayed draws another mask when the program changes that value.
 *   R          : device, T x n of type act, added after scaling, or NULL.
 *   X, Y, R    : element alignment, any leading dimension >= n; Y may be X or R.
 * T is at most 2^40, n at most 2^28, T ceil(n / 8) at most 2^44.
 * The mask: block b = t ceil(n / 8) + i / 8 of eight elements of row t takes the four 32-bit words of Philox 4x32-10 with
 * counter (b, offset), low words first, and key seed; element i takes the 16 bits number i mod 8 of them, the low half
 * of a word first, and is dropped where they are below D.
 */
ff_status ff_dropout(int64_t T, int64_t n, int act, const void* X, int64_t ldx, double p, uint64_t seed, uint64_t offset,
                     const uint64_t* offset_dev, const void* R, int64_t ldr, void* Y, int64_t ldy, void* stream);

/*
 * ff_glu_* -- a gated feed-forward block up to its down projection, both projections, the function and the product in one kernel:
 *   G = X Wg^T [+ Ag],   U = X Wu^T [+ Au],   H = f(G) U
 *   fn     : f, FF_GLU_SILU (g / (1 + exp -g)), FF_GLU_GELU (g times the normal distribution's integral up to g) or FF_GLU_GELU_TANH
 *            (g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2).
 *   X      : device, T x n;  Wg, Wu : device, F x n, one leading dimension ldw (halves of one weight, or two);
 *   Ag, Au : device, T x F, one leading dimension lda: what adapters on the projections add (ff_adapter_fwd on X); each may be NULL.
 *   H      : device, T x F.   G, U : device, T x F, one leading dimension ldg, kept for the backward; NULL to keep nothing.  fp32 for
 *            FF_F32; for FF_BF16 words of 16 bits that hold ten significant ones: from the highest bit on a sign, 6 bits of exponent
 *            (bias 37, 0 for subnormals) and 9 of mantissa, so that values from 1.5e-11 to 6.7e7 keep their digits; larger ones
 *            become infinite (a NaN the positive infinity).
 * ff_glu_bwd, from the gradient dH (T x F) of H:
 *   dU = dH f(G),   dG = dH U f'(G)                (T x F, one leading dimension lddg; also what the adapters' backwards take)
 *   dX = beta_dx dX + dG Wg + dU Wu                (skipped if NULL)
 *   dWg = beta_dw dWg + dG^T X,   dWu likewise     (F x n, one leading dimension lddw; skipped if both are NULL)
 *   G, U : as the forward kept them; X is then read for dWg and dWu alone, the weights for dX.  Without them (NULL) G and U
 *          are made again from X, the weights, Ag and Au, as the forward had them before their rounding.
 *          Where a word is infinite, what does not depend on the value it stands for is as it should be (f' is 1 or 0, f of a large
 *          negative G is 0, dH = 0 gives 0), and dH U and dH f(G) of the others are infinite.
 *   dG or dU may be dH, and dG may be G, dU may be U, with the same leading dimension.  beta = 0 does not read the output.
 *   workspace : device, 256-byte aligned, at least ff_glu_workspace bytes for the same T, n, F, act and the outputs wanted
 *          (FF_GLU_DX, FF_GLU_DW or both); not looked at without them.  It holds fp32 partial sums of products with few results.
 * All matrices but G and U of type act; n and F multiples of 8 (bf16) or 4 (fp32), at most 262144, T at most 2^28; 16-byte aligned, leading
 * dimensions multiples of 8 (4), at most 1048576.  Products accumulate in fp32; H, G, U, dG, dU, dX and the weights' gradients are
 * rounded once each (G and U as they are kept), and the products of the backward read dG and dU so.  Weights, X, dH, Ag and Au must be finite.
 * T = 0 writes nothing but dWg = beta_dw dWg and dWu.
 */
enum { FF_GLU_SILU = 0, FF_GLU_GELU = 1, FF_GLU_GELU_TANH = 2 };
enum { FF_GLU_DX = 1, FF_GLU_DW = 2 };
ff_status ff_glu_fwd(int64_t T, int64_t n, int64_t F, int act, int fn, const void* X, int64_t ldx, const void* Wg,
                     const void* Wu, int64_t ldw, const void* Ag, const void* Au, int64_t lda, void* H, int64_t ldh, void* G,
                     void* U, int64_t ldg, void* stream);
ff_status ff_glu_workspace(int64_t T, int64_t n, int64_t F, int act, int want, int64_t* bytes);
ff_status ff_glu_bwd(int64_t T, int64_t n, int64_t F, int act, int fn, const void* dH, int64_t lddh, const void* X, int64_t ldx,
                     const void* Wg, const void* Wu, int64_t ldw, const void* Ag, const void* Au, int64_t lda, const void* G,
                     const void* U, int64_t ldg, void* dG, void* dU, int64_t lddg, float beta_dx, void* dX, int64_t lddx,
                     float beta_dw, void* dWg, void* dWu, int64_t lddw, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * ff_xent_* -- cross entropy of a head's logits z = H W^T over a vocabulary of V entries, without keeping the logits:
 *   lse_t  = log sum_v exp z_tv,   loss_t = lse_t - z_t,target[t]
 *   P_tv   = (exp(z_tv - lse_t) - [v = target[t]]) dloss[t]
 *   dH     = beta_dh dH + scale P W,     dW = beta_dw dW + scale P^T H
 * A token whose target lies outside [0, V) has none: its loss is 0, its row of P is 0 whatever H holds, its lse is
 * still that of its logits.
 *   H, dH  : device, T x n of type act, W, dW : device, V x n of type act; n a multiple of 8 (bf16) or 4 (fp32), 16-byte
 *            aligned, leading dimensions multiples of 8 (4), at most 1048576.  beta = 0 does not read the output.
 *            The gradients multiply W by P and need it finite: an entry is switched off by a logit of the type's lowest
 *            value; minus infinity works for the loss alone.
 *   target : device, T int64.   loss, lse : device, T fp32.
 *   dloss  : device, T fp32, gradient of the result with respect to each token's loss; NULL for ones.
 *            `scale` multiplies the gradients (1 / counted tokens for a mean): P's rounding to bf16 is smallest where
 *            the weight of all tokens is in scale, or in a factor on the results, and dloss is NULL.
 *   workspace : device, 256-byte aligned, at least ff_xent_workspace bytes for the same T, n, V, act and the outputs wanted
 *            (FF_XENT_DH, FF_XENT_DW or both; 0: loss alone).  It holds P, in type act, for a piece of the tokens or of
 *            the vocabulary (at most 256 MiB, or 256 tokens where a longer piece of them is larger; with dW, 256 entries
 *            of all tokens where that is larger), fp32 partial sums of dH, and with dW a copy of H (two up to 128 tokens
 *            in bf16).
 * ff_xent_fwd  : loss and lse.
 * ff_xent_step : loss, lse and the gradients in one call, which computes the logits once (twice with dW where P does not
 *                fit one piece).
 * ff_xent_bwd  : the gradients from the lse of an earlier ff_xent_fwd on the same H, W: for programs that know dloss only
 *                after it.  It computes the logits again.  loss may be NULL; with the loss of that call the target's
 *                P keeps its digits where its probability is near one, as in ff_xent_step (from lse alone it carries
 *                lse's rounding).
 * dH == NULL or dW == NULL skips that output.  Arithmetic: products accumulate in fp32, softmax statistics are fp32, P is
 * rounded to type act before the products that read it (in ff_xent_step with bf16, after exp(z - max) was
 * rounded to fp16; up to 128 tokens in bf16, P is kept as the sum of two roundings).
 * With T = 0, dW = beta_dw dW.  V is at most 2^24 for the loss alone, 2^22 with a gradient.
 */
enum { FF_XENT_DH = 1, FF_XENT_DW = 2 };
ff_status ff_xent_workspace(int64_t T, int64_t n, int64_t V, int act, int want, int64_t* bytes);
ff_status ff_xent_fwd(int64_t T, int64_t n, int64_t V, int act, const void* H, int64_t ldh, const void* W, int64_t ldw,
                      const int64_t* target, float* loss, float* lse, void* workspace, int64_t workspace_bytes,
                      void* stream);
ff_status ff_xent_bwd(int64_t T, int64_t n, int64_t V, int act, const void* H, int64_t ldh, const void* W, int64_t ldw,
                      const int64_t* target, const float* lse, const float* loss, const float* dloss, float scale,
                      float beta_dh, void* dH, int64_t lddh, float beta_dw, void* dW, int64_t lddw, void* workspace,
                      int64_t workspace_bytes, void* stream);
ff_status ff_xent_step(int64_t T, int64_t n, int64_t V, int act, const void* H, int64_t ldh, const void* W, int64_t ldw,
                       const int64_t* target, const float* dloss, float scale, float* loss, float* lse, float beta_dh,
                       void* dH, int64_t lddh, float beta_dw, void* dW, int64_t lddw, void* workspace,
                       int64_t workspace_bytes, void* stream);

/*
 * ff_time_next_kernel -- instrumentation for benchmarks.  Arms this thread so
 * that the next hot-path call records the hipEvent_t `ev_start` just before and
 * `ev_stop` just after its main kernel (the fused forward, the fused backward,
 * or the merge), on that call's stream; the arming is then cleared.  Where a call
 * passes a side's coefficients through memory, that is the launches from the first
 * analysis to the last synthesis, two to four for every part that the call is split
 * into.  The reordering of the coefficients and the reduction of dC lie outside.
 * Passing NULL for both disarms.  Results are unaffected.
 */
ff_status ff_time_next_kernel(void* ev_start, void* ev_stop);

#ifdef __cplusplus
}
#endif

#endif /* FRAMEFT_H */
