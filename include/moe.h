/*
 * moe.h - C ABI of the MI355X (gfx950) MoE-layer library.
 *
 * One Mixture-of-Experts layer's forward pass, as defined in the paper's Sec. 2.1 (its training operators and low-rank adapters follow at the end):
 *   Eq. 1   s = softmax(W_r x)
 *   Eq. 2   T = top-k(s) = {(e_i, w_i)}
 *   Eq. 3   y = sum_i w_i * FFN_{e_i}(x)
 *   Eq. 4   FFN_e(x) = (SiLU(x W_gate_e) (.) x W_up_e) W_down_e
 * executed as the five stages of Sec. 3.1: route, permute into expert-contiguous
 * order (Sec. 3.5), fused gate+up grouped GEMM (Sec. 3.2-3.3), down grouped GEMM,
 * weighted un-permute / combine (Sec. 3.5, Eq. 3).
 *
 * Conventions common to every entry point
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The library never
 *     allocates, frees or keeps a pointer beyond the work it enqueues.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls only
 *     enqueue kernels; they never synchronise.  The caller keeps all buffers alive until
 *     the stream has drained.  No host<->device copy happens anywhere.
 *   - bf16 tensors are uint16 bit patterns, row-major, base pointer 16-byte aligned.
 *   - Stored weight matrices are [out, in] with the reduction dimension contiguous
 *     (Sec. 3.2's "E*N x K" flattened layout): W_r [E,d], W_gate,W_up [E,F,d], W_down [E,d,F].
 *     Eq. 4's "x W" is therefore x times the transpose of the stored matrix.
 *   - Notation: T tokens, d model dim, F expert FFN dim, E experts, k experts per token,
 *     R = T*k expanded rows, n_e rows routed to expert e.
 *   - Limits: 1 <= k <= E <= 256, d % 64 == 0, F % 64 == 0, T >= 0, T*k <= 2^30, and the
 *     activation buffers (x, x_perm, h: T*k*max(d,F) elements of 2 bytes) below 4 GiB: the GEMM
 *     kernels address their rows with 32-bit byte offsets.  Beyond: MOE_ERR_UNSUPPORTED.
 *     T == 0 returns MOE_OK and enqueues nothing (but moe_grouped_ffn_backward and moe_route_backward: gradients of weights
 *     of zero are written; and moe_dispatch: counts and offsets of zero).
 *   - Stream capture: the calls record kernel launches only and may be captured into a HIP
 *     graph; replays equal the eager result.  The first use of a GEMM kernel in a process sets
 *     a function attribute (its LDS size), which HIP does not allow during capture: run the
 *     call once eagerly with the same configuration before capturing it.
 *   - All argument checks run on the host before anything is enqueued: a call that returns
 *     an error has had no effect on device memory.  Errors are return codes only.
 */
#ifndef MOE_H_
#define MOE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MOE_OK = 0,
    MOE_ERR_NULL = -1,        /* a required pointer is NULL */
    MOE_ERR_SHAPE = -2,       /* T<0, k<1, k>E, E<1, d<1, F<1, unknown gating */
    MOE_ERR_ALIGN = -3,       /* a tensor base pointer is not 16-byte aligned (or a buffer not as far as its entry point asks) */
    MOE_ERR_WORKSPACE = -4,   /* workspace smaller than the matching *_workspace_size() */
    MOE_ERR_UNSUPPORTED = -5, /* E > 256, d % 64 != 0, F % 64 != 0, T*k > 2^30, or T*k*max(d,F)*2 bytes >= 4 GiB; further limits stand with the training and adapter operators */
    MOE_ERR_HIP = -6          /* a kernel launch reported a HIP error */
} moe_status;

typedef enum {
    MOE_GATE_SOFTMAX = 0,        /* w_i = softmax(z)[e_i]                      (Eq. 1-2) */
    MOE_GATE_SOFTMAX_RENORM = 1, /* w_i = softmax(z)[e_i] / sum_j softmax(z)[e_j]        */
    MOE_GATE_SIGMOID_NORM = 2    /* w_i = sigmoid(z_{e_i}) / sum_j sigmoid(z_{e_j})  (Sec. 3.4) */
} moe_gating;

/* moe_config.flags */
/* moe_forward folds the weighted combine (Eq. 3) into the down projection instead of launching
 * it as a fifth kernel (the paper's limitation 1): the workgroup that writes the last of a token's
 * k expert rows sums them, in slot order, from the bf16 rows in memory, so y is bit-identical to
 * moe_combine's whichever workgroup arrives last.  One launch fewer per layer; the GEMM
 * workgroups pay for it with latency-bound reads at their end, which costs more than the launch
 * it saves once T*k exceeds a few hundred rows (measured), so it is off unless asked for.
 * Needs packed weights and more than a handful of rows (the kernels that serve row-major weights
 * and the K-split kernel have no such epilogue): otherwise the flag is ignored. */
#define MOE_FLAG_FUSE_COMBINE 1

typedef struct {
    int32_t T, d, F, E, k;
    int32_t gating;       /* moe_gating */
    int32_t tile_m;       /* rows per block-schedule tile (Alg. 1's M); 0 = chosen from T*k/E */
    int32_t flags;        /* bit set of MOE_FLAG_*; unknown bits are refused (MOE_ERR_SHAPE) */
} moe_config;

/* Byte offsets of moe_forward's intermediates inside its workspace (all 256-byte aligned). */
typedef struct {
    size_t topk_idx;  /* int32 [T,k] */
    size_t topk_w;    /* float [T,k] */
    size_t counts;    /* int32 [E]   */
    size_t offsets;   /* int32 [E+1] */
    size_t row_of;    /* int32 [R]   */
    size_t src_of;    /* int32 [R]   */
    size_t x_perm;    /* zero-length: moe_forward reads x rows through src_of and writes no permuted copy */
    size_t h;         /* bf16  [R,F] */
    size_t y_perm;    /* bf16  [R,d] */
    size_t scratch;   /* internal: the router's, chunk histograms, block schedule */
    size_t total;     /* bytes needed */
} moe_workspace_layout;

const char* moe_status_string(moe_status s);

/* Tile height (Alg. 1's M) the library uses for this config: cfg->tile_m if non-zero
 * (must be 32, 64, 96, 128, 160, 192 or 256), else 256 (the GEMM kernels adapt to the rows each
 * block really holds), 128 for many experts of a few rows each at up to 128 tokens (kernels built
 * for two workgroups per CU), or 32 when there are so few rows in all that the down projection
 * is run by the K-split kernel.
 * Returns 0 for an invalid config. */
int32_t moe_tile_m(const moe_config* cfg);

/* Workspace sizes in bytes (0 for an invalid config).  Host only, no GPU needed. */
size_t moe_route_workspace_size(const moe_config* cfg);
size_t moe_permute_workspace_size(const moe_config* cfg);
size_t moe_ffn_workspace_size(const moe_config* cfg);
size_t moe_forward_workspace_size(const moe_config* cfg);
/* The workspace moe_forward needs: the same value as moe_forward_workspace_size(). */
size_t moe_workspace_size(const moe_config* cfg);
/* Fills *out with the layout moe_forward uses; returns MOE_OK or the config error. */
moe_status moe_forward_workspace_layout(const moe_config* cfg, moe_workspace_layout* out);
/* Name of the GEMM kernel instance moe_grouped_ffn launches for this config (stage 0: fused
 * gate+up, 1: down; packed != 0: with moe_pack_weights' layout), e.g. for matching profiler
 * output.  moe_forward launches the same, except that with few rows of packed weights (up to 512, or 1024) its gate+up is
 * routed_tile_kernel_mixed, which permutes by itself.  Returns a static string, NULL for an invalid config or stage. */
const char* moe_ffn_kernel_name(const moe_config* cfg, int32_t stage, int32_t packed);
/* Upper bound on Alg. 1's block count for tile height M: floor(R/M) + min(E, R); 0 for an
 * invalid config or M outside [1, 2^30]. */
int32_t moe_max_blocks(const moe_config* cfg, int32_t M);

/* Stage 1, router (Eq. 1-2, Sec. 3.4).
 *   x [T,d] bf16, W_r [E,d] bf16, bias [E] fp32 or NULL (added to the logits)
 *   -> topk_idx [T,k] int32, topk_w [T,k] fp32.
 * Logits z = W_r x + bias: exact products of the bf16 operands, accumulated in fp64.  Calls of many
 * logits sum them in integers instead, 30 bits below each row's largest element, with a proven bound on what is
 * left out, and go back to fp64 for what the bound cannot rule on: the choice, its order and its ties are those of the
 * fp64 logits in every case.  Weights are off by one rounding to fp32 (2^-24, relative) and, in those calls, by
 * 2^-24 more at most; only MOE_GATE_SOFTMAX on 2^19 logits (T*E) or more lets, on rows where the bound is looser
 * (elements a hundred times the others', logits in the hundreds), the experts that are not chosen carry up to
 * 2^-19 |x| |w| in their logits.  The
 * k experts are chosen by k rounds of arg-max over z with the winner masked; a tie goes to the
 * lower expert index; outputs are in selection order (descending score).  Weights follow
 * cfg->gating.  workspace: moe_route_workspace_size(cfg) bytes (partial logit tiles, integer digits of W_r). */
moe_status moe_route(const moe_config* cfg, const void* x, const void* W_r, const float* bias,
                     int32_t* topk_idx, float* topk_w, void* workspace, size_t ws_bytes, void* stream);

/* Stage 2, permutation into expert-contiguous order (Sec. 2.2, Sec. 3.5).
 *   topk_idx [T,k] (any valid assignment: values in [0,E), as Sec. 4.7 injects them)
 *   -> counts [E] (n_e), offsets [E+1] (exclusive prefix sum, offsets[E] = R),
 *      row_of [R] (row of flat slot j = t*k+i after a STABLE sort by expert id),
 *      src_of [R] (inverse: slot stored at row r), x_perm [R,d] = x[src_of[r]/k, :].
 * x and x_perm may both be NULL to compute the index arrays only.
 * An index outside [0,E) cannot be reported (that would need a device->host sync); it is
 * clamped into [0,E-1], so every row index the kernels produce stays inside the buffers. */
moe_status moe_permute(const moe_config* cfg, const void* x, const int32_t* topk_idx,
                       int32_t* counts, int32_t* offsets, int32_t* row_of, int32_t* src_of,
                       void* x_perm, void* workspace, size_t ws_bytes, void* stream);

/* moe_permute for callers that cannot allocate device memory and have no workspace to hand in
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * kernels and the same results as moe_permute, with the chunk histograms (the only scratch the
 * stage needs: ceil(R/1024) * E int32) in a file-scope device array of the library instead of a
 * workspace argument.  The array holds MOE_PERMUTE_STATIC_MAX_INTS int32 (256 KiB) on every GPU
 * the library is used on, for the life of the process.  A configuration with
 * ceil(T*k/1024) * E above that returns MOE_ERR_UNSUPPORTED.  The call allocates nothing and frees
 * nothing.  Nothing in the array has to start at zero (every entry that is read has been written
 * earlier in the same call), so it is never cleared; its contents after a call are unspecified.
 * All calls on one GPU share the one array: two calls whose kernels overlap on the same GPU
 * (different streams, or different host threads on different streams) race and give wrong
 * results; calls on one stream are ordered and safe. */
#define MOE_PERMUTE_STATIC_MAX_INTS 65536
moe_status moe_permute_static(const moe_config* cfg, const void* x, const int32_t* topk_idx,
                              int32_t* counts, int32_t* offsets, int32_t* row_of, int32_t* src_of,
                              void* x_perm, void* stream);

/* Alg. 1 on the device: blocks [max_blocks,2] int32 = (expert, b*M) in emission order,
 * *num_blocks (device int32) = sum_e ceil(n_e/M).  Entries past *num_blocks are untouched.
 * `blocks` must hold moe_max_blocks(cfg, M) pairs.  1 <= M <= 2^30, else MOE_ERR_SHAPE. */
moe_status moe_block_schedule(const moe_config* cfg, const int32_t* offsets, int32_t M,
                              int32_t* blocks, int32_t* num_blocks, void* stream);

/* One-time weight packing (the weights of an inference layer are static).  THE PACKED COPY IS
 * THE SERVING LAYOUT: the GEMM kernels are built around it, and a caller that serves traffic
 * should pack once at load time and pass W_packed from then on.  The row-major tensors of
 * Sec. 3.2 are accepted by every entry point as the interchange layout (same integers, floats
 * within the stated tolerance); the layer then takes up to 9 % longer, from one token to 1024 rows
 * per expert (single projections up to 25 %: the down projection at 256 rows per expert).
 * Sec. 3.2 stores each projection as a flattened E*N x K matrix; the GEMM kernels read it
 * through per-lane 16-byte loads whose lanes touch 32 different rows.  moe_pack_weights
 * re-orders the same bf16 values into the order those loads consume them, so that every load
 * instruction reads 1 KiB contiguous and a wavefront streams one contiguous region:
 *   unit = 16 bytes; order [expert][row block of 32][k step of 64][matrix][slot 0..3][lane 0..63];
 *   unit (rb, kt, m, s, lane) = W_m[expert][32 rb + lane%32][64 kt + 16 s + 8 (lane/32) .. +8];
 *   gate and up are interleaved (m = 0, 1) in the first 4*E*F*d bytes, the down projection
 *   (m = 0 only) follows.
 * `packed` must hold moe_packed_weights_size(cfg) bytes (= 6*E*d*F, the size of the three
 * weight tensors), 256-byte aligned.  A packed buffer depends on d, F and E only, not on T, k. */
size_t moe_packed_weights_size(const moe_config* cfg);
moe_status moe_pack_weights(const moe_config* cfg, const void* W_gate, const void* W_up, const void* W_down,
                            void* packed, void* stream);

/* Stages 3+4, expert FFN as two block-scheduled grouped GEMMs (Sec. 3.2, 3.3, Eq. 4).
 *   x_perm [R,d] bf16 expert-contiguous, offsets [E+1]
 *   W_gate, W_up [E,F,d] bf16, W_down [E,d,F] bf16
 *   W_packed: NULL, or moe_pack_weights' output for these weights; when it is given the kernels
 *             read only the packed copy and W_gate, W_up, W_down may be NULL
 *   -> h [R,F] bf16 = SiLU(x W_gate^T) (.) (x W_up^T)  (fp32 accumulate, SiLU and product in
 *      fp32 registers, one rounding to bf16), y_perm [R,d] bf16 = h W_down^T (fp32 accumulate).
 * The block schedule is built on the device from `offsets`; no host synchronisation. */
moe_status moe_grouped_ffn(const moe_config* cfg, const void* x_perm, const int32_t* offsets,
                           const void* W_gate, const void* W_up, const void* W_down, const void* W_packed,
                           void* h, void* y_perm, void* workspace, size_t ws_bytes, void* stream);

/* Stage 5, un-permute + weighted combine (Eq. 3, Sec. 3.5).
 *   y[t,:] = sum_{i<k} topk_w[t,i] * y_perm[row_of[t*k+i], :], fp32 accumulation in slot
 *   order, one rounding to bf16.  No atomics: results are bit-reproducible. */
moe_status moe_combine(const moe_config* cfg, const void* y_perm, const int32_t* row_of,
                       const float* topk_w, void* y, void* stream);

/* The whole layer: stages 1-5 enqueued back to back on `stream`, intermediates in
 * `workspace` at moe_forward_workspace_layout()'s offsets.  y [T,d] bf16.  W_packed as above.
 * The permutation stage builds the index arrays only: the gate+up GEMM fetches expert-contiguous
 * row r straight from x[src_of[r] / k] while it loads its token tile, so the permuted copy of x
 * (Sec. 3.1 step 2; the paper lists removing it as future work) is never written.  Results are
 * identical to moe_permute + moe_grouped_ffn on the materialised copy. */
moe_status moe_forward(const moe_config* cfg, const void* x, const void* W_r, const float* bias,
                       const void* W_gate, const void* W_up, const void* W_down, const void* W_packed,
                       void* y, void* workspace, size_t ws_bytes, void* stream);

/* moe_forward with timing hooks: `events` is an array of n_events hipEvent_t handles (as void*,
 * entries may be NULL, the array itself may be NULL when n_events == 0) recorded on `stream`
 *   [0] before the router, [1] after it, [2] after the permutation (index arrays; the row gather runs inside gate+up; with
 *   few rows of packed weights the whole permutation does: then nothing lies between [1] and [2], its time is in [2]-[3]),
 *   [3] after the fused gate+up GEMM, [4] after the down GEMM, [5] after the combine.
 * Entries beyond index 5 are ignored.  Everything else is exactly moe_forward (Sec. 3.1's
 * five stages; the per-stage breakdown mirrors the paper's Table 6). */
#define MOE_NUM_STAGE_EVENTS 6
moe_status moe_forward_staged(const moe_config* cfg, const void* x, const void* W_r, const float* bias,
                              const void* W_gate, const void* W_up, const void* W_down, const void* W_packed,
                              void* y, void* workspace, size_t ws_bytes, void* stream,
                              void* const* events, int32_t n_events);

/* ---- Training ---------------------------------------------------------------------------
 * The gated feed-forward block with what its backward pass needs, that backward pass, and the gradient
 * of the combine.  Rows are expert-contiguous as moe_permute leaves them; E = k = 1 with offsets {0, T}
 * is a dense block (or the expert that all tokens share).  Weights are the row-major tensors, which a training
 * program changes with every step.  A layer's step:
 *   moe_route, moe_permute, moe_grouped_ffn_train, moe_combine;
 *   moe_combine_backward, moe_grouped_ffn_backward; dx of a token = the sum of its k rows of dx_perm:
 *   moe_combine(dx_perm, row_of, weights of 1).  d_topk_w is what the router's gradient (moe_route_backward) starts from.
 * offsets are trusted as in moe_grouped_ffn: ascending, offsets[E] <= R.  Rows from offsets[E] on are
 * not written.  Where T == 0 the tensors of rows may be NULL.
 * Beyond the limits above: d, F <= 2^20 and E*d*F <= 2^36, else MOE_ERR_UNSUPPORTED.  No atomics: results are bit-reproducible. */

/* moe_grouped_ffn that keeps the two projections: g = x W_gate^T, u = x W_up^T [R,F] bf16 (rounded once from fp32),
 * h [R,F] = SiLU(g) (.) u from the fp32 values, y_perm [R,d] = h W_down^T.  h is not needed by the backward pass.
 * workspace: moe_ffn_workspace_size(cfg) bytes. */
moe_status moe_grouped_ffn_train(const moe_config* cfg, const void* x_perm, const int32_t* offsets,
                                 const void* W_gate, const void* W_up, const void* W_down,
                                 void* g, void* u, void* h, void* y_perm, void* workspace, size_t ws_bytes, void* stream);

/* flags of moe_grouped_ffn_backward */
#define MOE_GRAD_F32 1         /* dW_gate, dW_up, dW_down are fp32 tensors (else bf16) */
#define MOE_GRAD_ACCUMULATE 2  /* they are added to what the tensors hold (in fp32, one rounding), else written */

/* Gradients of moe_grouped_ffn_train at the kept g and u:
 *   dh = dy_perm W_down;  dg = dh (.) u (.) SiLU'(g),  du = dh (.) SiLU(g)
 *   dx_perm [R,d] = dg W_gate + du W_up
 *   dW_gate, dW_up [E,F,d] = dg^T x, du^T x;  dW_down [E,d,F] = dy^T h, over each expert's rows
 * dg, du and h = SiLU(g) (.) u (formed again) are rounded to bf16, the operands of the products that follow; all sums are fp32.
 * dx_perm and each dW may be NULL: it is then not computed.  An expert without rows (and T == 0) has weight
 * gradients of zero, which are written unless MOE_GRAD_ACCUMULATE is set.  Outputs must not overlap inputs; calls that may run at
 * the same time need a workspace each.
 * workspace: moe_ffn_backward_workspace_size(cfg) bytes (dg, du, h: 6*R*F, and partial sums of dx in small launches), 256-byte aligned. */
size_t moe_ffn_backward_workspace_size(const moe_config* cfg);
moe_status moe_grouped_ffn_backward(const moe_config* cfg, const void* x_perm, const int32_t* offsets,
                                    const void* W_gate, const void* W_up, const void* W_down,
                                    const void* g, const void* u, const void* dy_perm,
                                    void* dx_perm, void* dW_gate, void* dW_up, void* dW_down, int32_t flags,
                                    void* workspace, size_t ws_bytes, void* stream);

/* Gradients of moe_combine:  dy_perm[row_of[t*k+i],:] = topk_w[t,i] * dy[t,:] (one rounding to bf16),
 * d_topk_w[t,i] = <dy[t,:], y_perm[row_of[t*k+i],:]> (fp32).  row_of: moe_permute's (every row once).
 * dy_perm may be y_perm itself. */
moe_status moe_combine_backward(const moe_config* cfg, const void* dy, const void* y_perm, const int32_t* row_of,
                                const float* topk_w, void* dy_perm, float* d_topk_w, void* stream);

/* Gradient of moe_route: from d_topk_w [T,k] fp32 (of the weights that it gave for topk_idx) to x, W_r and the bias, at cfg->gating.
 *   dz = the gate's gradient: MOE_GATE_SOFTMAX p_e (G_e - sum_i p_i d_i) over all experts (p = softmax(z), G_e: d of the slot that chose e, else 0);
 *        MOE_GATE_SOFTMAX_RENORM w_i (d_i - sum_j w_j d_j) over the chosen; MOE_GATE_SIGMOID_NORM the same times 1 - sigmoid(z_i)
 *   dx [T,d] bf16 = dz W_r,  dW_r [E,d] = dz^T x (bf16, or fp32 with MOE_GRAD_F32),  dbias [E] fp32 = sum_t dz
 * z is formed again (fp32 sums; not for MOE_GATE_SOFTMAX_RENORM); dz enters the products as three bf16 numbers, all its 24 bits: an infinity in dz,
 * x or W_r comes out as NaN as a rule.
 * Of a token with one large weight dz is off as if every d were off by a few of its own fp32 roundings; weights that add up to one but for (k + 4) 2^-24 count as adding up to one.
 * dx, dW_r and dbias may be NULL: not computed.  MOE_GRAD_ACCUMULATE: dW_r and dbias are added to what the tensors hold.  x's whole gradient: moe_dispatch_backward
 * with this dx as base.  A slot whose index is outside 0 .. E-1 has no part in anything.  T == 0: dW_r and dbias of zero are written unless they are added to.
 * Limit: d <= 2^20.  Outputs must not overlap inputs.  workspace: moe_route_backward_workspace_size(cfg) bytes, 256-byte aligned, and no less for more
 * tokens of the same shape; calls that may run at the same time need one each. */
size_t moe_route_backward_workspace_size(const moe_config* cfg);
moe_status moe_route_backward(const moe_config* cfg, const void* x, const void* W_r, const float* bias, const int32_t* topk_idx, const float* topk_w,
                              const float* d_topk_w, void* dx, void* dW_r, float* dbias, int32_t flags, void* workspace, size_t ws_bytes, void* stream);

/* ---- Slots that may have no row ------------------------------------------------------------
 * Permutation and combine for a GPU that holds a share of the experts, or whose experts take a limited number of rows, with their gradients, and with what
 * a training step does beside them: gate weights applied on the way in, the residual, dropout.  Slot j = t*k+i has a row iff
 * e = topk_idx[j] - first is in 0 .. E-1 and fewer than `capacity` slots in front of it chose e; its row is offsets[e] plus that number (stable, as in moe_permute).
 * The rows are what moe_grouped_ffn and the training operators take, with the same T*k (their k <= E: T*k tokens with k = 1 say the same).
 * Limits: d % 8 == 0, d <= 2^20, k <= 256, E <= 256, T*k <= 2^30, first + E <= 2^31 - 1, else MOE_ERR_UNSUPPORTED (MOE_ERR_SHAPE for the last); sizes in bytes are
 * not limited.  No atomics on memory: results are bit-reproducible.  row_of below: moe_dispatch's; a number outside 0 .. T*k-1 is a slot without a row, and
 * no two slots may share one.  Tensors of [T*k,d] hold offsets[E] rows; what lies behind is neither read nor written.
 * The calls after moe_dispatch go by T, d and k of cfg.  topk_w may be NULL: weights of one.  Outputs
 * must not overlap inputs but where it is said. */
typedef struct {
    int32_t T, d, k;           /* tokens, width, slots per token */
    int32_t E, first;          /* experts held here: ids first .. first+E-1 */
    int32_t capacity;          /* rows that an expert takes at most, in order of slots; 0: all */
} moe_dispatch_config;

size_t moe_dispatch_workspace_size(const moe_dispatch_config* cfg);

/* counts [E] = slots that chose e (before the limit), offsets [E+1] = exclusive sums of the rows taken, row_of [T,k] (-1: none),
 * src_of [T*k]: slot of a row; rows [T*k,d] bf16 = topk_w[t,i] * x[t,:] (one rounding), or copies.  x and rows may both be NULL: the tables alone.
 * T == 0 writes counts and offsets of zero.  workspace: moe_dispatch_workspace_size(cfg) bytes; calls that may run at the same time need one each. */
moe_status moe_dispatch(const moe_dispatch_config* cfg, const void* x, const int32_t* topk_idx, const float* topk_w, int32_t* counts, int32_t* offsets,
                        int32_t* row_of, int32_t* src_of, void* rows, void* workspace, size_t ws_bytes, void* stream);

/* dx[t,:] = base[t,:] + sum_i topk_w[t,i] * drows[row_of[t,i],:] (fp32, slot order, one rounding); base may be NULL (0), and may be dx.
 * d_topk_w [T,k] fp32 = <x[t,:], drows[row_of[t,i],:]>, 0 without a row; may be NULL (then x may be, too). */
moe_status moe_dispatch_backward(const moe_dispatch_config* cfg, const void* x, const void* drows, const int32_t* row_of, const float* topk_w, const void* base,
                                 void* dx, float* d_topk_w, void* stream);

/* Dropout.  Element n of a tensor (t*d + c in the calls with tokens) is kept with probability 1 - p and divided by it; else it is zero, whatever it was.  The mask is
 * a function of (rng[0], rng[1], n): Philox4x32-10 with key rng[0] and counter (n / 8, rng[1]) gives 128 bits for eight elements, of which
 * element n takes 16 (n % 8) .. +15; it is dropped if they are below 65536 p.  p is taken in steps of 2^-16 (so is 1 - p): 0 <= p < 1 - 2^-17, else MOE_ERR_SHAPE.
 * rng: uint64 [2] ON THE DEVICE, seed and offset, so that a captured step draws another mask at each replay; the gradient's call has to find the
 * values that its forward call found.  It may be NULL where p == 0. */

/* y[t,:] = residual[t,:] + dropout(sum_i topk_w[t,i] * rows[row_of[t,i],:]): fp32, slot order, one rounding.  A token without rows gets its residual.
 * residual may be NULL (0), and may be y. */
moe_status moe_collect(const moe_dispatch_config* cfg, const void* rows, const int32_t* row_of, const float* topk_w, const void* residual, float p, const void* rng,
                       void* y, void* stream);

/* v = dropout(dy[t,:]):  drows[row_of[t,i],:] = topk_w[t,i] * v (one rounding),  d_topk_w[t,i] = <v, rows[row_of[t,i],:]> (fp32), 0 without a row; may be NULL (then rows
 * may be, too).  drows may be rows.  The residual's gradient is dy itself. */
moe_status moe_collect_backward(const moe_dispatch_config* cfg, const void* dy, const void* rows, const int32_t* row_of, const float* topk_w, float p,
                                const void* rng, void* drows, float* d_topk_w, void* stream);

/* y = residual + dropout(x) over n bf16 elements (n <= 2^40, any), residual may be NULL; y may be x or residual.  Its gradient is the same call on dy, without residual. */
moe_status moe_dropout(int64_t n, const void* x, const void* residual, float p, const void* rng, void* y, void* stream);

/* ---- Low-rank adapters of many requests beside a shared projection -------------------------
 * Serving requests that have each their own low-rank update of a projection (a shared expert's, a dense block's), in one call:
 *   y[t] = (base[t] +) x[t] W^T + scale[a] * (x[t] A[a]^T) B[a]^T,   a = adapter_of[t]
 * Tokens in any order and number per adapter; an id outside 0 .. adapters-1 (by convention -1) is a token without one.
 * Stored [out, in] as everywhere: W [N,K], A [adapters, rank, K], B [adapters, N, rank], bf16.  Adapters of a smaller rank are
 * padded with rows (columns) of zeros.  scale [adapters] fp32 or NULL (1).
 * x A^T is summed and scaled in fp32 and enters the product with B as two bf16 numbers (16 bits); the sum of all parts is rounded once.  (Hence an
 * infinity in B comes out as NaN as a rule, not as an infinity: it also meets the second number, which may be zero or of the other sign.)
 * Limits: N % 64 == 0, K % 64 == 0, N, K <= 2^20, rank % 8 == 0, 8 <= rank <= 128, adapters <= 65536, T*max(N,K)*2 bytes below
 * 4 GiB, else MOE_ERR_UNSUPPORTED.  T == 0 returns MOE_OK and enqueues nothing.  Every pointer 16-byte aligned but adapter_of and scale.
 * workspace: moe_adapter_workspace_size(cfg) bytes; calls that may run at the same time (other streams, graphs replayed side by side) need
 * one each.  y (h) must not overlap the inputs, but for base.  No atomics: results are bit-reproducible. */
typedef struct {
    int32_t T, N, K;           /* tokens, output and input features */
    int32_t adapters, rank;
} moe_adapter_config;

size_t moe_adapter_workspace_size(const moe_adapter_config* cfg);

/* base [T,N] bf16 or NULL: added before the rounding; may be y itself (e.g. the routed experts' result, to which the shared
 * expert's down projection is added).  W may be NULL: the adapters' part alone, for a projection that is computed elsewhere. */
moe_status moe_adapter_linear(const moe_adapter_config* cfg, const void* x, const void* W, const void* A, const void* B,
                              const float* scale, const int32_t* adapter_of, const void* base, void* y,
                              void* workspace, size_t ws_bytes, void* stream);

/* The first half of a gated block with adapters: h [T,N] = SiLU(gate) (.) up, gate and up being two such projections of x, with the
 * same adapter ids and scales; activation and product in fp32, one rounding. */
moe_status moe_adapter_gated_up(const moe_adapter_config* cfg, const void* x, const void* W_gate, const void* W_up,
                                const void* A_gate, const void* A_up, const void* B_gate, const void* B_up,
                                const float* scale, const int32_t* adapter_of, void* h,
                                void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_H_ */
