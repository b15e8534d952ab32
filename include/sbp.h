/*
 * sbp.h -- C ABI of the local-shard SBP linear layer for MI355X (gfx950).
 *
 * A linear layer Y = X W under an SBP (Split / Broadcast / Partial-sum)
 * signature runs, on each device, a local matrix product of that device's
 * shares of its operands (AutoDDL, Sec. 4.2, "Distributed Matrix
 * Multiplication based on SBP": the local matmul of the 3-D SBP rule).
 * This library runs rank r's local forward and backward products on one GPU
 * and tags each output with its SBP state.
 *
 * Supported signatures (the 1-D factors of the Sec. 4.2 rule, and three
 * that follow from linearity; a broadcast tensor's gradient is a partial
 * sum, Sec. 4.3 "Sources of Communication", and a partial sum's gradient is
 * broadcast):
 *
 *   name  X      W      -> Y     | dY     dX     dW
 *   DP    S(0)   B      -> S(0)  | S(0)   S(0)   P
 *   COL   B      S(1)   -> S(1)  | S(1)   P      S(1)
 *   KS    S(1)   S(0)   -> P     | B      S(1)   S(0)
 *   PB    P      B      -> P     | B      B      P
 *   BP    B      P      -> P     | B      P      B
 *   BB    B      B      -> B     | P      P      P
 *
 * PB, BP and BB divide no dimension: every device multiplies full-size
 * operands (its own partial of a P operand).
 *
 * Conventions (all functions):
 *   - Matrices are row-major with a leading dimension ld (elements between
 *     the starts of consecutive rows, ld >= cols). X is M x K, W is K x N,
 *     dY and Y are M x N, as global tensors.
 *   - Split(i) over p devices gives rank r the contiguous block
 *     [off, off + len) of axis i with len = D/p + (r < D%p), off =
 *     r*(D/p) + min(r, D%p) (the paper does not fix uneven splits; this is
 *     the balanced reading). Broadcast and Partial-sum shares span the full
 *     extent.
 *   - Every pointer in an sbp_view_t is a DEVICE pointer on the current HIP
 *     device. The caller owns every buffer; the library never copies inputs.
 *   - Return value: SBP_OK (0) or a negative SBP_ERR_* code. Every check
 *     except SBP_ERR_HIP happens on the host before any HIP call, so a
 *     rejected call has no effect on the device.
 *   - Compute calls are asynchronous on the given stream (0 = the null
 *     stream) and never synchronise. Inputs must stay valid, and outputs
 *     untouched, until the stream has run the call.
 *   - Memory: the library allocates nothing and keeps no device state.
 *     The linear calls take a caller-owned workspace (sbp_workspace_t) for
 *     the fp32 partials of split reductions; see below. Every call can be
 *     captured into a HIP graph, including the first on a stream.
 *   - Thread safety: calls on different host threads are safe. Two calls
 *     may share a workspace only if neither their launches can run at the
 *     same time nor the calls themselves: a call may enqueue several
 *     launches that pass data through it, so calls on one stream share one
 *     if the host makes them one after the other (a graph that was captured
 *     with it counts as a call wherever it is replayed), and host threads
 *     that make calls at the same time bring workspaces of their own.
 */
#ifndef SBP_H
#define SBP_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------ codes --- */
enum {
    SBP_OK = 0,
    SBP_ERR_NULL = -1,      /* a required pointer is NULL                       */
    SBP_ERR_LAYOUT = -2,    /* p < 1, r outside [0,p), bad kind/axis, or layouts
                               of one call disagree on p or r                    */
    SBP_ERR_SIGNATURE = -3, /* the input states form no supported signature     */
    SBP_ERR_SHAPE = -4,     /* inner dimensions disagree, ld < cols, a negative
                               or > 2^31-1 extent, or the output view is not the
                               local output shape                               */
    SBP_ERR_DTYPE = -5,     /* unknown dtype, inputs of mixed dtype, a
                               Partial-sum output that is not fp32, or a bf16
                               output of fp32 inputs                            */
    SBP_ERR_ALIAS = -6,     /* the output's memory overlaps an input's          */
    SBP_ERR_ALIGN = -7,     /* a data pointer is not aligned to its element size */
    SBP_ERR_HIP = -8,       /* a HIP call failed; see sbp_last_hip_error()      */
    SBP_ERR_WORKSPACE = -9  /* the split partials of the call's plan do not fit
                               the workspace it runs with                       */
};

/* ------------------------------------------------------------ types --- */
typedef enum { SBP_SPLIT = 0, SBP_BROADCAST = 1, SBP_PARTIAL = 2 } sbp_kind_t;

/* SBP state of a tensor on a 1-D mesh of p devices, seen from rank r.
 * axis is 0 or 1 for SBP_SPLIT and -1 otherwise. */
typedef struct {
    int32_t kind;
    int32_t axis;
    int32_t p;
    int32_t r;
} sbp_layout_t;

typedef enum { SBP_BF16 = 0, SBP_F32 = 1 } sbp_dtype_t;

/* SBP_GLOBAL: the view spans the whole global tensor and the library selects
 * rank r's share inside it (a strided sub-view, never a copy).
 * SBP_LOCAL: the view is exactly rank r's share.
 * SBP_ACCUMULATE (outputs only): the call adds its product to the output's
 * current contents instead of overwriting them -- gradient accumulation
 * over micro-batches (Sec. 5 splits each mini-batch into micro-batches and
 * accumulates their gradients). The output must be fp32 (else
 * SBP_ERR_DTYPE); each element becomes old + product with one fp32
 * rounding (the product itself summed in fp32 first). */
typedef enum { SBP_GLOBAL = 0, SBP_LOCAL = 1, SBP_ACCUMULATE = 2 } sbp_scope_t;

/* A strided 2-D view: element (i, j) is at data + i*ld + j (elements). */
typedef struct {
    void *data;
    int64_t rows;
    int64_t cols;
    int64_t ld;
    int32_t dtype; /* sbp_dtype_t */
    int32_t scope; /* sbp_scope_t; outputs are always local: SBP_ACCUMULATE
                      adds to them, any other value overwrites them */
} sbp_view_t;

/* Caller-owned device memory for split reductions. A product with a long
 * reduction and few output tiles runs faster with its reduction split over
 * several workgroups; each split writes an fp32 partial of the m x n output
 * (rows padded to a multiple of 4 floats: splits x m x 4 ceil(n / 4) x 4
 * bytes in all) that a second kernel adds up in split order. The linear calls take a workspace; data = NULL (or bytes = 0, or a
 * NULL sbp_workspace_t pointer) means none, and then no reduction is split.
 * With bytes >= SBP_WORKSPACE_BYTES every call gets the library's preferred
 * plan; a smaller workspace limits the splits to what fits (results are the
 * same up to fp32 summation order; identical for identical workspace
 * sizes). The library never reads the workspace's contents before writing
 * them, so it needs no clearing. data must be 16-byte aligned (else
 * SBP_ERR_ALIGN), must not overlap the call's inputs or outputs (else
 * SBP_ERR_ALIAS), and must not be used by another call at the same time. */
typedef struct {
    void *data;    /* device pointer on the current device, or NULL */
    int64_t bytes; /* its size in bytes (>= 0, else SBP_ERR_SHAPE)   */
} sbp_workspace_t;

#define SBP_WORKSPACE_BYTES ((int64_t)64 << 20)

/* Rank r's share of a tensor: rows [row_off, row_off+rows) x cols
 * [col_off, col_off+cols) of the global tensor. */
typedef struct {
    int64_t row_off;
    int64_t col_off;
    int64_t rows;
    int64_t cols;
} sbp_shard_t;

/* ------------------------------------------------------- host logic --- */

/* Rank l->r's share of a rows x cols tensor in state *l (Sec. 4.1: Split,
 * Broadcast and Partial-sum states; Fig. 5). Pure host function.
 * Errors: SBP_ERR_NULL, SBP_ERR_LAYOUT, SBP_ERR_SHAPE (negative extent). */
int sbp_shard_index(const sbp_layout_t *l, int64_t rows, int64_t cols,
                    sbp_shard_t *out);

/* Resolves the signature of Y = X W from the states of X and W (Sec. 4.2)
 * and writes the states of Y, dY, dX and dW (Sec. 4.3: a broadcast operand's
 * gradient is a partial sum; a split operand's gradient is split the same
 * way). Any of y, dy, dx, dw may be NULL. Pure host function.
 * Errors: SBP_ERR_NULL (x or w), SBP_ERR_LAYOUT, SBP_ERR_SIGNATURE. */
int sbp_signature(const sbp_layout_t *x, const sbp_layout_t *w,
                  sbp_layout_t *y, sbp_layout_t *dy, sbp_layout_t *dx,
                  sbp_layout_t *dw);

/* ----------------------------------------------------- device compute --- */

/* Forward local matmul Y_r = X_r W_r (Sec. 4.2, "local matmul").
 * X: M x K (or rank r's share), state *lx; W: K x N (or share), state *lw.
 * Y: rank r's local output, state written to *ly_out (may be NULL):
 *    DP m_r x N, COL M x n_r, KS M x N (Partial-sum, must be fp32);
 *    PB and BP M x N (Partial-sum, fp32), BB M x N (Broadcast).
 * Inputs bf16 or fp32 (same dtype); Y is fp32, or bf16 for bf16 inputs and
 * a Split/Broadcast output (rounded to nearest even from the fp32
 * accumulator). ws: workspace for a split reduction (may be NULL; see
 * sbp_workspace_t). */
int sbp_linear_fwd(const sbp_view_t *X, const sbp_layout_t *lx,
                   const sbp_view_t *W, const sbp_layout_t *lw, sbp_view_t *Y,
                   sbp_layout_t *ly_out, const sbp_workspace_t *ws,
                   hipStream_t stream);

/* Backward-data local matmul dX_r = dY_r W_r^T (Sec. 4.2: the redistributions
 * of the forward path have backward counterparts; Sec. 4.3).
 * dY: state *ldy (S(0) for DP, S(1) for COL, B for KS, PB and BP, P for
 *     BB); W: state *lw.
 * dX: rank r's local output, state to *ldx_out: DP m_r x K (S(0)),
 *     COL M x K (Partial-sum, fp32), KS M x k_r (S(1)); PB M x K (B), BP
 *     and BB M x K (Partial-sum, fp32).
 * ws as for sbp_linear_fwd. */
int sbp_linear_bwd_data(const sbp_view_t *dY, const sbp_layout_t *ldy,
                        const sbp_view_t *W, const sbp_layout_t *lw,
                        sbp_view_t *dX, sbp_layout_t *ldx_out,
                        const sbp_workspace_t *ws, hipStream_t stream);

/* Backward-weight local matmul dW_r = X_r^T dY_r (Sec. 4.3: a broadcast
 * weight receives partial-sum gradients).
 * X: state *lx; dY: state *ldy.
 * dW: rank r's local output, state to *ldw_out: DP K x N (Partial-sum,
 *     fp32), COL K x n_r (S(1)), KS k_r x N (S(0)); PB and BB K x N
 *     (Partial-sum, fp32), BP K x N (B).
 * ws as for sbp_linear_fwd. */
int sbp_linear_bwd_weight(const sbp_view_t *X, const sbp_layout_t *lx,
                          const sbp_view_t *dY, const sbp_layout_t *ldy,
                          sbp_view_t *dW, sbp_layout_t *ldw_out,
                          const sbp_workspace_t *ws, hipStream_t stream);

/* Both backward products of the linear, dX_r = dY_r W_r^T and
 * dW_r = X_r^T dY_r, in one call (one grouped launch when the planner
 * expects it to pay, else the two products in turn on `stream`). The two
 * products are independent -- each reads dY and one of X, W (Sec. 4.2
 * backward path, Sec. 4.3 gradient states) -- so in a grouped launch the
 * longer work items of one run while the shorter ones of the other fill the
 * remaining compute units. States, shapes, dtype rules and errors are those
 * of sbp_linear_bwd_data and sbp_linear_bwd_weight; the three input states
 * must form one signature (else SBP_ERR_SIGNATURE), and dX and dW must not
 * overlap (SBP_ERR_ALIAS). Results equal the two separate calls up to fp32
 * summation order. ws as for sbp_linear_fwd: a grouped launch holds the
 * partials of both products in it at once, two separate launches use it in
 * turn. */
int sbp_linear_bwd(const sbp_view_t *dY, const sbp_layout_t *ldy,
                   const sbp_view_t *X, const sbp_layout_t *lx,
                   const sbp_view_t *W, const sbp_layout_t *lw, sbp_view_t *dX,
                   sbp_layout_t *ldx_out, sbp_view_t *dW, sbp_layout_t *ldw_out,
                   const sbp_workspace_t *ws, hipStream_t stream);

/* For callers that cannot allocate device memory -- code being captured
 * into a HIP graph, tight serving loops, harnesses that forbid hipMalloc --
 * and so cannot bring a workspace: sbp_linear_bwd with the library's own
 * scratch in place of a caller workspace. The scratch is a static device
 * array of SBP_WORKSPACE_BYTES on each device (so the plans, kernels and
 * results are those of sbp_linear_bwd with a workspace of that size),
 * placed when the library's code is loaded on the device and held until
 * the process ends; the call itself allocates nothing, and neither does any
 * library routine it uses. A plan whose partials would not fit the scratch
 * is refused with SBP_ERR_WORKSPACE (plans are limited to it, so none
 * does). The scratch keeps the last call's partials; nothing in it needs
 * clearing, since every partial is written before it is read. Every call on
 * one device shares that device's scratch: calls that may overlap in time on
 * one device (different streams, host threads or processes sharing the
 * device's code object) race on it and must be ordered by the caller, e.g.
 * by issuing them on one stream. Arguments, states and errors are those of
 * sbp_linear_bwd. */
int sbp_linear_bwd_noalloc(const sbp_view_t *dY, const sbp_layout_t *ldy,
                           const sbp_view_t *X, const sbp_layout_t *lx,
                           const sbp_view_t *W, const sbp_layout_t *lw,
                           sbp_view_t *dX, sbp_layout_t *ldx_out, sbp_view_t *dW,
                           sbp_layout_t *ldw_out, hipStream_t stream);

/* ------------------------------------------- nd-SBP on device meshes --- */

/* Mesh axes an nd layout may have. */
#define SBP_MAX_MESH_DIMS 4

/* SBP state of a tensor on a d-dimensional device mesh, seen from the
 * device at mesh coordinate c: one Split / Broadcast / Partial-sum state
 * per mesh axis (Sec. 4.1, Listing 1: a placement hierarchy such as
 * (2, 3, 4) with one state per hierarchy level; Sec. 4.2: the 3-D rule
 * (S0:p0, B:p1, S1:p2) x (B:p0, S1:p1, S0:p2) -> (S0:p0, S1:p1, P:p2)).
 *   ndim     mesh axes d, 1..SBP_MAX_MESH_DIMS; entries a >= d are ignored
 *   kind[a]  sbp_kind_t on mesh axis a
 *   axis[a]  tensor axis (0 or 1) for SBP_SPLIT, else -1
 *   p[a]     devices along mesh axis a (>= 1)
 *   c[a]     this device's coordinate along mesh axis a, in [0, p[a])
 * The share of a tensor nests the splits in mesh-axis order: mesh axis 0
 * cuts the full extent into p[0] balanced blocks (the 1-D rule above), mesh
 * axis 1 cuts block c[0] into p[1] blocks, and so on; each tensor axis is cut
 * only by the mesh axes that split it. Broadcast and Partial-sum axes do not
 * cut. A 1-D layout (kind, axis, p, r) is the nd layout with d = 1,
 * c[0] = r. */
typedef struct {
    int32_t ndim;
    int32_t kind[SBP_MAX_MESH_DIMS];
    int32_t axis[SBP_MAX_MESH_DIMS];
    int32_t p[SBP_MAX_MESH_DIMS];
    int32_t c[SBP_MAX_MESH_DIMS];
} sbp_nd_layout_t;

/* Mesh coordinate of a device (Sec. 4.2, "Strategies for heterogeneous
 * interconnected networks"). Mesh axis a spans nodes[a] x gpus[a] devices:
 * nodes[a] compute nodes times gpus[a] GPUs of each node. Device (node, gpu)
 * -- node in [0, prod nodes), gpu in [0, prod gpus) -- has node-level digits
 * n_a and GPU-level digits g_a, both mixed-radix with mesh axis 0 varying
 * fastest (node = n_0 + nodes[0] (n_1 + nodes[1] (...)), likewise gpu), and
 * coordinate c[a] = n_a * gpus[a] + g_a. The paper's example
 * (S0:(1,2), B:(2,2)) on 2 nodes of 4 GPUs puts split 0 on GPUs (0,0),
 * (0,2), (1,0), (1,2): mesh axis 0 varies fastest within a node. For a
 * single-level mesh pass gpus = NULL (all 1) and the device rank as node.
 * Pure host function. Errors: SBP_ERR_NULL (nodes or c), SBP_ERR_LAYOUT
 * (ndim outside [1, SBP_MAX_MESH_DIMS], a factor < 1, or node / gpu outside
 * its range). */
int sbp_mesh_coords(int32_t ndim, const int32_t *nodes, const int32_t *gpus,
                    int64_t node, int64_t gpu, int32_t *c);

/* The device's share of a rows x cols tensor in nd state *l (nested splits,
 * as described at sbp_nd_layout_t). Pure host function.
 * Errors: SBP_ERR_NULL, SBP_ERR_LAYOUT (bad ndim, p, c, kind or axis),
 * SBP_ERR_SHAPE (negative extent). */
int sbp_nd_shard_index(const sbp_nd_layout_t *l, int64_t rows, int64_t cols,
                       sbp_shard_t *out);

/* Resolves the nd signature of Y = X W (Sec. 4.2: the 3-D rule factors
 * into one 1-D signature per mesh axis) and writes the nd states of Y, dY,
 * dX and dW (Sec. 4.3 gradient states, per axis). Each mesh axis must carry
 * one of the 1-D signatures of the table at the top of this file; an axis
 * with X and W both Broadcast (BB) replicates the product, and the
 * gradients are partial sums on it. The layouts must agree on ndim, p and
 * c. Any of y, dy, dx, dw may be NULL. Pure host function.
 * Errors: SBP_ERR_NULL (x or w), SBP_ERR_LAYOUT, SBP_ERR_SIGNATURE. */
int sbp_nd_signature(const sbp_nd_layout_t *x, const sbp_nd_layout_t *w,
                     sbp_nd_layout_t *y, sbp_nd_layout_t *dy,
                     sbp_nd_layout_t *dx, sbp_nd_layout_t *dw);

/* nd forms of the four compute calls: the device's local products on its
 * nd shares, on the same kernels. Views, dtypes, scopes, workspaces, streams
 * and errors are those of the 1-D calls, with nd layouts in place of 1-D ones (all
 * layouts of one call agree on ndim, p and c, else SBP_ERR_LAYOUT).
 * Local output shapes: X_r is the nd share of X, and so on; Y_r = X_r W_r,
 * dX_r = dY_r W_r^T, dW_r = X_r^T dY_r. An output is Partial-sum -- and must
 * be fp32 -- when any mesh axis leaves it Partial-sum (Y under a KS, PB or
 * BP axis, dX under a COL, BP or BB axis, dW under a DP, PB or BB axis). */
int sbp_nd_linear_fwd(const sbp_view_t *X, const sbp_nd_layout_t *lx,
                      const sbp_view_t *W, const sbp_nd_layout_t *lw,
                      sbp_view_t *Y, sbp_nd_layout_t *ly_out,
                      const sbp_workspace_t *ws, hipStream_t stream);
int sbp_nd_linear_bwd_data(const sbp_view_t *dY, const sbp_nd_layout_t *ldy,
                           const sbp_view_t *W, const sbp_nd_layout_t *lw,
                           sbp_view_t *dX, sbp_nd_layout_t *ldx_out,
                           const sbp_workspace_t *ws, hipStream_t stream);
int sbp_nd_linear_bwd_weight(const sbp_view_t *X, const sbp_nd_layout_t *lx,
                             const sbp_view_t *dY, const sbp_nd_layout_t *ldy,
                             sbp_view_t *dW, sbp_nd_layout_t *ldw_out,
                             const sbp_workspace_t *ws, hipStream_t stream);
int sbp_nd_linear_bwd(const sbp_view_t *dY, const sbp_nd_layout_t *ldy,
                      const sbp_view_t *X, const sbp_nd_layout_t *lx,
                      const sbp_view_t *W, const sbp_nd_layout_t *lw,
                      sbp_view_t *dX, sbp_nd_layout_t *ldx_out,
                      sbp_view_t *dW, sbp_nd_layout_t *ldw_out,
                      const sbp_workspace_t *ws, hipStream_t stream);

/* --------------------------------------- gated feed-forward block --- */

/* act(x): SILU x sigmoid(x); GELU, the Gaussian error linear unit in its tanh form,
 * 0.5 x (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))); RELU max(x, 0). */
typedef enum { SBP_ACT_SILU = 0, SBP_ACT_GELU = 1, SBP_ACT_RELU = 2 } sbp_act_t;

/* The first half of a gated feed-forward block on rank r's shares,
 *     H = act(X Wg) * (X Wu)   (element-wise product),
 * both projections, the activation and the product in one kernel for bf16. X: M x K,
 * state *lx; Wg, Wu: K x N, both in state *lw. The product with the down projection is
 * an ordinary linear (sbp_linear_fwd on H).
 *
 * Signatures: those of Y = X W whose Y is no partial sum -- DP, COL and BB (an
 * activation of a partial sum is no partial sum of activations); else
 * SBP_ERR_SIGNATURE. H takes Y's state, dH dY's, dX and the weights' gradients
 * dX's and dW's:
 *     DP   H S(0)   dH S(0)   dX S(0)   dWg, dWu P
 *     COL  H S(1)   dH S(1)   dX P      dWg, dWu S(1)
 *     BB   H B      dH P      dX P      dWg, dWu P
 *
 * sbp_gated_fwd: H, and with G and U (both or neither NULL) the projections
 * G = X Wg, U = X Wu for the backward pass. Inputs bf16 or fp32; H, G and U have the
 * inputs' dtype (SBP_ERR_DTYPE) and the local shape. H is computed from the fp32 sums,
 * not from the rounded G and U. fp32 calls need G and U (SBP_ERR_NULL).
 *
 * sbp_gated_bwd: from dH, G and U
 *     dU = dH * act(G),  dG = dH * U * act'(G),
 *     dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU.
 * G and U: H's state, as the forward call left them. dG, dU: local m x n buffers of
 * the inputs' dtype that the call fills (bf16: rounded, as the operands of the
 * products, whose fp32 results carry that rounding too). dX, dWg, dWu: fp32, or for bf16
 * inputs bf16 where they are no partial sum of several devices (a sum over one device
 * is the tensor); SBP_ACCUMULATE adds to fp32 contents. dWg and dWu have one dtype. dX is
 * rounded once, from the sum of both products (twice, once per product, where an fp32
 * operand's leading dimension is 2^21 or more). bf16 calls are fastest with K, N, every
 * operand's start (16 bytes) and leading dimension multiples of 8, one leading dimension of
 * Wg and Wu, and one of dG and dU; with others the operands pass through registers (8192 x
 * 8192 with 8192 x 4096 weights: 1.86 ms, and 2.44 where Wu's rows are longer than Wg's).
 *
 * No output may overlap an input or another output. ws as for sbp_linear_fwd. Errors:
 * those of the linear calls; SBP_ERR_SHAPE also for an unknown act, for outputs of 2^22
 * tiles of 64 x 64 or more, and for dX, dWg and dWu of 2^23 such tiles together. */
int sbp_gated_fwd(const sbp_view_t *X, const sbp_layout_t *lx, const sbp_view_t *Wg,
                  const sbp_view_t *Wu, const sbp_layout_t *lw, int32_t act,
                  sbp_view_t *H, sbp_layout_t *lh_out, sbp_view_t *G, sbp_view_t *U,
                  const sbp_workspace_t *ws, hipStream_t stream);
int sbp_gated_bwd(const sbp_view_t *dH, const sbp_layout_t *ldh, const sbp_view_t *X,
                  const sbp_layout_t *lx, const sbp_view_t *Wg, const sbp_view_t *Wu,
                  const sbp_layout_t *lw, int32_t act, const sbp_view_t *G,
                  const sbp_view_t *U, sbp_view_t *dG, sbp_view_t *dU, sbp_view_t *dX,
                  sbp_layout_t *ldx_out, sbp_view_t *dWg, sbp_view_t *dWu,
                  sbp_layout_t *ldw_out, const sbp_workspace_t *ws, hipStream_t stream);
/* nd forms: one of DP, COL and BB on every mesh axis. */
int sbp_nd_gated_fwd(const sbp_view_t *X, const sbp_nd_layout_t *lx, const sbp_view_t *Wg,
                     const sbp_view_t *Wu, const sbp_nd_layout_t *lw, int32_t act,
                     sbp_view_t *H, sbp_nd_layout_t *lh_out, sbp_view_t *G, sbp_view_t *U,
                     const sbp_workspace_t *ws, hipStream_t stream);
int sbp_nd_gated_bwd(const sbp_view_t *dH, const sbp_nd_layout_t *ldh,
                     const sbp_view_t *X, const sbp_nd_layout_t *lx,
                     const sbp_view_t *Wg, const sbp_view_t *Wu,
                     const sbp_nd_layout_t *lw, int32_t act, const sbp_view_t *G,
                     const sbp_view_t *U, sbp_view_t *dG, sbp_view_t *dU,
                     sbp_view_t *dX, sbp_nd_layout_t *ldx_out, sbp_view_t *dWg,
                     sbp_view_t *dWu, sbp_nd_layout_t *ldw_out,
                     const sbp_workspace_t *ws, hipStream_t stream);

/* ------------------------------ attention core under a head split --- */

/* A strided 4-D view [batch][heads][rows][cols]: element (b, h, i, j) is at
 * data + b*stride_b + h*stride_h + i*ld + j (elements). Views into a fused
 * activation -- e.g. the Q, K or V part of a QKV projection output laid out
 * [batch][seq][3][heads][head_dim] -- have stride_h = head_dim and ld =
 * 3*heads*head_dim. scope: SBP_GLOBAL (inputs) -- heads counts all H heads
 * and the call takes rank r's heads; SBP_LOCAL -- heads counts rank r's
 * heads only; outputs always hold rank r's heads (SBP_ACCUMULATE adds to an
 * fp32 output, as for the 2-D calls). */
typedef struct {
    void *data;
    int64_t batch, heads, rows, cols;
    int64_t stride_b, stride_h, ld;
    int32_t dtype; /* sbp_dtype_t */
    int32_t scope; /* sbp_scope_t */
} sbp_view4_t;

/* Multi-head attention reduces to batched matrix products (Sec. 2). Under a
 * split of the head dimension over p devices (heads split(H, p, r), the
 * balanced rule), every operand and output is Split on heads and each
 * device multiplies its own heads: one product per (batch, local head), no
 * partial sums. Inputs are bf16 (SBP_ERR_DTYPE otherwise); outputs bf16
 * (rounded to nearest even) or fp32. Softmax, its scale and masking are not
 * part of these calls.
 *
 *   sbp_attn_scores       S  = Q K^T    Q: [B][H][Sq][D], K: [B][H][Sk][D]
 *                                       -> S: [B][H_r][Sq][Sk]
 *   sbp_attn_context      O  = P V      P: [B][H][Sq][Sk], V: [B][H][Sk][D]
 *                                       -> O: [B][H_r][Sq][D]
 *   sbp_attn_scores_bwd   dQ = dS K, dK = dS^T Q (dS like S; dQ like Q, dK
 *                         like K, each over rank r's heads)
 *   sbp_attn_context_bwd  dP = dO V^T, dV = P^T dO (dO like O; dP like P, dV
 *                         like V)
 *
 * Errors: SBP_ERR_NULL, SBP_ERR_LAYOUT (p < 1 or r outside [0, p)),
 * SBP_ERR_SHAPE (extents that disagree, ld < cols, a negative or too large
 * extent or stride, an output whose elements overlap one another, or an
 * output of the wrong shape), SBP_ERR_DTYPE, SBP_ERR_ALIGN, SBP_ERR_ALIAS
 * (an output's span overlaps an input's or the other output's span),
 * SBP_ERR_HIP. Batched products never split their reduction, so these calls
 * take no workspace. */
int sbp_attn_scores(const sbp_view4_t *Q, const sbp_view4_t *K, sbp_view4_t *S,
                    int32_t p, int32_t r, hipStream_t stream);
int sbp_attn_context(const sbp_view4_t *P, const sbp_view4_t *V, sbp_view4_t *O,
                     int32_t p, int32_t r, hipStream_t stream);
int sbp_attn_scores_bwd(const sbp_view4_t *dS, const sbp_view4_t *Q,
                        const sbp_view4_t *K, sbp_view4_t *dQ, sbp_view4_t *dK,
                        int32_t p, int32_t r, hipStream_t stream);
int sbp_attn_context_bwd(const sbp_view4_t *dO, const sbp_view4_t *P,
                         const sbp_view4_t *V, sbp_view4_t *dP, sbp_view4_t *dV,
                         int32_t p, int32_t r, hipStream_t stream);

/* ------------------------------------------------- softmax attention --- */

/* What a query sees, and the scores' scale. len_q, len_k: device arrays of one
 * int32 per sequence (its rows of Q, and of K and V, that are in use; read when the
 * call runs, clamped to [0, rows]), or NULL for all rows. Query i of a sequence sees
 * key j when
 *     i < len_q,  j < len_k,
 *     causal:      j <= i + len_k - len_q   (the last query sees the last key)
 *     window > 0:  j >  i + len_k - len_q - window. */
typedef struct {
    float scale;      /* 2^-100 to 2^100 (else SBP_ERR_SHAPE); usually 1/sqrt(D) */
    int32_t causal;   /* 0 or 1 */
    int32_t window;   /* >= 0; 0: none */
    const int32_t *len_q;
    const int32_t *len_k;
} sbp_attn_opts_t;

/* Attention of rank r's heads without scores or probabilities in memory.
 *
 *   sbp_attn_core_fwd   O_i = sum_j P_ij V_j,  P_ij = exp(scale Q_i.K_j - lse_i),
 *                       lse_i = log sum_j exp(scale Q_i.K_j), over the keys j that
 *                       query i sees
 *   sbp_attn_core_bwd   from dO, O and lse: dV = P^T dO, dS = P (dO V^T - rowsum(dO O)),
 *                       dQ = scale dS K, dK = scale dS^T Q, with P recomputed
 *
 * Q, dO, O, dQ: [B][H][Sq][D]; K, V, dK, dV: [B][Hk][Sk][D]; lse: [B][H][Sq][1], fp32.
 * H is a multiple of Hk: query heads h G .. h G + G - 1 (G = H / Hk) share key head h,
 * whose gradients sum over them. 1 <= D <= 128. Q, K, V and dO are bf16; O and the
 * gradients bf16 (rounded to nearest even) or fp32; SBP_ACCUMULATE adds to an fp32
 * gradient (not to O or lse: SBP_ERR_SHAPE). Scores, row statistics and sums are fp32;
 * P and dS are rounded to bf16 as operands of the matrix products, so fp32 outputs
 * carry that rounding too.
 * The forward call takes finite scores of any size. The backward call recomputes P
 * from lse, whose 24 bits leave it off by a factor of up to exp(2^-22 |lse|): 2^-10 of it
 * where the scores, scaled, reach 2^12, a sixteenth at 2^18, and no use from 2^22 on (past
 * 2^28 P may overflow).
 *
 * Head split: key heads split over p devices by the balanced rule, query heads with
 * them (rank r has G per key head of its share). Q, K and V share one scope; dO, O
 * and lse may be GLOBAL or LOCAL. Outputs hold rank r's heads. Every operand is Split
 * on heads; nothing is a partial sum.
 *
 * Rows that see no key get O = 0, lse = -infinity and dQ = 0, whatever the other rows
 * hold (accumulated gradients stay as they are); so do rows past len_q and, in dK and dV,
 * keys past len_k, whose inputs are never read. Else a non-finite K, V, Q or dO row within
 * the lengths may reach every row of its head and sequence, also those that do not see it
 * or that it does not see. lse may be NULL in the forward call.
 *
 * ws: the forward call uses a workspace, if it has one, to split the keys of few rows
 * over workgroups. The backward call needs 8 bytes per query row of the rank
 * (8 B H_r Sq, rounded up to 32), else SBP_ERR_WORKSPACE, and splits with the rest.
 * Results are the same up to fp32 summation order and identical for identical
 * workspace sizes.
 *
 * Errors: those of the calls above; SBP_ERR_SHAPE also for D outside [1, 128], H not a
 * multiple of Hk, more than 2^29 rows of a sequence, or more of them in all than a
 * launch covers (B H_r Sq > 2^28 - 16, or 2^24 tiles of 32 keys or of 32 rows of a
 * group; in the backward call 2^24 tiles of 64 keys and of 64 rows of a group, taken
 * together). Outputs may interleave in one buffer
 * (dQ, dK and dV as parts of a fused gradient) when their strides agree and their
 * columns do not meet. */
int sbp_attn_core_fwd(const sbp_view4_t *Q, const sbp_view4_t *K, const sbp_view4_t *V,
                      const sbp_attn_opts_t *opts, sbp_view4_t *O, sbp_view4_t *lse,
                      int32_t p, int32_t r, const sbp_workspace_t *ws,
                      hipStream_t stream);
int sbp_attn_core_bwd(const sbp_view4_t *dO, const sbp_view4_t *Q,
                      const sbp_view4_t *K, const sbp_view4_t *V, const sbp_view4_t *O,
                      const sbp_view4_t *lse, const sbp_attn_opts_t *opts,
                      sbp_view4_t *dQ, sbp_view4_t *dK, sbp_view4_t *dV, int32_t p,
                      int32_t r, const sbp_workspace_t *ws, hipStream_t stream);

/* --------------------------------------------------- rotary positions --- */

/* Which columns of a head's first `dim` make a pair: HALVES (i, i + dim / 2), PAIRS
 * (2 i, 2 i + 1), for i in [0, dim / 2). */
typedef enum { SBP_ROPE_HALVES = 0, SBP_ROPE_PAIRS = 1 } sbp_rope_order_t;

/* Frequency of pair i, radians a position: f_i = base^(-2 i / dim), and for contexts that are
 * `factor` times as long as the `context` a model was trained on
 *   LINEAR    f_i / factor
 *   BASE      base factor^(dim / (dim - 2)) in place of base (dim 2: base itself)
 *   BY_TURNS  f_i w + f_i / factor (1 - w), w = (n_i - low) / (high - low) limited to [0, 1],
 *             where n_i = context f_i / 2 pi are pair i's turns over the context
 *   BY_PAIRS  f_i (1 - w) + f_i / factor w, w = (i - a) / max(b - a, 0.001) limited to [0, 1],
 *             a = max(0, floor(at(high))), b = min(dim - 1, ceil(at(low))), where at(n) =
 *             dim ln(context / (2 pi n)) / (2 ln base) is the pair with n turns */
typedef enum { SBP_ROPE_PLAIN = 0, SBP_ROPE_LINEAR = 1, SBP_ROPE_BASE = 2,
               SBP_ROPE_BY_TURNS = 3, SBP_ROPE_BY_PAIRS = 4 } sbp_rope_scaling_t;

/* The dim / 2 frequencies as turns a position, in units of 2^-64 turn, to HOST memory; the
 * caller copies them to the device once. The angle of a position is a product modulo 2^64, so
 * far positions lose nothing: at t it is off by t 2^-62 turns at most, for a factor below 1 by
 * 1 / factor times that (the frequencies, up to 1 / factor, are computed in the host's long
 * double; for factors from 2^-32 on and high >= 2 low). Pure host function. Errors:
 * SBP_ERR_NULL, SBP_ERR_SHAPE (dim odd or outside [2, 128], base <= 1 or not finite, an unknown
 * scaling; for a scaling factor <= 0; BY_TURNS and BY_PAIRS context <= 0, low <= 0 or high <= low;
 * or a number that is not finite). */
int sbp_rope_turns(int32_t dim, double base, int32_t scaling, double factor, double low,
                   double high, double context, uint64_t *turns);

/* A rotation: the table of sbp_rope_turns in device memory, and its dim. `mul` multiplies the
 * rotated columns (1: a pure rotation). */
typedef struct {
    const uint64_t *turns;
    int32_t dim;      /* even, 2 .. the head dimension; columns past it are copied */
    int32_t order;    /* sbp_rope_order_t */
    float mul;        /* finite */
} sbp_rope_t;

/* The rows' positions, any int32, read when the call runs. per_row: row i of sequence b is at
 * pos[b ld + i]; else at pos[b ld] + i. A NULL sbp_places_t: at i. */
typedef struct {
    const int32_t *pos;
    int64_t ld;
    int32_t per_row;
} sbp_places_t;

/* Rotation of rank r's heads of Q and K by the positions of their rows, in one launch (K and Ko
 * may be NULL). At position t, with c = mul cos(t f_i) and s = mul sin(t f_i), pair i becomes
 *   sbp_rope_fwd   y1 = x1 c - x2 s,  y2 = x2 c + x1 s
 *   sbp_rope_bwd   dx1 = dy1 c + dy2 s,  dx2 = dy2 c - dy1 s
 * Q: [B][H][S][D], K: [B][Hk][S][D], one scope; heads split as for softmax attention (without
 * K: the heads of Q by the balanced rule). 1 <= D <= 128. Outputs hold rank r's heads.
 * Inputs bf16 or fp32 (one dtype); outputs of one dtype, the inputs', or fp32 for bf16 inputs
 * (SBP_ERR_DTYPE; SBP_ACCUMULATE: SBP_ERR_SHAPE). Angles, cosines and products are fp32 or
 * better, each output is rounded once. An output may be the rank's part of its own input
 * (the same address, strides and dtype: in place); else no output may overlap an input or the
 * other output, but for outputs that interleave as those of sbp_attn_core_bwd may.
 * Errors: those of the attention calls; SBP_ERR_SHAPE also for more than 2^29 rows of a
 * sequence, or 2^31 / ((D + 23) / 8) rows over the rank's heads. */
int sbp_rope_fwd(const sbp_view4_t *Q, const sbp_view4_t *K, const sbp_rope_t *rope,
                 const sbp_places_t *at, sbp_view4_t *Qo, sbp_view4_t *Ko, int32_t p, int32_t r,
                 hipStream_t stream);
int sbp_rope_bwd(const sbp_view4_t *dQo, const sbp_view4_t *dKo, const sbp_rope_t *rope,
                 const sbp_places_t *at, sbp_view4_t *dQ, sbp_view4_t *dK, int32_t p, int32_t r,
                 hipStream_t stream);

/* --------------------------------------- paged cache of keys and values --- */

/* A cache is two views [pages][heads][tokens of a page][D], one of keys and one of values, of
 * any strides (a page's tokens or its heads outside). Token t of sequence b is row t % P
 * of page table[b table_ld + t / P], P tokens a page. All arrays are device memory, read when a
 * call runs. The new tokens' rows (of Q, K, V and O) are
 *   padded   row_q NULL: views of `seqs` batches, sequence b the first len_q[b] rows of batch b
 *            (limited to [0, rows]; len_q NULL: all)
 *   packed   views of one batch, sequence b rows row_q[b] .. row_q[b + 1] - 1, limited to the
 *            view. row_q must not descend (else what the rows hold is not defined, but nothing
 *            outside the views and the workspace is touched). len_q must be NULL. Rows of no
 *            sequence are never read or written.
 * len_k[b]: tokens that sequence b has in the cache once its n new ones are there, so that new
 * token i is at place len_k[b] - n + i. Not more than width P, the table's room: past that the two
 * calls differ. sbp_paged_append counts places from len_k as it is (rotates by them, and stores
 * those in the room); sbp_paged_attn takes width P for it everywhere, also in its masks, which
 * then see the new tokens at the room's last places. sbp_paged_attn chooses its kernel for the
 * room: a table cut to the width that a step's longest sequence needs serves short ones better. */
typedef struct {
    const int32_t *table;
    int64_t table_ld;     /* >= width */
    int32_t seqs, width;  /* sequences; entries of a table row: width P tokens at most */
    const int32_t *len_k; /* [seqs] */
    const int32_t *len_q; /* [seqs], or NULL */
    const int32_t *row_q; /* [seqs + 1], or NULL */
} sbp_pages_t;

/* Stores the new tokens' keys and values in the cache. With `rope` the keys are rotated on
 * the way by their places, and with Q and Qo (both or neither NULL) Q's rows by theirs, all in
 * one launch. Without `rope` Q must be NULL.
 * K, V: [B][Hk][S][D] and Q: [B][H][S][D], of one scope, bf16; Kc, Vc: the cache, bf16, of one
 * scope, which may be another (LOCAL: rank r's heads). Qo: rank r's heads, bf16 or fp32; it
 * may be the rank's part of Q itself. Heads split as for softmax attention.
 * Tokens at places outside [0, width P), or on a page outside [0, pages), are not stored; nothing
 * else of the cache is written. Two tokens of one call must not share a row of the cache (it
 * would hold parts of either). Qo's rows past len_q stay as they are.
 * Errors: those of the attention calls; SBP_ERR_SHAPE also for P < 1, width P > 2^29, more than
 * 2^20 sequences, more rows over the heads of Q, K and V than sbp_rope_fwd takes, or rows that do
 * not fit `seqs`; SBP_ERR_ALIAS also for a cache that overlaps another operand or whose own
 * elements overlap. */
int sbp_paged_append(const sbp_view4_t *K, const sbp_view4_t *V, const sbp_pages_t *pages,
                     const sbp_rope_t *rope, sbp_view4_t *Kc, sbp_view4_t *Vc,
                     const sbp_view4_t *Q, sbp_view4_t *Qo, int32_t p, int32_t r,
                     hipStream_t stream);

/* Softmax attention of the new tokens over the cache (sbp_attn_core_fwd's formulas): query i
 * of the n new ones of a sequence sees key j when
 *     j < len_k
 *     causal:      j <= i + len_k - n
 *     window > 0:  j >  i + len_k - n - window
 * with len_k limited to [0, width P] in all three,
 * and j's page is in [0, pages): keys on other pages are not seen. Entries of the table whose
 * keys no query of the sequence sees are not read.
 * Q: [B][H][S][D] bf16; Kc, Vc: [pages][Hk][P][D] bf16, of Q's scope; H a multiple of Hk,
 * 1 <= D <= 128; O and lse (fp32, may be NULL) as in sbp_attn_core_fwd, rounding and
 * scores' size too. Rows that see no key, and padded rows past len_q, get O = 0, lse = -infinity.
 * A non-finite K, V or Q row that some query of its sequence sees may reach every row of its
 * head and sequence; cache rows that no query of the sequence sees are not read.
 * ws: splits the work into equal parts, if there is one; results are the same up to fp32
 * summation order, and identical for identical lengths and workspace sizes.
 * Errors: those of sbp_attn_core_fwd and sbp_paged_append. */
int sbp_paged_attn(const sbp_view4_t *Q, const sbp_view4_t *Kc, const sbp_view4_t *Vc,
                   const sbp_pages_t *pages, float scale, int32_t causal, int32_t window,
                   sbp_view4_t *O, sbp_view4_t *lse, int32_t p, int32_t r,
                   const sbp_workspace_t *ws, hipStream_t stream);

/* ------------------------------------- cost model and strategy search --- */

/* Collectives of the alpha-beta model (Sec. 3.1, Table 2). */
enum {
    SBP_COLL_ALLREDUCE = 0,      /* (2p-1) alpha + 2 (p-1)/p n beta          */
    SBP_COLL_ALLGATHER = 1,      /* (p-1) alpha + (p-1)/p n beta             */
    SBP_COLL_REDUCESCATTER = 2,  /* (p-1) alpha + (p-1)/p n beta             */
    SBP_COLL_ALLTOALL = 3        /* (p-1) alpha + n beta                     */
};

/* Time of one collective over p devices for an n-byte message (the input
 * of ReduceScatter, the output of the others, per device), latency alpha
 * (seconds) and inverse bandwidth beta (seconds per byte): the formulas of
 * Table 2 as printed. Pure host function. Errors: SBP_ERR_NULL,
 * SBP_ERR_LAYOUT (p < 1, unknown collective), SBP_ERR_SHAPE (negative n,
 * alpha or beta). */
int sbp_collective_cost(int32_t coll, int32_t p, double n, double alpha, double beta,
                        double *cost);

/* Time to redistribute a tensor of `bytes` (global size) from 1-D state
 * *from to 1-D state *to on the same p devices (Sec. 4.2 redistributions,
 * Sec. 4.3 "Sources of Communication"): S(i)->S(j), i != j: AlltoAll of
 * bytes/p; S->B: AllGather of bytes; P->S: ReduceScatter of bytes; P->B:
 * AllReduce of bytes; every other change (B->S, B->P, S->P) and no change:
 * 0 (local). *coll_out, if not NULL, receives the collective used, or -1.
 * Errors: SBP_ERR_NULL, SBP_ERR_LAYOUT (bad states, p mismatch),
 * SBP_ERR_SHAPE. */
int sbp_boxing_cost(const sbp_layout_t *from, const sbp_layout_t *to, double bytes,
                    double alpha, double beta, double *cost, int32_t *coll_out);

/* Signature ids for the search: the rows of the table at the top of this
 * file, in order. */
enum { SBP_SIG_DP = 0, SBP_SIG_COL = 1, SBP_SIG_KS = 2, SBP_SIG_PB = 3, SBP_SIG_BP = 4,
       SBP_SIG_BB = 5 };

/* A chain of linear layers Y_l = X_l W_l (X_l: M x K[l], W_l: K[l] x N[l])
 * on a 1-D mesh of p devices, one signature per layer. Between layers the
 * previous output (M x N[l] elements; M is the same for every layer) is
 * redistributed from layer l's output state to layer l+1's input state; an
 * op between the two (an activation function, the attention core, which
 * maps 3 x hidden to hidden columns) keeps the state, so K[l+1] may differ
 * from N[l]. The network input (M x K[0]) starts in state (in_kind,
 * in_axis) and the last output must end in (out_kind, out_axis). A
 * Partial-sum output is never fed on as is (a nonlinearity separates the
 * layers), so signatures with a Partial-sum X (PB) are not allowed. */
typedef struct {
    int32_t layers;
    int32_t p;
    double alpha, beta;          /* seconds, seconds per byte */
    const int64_t *M, *K, *N;    /* per layer */
    double act_bytes;            /* bytes per activation element */
    double grad_bytes;           /* bytes per weight-gradient element */
    int32_t in_kind, in_axis, out_kind, out_axis;
    uint32_t allowed;            /* bit s: signature s may be chosen */
} sbp_chain_t;

/* Communication time of one training step of the chain under signatures
 * sigs[0..layers): for every activation redistribution, its forward cost
 * plus the backward cost of moving the gradient the other way (the dual
 * states: grad of S(i) is S(i), of B is P, of P is B), plus an AllReduce of
 * every weight gradient left Partial-sum (Sec. 4.3). Pure host function.
 * Errors: SBP_ERR_NULL, SBP_ERR_SHAPE (layers < 1, extents), SBP_ERR_LAYOUT
 * (p, boundary states), SBP_ERR_SIGNATURE (a signature not allowed). */
int sbp_chain_cost(const sbp_chain_t *net, const int32_t *sigs, double *cost);

/* Coordinate-descent search (Sec. 4.4): from an initial guess, each sweep
 * sets every layer in turn to the allowed signature that minimises the
 * chain cost with the others fixed (a change only on strict improvement, so
 * the cost never rises); at a fixed point the run restarts from a new
 * random guess, and the best strategy of `restarts` runs (>= 1; the first
 * starts from all-DP where allowed) is returned in sigs_out with its cost.
 * sweep_costs (may be NULL) receives, run after run, each run's starting
 * cost followed by its cost after every sweep, up to max_sweeps entries;
 * within a run the values strictly decrease until the final sweep, which
 * changes nothing and repeats the previous value. *sweeps_out (may be
 * NULL) receives the total count of entries.
 * Random guesses come from splitmix64 seeded with `seed`. Pure host
 * function. Errors: those of sbp_chain_cost, SBP_ERR_SHAPE (restarts < 1). */
int sbp_search_strategy(const sbp_chain_t *net, int32_t restarts, uint64_t seed,
                        int32_t *sigs_out, double *cost_out, double *sweep_costs,
                        int32_t max_sweeps, int32_t *sweeps_out);

/* --------------------------------------------------------- utilities --- */

/* Static description of an error code (never NULL). */
const char *sbp_strerror(int code);

/* hipError_t of the last SBP_ERR_HIP returned on the calling thread
 * (0 if none). */
int sbp_last_hip_error(void);

/* Kernel plan the library would use for a local product of m x n outputs
 * over a reduction of k with 16-byte aligned operands and tight leading
 * dimensions, for input dtype in_dtype, output dtype out_dtype and operand
 * orientation op (0 forward, 1 backward-data, 2 backward-weight). Writes
 * the tile rows and columns, the number of reduction splits and the kernel
 * (3 fp32, else the bf16 instance code of sbp_set_plan_override), as
 * planned with a workspace of SBP_WORKSPACE_BYTES. For benchmarks and
 * tests; pure host function.
 * Errors: SBP_ERR_NULL, SBP_ERR_SHAPE, SBP_ERR_DTYPE. */
int sbp_plan(int op, int64_t m, int64_t n, int64_t k, int32_t in_dtype,
             int32_t out_dtype, int32_t *tile_m, int32_t *tile_n,
             int32_t *splits, int32_t *kernel);

/* Plan of sbp_linear_bwd for bf16 inputs with 16-byte aligned operands and
 * tight leading dimensions: the backward-data product is md x nd over a
 * reduction of kd with output dtype out_d, the backward-weight product
 * mw x nw over kw with out_w. Writes whether both run as one grouped launch,
 * the tile of the backward-data product (shared when grouped), and the
 * splits of each product, as planned with a workspace of
 * SBP_WORKSPACE_BYTES. Pure host function. Errors: SBP_ERR_NULL, SBP_ERR_SHAPE, SBP_ERR_DTYPE. */
int sbp_plan_bwd(int64_t md, int64_t nd, int64_t kd, int32_t out_d, int64_t mw,
                 int64_t nw, int64_t kw, int32_t out_w, int32_t *grouped,
                 int32_t *tile_m, int32_t *tile_n, int32_t *splits_d,
                 int32_t *splits_w);

/* Per-kernel timing for benchmarks. After sbp_profile_begin(capacity), the
 * first `capacity` kernels that the library launches from the calling
 * thread are each bracketed by a HIP event pair recorded with the dispatch
 * itself (hipExtLaunchKernelGGL). sbp_profile_end stops recording, waits for
 * those events, writes each kernel's duration in microseconds to us[i] and
 * its name (NUL-terminated, at most name_len bytes) to names + i*name_len
 * (either may be NULL), and returns the number of kernels recorded, or
 * SBP_ERR_HIP. Not for use while a stream is being captured into a graph. */
int sbp_profile_begin(int capacity);
int sbp_profile_end(float *us, char *names, int name_len);

/* Thread-local override of the bf16 plan for subsequent calls on this
 * thread (tests and tuning). tile_m x tile_n is one of 256x256, 256x192,
 * 256x128, 128x256, 128x128, 128x64, 64x128, 64x64; splits >= 1. kernel
 * selects the instance:
 *   0, 1  the tile's default pipelined direct-to-LDS instance (256x192:
 *         eight waves as 4 x 2, two stages; as many 256 x 192 tiles as
 *         compute units for a 4096 x 3072 output);
 *   2     the generic kernel;
 *   4     pipelined with two stages (128x128, 128x64, 64x128, 64x64: two or
 *         more workgroups per compute unit);
 *   5     pipelined, eight waves in two reduction groups, output staged in
 *         LDS (256x128, 128x256, 128x128, 128x64, 64x128, 64x64);
 *   6     pipelined, row-quad epilogue: MFMA operands swapped so each lane
 *         stores 4 consecutive outputs of a row from registers (256x256, and
 *         128x128 with two stages);
 *   7     as 5 with the row-quad epilogue (256x128, 128x256, 128x128, 128x64,
 *         64x128, 64x64);
 *   8     pipelined with 32-wide reduction stages, five in LDS (256x256);
 *   9     as 5 with 32-wide reduction stages, six (256x128, 128x256) or
 *         eight (128x128) in LDS;
 *   10    as 5 with two stages, two workgroups per compute unit (128x128);
 *   11    pipelined with deep prefetch for operand streams that HBM latency
 *         bounds: six stages (128x64, 64x128) or eight (64x64) in LDS;
 *   12    as 5 with 128-wide reduction stages, two (128x128), three
 *         (128x64, 64x128) or four (64x64) in LDS: half the barriers and
 *         twice the bytes per operand row of 64-wide stages;
 *   13    as 12 with the row-quad epilogue.
 * wgs_per_cu > 0 makes the launch persistent: at most wgs_per_cu workgroups
 * per compute unit, each taking every G-th work item (0 = one workgroup per
 * item; the grouped backward launch always runs one per item). A call whose
 * operands the pipelined kernel cannot read runs the generic kernel, where
 * 256x256 and 256x192 become 256x128; splits are clamped to the reduction
 * blocks and to the call's workspace. An unsplit product that is added to its
 * output (SBP_ACCUMULATE) exists for codes 1 (256x256, 256x192, 64x64), 4, 12
 * and 2 only: under another code it runs code 4 or 1 of its tile, else 2.
 * tile_m = 0 clears the override.
 * Errors: SBP_ERR_SHAPE for a (tile, kernel) pair not listed above,
 * splits < 1, or wgs_per_cu outside [0, 8]. */
int sbp_set_plan_override(int32_t tile_m, int32_t tile_n, int32_t splits,
                          int32_t kernel, int32_t wgs_per_cu);

/* Thread-local choice of how sbp_linear_bwd runs its two products (tuning):
 * mode 0 = the library's choice, 1 = two launches, one per product, 2 = one
 * grouped launch on the tile and kernel of sbp_set_plan_override (which must
 * be set, else mode 2 acts as 0), with that override's splits for the
 * backward-data product and splits_w for the backward-weight product.
 * Clearing the plan override (tile_m = 0) also resets this to mode 0.
 * Errors: SBP_ERR_SHAPE for a mode outside [0, 2] or splits_w < 1. */
int sbp_set_bwd_override(int32_t mode, int32_t splits_w);

/* Restricts the plan override of sbp_set_plan_override to the products of
 * the orientations in mask (bit 0 forward / Y = X W, bit 1 backward-data /
 * A B^T, bit 2 backward-weight / A^T B); the others keep their own plans
 * (tuning one product of a two-product call). Clearing the plan override
 * (tile_m = 0) resets the mask to 7. Errors: SBP_ERR_SHAPE for a mask
 * outside [1, 7]. */
int sbp_set_override_orients(int32_t mask);

#ifdef __cplusplus
}
#endif

#endif /* SBP_H */
