/*
 * brownout_moe.h -- C ABI of the grouped ("full-brownout") MoE layer forward
 * for AMD Instinct MI355X (gfx950).
 *
 * The layer (paper: Sec. 2.1 for the top-K MoE layer, Eq. 1-2 in Sec. 4.2 for
 * the expert-to-group map, the closing paragraphs of Sec. 4.3 and Sec. 4.4 for
 * how the map is used while serving): a gate picks each token's top-k experts
 * among E; a map g sends expert e to united expert g(e) of G; under full
 * brownout every picked expert is served by its united expert. A token whose
 * picks share a united expert calls it once with the sum of their gate
 * weights. The output is
 *
 *     out_t = sum over distinct groups r of t's picks of gamma_{t,r} * FFN_r(x_t)
 *             (+ shared-expert FFN(x_t) when the layer has shared experts)
 *
 * with FFN_r a SwiGLU expert, y = W_down (silu(W_gate a) * (W_up a)).
 *
 * Four calls make one forward, enqueued on one stream with no host sync:
 *   brownout_moe_route     gate logits, softmax, top-k, map, per-group merge
 *   brownout_moe_dispatch  per-group histogram, prefix, stable permutation, row gather
 *   brownout_moe_ffn       grouped SwiGLU FFN over the united experts
 *   brownout_moe_combine   gate-weighted sum back into token order
 * For up to 16 tokens one call does the same (brownout_moe_few). The experts may be held
 * in 4 bits (bmoe_w4; brownout_moe_w4_ffn in place of brownout_moe_ffn, or brownout_moe_few),
 * or in 8 bits with the activations rounded to 8 bits by token (bmoe_w8; brownout_moe_w8_ffn).
 * brownout_moe_balance measures how evenly the router's picks fall, with its gradient by the logits.
 * brownout_moe_pre_norm and brownout_moe_post_norm are the layer's two ends in a residual block.
 *
 * Conventions for every call:
 *   - Tensor pointers are DEVICE pointers, row-major, owned by the caller. The
 *     library allocates and frees nothing at run time. Its only device memory
 *     is two fixed arrays of its code object, one copy per GPU: 64 KiB of
 *     zeros that the FFN's copies of padding rows read, and the workspace of
 *     brownout_moe_dispatch_noalloc. On the host it caches per-device facts
 *     (CU count, those arrays' addresses, kernel attributes set once).
 *   - Weights use the [out, in] layout: W_gate/W_up [n, d_ff, d], W_down [n, d, d_ff].
 *   - Every call checks its arguments on the host before it enqueues anything;
 *     on error it returns a BMOE_ERR_* code and writes nothing. Launch failures
 *     return BMOE_ERR_HIP. Calls are asynchronous on `stream` (a hipStream_t;
 *     NULL is the default stream); outputs are valid once the stream has
 *     reached them.
 *   - Pointers to float/bf16 tensors that kernels read or write 16 bytes at a
 *     time (x, x_perm, w_*, h, y, out, y_shared) must be 16-byte aligned; d and
 *     d_ff must be multiples of 8.
 *   - T == 0 is a no-op that returns BMOE_OK.
 *   - Inputs must be finite.
 */
#ifndef BROWNOUT_MOE_H
#define BROWNOUT_MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define BMOE_API __attribute__((visibility("default")))
#else
#define BMOE_API
#endif

#define BMOE_MAX_EXPERTS 256 /* E <= 256, hence G <= 256 */
#define BMOE_MAX_TOPK 16     /* top_k <= 16 */

/* Route decides every token whose fast fp32 logits leave any two of its top
 * (k+1) values closer than this gap (2^-14) again from float64 logits; see
 * brownout_moe_route. The gap is far above the error of the fp32 logits (a few
 * 1e-6 at d = 4096), so every pair the fp32 logits order is ordered the same
 * way by the float64 ones. */
#define BMOE_ROUTE_RECHECK_GAP (1.0f / 16384.0f)

typedef enum bmoe_status {
    BMOE_OK = 0,
    BMOE_ERR_NULL = 1,        /* a required pointer is NULL                       */
    BMOE_ERR_SHAPE = 2,       /* a size is out of range                            */
    BMOE_ERR_ALIGN = 3,       /* a pointer is not 16-byte aligned                  */
    BMOE_ERR_MAP = 4,         /* an expert-to-group map entry is outside [0, G)    */
    BMOE_ERR_UNSUPPORTED = 5, /* unknown dtype, or a mode this build does not do  */
    BMOE_ERR_WORKSPACE = 6,   /* workspace missing or too small                    */
    BMOE_ERR_HIP = 7          /* the HIP runtime reported an error at launch       */
} bmoe_status;

typedef enum bmoe_dtype {
    BMOE_F32 = 0,  /* float activations and weights                        */
    BMOE_BF16 = 1  /* bf16 activations and weights, fp32 accumulation      */
} bmoe_dtype;

typedef enum bmoe_stage {
    BMOE_STAGE_ROUTE = 0,
    BMOE_STAGE_DISPATCH = 1,
    BMOE_STAGE_FFN = 2,
    BMOE_STAGE_COMBINE = 3,
    BMOE_STAGE_DOWN_COMBINE = 4, /* brownout_moe_ffn_down_combine */
    BMOE_STAGE_FEW = 5           /* brownout_moe_few */
} bmoe_stage;

/* Shape of one layer. */
typedef struct bmoe_desc {
    int32_t T;           /* tokens, >= 0                                          */
    int32_t d;           /* model width, multiple of 8                            */
    int32_t E;           /* routed experts, 1..256                                */
    int32_t top_k;       /* experts per token, 1..min(E, 16)                      */
    int32_t G;           /* united experts (groups), 1..E                         */
    int32_t d_ff;        /* SwiGLU width of a united expert, multiple of 8        */
    int32_t d_ff_shared; /* width of the always-on shared FFN, 0 = none           */
    int32_t norm_topk;   /* 1: the k gate weights are renormalised to sum to 1    */
    int32_t dtype;       /* bmoe_dtype                                            */
} bmoe_desc;

/* Host-only checks (no HIP call). */
BMOE_API bmoe_status bmoe_validate(const bmoe_desc* desc);
/* e2g_host[E] (host memory): every entry in [0, G). The map is a static
 * per-layer artifact (Sec. 4.3-4.4); kernels assume a validated map. */
BMOE_API bmoe_status bmoe_validate_map(const int32_t* e2g_host, int32_t E, int32_t G);
/* Workspace bytes a stage needs for `desc` (0: none). */
BMOE_API size_t bmoe_workspace_bytes(const bmoe_desc* desc, int32_t stage);
/* Static string for a status code. */
BMOE_API const char* bmoe_status_str(bmoe_status status);
/* Library version, e.g. 10000 for 1.0.0. */
BMOE_API int32_t bmoe_version(void);

/*
 * bmoe_partial_segment_map -- host only: the segment map of partial brownout.
 * Paper: Sec. 2.2 (zero, partial and full brownout), Sec. 5 baselines
 * (threshold 1.0 keeps every original expert, 0 substitutes every call),
 * Sec. 4.3 closing paragraph (only eligible cold calls are replaced through
 * the saved map), Sec. 4.5 (the controller moves the threshold).
 *
 * Hot experts: the longest run of experts in order of decreasing freq (ties:
 * lower index first) whose cumulative freq / sum(freq) is <= theta + 1e-9.
 * Segments: the hot experts in ascending index (each with its own FFN), then
 * the united experts with at least one cold member in ascending group index.
 * The layer runs over the segments with e2s in place of e2g and S = *n_seg
 * in place of G (the weights of segment s stacked at index s).
 *
 * freq[E] double (calibration routing frequencies: finite, >= 0, positive
 * sum), e2g[E] int32 in [0, G), theta in [0, 1]; all HOST memory. Outputs,
 * host memory: e2s[E] int32; seg_kind[E] int32 (0: a hot expert's own FFN,
 * 1: a united expert) and seg_id[E] int32 (that expert or group), first
 * *n_seg entries valid; *n_seg in 1..E. Errors: BMOE_ERR_NULL,
 * BMOE_ERR_SHAPE (sizes, theta, frequencies), BMOE_ERR_MAP (e2g); nothing
 * is written on error.
 */
BMOE_API bmoe_status bmoe_partial_segment_map(const double* freq, const int32_t* e2g, int32_t E, int32_t G,
                                             double theta, int32_t* e2s, int32_t* seg_kind, int32_t* seg_id,
                                             int32_t* n_seg);

/*
 * brownout_moe_route -- the gate and the substitution by united experts.
 * Paper: Sec. 2.1 (gating scores g_i of the top-K experts), Eq. 2 (the map),
 * Sec. 4.3 last paragraph before Algorithm 1 (the gate still picks the
 * experts; picked experts are replaced by their united expert).
 *
 *   z[t,e]   = x[t,:] . w_router[e,:] + bias[e]          (or logits_in[t,e])
 *   p[t,:]   = softmax over all E of z[t,:]
 *   slot i   = the i-th largest z[t,:] (ties: lower expert index first)
 *   topk_idx[t,i] = that expert; topk_w[t,i] = its p (divided by the sum of
 *                   the k values when desc->norm_topk)
 *   slot_group[t,i] = e2g[topk_idx[t,i]] if no earlier slot of t has that
 *                   group, else -1;
 *   slot_gate[t,i]  = sum of topk_w[t,j] over j >= i with the same group when
 *                   slot_group[t,i] >= 0, else 0.
 *
 * x [T,d] (dtype), w_router [E,d] (dtype), bias [E] float or NULL, e2g [E]
 * int32 (validated map), logits_in [T,E] float or NULL. When logits_in is
 * set, x, w_router and bias are not used (they may be NULL) and selection
 * runs on those exact values.
 * Otherwise the logits are computed in fp32 (bf16: MFMA); a token whose fp32
 * top-(k+1) values have an adjacent gap below BMOE_ROUTE_RECHECK_GAP has its
 * candidate experts re-evaluated in float64 and is selected on those.
 * Outputs: topk_idx, slot_group [T,k] int32; topk_w, slot_gate [T,k] float;
 * logits_out [T,E] float or NULL (the fp32 logits, bias included).
 * No workspace.
 */
BMOE_API bmoe_status brownout_moe_route(const bmoe_desc* desc, const void* x, const void* w_router,
                               const float* bias, const float* logits_in, const int32_t* e2g,
                               int32_t* topk_idx, float* topk_w, int32_t* slot_group,
                               float* slot_gate, float* logits_out, void* stream);

/*
 * brownout_moe_dispatch -- group rows for the united experts (Eq. 2: the sets
 * G_r of the map, here filled with (token, group) pairs).
 *
 *   counts[r]   = number of tokens with a valid slot of group r
 *   offsets     = exclusive prefix of counts, offsets[G] = N (total rows)
 *   rows of group r are offsets[r] .. offsets[r+1]-1, in ascending token order
 *   perm_token[row] = token of that row; slot_row[t,i] = row of slot (t,i), or -1
 *   x_perm[row,:]   = x[perm_token[row],:]  (bit copy)
 *
 * slot_group [T,k] int32 as written by brownout_moe_route (entries outside
 * [-1, G) count as -1). x [T,d] (dtype). counts [G], offsets [G+1],
 * perm_token [T*k], slot_row [T,k] int32; x_perm [T*k, d] (dtype). Rows at
 * and beyond N are left unspecified.
 * x_perm NULL: the permutation only (counts, offsets, perm_token, slot_row);
 * no row is copied and x is not read (it may be NULL). This is the first half
 * of the fused path, whose FFN gathers its rows from x through perm_token
 * (brownout_moe_ffn_gather).
 * workspace: bmoe_workspace_bytes(desc, BMOE_STAGE_DISPATCH) bytes, 256-byte
 * aligned, ALL ZERO before the first call that uses it; every call leaves it
 * all zero again when it completes on the stream. Two calls that share a
 * workspace must not overlap in time. A call that finds the workspace not
 * zero (for example after an earlier call on it was cut short) writes the
 * "no rows" result instead: counts all 0, offsets[0..G-1] = 0 and
 * offsets[G] = -1 (the sentinel to check), every slot_row -1, no row copied;
 * the FFN and combine then see no rows. It still leaves the workspace zero.
 * Implementation: a histogram with LDS atomics and a single-pass decoupled
 * look-back scan across token tiles, then a 128-bit row gather; at most 256
 * tokens (one tile) take one kernel in which every workgroup rebuilds the
 * tile's histogram and prefix in LDS before gathering its tokens' rows.
 */
BMOE_API bmoe_status brownout_moe_dispatch(const bmoe_desc* desc, const int32_t* slot_group,
                                  const void* x, int32_t* counts, int32_t* offsets,
                                  int32_t* perm_token, int32_t* slot_row, void* x_perm,
                                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * brownout_moe_dispatch_noalloc -- brownout_moe_dispatch for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation): the same kernels and results, but
 * the workspace is a device array inside the library, one per GPU, of
 * BMOE_DISPATCH_SCRATCH_BYTES bytes, held until the process ends. The call
 * allocates nothing; each call first clears the array with a kernel (no
 * memset, so it may be captured into a graph). Arguments as for
 * brownout_moe_dispatch without the workspace. Shapes whose workspace
 * (bmoe_workspace_bytes(desc, BMOE_STAGE_DISPATCH)) exceeds the array return
 * BMOE_ERR_WORKSPACE before anything is enqueued. Every call on one GPU uses
 * that GPU's array, which keeps the last call's contents: two calls on one GPU
 * that overlap in time (other streams, other threads) race and must not be
 * made. The device is the current HIP device.
 */
#define BMOE_DISPATCH_SCRATCH_BYTES 1048576
BMOE_API bmoe_status brownout_moe_dispatch_noalloc(const bmoe_desc* desc, const int32_t* slot_group,
                                          const void* x, int32_t* counts, int32_t* offsets,
                                          int32_t* perm_token, int32_t* slot_row, void* x_perm,
                                          void* stream);

/*
 * brownout_moe_ffn -- grouped SwiGLU FFN (Sec. 2.1 "small FFNs"; SwiGLU form).
 * Segment s covers rows offsets[s] .. offsets[s+1]-1 of a and uses united
 * expert s:
 *   h[row,:] = silu(a[row,:] W_gate[s]^T) * (a[row,:] W_up[s]^T)   (stored in dtype)
 *   y[row,:] = h[row,:] W_down[s]^T                                  (stored in dtype)
 * dtype: bmoe_dtype. offsets [n_seg+1] int32 in DEVICE memory (as written by
 * dispatch; non-decreasing, offsets[n_seg] <= rows_cap; rows beyond rows_cap
 * are never touched). a [rows_cap, d]; w_gate, w_up [n_seg, d_ff, d];
 * w_down [n_seg, d, d_ff]; h [rows_cap, d_ff] (scratch the caller owns);
 * y [rows_cap, d]. n_seg in 1..256. bf16: MFMA, fp32 accumulation.
 * offsets[0] need not be 0: a sub-range of segments runs alone when the
 * caller passes offsets + s0 and the weights of segments s0.. (one rank's
 * block of united experts under expert parallelism); other rows stay untouched.
 * The shared experts of a layer run through this call too, with n_seg = 1,
 * offsets = {0, T}, a = x.
 * workspace (optional, device memory, 256-byte aligned): the large bf16
 * GEMMs run one workgroup per CU, each taking whole output tiles in turn;
 * NULL keeps every tile whole. With at least bmoe_workspace_bytes(desc,
 * BMOE_STAGE_FFN) bytes (the size depends on the current device) they may
 * also split the K loop of the last tiles so every CU gets the same work;
 * the partial sums of a split tile meet in the workspace in a fixed order,
 * so results stay deterministic (they may differ in the last bits from the
 * NULL-workspace path). Contents need no
 * initialisation and are not preserved; calls that can overlap in time must
 * not share a workspace. A non-NULL workspace below the size is
 * BMOE_ERR_WORKSPACE. The K loops are split only when whole tiles would leave
 * the CUs idle for more than 48 K-steps (of 64 columns) on average
 * (brownout_moe_ffn_ex takes that threshold as an argument).
 */
BMOE_API bmoe_status brownout_moe_ffn(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                             int32_t d_ff, const int32_t* offsets, const void* a,
                             const void* w_gate, const void* w_up, const void* w_down, void* h,
                             void* y, void* workspace, size_t workspace_bytes, void* stream);

/* brownout_moe_ffn with the stream-K split threshold given explicitly: with a
 * workspace, the K loops of the last tiles are split when whole tiles would
 * leave the CUs idle for more than split_min_idle K-steps (of 64 columns) on
 * average; 0 splits whenever any CU would idle, -1 takes the default (48).
 * Values below -1 or above 2^20 are BMOE_ERR_SHAPE. The result is the same
 * layer as brownout_moe_ffn's within the rounding of the split sums. */
BMOE_API bmoe_status brownout_moe_ffn_ex(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                int32_t d_ff, const int32_t* offsets, const void* a,
                                const void* w_gate, const void* w_up, const void* w_down, void* h,
                                void* y, void* workspace, size_t workspace_bytes,
                                int32_t split_min_idle, void* stream);

/* The two grouped GEMMs of brownout_moe_ffn, callable on their own (same
 * arguments and rules as brownout_moe_ffn):
 *   brownout_moe_ffn_gate_up: h = silu(a W_gate[s]^T) * (a W_up[s]^T)
 *   brownout_moe_ffn_down:    y = h W_down[s]^T                                   */
BMOE_API bmoe_status brownout_moe_ffn_gate_up(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                     int32_t d_ff, const int32_t* offsets, const void* a,
                                     const void* w_gate, const void* w_up, void* h, void* workspace,
                                     size_t workspace_bytes, void* stream);
BMOE_API bmoe_status brownout_moe_ffn_down(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                  int32_t d_ff, const int32_t* offsets, const void* h,
                                  const void* w_down, void* y, void* workspace, size_t workspace_bytes,
                                  void* stream);

/* Fused gather (the same FFN, Sec. 2.1, without the x_perm copy): the gate/up
 * GEMM reads row r of its activations as a[a_rows[r], :] instead of a[r, :],
 * straight from the token rows: with a = x [T, d], a_count = T and a_rows =
 * the perm_token that brownout_moe_dispatch wrote (with x_perm NULL there),
 * the results are bit-identical to dispatch's x_perm followed by
 * brownout_moe_ffn. a_rows [rows_cap] int32 in DEVICE memory; entries are
 * clamped into [0, a_count) (never read out of bounds); a [a_count, d]
 * (dtype), 16-byte aligned; a_count * d * element size must stay below
 * 2^32 bytes (BMOE_ERR_SHAPE otherwise). NULL a_rows with rows_cap > 0 is
 * BMOE_ERR_NULL. Every other argument and rule as brownout_moe_ffn /
 * brownout_moe_ffn_gate_up; the down GEMM is unchanged (h is already in row
 * order). */
BMOE_API bmoe_status brownout_moe_ffn_gather(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                    int32_t d_ff, const int32_t* offsets, const int32_t* a_rows,
                                    int32_t a_count, const void* a, const void* w_gate, const void* w_up,
                                    const void* w_down, void* h, void* y, void* workspace,
                                    size_t workspace_bytes, void* stream);
BMOE_API bmoe_status brownout_moe_ffn_gate_up_gather(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d,
                                            int32_t d_ff, const int32_t* offsets, const int32_t* a_rows,
                                            int32_t a_count, const void* a, const void* w_gate,
                                            const void* w_up, void* h, void* workspace,
                                            size_t workspace_bytes, void* stream);

/*
 * Grouping search (Sec. 4.3): what a candidate map costs in distillation
 * error. The member experts' outputs f_e(x) and the united experts' outputs
 * f_u(x) on the calibration tokens come from brownout_moe_ffn_gather with one
 * segment per expert (rows e*T .. e*T+T-1 read token t = row mod T).
 *
 * brownout_moe_united_init -- the united experts' starting point: each united
 * matrix is the element-wise average of its members' matrices (the parameter
 * average the paper starts distillation from, Sec. 4.3, after Eq. 5).
 *   w_*_u[r] = (sum over e with e2g[e] == r, ascending e, of w_*_e[e]) / count
 * e2g [E] int32 in DEVICE memory (entries outside [0, G) belong to no group);
 * w_gate_e, w_up_e [E, d_ff, d], w_down_e [E, d, d_ff]; w_gate_u, w_up_u
 * [G, d_ff, d], w_down_u [G, d, d_ff] (dtype; bf16: fp32 sum, rounded once;
 * f32: fp64 sum). An empty group gets zeros. E, G in 1..256.
 */
BMOE_API bmoe_status brownout_moe_united_init(int32_t dtype, int32_t E, int32_t G, int32_t d, int32_t d_ff,
                                     const int32_t* e2g, const void* w_gate_e, const void* w_up_e,
                                     const void* w_down_e, void* w_gate_u, void* w_up_u, void* w_down_u,
                                     void* stream);

/*
 * brownout_moe_distill_mse -- distillation error of every group and the
 * layer total (Eq. 5, Eq. 3 and Eq. 6):
 *   alpha_e  = w_e / (sum of w over e's group)  (equal weights if that sum is 0)
 *   t_r(x_t) = sum over the members e of r of alpha_e y_expert[e*T + t, :]
 *   mse[r]   = mean over t < T and j < d of (y_united[r*T + t, j] - t_r(x_t)[j])^2
 *   *mse_total = sum over r of beta_r mse[r],  beta_r = sum of w over r's members
 * (the reward of the grouping search is -*mse_total). An empty group has
 * mse 0 and beta 0. e2g [E] int32 and w_freq [E] float (routing frequencies)
 * in DEVICE memory; y_expert [E*T, d], y_united [G*T, d] (dtype, 16-byte
 * aligned); mse [G] double, mse_total (nullable) double, in DEVICE memory.
 * Targets in fp32, squares accumulated in fp64 in a fixed order: results are
 * deterministic. workspace: at least BMOE_DISTILL_WS_BYTES bytes of device
 * memory, 8-byte aligned, contents need no initialisation (calls that can
 * overlap must not share one). T == 0 writes nothing.
 */
#define BMOE_DISTILL_WS_BYTES 32768
BMOE_API bmoe_status brownout_moe_distill_mse(int32_t dtype, int32_t E, int32_t G, int32_t T, int32_t d,
                                     const int32_t* e2g, const float* w_freq, const void* y_expert,
                                     const void* y_united, double* mse, double* mse_total, void* workspace,
                                     size_t workspace_bytes, void* stream);

/*
 * brownout_moe_ffn_down_combine -- the down projection with the combine folded
 * into its epilogue (the fused MoE operator of Sec. 4.1; the layer output of
 * Sec. 2.1). Writes the same y as brownout_moe_ffn_down and the same out, bit
 * for bit, as brownout_moe_combine on that y (fp32 fmaf of slot gate and bf16
 * y over the token's valid slots in slot order, + y_shared, one RNE rounding),
 * whatever order the tiles finish in: each tile's epilogue counts its rows per
 * (token, 128-column chunk), and the row that completes a token's chunk forms
 * that chunk of out from the token's rows of y.
 * desc: the layer (G segments, d, d_ff, top_k, dtype). offsets [G+1], h
 * [T*k, d_ff], w_down [G, d, d_ff], y [T*k, d], perm_token [T*k], slot_row
 * [T,k], slot_gate [T,k] (as written by route and dispatch), y_shared [T,d] or
 * NULL, out [T,d]. workspace: bmoe_workspace_bytes(desc,
 * BMOE_STAGE_DOWN_COMBINE) bytes (4 * T * ceil(d/128)), 256-byte aligned, ALL
 * ZERO before the first call; every call leaves it zero; calls that share one
 * must not overlap. The fold runs on the 256-row bf16 GEMM tiles with d a
 * multiple of 128 (every tile whole: no stream-K split); other shapes run the
 * down projection and then the combine kernel, with the same results.
 */
BMOE_API bmoe_status brownout_moe_ffn_down_combine(const bmoe_desc* desc, const int32_t* offsets, const void* h,
                                          const void* w_down, void* y, const int32_t* perm_token,
                                          const int32_t* slot_row, const float* slot_gate,
                                          const void* y_shared, void* out, void* workspace,
                                          size_t workspace_bytes, void* stream);

/*
 * brownout_moe_combine -- weighted sum back into token order (Sec. 2.1: the
 * layer output is the gate-weighted sum of the expert outputs).
 *   out[t,:] = sum over i ascending with slot_row[t,i] >= 0 of
 *              slot_gate[t,i] * y_perm[slot_row[t,i],:]  (+ y_shared[t,:])
 * fp32 accumulation, stored in dtype. slot_row [T,k] int32, slot_gate [T,k]
 * float, y_perm [T*k, d], y_shared [T,d] or NULL, out [T,d]. Rows of y_perm
 * named by slot_row must be < T*k.
 */
BMOE_API bmoe_status brownout_moe_combine(const bmoe_desc* desc, const int32_t* slot_row,
                                 const float* slot_gate, const void* y_perm,
                                 const void* y_shared, void* out, void* stream);

/*
 * Norms around the layer: the RMS norm that makes the layer's input, and the
 * one that returns its output to the residual stream.
 *
 * brownout_moe_pre_norm:
 *   out[t,:] = rms(x[t,:]) * w,   rms(v) = v / sqrt(mean over j of v_j^2 + eps)
 * brownout_moe_post_norm:
 *   n[t,:] = rms(y[t,:]) * w_post  (norm_y 1)   or   y[t,:]  (norm_y 0)
 *   r[t,:] = res_scale * x[t,:] + gate * n[t,:]
 *   a[t,:] = rms(r[t,:]) * w_next   (when a is not NULL: the next block's norm;
 *            it reads r before r is rounded to dtype)
 * x, y, out, r, a [T,d] and w, w_post, w_next [d] in dtype; a NULL w, w_post or
 * w_next stands for ones (w_post must be NULL when norm_y is 0, w_next when a
 * is). gate by gate_mode: BMOE_GATE_NONE (NULL, 1), BMOE_GATE_CHANNEL ([d] in
 * dtype), BMOE_GATE_TOKEN ([T] float) or BMOE_GATE_FULL ([T,d] in dtype).
 * Sums in fp32 over the whole row, one rounding at each output. Every tensor
 * except the per-token gate is 16-byte aligned. d is at most 32768; eps in
 * [1e-12, 1]; res_scale finite. An output may be one of the input tensors of
 * its shape (the residual stream updated in place); any other memory shared with
 * an input, or by r and a, is BMOE_ERR_UNSUPPORTED. No workspace.
 */
typedef enum bmoe_gate_mode {
    BMOE_GATE_NONE = 0,
    BMOE_GATE_CHANNEL = 1,
    BMOE_GATE_TOKEN = 2,
    BMOE_GATE_FULL = 3
} bmoe_gate_mode;
#define BMOE_NORM_MAX_D 32768
BMOE_API bmoe_status brownout_moe_pre_norm(int32_t dtype, int32_t T, int32_t d, float eps, const void* x,
                                  const void* w, void* out, void* stream);
BMOE_API bmoe_status brownout_moe_post_norm(int32_t dtype, int32_t T, int32_t d, float eps, int32_t norm_y,
                                   float res_scale, int32_t gate_mode, const void* y, const void* x,
                                   const void* w_post, const void* gate, void* r, const void* w_next, void* a,
                                   void* stream);

/*
 * Weights held in 4 bits with group scales. A matrix stack [n, N, K] (K: the
 * summed columns, a multiple of 8) is held as
 *   codes  [n, N, P] uint8, P = 16 * ceil(K/32): byte b of a row holds column 2b
 *          in its low four bits and column 2b+1 in its high four; the bytes past
 *          K/2 are padding, their values do not matter;
 *   scales [n, N, ceil(K/group)] bf16 (finite, or NaN for weights that are not numbers),
 *          group 32, 64 or 128;
 *   zeros  [n, N, ceil(K/group)] uint8, or NULL: every zero point is 8.
 * Column k of a row stands for  w = scale[k / group] * (code[k] - zero[k / group]).
 * Products are exact in fp32 (bf16 activations on MFMA against code + 16, whose
 * offset the sum of the activations takes back), sums in fp32, the group's sum
 * is scaled in fp32. codes 16-byte aligned, scales 2-byte.
 */
#define BMOE_W4_ROW_BYTES(K) (((K) + 31) / 32 * 16)
typedef struct bmoe_w4 {
    const uint8_t* codes;
    const void* scales;   /* bf16 */
    const uint8_t* zeros; /* or NULL */
    int32_t group;        /* 32, 64 or 128 */
} bmoe_w4;

/*
 * brownout_moe_w4_quantize -- rounds w [n, N, K] (dtype) to that format. Per
 * group of a row: without zeros, scale = max|w| / 7, code = 8 + round(w / scale)
 * in 1..15; with zeros, scale = (max - min) / 15 over the group's values and 0,
 * zero = round(-min / scale), code = zero + round(w / scale) clamped to 0..15.
 * The scale is rounded to bf16 first, and w is divided by the rounded one;
 * rounding is to nearest even. A group of zeros has scale 0 and codes 8 (0 and
 * zero 0 with zeros). A group with a value that is not finite has scale NaN and the
 * codes of a group of zeros: all of its weights read NaN, and so do the products with
 * them. Padding bytes are written 0x88. Outputs as above.
 */
BMOE_API bmoe_status brownout_moe_w4_quantize(int32_t dtype, int32_t n, int32_t N, int32_t K, int32_t group,
                                     const void* w, uint8_t* codes, void* scales, uint8_t* zeros, void* stream);

/*
 * Grouped products with 4-bit weights, for few rows per segment (each pass over
 * a segment's weights serves up to 32 of its rows). dtype: BMOE_BF16 (the
 * activations' and outputs'; others are BMOE_ERR_UNSUPPORTED). Segments as in
 * brownout_moe_ffn: segment s covers rows offsets[s] .. offsets[s+1]-1; rows of
 * no segment are left as they are. a_rows as in brownout_moe_ffn_gather, or NULL
 * (row r reads a[r]; a then has rows_cap rows and a_count is not used). A product's output
 * shares no memory with its input (BMOE_ERR_UNSUPPORTED; w4_ffn's y may with a). No workspace.
 *   brownout_moe_w4_matmul   y[row,:] = a[row,:] W[s]^T                 W [n_seg, N, K]
 *   brownout_moe_w4_gate_up  h[row,:] = silu(a[row,:] Wg[s]^T) * (a[row,:] Wu[s]^T)
 *                            Wg, Wu [n_seg, d_ff, d], the same group and both with or without zeros
 *   brownout_moe_w4_ffn      gate_up, then y[row,:] = h[row,:] Wd[s]^T   Wd [n_seg, d, d_ff]
 *                            (from the stored h: rounded to dtype, as in brownout_moe_ffn)
 * A result that leaves fp32 on the way though it is finite itself (activations near the
 * largest value), or that an infinite h makes infinite, is what the definition gives.
 * Long segments are multiplied right but not fast: bf16 weights and brownout_moe_ffn are
 * faster from about 70 rows a segment on.
 */
BMOE_API bmoe_status brownout_moe_w4_matmul(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t N, int32_t K,
                                   const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                   const bmoe_w4* w, void* y, void* stream);
BMOE_API bmoe_status brownout_moe_w4_gate_up(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                    const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                    const bmoe_w4* w_gate, const bmoe_w4* w_up, void* h, void* stream);
BMOE_API bmoe_status brownout_moe_w4_ffn(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                const bmoe_w4* w_gate, const bmoe_w4* w_up, const bmoe_w4* w_down, void* h, void* y,
                                void* stream);

/*
 * brownout_moe_few -- the whole layer for 1 to BMOE_FEW_MAX_TOKENS tokens: the
 * results of route, dispatch, FFN, the shared experts and combine, without the
 * permutation and its buffers. Every token of a reached segment shares one read
 * of the segment's weights.
 *   topk_idx, topk_w, slot_group, slot_gate [T,k] as brownout_moe_route writes them
 *   out[t,:] = sum over the valid slots i of t, segments ascending, of
 *              W_down[g] (slot_gate[t,i] * silu(W_gate[g] x_t) * (W_up[g] x_t))
 *              (+ W_down_sh (silu(W_gate_sh x_t) * (W_up_sh x_t)))
 * The hidden values are held to 16 bits of significand (bf16 layers) or in fp32,
 * the sum over experts in fp32; out is rounded once.
 * x, out [T,d] (dtype). weights: w_router, bias, e2g as in brownout_moe_route;
 * the six matrices either all plain (dtype, group 0; scales and zeros NULL) or
 * all in 4 bits (dtype BMOE_BF16; `w` the codes, the same group for all six, and
 * zeros for all or none). The *_sh matrices are read when d_ff_shared > 0.
 * T above BMOE_FEW_MAX_TOKENS is BMOE_ERR_SHAPE.
 * workspace: bmoe_workspace_bytes(desc, BMOE_STAGE_FEW) bytes, 256-byte aligned,
 * no initialisation; calls that can overlap in time must not share one.
 */
#define BMOE_FEW_MAX_TOKENS 16
typedef struct bmoe_matrix {
    const void* w;
    const void* scales;
    const uint8_t* zeros;
} bmoe_matrix;
typedef struct bmoe_few_weights {
    const void* w_router;
    const float* bias;
    const int32_t* e2g;
    bmoe_matrix gate, up, down, gate_sh, up_sh, down_sh;
    int32_t group; /* 0: plain weights; 32, 64 or 128: 4-bit weights */
} bmoe_few_weights;
BMOE_API bmoe_status brownout_moe_few(const bmoe_desc* desc, const bmoe_few_weights* weights, const void* x,
                             int32_t* topk_idx, float* topk_w, int32_t* slot_group, float* slot_gate, void* out,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * Rows held in 8 bits with one scale each: weights [n, N, K] by output channel, activations
 * [rows, K] by token. A stack of rows of K values (K a multiple of 8, at most BMOE_W8_MAX_K) is
 *   codes  [rows, P] int8, P = 128 * ceil(K/128): the codes of a row, then zeros
 *   scales [rows] float
 * and stands for x = scale * code. Both 16-byte aligned. Where they were made elsewhere, scales may
 * have either sign; codes of -128 may be in one operand of a product (in both, sums of K =
 * BMOE_W8_MAX_K can leave int32).
 *
 * brownout_moe_w8_quantize -- rounds x [rows, K] (dtype) to that format: scale = max|x| / 127 in
 * fp32, code = round(x / scale) to nearest even, of the true quotient. A row whose scale would be
 * below 2^-120 (zeros, say) has scale 0 and codes 0. A row with a value that is not finite has
 * scale NaN and codes 0: all of it reads NaN, and so does every product with it. rows at most
 * 2^30; outputs share no memory with x (BMOE_ERR_UNSUPPORTED).
 */
#define BMOE_W8_MAX_K 131072
#define BMOE_W8_ROW_BYTES(K) (((K) + 127) / 128 * 128)
typedef struct bmoe_w8 {
    const int8_t* codes;
    const float* scales;
} bmoe_w8;
BMOE_API bmoe_status brownout_moe_w8_quantize(int32_t dtype, int32_t rows, int32_t K, const void* x, int8_t* codes,
                                     float* scales, void* stream);

/*
 * Grouped products in 8-bit integers. dtype: BMOE_BF16 (the activations' and outputs'; others are
 * BMOE_ERR_UNSUPPORTED). Segments as in brownout_moe_ffn: segment s covers rows offsets[s] ..
 * offsets[s+1]-1; rows of no segment are left as they are. Row r reads a[a_rows[r]] (entries
 * clamped into [0, a_count), the codes below 2^32 bytes), or a[r] with a_rows NULL (a then has
 * rows_cap rows and a_count is not used). The activations are given as a (dtype; the call rounds
 * them to 8 bits, each row once however many rows read it) or as a8 (rounded already); the other
 * is NULL.
 *   brownout_moe_w8_matmul   y[row, n] = sa[row] * sw[s, n] * sum_k qa[row, k] * qw[s, n, k]    W [n_seg, N, K]
 *   brownout_moe_w8_gate_up  h[row, :] = silu(gate[row, :]) * up[row, :], two such products      [n_seg, d_ff, d]
 *   brownout_moe_w8_ffn      gate_up, then y from the stored h (rounded to dtype, as in
 *                            brownout_moe_ffn, then to 8 bits by row) and w_down                 [n_seg, d, d_ff]
 * The sums are exact (int32); a product is rounded to fp32 three times and once to dtype. N and d
 * are multiples of 8. An output shares no memory with the input of its product
 * (BMOE_ERR_UNSUPPORTED; w8_ffn's y may with a).
 * workspace (256-byte aligned, no initialisation, not preserved; calls that can overlap in time must
 * not share one): at least bmoe_w8_workspace_bytes(a_count, K, rows_cap, d_ff, 0) bytes, a_count 0
 * where a8 is given (rows_cap where a_rows is NULL), K the columns of a, d_ff 0 but for w8_ffn.
 * With the size for split 1, which depends on the current device, the K loops of the last large
 * tiles may be split, as in brownout_moe_ffn; the results are the same bits.
 */
BMOE_API size_t bmoe_w8_workspace_bytes(int32_t a_count, int32_t K, int32_t rows_cap, int32_t d_ff, int32_t split);
BMOE_API bmoe_status brownout_moe_w8_matmul(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t N, int32_t K,
                                   const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                   const bmoe_w8* a8, const bmoe_w8* w, void* y, void* workspace,
                                   size_t workspace_bytes, void* stream);
BMOE_API bmoe_status brownout_moe_w8_gate_up(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                    const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                    const bmoe_w8* a8, const bmoe_w8* w_gate, const bmoe_w8* w_up, void* h,
                                    void* workspace, size_t workspace_bytes, void* stream);
BMOE_API bmoe_status brownout_moe_w8_ffn(int32_t dtype, int32_t n_seg, int32_t rows_cap, int32_t d, int32_t d_ff,
                                const int32_t* offsets, const int32_t* a_rows, int32_t a_count, const void* a,
                                const bmoe_w8* a8, const bmoe_w8* w_gate, const bmoe_w8* w_up, const bmoe_w8* w_down,
                                void* h, void* y, void* workspace, size_t workspace_bytes, void* stream);

/*
 * brownout_moe_balance -- how evenly the router's picks fall on the experts, or on the groups that
 * a map makes of them. Over the tokens that count (valid[t] != 0; all of them with valid NULL), V
 * in number:
 *   p_t = softmax(logits_t),  lse_t = log(sum over e of exp(logits_te))
 *   counts[e] = picks of expert e among topk_idx,  counts[E] = V
 *   prob[e]   = mean of p_te
 *   F_r       = (sum of counts[e] over the experts of group r) / (k V)
 *   losses[0] = G * sum over e of F_{e2g[e]} * prob[e]     (1 where picks and probabilities are even)
 *   losses[1] = mean of lse_t^2                            (the z loss)
 * brownout_moe_balance_grad -- the gradient of d_losses[0] losses[0] + d_losses[1] losses[1] by the
 * logits, the counts held constant:
 *   d_logits[t,e] = (d_losses[0] G / V) p_te (F_{e2g[e]} - sum over j of F_{e2g[j]} p_tj)
 *                   + d_losses[1] (2 / V) lse_t p_te,   0 for tokens that do not count
 * logits [T,E] float (as brownout_moe_route writes them), topk_idx [T,k] int32 (entries outside
 * [0, E) pick nothing; a repeated one counts each time), valid [T] uint8 or NULL, e2g [E] int32
 * (entries outside [0, G) belong to no group and add nothing) or NULL (groups are the experts: G
 * must be E). All in DEVICE memory. Outputs: losses [2], prob [E] float, counts [E+1] int32;
 * d_logits [T,E] float, which may be logits itself (other shared memory is BMOE_ERR_UNSUPPORTED).
 * Logits of tokens that do not count may hold anything. -infinity is an expert of probability 0; a
 * token of nothing else has no probabilities, adds nothing to the losses and gets gradient 0,
 * though it counts in V. With V == 0 losses and prob are 0 (T == 0 writes nothing). Sums in a
 * fixed order: results are deterministic. E in 1..256, k in 1..16, G in 1..256.
 * workspace: bmoe_balance_workspace_bytes(T, E) bytes (0 for few tokens), 8-byte aligned. Its
 * first BMOE_BALANCE_ZERO_BYTES bytes (arrival counters) are zero before the first call that uses
 * it; every call leaves them zero; the rest needs no initialisation. Calls that can overlap in
 * time must not share one.
 */
#define BMOE_BALANCE_ZERO_BYTES 64
BMOE_API size_t bmoe_balance_workspace_bytes(int32_t T, int32_t E);
BMOE_API bmoe_status brownout_moe_balance(int32_t T, int32_t E, int32_t k, int32_t G, const float* logits,
                                 const int32_t* topk_idx, const uint8_t* valid, const int32_t* e2g, float* losses,
                                 int32_t* counts, float* prob, void* workspace, size_t workspace_bytes, void* stream);
BMOE_API bmoe_status brownout_moe_balance_grad(int32_t T, int32_t E, int32_t k, int32_t G, const float* logits,
                                      const uint8_t* valid, const int32_t* e2g, const int32_t* counts,
                                      const float* d_losses, float* d_logits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BROWNOUT_MOE_H */
