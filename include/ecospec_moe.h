/*
 * ecospec_moe.h -- C ABI of the MoE verification pass on MI355X (gfx950).
 *
 * The library computes, for one MoE layer, what a speculative-decoding
 * verifier must do for T draft tokens (EcoSpec, arXiv 2607.12696):
 *   router top-k          -> moe_route_topk (or moe_route_topk_hidden from x,
 *                            moe_route_topk_grouped for group-limited routing)
 *   expert union, Eq. 1   -> moe_expert_union (moe_route_union: route + union in one call)
 *   grouped SwiGLU experts streaming every activated expert's weights from
 *   HBM once, gate-weighted combine -> moe_verify_layer
 * and, on the host, the cost-aware draft-tree selection of Section 4.2
 * (Eq. 7-9, Algorithm 1) -> moe_select_tree.
 *
 * Conventions for every call:
 *   - Device pointers point to HIP device memory owned by the caller.  The
 *     library never allocates or frees memory and never synchronises; all
 *     device work is enqueued on `stream` (a hipStream_t; NULL is the null
 *     stream).  Calls are stateless and may run concurrently on different
 *     streams with different buffers.
 *   - Argument errors are detected on the host before anything is enqueued
 *     and return MOE_ERR_INVALID_ARG (or MOE_ERR_UNSUPPORTED for shapes the
 *     kernels do not handle, MOE_ERR_WORKSPACE for a short workspace).  A
 *     failed launch returns MOE_ERR_HIP.  Contents of device arrays are
 *     preconditions, not checked: e.g. topk_idx entries must lie in [0, E).
 *     A violated precondition gives unspecified results but no access
 *     outside the buffers described here.
 *   - Integers are int32, row-major, no padding.  bf16 values are stored as
 *     their 16-bit patterns.
 */
#ifndef ECOSPEC_MOE_H
#define ECOSPEC_MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MOE_OK = 0,
    MOE_ERR_INVALID_ARG = 1,
    MOE_ERR_UNSUPPORTED = 2,
    MOE_ERR_WORKSPACE = 3,
    MOE_ERR_HIP = 4
} moe_status_t;

/* Gate-weight rule applied to the k selected router logits l_0..l_{k-1}. */
typedef enum {
    MOE_SCORE_SOFTMAX = 0, /* w_j = exp(l_j - max) / sum_i exp(l_i - max)        */
    MOE_SCORE_SIGMOID = 1  /* w_j = sigmoid(l_j) / sum_i sigmoid(l_i)            */
} moe_score_t;

/* Expert weight storage.  Every matrix is stored out x in with the input
 * (reduction) dimension contiguous: W_gate, W_up are [d_ff][d], W_down is
 * [d][d_ff]; experts are stacked along a leading [E] dimension. */
typedef enum {
    MOE_W_BF16 = 0,          /* bf16 [E][N][K]                                               */
    MOE_W_FP8_E4M3_B128 = 1, /* OCP e4m3fn codes u8 [E][N][K], fp32 scales [E][N/128][K/128];
                                weight = e4m3fn(q[n][c]) * s[n/128][c/128]                      */
    MOE_W_MXFP4 = 2          /* OCP MXFP4: e2m1 codes packed two per byte u8 [E][N][K/2], the
                                low nibble holding the even K index; e8m0 scale codes u8
                                [E][N][K/32]; weight = e2m1 * 2^(code-127)                      */
} moe_wfmt_t;

/* Draft-selection scores (Section 4.2 and the ablation of Section 5.4). */
typedef enum {
    MOE_SEL_COST_RATIO = 0,  /* Eq. 9:  P / (DeltaCost + eps), buffer updated (Algorithm 1) */
    MOE_SEL_CONFIDENCE = 1,  /* P alone: the confidence-driven baseline                     */
    MOE_SEL_GLOBAL_COST = 2, /* Eq. 10: P / (|E_traj| + eps), buffer never consulted        */
    MOE_SEL_COST_DIFF = 3    /* P - lambda * DeltaCost                                      */
} moe_sel_mode_t;

/* Expert activation.  MOE_ACT_SWIGLU: h = silu(g) * u.  MOE_ACT_SWIGLU_OAI:
 * the clamped form of the GPT-OSS family (the GPT-OSS-120B rows of the
 * paper's tables): g = min(g, limit), u = clamp(u, -limit, limit),
 * h = g * sigmoid(alpha * g) * (u + 1). */
typedef enum {
    MOE_ACT_SWIGLU = 0,
    MOE_ACT_SWIGLU_OAI = 1
} moe_act_t;

/* Precision of the projections' inputs (x for gate/up, the activation rows h
 * for down).  MOE_ACTQ_BF16: x as given, h rounded to bf16, exact products.
 * MOE_ACTQ_MXFP8 (opt-in; MOE_W_MXFP4 weights only): both inputs quantised to
 * OCP MX FP8 and multiplied on the scaled FP4 x FP8 matrix-core instruction.
 * A row is taken in blocks of 32 consecutive elements (the OCP MX block, and
 * the K block the instruction's scales apply to).  A block's scale is 2^E,
 * E = floor(log2(max |v|)) - 8 clamped to [-127, 127] (-127 for an all-zero
 * block); each element becomes the e4m3fn value nearest to v / 2^E, ties to
 * the even code, magnitudes from 448 up saturating to 448.  The paper keeps
 * activations exact; this mode trades a few percent of y (relative to
 * max |y|) for matrix-core work without weight decoding. */
typedef enum {
    MOE_ACTQ_BF16 = 0,
    MOE_ACTQ_MXFP8 = 1
} moe_actq_t;

/* Weights of one MoE layer, in the streaming layout written by
 * moe_pack_weights; all pointers are device pointers.  The scale pointers
 * are NULL for MOE_W_BF16.  The sh_* fields describe one always-on shared
 * expert (packed the same way, E = 1) with gate weight 1 that every token
 * uses; all sh_* weight pointers NULL means no shared expert.
 * act / alpha / limit select the activation (moe_act_t; alpha and limit are
 * read for MOE_ACT_SWIGLU_OAI only, finite, limit > 0).  b_gate, b_up
 * [E][d_ff] and b_down [E][d] are optional fp32 biases of the routed experts
 * (NULL: none; 16-byte aligned): g and u get b_gate, b_up before the
 * activation and each expert output gets b_down before the gate weight.
 * The shared expert takes the activation but no biases.  act_fmt selects the
 * precision of the projection inputs (moe_actq_t; MOE_ACTQ_MXFP8 needs
 * MOE_W_MXFP4, else MOE_ERR_UNSUPPORTED).  A zero-initialised struct tail
 * (act 0, NULL biases, act_fmt 0, down_paired 0) is the plain SwiGLU layer
 * with W_down packed by moe_pack_weights; callers zero-initialise the whole
 * struct, since fields are only ever added at its end.
 * w_up == NULL means W_gate and W_up were packed together by
 * moe_pack_gate_up into w_gate (likewise sh_up == NULL with sh_gate set);
 * s_up (sh_s_up) still points to the up scales.  down_paired = 1 means
 * w_down and sh_down were packed by moe_pack_down (0: moe_pack_weights; any
 * other value is MOE_ERR_INVALID_ARG).
 * Requirements: d % 32 == 0, d_ff % 32 == 0, and for FP8 d % 128 == 0 and
 * d_ff % 128 == 0; each packed matrix below 2 GiB; 16-byte aligned pointers.
 * Other shapes return MOE_ERR_UNSUPPORTED. */
typedef struct {
    int fmt; /* moe_wfmt_t */
    int d, d_ff, E;
    const void *w_gate, *w_up, *w_down;
    const void *s_gate, *s_up, *s_down;
    const void *sh_gate, *sh_up, *sh_down;
    const void *sh_s_gate, *sh_s_up, *sh_s_down;
    int act; /* moe_act_t */
    float alpha, limit;
    const float *b_gate, *b_up, *b_down;
    int act_fmt; /* moe_actq_t */
    int down_paired;
} moe_weights_t;

/* Routing of T tokens (device pointers).  Slot s = t*k + j is the j-th
 * expert of token t.  topk_idx and topk_w are moe_route_topk's output; the
 * union and grouping arrays are moe_expert_union's output for that topk_idx.
 * moe_verify_layer reads topk_idx and topk_w and writes the union and
 * grouping arrays itself (the same values moe_expert_union gives), so they
 * need not be filled before the call. */
typedef struct {
    int T, k, E;
    const int32_t *topk_idx; /* [T][k] */
    const float *topk_w;     /* [T][k] */
    int32_t *counts;         /* [E]    */
    int32_t *union_ids;      /* [E]    */
    int32_t *n_unique;       /* [1]    */
    int32_t *offsets;        /* [E+1]  */
    int32_t *perm;           /* [T*k]  */
} moe_routing_t;

/*
 * moe_route_topk followed by moe_expert_union in one call (the two kernels,
 * enqueued back to back).  Same arguments, limits and results as the two
 * calls: logits [T][E] fp32 in; topk_idx, topk_w [T][k] and counts,
 * union_ids, n_unique, offsets, perm out.
 */
moe_status_t moe_route_union(const float *logits, int T, int E, int k, int score, int32_t *topk_idx, float *topk_w,
                             int32_t *counts, int32_t *union_ids, int32_t *n_unique, int32_t *offsets, int32_t *perm,
                             void *stream);

/*
 * Weight packing (done once, when a model is loaded).  Converts E stacked
 * N x K matrices of one tensor (W_gate or W_up: N = d_ff, K = d; W_down:
 * N = d, K = d_ff) from the interchange layout of moe_wfmt_t into the
 * streaming layout the verify kernels read:
 *   K is padded with zero codes to Kp = the next multiple of 128; each
 *   matrix is a row-major grid of blocks of 16 rows x 128 elements, block
 *   (rb, kb) at byte offset (rb*Kp/128 + kb) * B, with B = 4096 (bf16), 2048
 *   (FP8) or 1024 (MXFP4); a block is B/1024 vectors of 1 KiB and the 16
 *   bytes at offset 16*l of vector i (l = c + 16*g, c < 16, g < 4) hold
 *   the weights of row rb*16 + c from element kb*128 + 32*g + i*32*1024/B on,
 *   i.e. exactly the matrix-core operand fragment of lane l.
 *   FP8 scales keep their [N/128][K/128] layout (copied).  MXFP4 scales
 *   become [N/16][ceil(Kp/512)][64][4] bytes: in quad q of row tile rb,
 *   the 4 bytes of lane l = c + 16*g are the codes of row rb*16 + c for the
 *   32-element chunks (4q + j)*4 + g, j = 0..3 (127 in the padding).
 * w, s: device pointers in the interchange layout; w_packed, s_packed:
 * device buffers of the sizes moe_packed_size returns (s may be NULL for
 * bf16).  Requirements: N % 16 == 0, K % 32 == 0 (FP8: N, K % 128 == 0).
 */
moe_status_t moe_packed_size(int fmt, int E, int N, int K, size_t *weight_bytes, size_t *scale_bytes);

/*
 * W_gate and W_up (both E x N x K, N = d_ff, K = d) packed as one pair: the
 * streaming layout of moe_pack_weights, except that block (rb, kb) of the
 * pair is the gate block (B bytes) immediately followed by the up block, so
 * the verify kernel streams both tiles of a step as one contiguous run.
 * w_packed: 2 * weight_bytes of moe_packed_size (per pair of matrices);
 * s_gate_packed, s_up_packed: scale_bytes each (NULL for bf16), laid out as
 * moe_pack_weights lays them out.  A layer packed this way passes w_gate =
 * w_packed and w_up = NULL in moe_weights_t.  Requirements as for
 * moe_pack_weights, and 2 * weight_bytes / E below 2 GiB.
 */
moe_status_t moe_pack_gate_up(int fmt, int E, int N, int K, const void *w_gate, const void *s_gate, const void *w_up,
                              const void *s_up, void *w_packed, void *s_gate_packed, void *s_up_packed, void *stream);

/*
 * W_down (E x N x K, N = d, K = d_ff) with the two 16-row tiles that one
 * down wavefront streams interleaved: the streaming layout of
 * moe_pack_weights, except that block (2p + j, kb), j = 0, 1, sits at byte
 * offset ((p*Kp/128 + kb)*2 + j) * B, so the pair's blocks of one K step
 * form one contiguous run.  Same sizes as moe_pack_weights; the scales are
 * laid out exactly as moe_pack_weights lays them out.  A layer packed this
 * way sets down_paired = 1 in moe_weights_t (for w_down and sh_down alike).
 * Requirements as for moe_pack_weights, and N % 32 == 0
 * (MOE_ERR_UNSUPPORTED otherwise).
 */
moe_status_t moe_pack_down(int fmt, int E, int N, int K, const void *w, const void *s, void *w_packed, void *s_packed,
                           void *stream);
moe_status_t moe_pack_weights(int fmt, int E, int N, int K, const void *w, const void *s, void *w_packed,
                              void *s_packed, void *stream);

/*
 * Router top-k (Section 1: each token goes to a top-k subset of experts;
 * Table 13 gives k per model).
 *   logits   [T][E] fp32, device.
 *   topk_idx [T][k] out: for each token, the experts in routing order --
 *            larger logit first, equal logits (-0 == +0) by lower expert
 *            index, NaN after every number -- slot j holding rank j.
 *   topk_w   [T][k] out: gate weights by `score`, computed in fp32.
 * Limits: T >= 1, 1 <= E <= 1024, 1 <= k <= min(E, 64).
 */
moe_status_t moe_route_topk(const float *logits, int T, int E, int k, int score, int32_t *topk_idx,
                            float *topk_w, void *stream);

/*
 * Group-limited router top-k: the routing rule of the DeepSeek-V3 family (the
 * DeepSeek-V3.1 rows of Tables 1-13; Section 1 only fixes that each token goes
 * to a top-k subset of experts).  Per token, from the fp32 logits l:
 *   s_e = sigmoid(l_e), c_e = s_e + bias_e (bias NULL: zero);
 *   the E experts form n_group contiguous groups of E / n_group; a group's
 *   score is the sum of its two highest c (in routing order: NaN below every
 *   number, so it only counts in a group with fewer than two numbers);
 *   the topk_group groups of highest score stay eligible (ties: lower group);
 *   the k eligible experts of highest c are selected, in order (ties: lower
 *   index), slot j holding rank j;
 *   topk_w[j] = scale * s_j / sum_i s_i over the selected, in fp32.
 *   logits [T][E], bias [E], topk_idx / topk_w [T][k]: fp32 / int32 device.
 * Limits: T >= 1, 1 <= E <= 1024, 1 <= n_group <= 64, E % n_group == 0,
 * E / n_group >= 2, 1 <= topk_group <= n_group, 1 <= k <= min(64,
 * topk_group * E / n_group), scale finite; else MOE_ERR_INVALID_ARG.
 */
moe_status_t moe_route_topk_grouped(const float *logits, const float *bias, int T, int E, int k, int n_group,
                                    int topk_group, float scale, int32_t *topk_idx, float *topk_w, void *stream);

/*
 * Router from hidden states (Section 1: the router scores every expert for
 * each token, and the token goes to the top-k of them): logits = x . W_r^T,
 * then the same top-k and gate weights as moe_route_topk.
 *   x         [T][d] bf16, device, 16-byte aligned.
 *   w_router  [E][d] bf16, device, 16-byte aligned.
 *   topk_idx, topk_w: as for moe_route_topk, ranked on the logits below.
 *   logits    [T][E] fp32 out, device, or NULL: the router logits the top-k
 *             was taken on.  Each is the exact bf16 products summed in fp32;
 *             the reduction order is fixed (within 512-wide slices of d on
 *             the matrix cores, then over the slices in order), so results
 *             are deterministic, but they are not the sequential fp32 sum.
 *   workspace device scratch of moe_router_workspace_size bytes, 16-byte
 *             aligned; its contents on entry do not matter.
 * Limits: T >= 1, 1 <= E <= 1024, 1 <= k <= min(E, 64); d % 32 == 0 and x,
 * W_r each below 2 GiB (else MOE_ERR_UNSUPPORTED).  Two kernels on `stream`,
 * no allocation.
 */
moe_status_t moe_router_workspace_size(int T, int d, int E, size_t *bytes);
moe_status_t moe_route_topk_hidden(const void *x, const void *w_router, int T, int d, int E, int k, int score,
                                   int32_t *topk_idx, float *topk_w, float *logits, void *workspace,
                                   size_t workspace_bytes, void *stream);

/*
 * Expert union and grouping (Section 3, Eq. 1: the verifier must fetch the
 * union of the experts routed to by all verified tokens).
 *   topk_idx  [T][k] in (entries in [0, E)).
 *   counts    [E]    out: slots routed to each expert.
 *   union_ids [E]    out: experts with counts > 0 in ascending order, then -1.
 *   n_unique  [1]    out: U, the number of distinct experts.
 *   offsets   [E+1]  out: offsets[u] = first grouped position of union member
 *                    u; offsets[u] = T*k for u >= U.
 *   perm      [T*k]  out: slot at each grouped position; slots are ordered by
 *                    (expert, slot), i.e. a stable counting sort.
 * Limits: T >= 1, 1 <= k <= 64, 1 <= E <= 1024, T*k <= 2^24.
 */
moe_status_t moe_expert_union(const int32_t *topk_idx, int T, int k, int E, int32_t *counts,
                              int32_t *union_ids, int32_t *n_unique, int32_t *offsets, int32_t *perm,
                              void *stream);

/*
 * Bytes of device workspace moe_verify_layer needs for T tokens and top-k.
 * MOE_ERR_UNSUPPORTED when a call could hold more than 4096 token groups
 * (one per distinct expert, plus one per further 64 tokens of an expert):
 * 1025 + ceil((T*k + T) / 64) > 4096.
 */
moe_status_t moe_verify_workspace_size(const moe_weights_t *w, int T, int k, size_t *bytes);

/*
 * MoE verification layer (Section 3; Fig. 1(a): cost grows with the number
 * of distinct experts).  For every token t:
 *   y[t] = sum_j topk_w[t][j] * FFN_{topk_idx[t][j]}(x[t])  (+ FFN_shared(x[t]))
 *   FFN_e(x) = W_down[e] (silu(W_gate[e] x) * (W_up[e] x))
 * Each distinct routed expert (and the shared one) is streamed from HBM once
 * per call for up to 64 of its tokens (once per 64 tokens beyond that).  A
 * token may name an expert more than once: every slot counts, and where an
 * expert so gets more slots than T, it is streamed once per T of them (T
 * rounded up to a multiple of 16, at most 64).
 *   x  [T][d] bf16 in, y [T][d] bf16 out (may not alias x), device.
 *   r  routing for the same T, k, E: topk_idx and topk_w in (moe_route_topk);
 *      counts, union_ids, n_unique, offsets and perm out, the union of the
 *      routed experts and the grouping of the slots by expert (Eq. 1), as
 *      moe_expert_union computes them (their contents on entry do not matter).
 *   workspace: device buffer of at least moe_verify_workspace_size bytes,
 *   256-byte aligned; its contents on entry do not matter.
 * Arithmetic: weights decoded exactly to bf16, bf16 matrix cores with fp32
 * accumulation, FP8 block scales applied to fp32 partial sums, the SwiGLU
 * intermediate rounded to bf16, y rounded to bf16.  With act_fmt =
 * MOE_ACTQ_MXFP8 (MXFP4 weights) x and the SwiGLU intermediate are quantised
 * to MX FP8 instead (moe_actq_t) and multiplied on the scaled FP4 x FP8
 * matrix cores, fp32 accumulation.  Deterministic: the same inputs give
 * bit-identical y.
 * Limits: T*d*2, (T*k + T)*d_ff*2 and (T*k + T)*d*4 bytes each below 2 GiB
 * (else MOE_ERR_UNSUPPORTED), plus those of moe_verify_workspace_size.
 */
moe_status_t moe_verify_layer(const void *x, const moe_weights_t *w, const moe_routing_t *r, void *y,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * moe_verify_layer without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, results and limits as
 * moe_verify_layer; the workspace is a fixed array of the library of
 * MOE_NOALLOC_SCRATCH_BYTES per GPU (each GPU the library runs on holds its
 * own copy until the process ends).  A call whose moe_verify_workspace_size
 * exceeds it returns MOE_ERR_WORKSPACE (moe_last_error says how much it
 * needs), before anything is enqueued.  Nothing is allocated, freed or
 * cleared.  All calls on one GPU share the array and it keeps the last call's
 * contents: calls ordered on one stream are safe, calls that overlap on one
 * GPU (other streams, unordered host threads) race.  DeepSeek-V3.1-shaped FP8
 * layers fit up to about T = 96 tokens, Qwen3-shaped bf16 layers up to about
 * T = 128.
 */
#define MOE_NOALLOC_SCRATCH_BYTES (64u << 20)
moe_status_t moe_verify_layer_noalloc(const void *x, const moe_weights_t *w, const moe_routing_t *r, void *y,
                                      void *stream);

/*
 * moe_verify_layer with timing marks: identical work and arguments, and in
 * addition records the caller's events on `stream` around its kernels:
 *   events[0] before the gate/up expert kernel, events[1] after it (before
 *   its fix-up kernel), events[2] before the down expert kernel, events[3]
 *   after it (before the combine kernel), events[4] after the combine kernel.
 * With MX activations events[0] precedes the kernel that quantises x (which
 * for some calls of more than 64 tokens builds the union and the token-group
 * plan as well); without, the union of a call of more than 64 tokens is built
 * before events[0].  Calls of up to 16 tokens without MX activations, d and
 * d_ff up to 8192, have no fix-up kernel: nothing runs between events[1] and
 * events[2].
 * events is an array of 5 hipEvent_t handles created by the caller (any
 * entry may be NULL to skip that mark).
 */
moe_status_t moe_verify_layer_timed(const void *x, const moe_weights_t *w, const moe_routing_t *r, void *y,
                                    void *workspace, size_t workspace_bytes, void *stream, void *const *events);

/*
 * Cost-aware draft-tree selection on the host (Section 4.2, Eq. 7-9,
 * Algorithm 1 in the appendix; Eq. 10 of Section 5.4 for the global mode).
 *   n       number of tree nodes; parent[n] (-1 for the root, parent ids
 *           smaller than the child's), P[n] cumulative path probability.
 *   pred    [n][L][K] predicted expert ids per node and layer (Eq. 4), each
 *           in [0, E).
 *   B0      initial buffer as a bitset [L][ceil(E/64)] uint64 (bit e of word
 *           e/64 set = expert e of that layer already covered), or NULL.
 *   budget  number of nodes to select (gamma); fewer if n < budget.
 *   eps     the epsilon of Eq. 9/10; lambda weights the cost in COST_DIFF.
 *   selected       [budget] out: node ids in pick order.
 *   marginal_cost  [budget] out or NULL: number of (layer, expert) pairs of
 *                  the pick's path not covered by B0 and earlier picks.
 *   n_selected     out or NULL: number of entries written.
 * The score of every unselected node is computed each round; ties go to the
 * shallower node, then to the lower id, so the result is prefix-closed.
 * Host memory only; limits: n <= 65536, L*K <= 65536, E <= 4096.
 */
moe_status_t moe_select_tree(int n, const int32_t *parent, const double *P, int L, int K,
                             const int32_t *pred, int E, const uint64_t *B0, int budget, double eps,
                             double lambda, int mode, int32_t *selected, int32_t *marginal_cost,
                             int32_t *n_selected);

/*
 * The rest of a layer's verification step: the norm that makes x from the
 * residual stream, and the attention of the draft tokens.  In the verification
 * pass the T selected tokens of a draft tree go through the layer at once
 * ("a tree attention mask", Section 5.1): each attends to everything cached of
 * its sequence and, of the drafts, to its own ancestors and itself.  The
 * drafts' keys and values are therefore passed beside the cache, and only the
 * tokens that the verification accepts are appended to it.
 */

/* 8-bit output of moe_add_rmsnorm: OCP e4m3fn codes q [T][d], and scales.
 * The value of a code is e4m3fn(q) * scale, scale being that of its group. */
typedef enum {
    MOE_Q_NONE = 0,
    MOE_Q_FP8_GROUP = 1, /* fp32 scales [T][ceil(d/128)], one per 128 consecutive elements (the last
                            group may be shorter)                                                     */
    MOE_Q_MXFP8 = 2,     /* OCP MX: e8m0 codes u8 [T][d/32], by the rule of moe_actq_t                */
    MOE_Q_FP8_ROW = 3    /* fp32 scales [T][1], one per row                                           */
} moe_qfmt_t;

/*
 * Residual addition and root-mean-square norm.  Per row, in fp32:
 *   v = x + residual (x alone if residual is NULL);  sum = bf16(v);
 *   u = v / sqrt(mean(v^2) + eps) * weight;  y = bf16(u);
 *   q = the 8-bit form of u: fp32 scale = max(max |u|, 2^-100) / 448 over the
 *   group, code = e4m3fn(u / scale), magnitudes from 448 up saturating; or MX.
 * v and u are not rounded on the way: y and q come from the unrounded sum.
 * The mean is right for rows of any size, also where v^2 is past fp32's range.
 *   x, residual, sum, y [T][d] bf16, weight [d] bf16; q, scales by qfmt.
 *   sum, y or q may be NULL (q and scales exactly when qfmt is MOE_Q_NONE),
 *   not all three.  sum may be the buffer of x or of residual, and y that of
 *   x; other overlaps are not allowed.
 * Limits: T >= 1; T <= 2^21, d % 32 == 0 and d <= 16384 (else
 * MOE_ERR_UNSUPPORTED), finite eps >= 0; all pointers 16-byte aligned (scales:
 * 4).  One kernel, deterministic.
 */
moe_status_t moe_add_rmsnorm(const void *x, const void *residual, const void *weight, int T, int d, float eps,
                             int qfmt, void *sum, void *y, void *q, void *scales, void *stream);

/* Draft tokens of one call: N tokens of B sequences, sequence b having tokens
 * token_offsets[b] .. token_offsets[b+1] - 1 (token_offsets[0] = 0,
 * token_offsets[B] = N, none decreasing; at most 64 tokens a sequence; a
 * sequence may have none).  Bit j of mask[t] set: token t attends to the j-th
 * token of its sequence, itself included (bits past the sequence's tokens are
 * ignored).  mask NULL: every token attends to itself and those before it.
 * What a token does not attend to has no effect on it, infinities and NaN
 * among it.  A token that attends to nothing at all gets zeros, and -inf as
 * its log-sum.  Device pointers. */
typedef struct {
    int N, B;
    const int32_t *token_offsets; /* [B+1] */
    const uint64_t *mask;         /* [N] or NULL */
} moe_drafts_t;

/* Latent cache: one row of r + p bf16 a token (latent part, then rotary part,
 * shared by all heads) in pages of `page` tokens.  Token i of sequence b is
 * row i % page of page block_table[b][i / page]; cache_len[b] tokens are
 * cached (0 <= cache_len[b] <= max_blocks * page).  Requirements: r = 512,
 * p = 64 (else MOE_ERR_UNSUPPORTED); page 16, 32, 64 or 128; n_pages >= 1;
 * max_blocks * page <= 2^30; pages 16-byte aligned. */
typedef struct {
    int r, p;
    int n_pages, page, max_blocks;
    const void *pages;          /* [n_pages][page][r+p] bf16 */
    const int32_t *block_table; /* [B][max_blocks], entries in [0, n_pages) */
    const int32_t *cache_len;   /* [B] */
} moe_latent_cache_t;

/*
 * Latent attention, absorbed form: keys and values are the latent rows
 * themselves, and the key and value expansions are folded into the products
 * before and after the call.  For token t of sequence b and head h, over the
 * cached rows of b and the drafts that t attends to:
 *   s_j = scale * q[t][h] . c_j            (r + p elements)
 *   o[t][h] = sum_j softmax(s)_j c_j[0:r],   lse[t][h] = log sum_j exp(s_j)
 *   q [N][H][r+p], kv_new [N][r+p] (the drafts' rows), o [N][H][r]: bf16;
 *   lse [N][H] fp32 or NULL.
 *   workspace: device scratch of moe_latent_attn_workspace_size bytes, 256-byte
 *   aligned; its contents on entry do not matter.  The size for N and B is
 *   enough for every call of no more tokens and sequences (same cache, same H).
 * Arithmetic: bf16 products summed in fp32, softmax in fp32, the weights
 * exp(s - max) rounded to bf16 for the value product, fp32 sums, one rounding
 * to bf16 at the end.  Deterministic.
 * Limits: 1 <= H <= 1024, 1 <= B <= 1024, 1 <= N <= 64 * B, N * H <= 2^24,
 * scale finite.
 */
moe_status_t moe_latent_attn_workspace_size(const moe_latent_cache_t *cache, int N, int B, int H, size_t *bytes);
moe_status_t moe_latent_attn(const moe_latent_cache_t *cache, const moe_drafts_t *drafts, const void *q,
                             const void *kv_new, int H, float scale, void *o, float *lse, void *workspace,
                             size_t workspace_bytes, void *stream);

/*
 * Latent attention, expanded form, for prompts: every head has its own keys
 * and values, expanded from the latent rows by the caller's products, beside
 * the shared rotary part.  Sequence b has queries q_offsets[b] ..
 * q_offsets[b+1] - 1 and keys kv_offsets[b] .. kv_offsets[b+1] - 1 (both from 0
 * to N and M, none decreasing); its i-th query of n attends to the first
 * i + 1 + (m - n) of its m keys (the queries are the last n of m tokens).  A
 * query that attends to nothing gets zeros, and -inf as its log-sum; keys past
 * a query's have no effect on it, infinities and NaN among them.
 *   s_j = scale * (q[t][h][0:dn] . k_j[h] + q[t][h][dn:] . k_rope_j)
 *   o[t][h] = sum_j softmax(s)_j v_j[h],  lse[t][h] = log sum_j exp(s_j)
 *   q [N][H][dn+p], k_rope [M][p], o [N][H][dv]: bf16; lse [N][H] fp32 or NULL.
 *   k: head h of key j is the dn elements from k + j * k_stride + h * k_head
 *   on (strides in elements), v the same with dv elements; so both may be
 *   parts of one expansion's output.
 *   max_tokens: at least the most queries of a sequence.
 * Arithmetic as for moe_latent_attn.  No workspace.
 * Limits: dn = dv = 128, p = 64 (else MOE_ERR_UNSUPPORTED); 1 <= H <= 1024,
 * 1 <= B <= 1024, N, M >= 1, scale finite; strides multiples of 8, 16-byte
 * aligned pointers; k_stride, v_stride <= 2^23, N * H <= 2^30 and B * H *
 * max_tokens <= 2^30 (else MOE_ERR_UNSUPPORTED).
 */
typedef struct {
    int N, M, B, H, dn, p, dv, max_tokens;
    const int32_t *q_offsets, *kv_offsets; /* [B+1] each */
    const void *q, *k, *k_rope, *v;
    int64_t k_stride, k_head, v_stride, v_head;
    float scale;
} moe_prompt_t;

moe_status_t moe_latent_prompt(const moe_prompt_t *a, void *o, float *lse, void *stream);

/* Key/value cache of grouped-query attention in 8 bits: OCP e4m3fn codes in
 * pages of `page` tokens, with one fp32 scale for the keys and one for the
 * values of each page and head.  Paging as in moe_latent_cache_t.  A page
 * holds, per head, its keys token by token and its values element by element
 * (each element's tokens side by side: the operand order of the value
 * product).  The scales of pages in use are finite and at least
 * 2^-126.
 * Requirements: D 64 or 128 (else MOE_ERR_UNSUPPORTED); page 16, 32, 64 or
 * 128; 1 <= Hkv <= 256; max_blocks * page <= 2^30; k and v 16-byte aligned. */
typedef struct {
    int Hkv, D;
    int n_pages, page, max_blocks;
    uint8_t *k;                 /* [n_pages][Hkv][page][D] */
    uint8_t *v;                 /* [n_pages][Hkv][D][page] */
    float *k_scale, *v_scale;   /* [n_pages][Hkv] */
    const int32_t *block_table; /* [B][max_blocks], entries in [0, n_pages) */
    const int32_t *cache_len;   /* [B] */
} moe_cache_t;

/*
 * Append to the 8-bit cache.  Sequence b's new tokens are entries
 * token_offsets[b] .. token_offsets[b+1] - 1 of rows [N] (rows NULL: the
 * entries themselves), each the index of a row of k_new, v_new [n_rows][Hkv][D]
 * bf16; they go to positions cache_len[b] on.  (After a verification: rows of
 * the accepted path.)  Per touched page and head, for keys and values alike:
 *   need = the smallest power of two >= max |new value| / 448, at least 2^-126
 *          (infinities and NaN left out of the maximum);
 *   scale = need if the page begins with a new token, else max(scale, need);
 *   where the scale grows, the codes of the page's other slots are coded
 *   again: e4m3fn(value of the code / new scale), ties to even;
 *   new codes are e4m3fn(value / scale), infinities saturating to 448.
 * So a page's values stay exact multiples of their codes' grid however often
 * its scale grows, up to the smallest codes.  cache_len is not changed.  A
 * position past max_blocks * page is dropped.  No two sequences may share a
 * page that is written.
 * max_tokens: at least the most new tokens of a sequence.
 * Limits: N, n_rows, B >= 1, B <= 1024; k_new, v_new 16-byte aligned;
 * a launch of more than 2^31 threads is MOE_ERR_UNSUPPORTED, which
 * (N + 2 * B * page) * Hkv * D <= 2^35 rules out.  One kernel,
 * deterministic.
 */
moe_status_t moe_cache_append(const moe_cache_t *cache, const void *k_new, const void *v_new, int n_rows,
                              const int32_t *rows, int N, int B, const int32_t *token_offsets, int max_tokens,
                              void *stream);

/*
 * The same behind a moe_pages_update: entry i goes to row slots[i] of the
 * pages, and cache_len and block_table are not read.  A sequence whose first
 * slot lies outside [0, n_pages * page) gets nothing, as one that the update
 * refused; where it kept fewer tokens than it had, the new ones follow those.
 * slots [N] int64, 8-byte aligned: a sequence's slots on one page follow each
 * other, and the first on each of its further pages is that page's first row.
 */
moe_status_t moe_cache_append_slots(const moe_cache_t *cache, const void *k_new, const void *v_new, int n_rows,
                                    const int32_t *rows, int N, int B, const int32_t *token_offsets, int max_tokens,
                                    const int64_t *slots, void *stream);

/*
 * Grouped-query attention of draft tokens over the 8-bit cache and the drafts
 * themselves.  Query head h uses key/value head h / (H / Hkv).
 *   s_j = scale * q[t][h] . k_j,  o[t][h] = sum_j softmax(s)_j v_j,
 *   lse[t][h] = log sum_j exp(s_j), over the cached tokens (code value times
 *   its page's scale) and the drafts that t attends to (k_new, v_new).
 *   q, o [N][H][D], k_new, v_new [N][Hkv][D]: bf16; lse [N][H] fp32 or NULL.
 *   workspace: device scratch of moe_cache_attn_workspace_size bytes, 256-byte
 *   aligned; its contents on entry do not matter.  The size for N and B is
 *   enough for every call of no more tokens and sequences (same cache, same H).
 * Arithmetic: codes are exact in bf16; the keys' scale multiplies the fp32
 * scores, the values' scale the bf16 codes (its power of two, exact) and the
 * fp32 softmax weights (the rest); otherwise as for moe_latent_attn.
 * Deterministic.
 * Limits: H % Hkv == 0, H <= 1024, 1 <= B <= 1024, 1 <= N <= 64 * B,
 * N * H <= 2^24, scale finite.
 */
moe_status_t moe_cache_attn_workspace_size(const moe_cache_t *cache, int N, int B, int H, size_t *bytes);
moe_status_t moe_cache_attn(const moe_cache_t *cache, const moe_drafts_t *drafts, const void *q, const void *k_new,
                            const void *v_new, int H, float scale, void *o, float *lse, void *workspace,
                            size_t workspace_bytes, void *stream);

/*
 * The two ends of a decoding step: pages and prompts in, log probabilities
 * out.  A call runs on its stream's device, whichever is the current one.
 * Nothing that a call writes may overlap anything else that it is given
 * (MOE_ERR_INVALID_ARG).
 */

/* Pages of B sequences, for caches paged as in moe_latent_cache_t (one update
 * serves the caches of all layers that share the table).  Sequence b has
 * cache_len[b] tokens in the first ceil(cache_len[b] / page) pages of its row
 * of block_table; free_pages[0 .. n_free - 1] are the pages that nobody has.
 * No page is in two places.  page 16, 32, 64 or 128; n_pages, max_blocks >= 1;
 * max_blocks * page <= 2^30; 1 <= B <= 1024. */
typedef struct {
    int B, n_pages, page, max_blocks;
    int32_t *block_table;     /* [B][max_blocks] */
    const int32_t *cache_len; /* [B] */
    int32_t *free_pages;      /* [n_pages] */
    const int32_t *n_free;    /* [1] */
} moe_page_pool_t;

/*
 * Pages for what a step changes: sequence b keeps its first keep_len[b] tokens
 * (keep_len NULL: all; more than cache_len[b] means all) and gets n_b =
 * token_offsets[b+1] - token_offsets[b] new ones behind them.  A request that
 * ended keeps none and gets none; one that takes its place keeps none and gets
 * its prompt.
 *   have = ceil(cache_len[b] / page), want = ceil((keep + n_b) / page);
 *   where want < have, pages want .. have - 1 of the sequence are returned:
 *     the returned pages of all sequences, in order, go behind the free ones;
 *   where want > have, the sequence takes want - have pages, from the end of
 *     that list, in order of the sequences;
 *   a sequence of want > max_blocks is refused and counts for nothing; one
 *   whose last page, counted with all that the sequences before it ask for,
 *   is past what the list holds, is refused, and so are those behind it that
 *   ask for any.  A refused sequence stays as it was, with cache_len[b] tokens
 *   and its pages.
 *   token_offsets [B+1]: from 0 to at most N, none decreasing.
 *   block_table, free_pages: updated in place (what free_pages holds from
 *   *n_free_out on is left over and means nothing).
 *   new_len [B] out: keep + n_b, cache_len[b] where refused.  n_free_out,
 *   refused [1] out: the free pages left, and the refused sequences.
 *   slots [N] (int64), positions [N] out: token t of sequence b, the i-th new
 *   one, is at position keep + i, row `slots[t]` of the pages taken as one
 *   array of n_pages * page rows.  Both are -1 for tokens of a refused
 *   sequence and for entries from token_offsets[B] on.  Each may be NULL.
 * new_len and n_free_out are buffers of their own (not cache_len, keep_len or
 * n_free): the update reads the old counts throughout.  The same call again, on
 * the same counts, gives the same results; so an update whose new counts are not
 * taken over has changed nothing.  The new tokens go where slots says
 * (moe_latent_append, moe_cache_append_slots).  moe_cache_append would put
 * them behind cache_len[b]: not where fewer are kept, and for a refused sequence
 * into pages that are not its own.
 *   1 <= N <= 2^30.  One kernel, deterministic.
 */
moe_status_t moe_pages_update(const moe_page_pool_t *pool, const int32_t *keep_len, const int32_t *token_offsets, int N,
                              int32_t *new_len, int32_t *n_free_out, int32_t *refused, int64_t *slots,
                              int32_t *positions, void *stream);

/*
 * Rows of new tokens into the latent cache: row slots[i] of the pages, taken as
 * one array of n_pages * page rows, becomes row rows[i] (rows NULL: i) of
 * kv_new [n_rows][r+p] bf16.  A slot outside [0, n_pages * page) drops its
 * entry; no slot within is given twice.  pages [n_pages][page][r+p] bf16, as in
 * moe_latent_cache_t; slots [N] int64 (moe_pages_update's), rows [N].
 * Requirements: r = 512, p = 64 (else MOE_ERR_UNSUPPORTED); page 16, 32, 64 or
 * 128; pages and kv_new 16-byte aligned; N, n_rows >= 1, N <= 2^24 (else
 * MOE_ERR_UNSUPPORTED).  One kernel.
 */
moe_status_t moe_latent_append(void *pages, int n_pages, int page, int r, int p, const void *kv_new, int n_rows,
                               const int32_t *rows, int N, const int64_t *slots, void *stream);

/*
 * Grouped-query attention of whole prompts.  Sequence b has queries
 * q_offsets[b] .. q_offsets[b+1] - 1 and keys kv_offsets[b] .. kv_offsets[b+1] - 1
 * (both from 0 to at most N and M, none decreasing); its i-th query of n attends
 * to the first i + 1 + (m - n) of its m keys (the queries are the last n of m
 * tokens).  A query that attends to nothing gets zeros, and -inf as its
 * log-sum; keys past a query's have no effect on it, infinities and NaN among
 * them.  Query head h uses key/value head h / (H / Hkv).
 *   s_j = scale * q[t][h] . k_j,  o[t][h] = sum_j softmax(s)_j v_j,
 *   lse[t][h] = log sum_j exp(s_j)
 *   q: head h of query t is the D elements from q + t * q_stride + h * q_head
 *   on (strides in elements), k and v likewise by key and key/value head: parts
 *   of one projection's output may be passed as they lie.
 *   o [N][H][D] bf16; lse [N][H] fp32 or NULL.  Rows from q_offsets[B] on are
 *   left as they were.
 *   max_tokens: at least the most queries of a sequence.  The launch has
 *   workgroups for that many of each, and whether long keys are cut into chunks
 *   follows from them: a number far above the most costs time.
 *   workspace: device scratch of moe_grouped_prompt_workspace_size bytes, 256-byte
 *   aligned; its contents on entry do not matter.  The size depends on D alone.
 * Arithmetic as for moe_latent_attn.  Deterministic: the same call gives the
 * same bits; in another batch a sequence's keys may be summed in other chunks.
 * Limits: D 64 or 128 (else MOE_ERR_UNSUPPORTED); 1 <= Hkv <= 256, H % Hkv == 0,
 * H <= 1024, 1 <= B <= 1024, N, M >= 1, scale finite; strides >= 0 and multiples
 * of 8, 16-byte aligned pointers; k_stride, v_stride <= 2^23, N * H <= 2^30 and
 * B * H * max_tokens <= 2^30 (else MOE_ERR_UNSUPPORTED).
 */
typedef struct {
    int N, M, B, H, Hkv, D, max_tokens;
    const int32_t *q_offsets, *kv_offsets; /* [B+1] each */
    const void *q, *k, *v;
    int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head;
    float scale;
} moe_grouped_prompt_t;

moe_status_t moe_grouped_prompt_workspace_size(int D, size_t *bytes);
moe_status_t moe_grouped_prompt(const moe_grouped_prompt_t *a, void *o, float *lse, void *workspace,
                                size_t workspace_bytes, void *stream);

/* Type of the logits. */
typedef enum {
    MOE_F32 = 0,
    MOE_BF16 = 1
} moe_dtype_t;

/*
 * Log probabilities from logits: what a verification accepts drafts by, and
 * what an answer reports.  Per row of V logits l, with s = scale * l (scale: the
 * inverse temperature):
 *   lse = log sum_j exp(s_j),  p_j = exp(s_j - lse),
 *   logprob[m] = s_t - lse for each given token t = tokens[m] (-inf for a t
 *     outside [0, V): a place that is not used),
 *   entropy = -sum_j p_j log p_j,
 *   top_idx, top_logprob: the k tokens of largest logit, larger first, equal
 *     ones (-0 == +0) by lower index, NaN after every number.
 * A logit of -inf has probability 0.  A row of nothing else has lse and all log
 * probabilities -inf, and entropy 0.  A NaN among the logits, or a scaled one of
 * +inf, makes the row's lse, entropy and log probabilities NaN (those of unused
 * places stay -inf).
 *   logits: row n is the V elements from logits + n * stride on (stride in
 *   elements, >= V; any alignment of the type); dtype: moe_dtype_t.
 *   tokens [N][M], logprob [N][M] (both NULL exactly when M is 0), lse and
 *   entropy [N], each or NULL, top_idx [N][k], top_logprob [N][k] (top_idx NULL
 *   exactly when k is 0; top_logprob may be NULL).
 *   workspace: device scratch of moe_token_logprobs_workspace_size bytes,
 *   256-byte aligned; its contents on entry do not matter.  The size is 2.2 MB
 *   for any number of rows.
 * Arithmetic: exponentials in fp32, relative to the largest logits so far, their
 * sum in fp64; the logits are read once.  Deterministic.
 * Limits: 1 <= N <= 2^22, 1 <= V <= 2^24, 0 <= k <= min(V, 64), 0 <= M <= 65536,
 * N * M <= 2^30, scale finite and > 0, at most 2^126 (else
 * MOE_ERR_UNSUPPORTED).  One or two kernels.
 */
moe_status_t moe_token_logprobs_workspace_size(int N, size_t *bytes);
moe_status_t moe_token_logprobs(const void *logits, int dtype, int64_t stride, int N, int V, float scale,
                                const int32_t *tokens, int M, int k, float *logprob, float *lse, float *entropy,
                                int32_t *top_idx, float *top_logprob, void *workspace, size_t workspace_bytes,
                                void *stream);

/* Static description of a status code. */
const char *moe_status_string(moe_status_t status);

/* Message of the last HIP error seen by this thread (empty if none). */
const char *moe_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ECOSPEC_MOE_H */
