/*
 * vmoe.h -- C ABI of libvmoe: one adaptation step of T concurrent V-MoE expert
 * layers on one NVIDIA GB300 (sm_103a).
 *
 * The method is AdaSprite's multi-task V-MoE co-adaptation (arxiv 2608.16188):
 * the experts of T V-MoEs form one pool (Section 2.2, "MoE merging"); each
 * task keeps its own router and experts and its tokens are routed to their
 * most relevant experts (Section 2.1) under per-expert capacity limits
 * (Challenge #1 in Section 1, Section 2.3.1); the experts of all tasks run
 * concurrently (Section 3.2, expert parallelism) and only the visual
 * experts are adapted (Section 3.1, specification-based tuning).  Here every
 * stage is one grouped launch over all T*E (task, expert) groups.
 *
 * One step is:
 *   vmoe_route     logits = x W_r + bias; softmax; top-k; capacity scan
 *   vmoe_dispatch  Xe  = gather(x)               (padding rows zero)
 *   vmoe_expert_fwd H = Xe W1, A = GELU(H), Ye = A W2
 *   vmoe_combine   y   = sum_j gate_j * Ye[e_j, s_j]
 *   vmoe_dispatch  dYe = gate * gather(dY)
 *   vmoe_expert_bwd dH = (dYe W2^T) * GELU'(H), dXe = dH W1^T,
 *                  dW1 = Xe^T dH, dW2 = A^T dYe
 *   vmoe_combine   dX  = sum_j dXe[e_j, s_j]
 *   vmoe_router_bwd dgate, dlogits, dW_r, dbias; dX += dlogits W_r^T
 * vmoe_gate and vmoe_gate_bwd stand in the places of vmoe_route and vmoe_router_bwd for
 * routers with scores, groups of experts and a bias for balance (vmoe_gate_bias).
 * Around it, in training: vmoe_balance and vmoe_balance_bwd (the routers' balance
 * losses), vmoe_block_norm and vmoe_block_norm_bwd (a block's norms, gate and
 * residual), vmoe_head_loss and vmoe_head_loss_bwd (a head over a vocabulary, cross
 * entropy and distillation), vmoe_adamw (the update).
 *
 * Conventions for every entry point:
 *  - Ownership: every array argument is caller-owned DEVICE memory (except
 *    the vmoe_problem struct, read on the host), row-major and contiguous in
 *    the layout stated, with a base address aligned to 16 bytes.  The library
 *    allocates no device memory and keeps no state between calls other than
 *    the device status word (vmoe_device_status) and the optional trace.
 *  - Execution: calls enqueue kernels on `cuda_stream` (a cudaStream_t; NULL
 *    is the legacy default stream) and return without synchronising.
 *  - Errors: arguments are checked on the host before any launch; an invalid
 *    argument returns VMOE_ERR_INVALID and an unsupported shape
 *    VMOE_ERR_UNSUPPORTED, in both cases with nothing launched.  A failed
 *    launch returns VMOE_ERR_CUDA.  Device data is trusted: loads are clamped
 *    to [0, C], and expert indices or slots out of range are undefined
 *    behaviour.
 *  - Determinism: results are bitwise reproducible run to run (no atomics in
 *    any reduction but of whole numbers, fixed summation orders).
 *  - Host threads: entry points may be called from several host threads at
 *    once, each with its own stream and arrays; the kernel trace is kept per
 *    host thread.  The exception is vmoe_expert_bwd_static_scratch, whose
 *    calls share one device array (see there).
 *  - Dtypes: x, dY, weights and all activations use p->dtype (fp32 or bf16);
 *    W_r, bias, logits and gates are always fp32.  bf16 contractions
 *    accumulate in fp32 on the tcgen05 tensor cores; fp32 runs on CUDA cores, but for
 *    the head's products (three bf16 parts of each value).
 *
 * Shapes (t < T tasks, n < N tokens per task, e < E experts per task,
 * j < k choices, s < C capacity slots, g = t*E + e):
 *   x, y, dY, dX [T,N,d]   W_r [T,d,E]   bias [T,E]   logits [T,N,E]
 *   expert_idx, gate, slot [T,N,k]   load [T,E]
 *   Xe, Ye, dYe, dXe [T,E,C,d]   H, A [T,E,C,f]
 *   W1, dW1 [T,E,d,f]   W2, dW2 [T,E,f,d]
 */
#ifndef VMOE_H
#define VMOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define VMOE_VERSION 1

typedef enum {
    VMOE_OK = 0,
    VMOE_ERR_INVALID = -1,        /* bad argument; nothing launched */
    VMOE_ERR_UNSUPPORTED = -2,    /* valid but unsupported shape; nothing launched */
    VMOE_ERR_CUDA = -3,           /* a CUDA runtime call or launch failed */
    VMOE_ERR_DEVICE_TIMEOUT = -4  /* a kernel gave up a bounded wait (vmoe_device_status) */
} vmoe_status;

typedef enum { VMOE_F32 = 0, VMOE_BF16 = 1 } vmoe_dtype;

enum {
    VMOE_LOGITS_IN = 1u << 0, /* vmoe_route reads `logits` instead of computing them */
    VMOE_NO_RENORM = 1u << 1, /* gate = softmax probability (V-MoE); default renormalises over top-k */
    VMOE_GELU_TANH = 1u << 2, /* tanh-approximate GELU; default is the exact erf form */
    VMOE_DLOGITS_ADD = 1u << 3 /* vmoe_router_bwd adds to the gradients that `dlogits` holds */
};

/* The problem statement: T tasks, each with N tokens of width d_model, its own
 * router and E experts of hidden width d_ff; top-k routing with capacity
 * C = ceil(capacity_factor * k * N / E) clamped to [1, N], or `capacity` when
 * it is > 0.  Limits: T, N, E >= 1; 1 <= k <= min(E, 8); E <= 256;
 * T*E <= 1024; d_model % 8 == 0.  The bf16 expert path also needs d_model and
 * d_ff to be multiples of 128 (VMOE_ERR_UNSUPPORTED otherwise). */
typedef struct {
    int32_t T, N, d_model, d_ff, E, k;
    double capacity_factor;
    int32_t capacity;
    vmoe_dtype dtype;
    uint32_t flags;
} vmoe_problem;

/* Library version (VMOE_VERSION). */
int vmoe_version(void);

/* Human-readable name of a vmoe_status value (static storage). */
const char *vmoe_status_string(int status);

/* The capacity C the library uses for `p` (capacity rule above), or a negative
 * vmoe_status if `p` is invalid.  Host only; no device work. */
int vmoe_problem_capacity(const vmoe_problem *p);

/* Routing: top-k softmax gating with per-expert capacity (Section 2.1 routing
 * to the most relevant experts; capacity limits of Challenge #1; sequential
 * assignment of Section 3.3.1).
 *   x          [T,N,d] p->dtype           input tokens (unused with VMOE_LOGITS_IN; may be NULL then)
 *   w_router   [T,d,E] fp32               per-task router (unused with VMOE_LOGITS_IN)
 *   logit_bias [T,E]   fp32, nullable     per-task additive logit bias
 *   logits     [T,N,E] fp32               output, or input with VMOE_LOGITS_IN
 *   expert_idx [T,N,k] int32 out          the k largest logits, descending, ties to the lower index
 *   gate       [T,N,k] fp32 out           softmax probability of each choice, divided by the
 *                                         top-k probability mass unless VMOE_NO_RENORM
 *   slot       [T,N,k] int32 out          position in the expert's buffer, -1 if dropped: in
 *                                         choice-major order (all first choices in token order,
 *                                         then all second choices, ...) the s-th assignment to an
 *                                         expert gets slot s while s < C
 *   load       [T,E]   int32 out          kept assignments per expert = min(count, C)
 * Logits are accumulated in fp32.  A NaN logit is treated as -inf when the
 * experts are chosen (indices stay in range); its gates are unspecified. */
int vmoe_route(const vmoe_problem *p, const void *x, const float *w_router,
               const float *logit_bias, float *logits, int32_t *expert_idx, float *gate,
               int32_t *slot, int32_t *load, void *cuda_stream);

/* Dispatch (permute into expert-contiguous buffers for the grouped expert
 * launch of Section 3.2): dst[t,e,s,:] = w * src[t,n,:] for the kept choice
 * (n, j) with expert_idx = e and slot = s, w = weight[t,n,j] or 1 if weight
 * is NULL; rows s >= load[t,e] of dst are written as zero.
 *   src [T,N,d] p->dtype, weight [T,N,k] fp32 nullable, expert_idx/slot [T,N,k],
 *   load [T,E], dst [T,E,C,d] p->dtype (every element written).
 * The weighted product is formed in fp32 and rounded to p->dtype. */
int vmoe_dispatch(const vmoe_problem *p, const void *src, const float *weight,
                  const int32_t *expert_idx, const int32_t *slot, const int32_t *load,
                  void *dst, void *cuda_stream);

/* Expert FFN forward over all T*E groups in one grouped launch per layer
 * (Section 2.1: the ViT MLP block becomes experts; no bias terms):
 *   H = Xe W1, A = GELU(H), Ye = A W2, per group g for its rows s < load[g].
 *   xe [T,E,C,d], w1 [T,E,d,f], w2 [T,E,f,d], load [T,E] int32
 *   h, a [T,E,C,f] out, ye [T,E,C,d] out -- rows s >= load[g] are not written.
 * Rows s >= load[g] of xe are padding: their contents (NaN included) reach no
 * output.  load[g] is clamped to [0, C].
 * bf16: fp32 accumulation; A is GELU of the fp32 accumulator, H and A are
 * stored rounded to bf16. */
int vmoe_expert_fwd(const vmoe_problem *p, const void *xe, const void *w1, const void *w2,
                    const int32_t *load, void *h, void *a, void *ye, void *cuda_stream);

/* Device bytes of scratch vmoe_expert_bwd needs for `p`, or 0 if `p` is
 * invalid.  Host only.  It holds dH: T*E*C*d_ff fp32 elements for fp32
 * problems; for bf16, 2*T*E*C*d_ff bf16 elements, dH kept as a bf16 value plus
 * its bf16 residual so the weight gradients of small groups stay accurate. */
size_t vmoe_expert_bwd_workspace_size(const vmoe_problem *p);

/* The smallest workspace vmoe_expert_bwd accepts for `p`, or 0 if `p` is
 * invalid.  Host only.  fp32: the full size above.  bf16: one group's dH (2C
 * rows, rounded up to 8) plus 8*T*E bytes (rounded up to 256) for the plan of a
 * sliced run -- see vmoe_expert_bwd. */
size_t vmoe_expert_bwd_min_workspace_size(const vmoe_problem *p);

/* Expert FFN backward (adaptation of the expert weights, Section 3.1), the
 * gradient of <dY, y> through the expert path with routing and gates fixed:
 *   dH = (dYe W2^T) * GELU'(H), dXe = dH W1^T, dW1 = Xe^T dH, dW2 = A^T dYe,
 * the weight gradients summing over each group's rows s < load[g].
 *   xe [T,E,C,d], h, a [T,E,C,f] (from vmoe_expert_fwd), w1, w2, dye [T,E,C,d]
 *   (= vmoe_dispatch(dY, gate)), load [T,E]
 *   dxe [T,E,C,d] out (rows >= load not written), dw1 [T,E,d,f] out, dw2 [T,E,f,d] out
 *   (every element written; zero for a group with load 0)
 *   Rows s >= load[g] of xe, h, a and dye are padding: their contents (NaN
 *   included) reach no output.
 *   workspace: caller-owned device scratch, 16-byte aligned, its contents
 *   clobbered.  With vmoe_expert_bwd_workspace_size(p) bytes or more, dH of
 *   every group fits and the call is asynchronous.  bf16 problems also accept
 *   less, down to vmoe_expert_bwd_min_workspace_size(p): the groups are then
 *   placed in slices whose dH fits (the cross-task DP of vmoe_plan_slices,
 *   Section 3.2.1, each group's footprint its dH rows, its lifespan its load)
 *   and dA, dX and dW1 run slice by slice.  That path reads `load` back to the
 *   host first and synchronises `cuda_stream` (once); it then launches dW2 and
 *   plans one slice at a time, each slice's kernels queued as soon as it is
 *   placed, and returns when the last slice is queued.  The results are
 *   bitwise the same either way.  Less than the minimum, or NULL, returns
 *   VMOE_ERR_INVALID. */
int vmoe_expert_bwd(const vmoe_problem *p, const void *xe, const void *h, const void *a,
                    const void *w1, const void *w2, const void *dye, const int32_t *load,
                    void *dxe, void *dw1, void *dw2, void *workspace, size_t workspace_bytes,
                    void *cuda_stream);

/* Size in bytes of the device array behind vmoe_expert_bwd_static_scratch. */
#define VMOE_STATIC_SCRATCH_BYTES (64u << 20)

/* vmoe_expert_bwd without a caller-supplied workspace, for callers that cannot
 * allocate device memory: a plug-in whose host framework owns every device
 * buffer, or a deployment that allows no device allocation after start-up.
 * The paper has no counterpart; this is a packaging choice of the library.
 *   Arguments, layouts and results are those of vmoe_expert_bwd.  The dH
 *   scratch is a 64 MiB array compiled into the library, which every GPU that
 *   loads the library holds until the process exits; the call itself allocates
 *   nothing.  When vmoe_expert_bwd_workspace_size(p) <= VMOE_STATIC_SCRATCH_BYTES,
 *   dH of every group fits and the call is asynchronous like vmoe_expert_bwd.
 *   Otherwise a bf16 problem runs in slices planned to fit the array (as
 *   vmoe_expert_bwd with a smaller workspace): that path reads `load` back to
 *   the host and synchronises `cuda_stream`.  The call returns
 *   VMOE_ERR_UNSUPPORTED, with nothing launched, only when even
 *   vmoe_expert_bwd_min_workspace_size(p) exceeds the array: an fp32 problem
 *   whose dH is larger than the array, or a bf16 problem one of whose groups
 *   alone does not fit.  The first call on a device looks up the array's
 *   device address (cudaGetSymbolAddress) with that device current and caches
 *   it; make that first call before any stream capture.  Every call on a
 *   device shares the one array, which keeps whatever the last call left in
 *   it, so calls whose kernels overlap on the GPU (other streams, other host
 *   threads) race and corrupt each other's dH; issue them in order on one
 *   stream. */
int vmoe_expert_bwd_static_scratch(const vmoe_problem *p, const void *xe, const void *h,
                                   const void *a, const void *w1, const void *w2, const void *dye,
                                   const int32_t *load, void *dxe, void *dw1, void *dw2,
                                   void *cuda_stream);

/* Attention experts (Section 2.1: V-MoE expertizes the ViT's attention as well
 * as its MLP; Section 3.2.1's memory estimator gives such an expert buffers of
 * order T d_k for Q / K / V and T^2 for the scores).  The paper gives no more;
 * the library's reading: each (task, expert) group g owns W_qkv [d, 3 H 64]
 * (column blocks Q | K | V, head h at columns h * 64 of each) and W_o [H 64, d],
 * and runs H-head softmax attention, head dimension 64, among its L = load[g]
 * routed tokens only (the rows [0, L) of xe, as dispatched by vmoe_dispatch):
 *   QKV = Xe W_qkv;  per head  S = Q_h K_h^T / 8,  P = softmax over the L keys
 *   (row maximum subtracted),  O_h = P V_h;  Ye = O W_o,
 * then vmoe_combine gate-weights Ye back to token order as for the FFN.
 * bf16 only, H even, d % 128 == 0, C <= 512 (else VMOE_ERR_UNSUPPORTED);
 * p->d_ff is not used.  Sums accumulate in fp32; P is rounded to bf16 for the
 * P V product; no atomics.  Rows s >= load[g] of xe (and of dye, qkv, o in the
 * backward) are padding, reach no output and are not written.
 *   xe [T,E,C,d], wqkv [T,E,d,3H64], wo [T,E,H64,d] in; qkv [T,E,C,3H64],
 *   o [T,E,C,H64] bf16 and lse [T,E,H,C] fp32 (each row's log-sum-exp of the
 *   scaled scores, kept for the backward) out; ye [T,E,C,d] out. */
int vmoe_attn_expert_fwd(const vmoe_problem *p, int heads, const void *xe, const void *wqkv,
                         const void *wo, const int32_t *load, void *qkv, void *o, float *lse, void *ye,
                         void *cuda_stream);

/* Workspace of vmoe_attn_expert_bwd in bytes (dO and dQKV in bf16, then the row
 * sums D of dO * O in fp32), or 0 for an invalid or unsupported problem. */
size_t vmoe_attn_expert_bwd_workspace_size(const vmoe_problem *p, int heads);

/* Backward of vmoe_attn_expert_fwd with routing and gates fixed: the gradient
 * of <dYe, Ye> per group,
 *   dO = dYe W_o^T,  dW_o = O^T dYe,  D = rowsum(dO * O) per head,
 *   dS = P * (dO_h V_h^T - D),  dQ_h = dS K_h / 8,  dK_h = dS^T Q_h / 8,  dV_h = P^T dO_h,
 *   dXe = dQKV W_qkv^T,  dW_qkv = Xe^T dQKV,
 * P rebuilt from qkv and lse, D formed from the stored o.  The attention core's
 * products take fp16 operands, each staged tile of Q, K, V and dO scaled by a
 * power of two (exact for bf16 values down to 2^-29 of the tile's largest), so P
 * and dS enter dV, dQ and dK with 11 significant bits; for C > 128, dQ instead
 * takes bf16 operands and dS as a bf16 value plus its residual.  A row of Q or dO
 * that is infinite, NaN or 2^29 times the others thus reaches dK and dV of its
 * whole group and head, and, for C <= 128, the other rows' dQ.  Sums accumulate in
 * fp32.  Inputs as written by the forward (xe, qkv, o, lse) and dye [T,E,C,d]
 * (vmoe_dispatch of dY with the gates); outputs dxe [T,E,C,d] (rows >= load not
 * written), dwqkv [T,E,d,3H64] and dwo [T,E,H64,d] (zero for an
 * empty group).  workspace: caller-owned device scratch of at least
 * vmoe_attn_expert_bwd_workspace_size(p, heads) bytes (else VMOE_ERR_INVALID),
 * its contents clobbered.  Asynchronous on `cuda_stream`. */
int vmoe_attn_expert_bwd(const vmoe_problem *p, int heads, const void *xe, const void *qkv,
                         const void *o, const float *lse, const void *wqkv, const void *wo,
                         const void *dye, const int32_t *load, void *dxe, void *dwqkv, void *dwo,
                         void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Combine back to token order: dst[t,n,:] = sum over kept choices j (slot >= 0)
 * of w * src[t, expert_idx_j, slot_j, :], w = weight[t,n,j] or 1 if NULL,
 * summed in fp32 in the order j = 0..k-1 and rounded once; a token with every
 * choice dropped gets zero.
 *   src [T,E,C,d], weight [T,N,k] fp32 nullable, expert_idx/slot [T,N,k],
 *   dst [T,N,d] out.  The forward uses weight = gate, the backward (dX) NULL. */
int vmoe_combine(const vmoe_problem *p, const void *src, const float *weight,
                 const int32_t *expert_idx, const int32_t *slot, void *dst, void *cuda_stream);

/* Router backward (Section 3.1 adapts the visual module, its gating network
 * included; Section 2.1 defines the gates as a softmax of the router logits).
 * With the routing held fixed (expert_idx, slot from vmoe_route), the gradient
 * of <dY, y> with y = sum_j gate_j Ye[e_j, s_j]:
 *   dgate[t,n,j]   = <dY[t,n], Ye[t,e_j,s_j]> for a kept choice, 0 if dropped;
 *   dlogits[t,n,e] = softmax backward: with s = sum_j gate_j dgate_j,
 *     renormalised gates:  dlogits[e_j] = gate_j (dgate_j - s), 0 elsewhere;
 *     VMOE_NO_RENORM:      dlogits[e]   = p_e (dgate(e) - s), p = softmax(logits)
 *                          and dgate(e) = dgate_j if e = e_j, else 0;
 *   dw_router[t]   = x[t]^T dlogits[t]      (sum over the N tokens of task t);
 *   dbias[t,e]     = sum_n dlogits[t,n,e];
 *   dx[t,n,:]     += W_r[t] dlogits[t,n]    (summed in fp32, rounded once).
 * Inputs: x, dY [T,N,d] and Ye [T,E,C,d] in p->dtype (Ye is the expert output
 * of vmoe_expert_fwd); w_router [T,d,E], logits [T,N,E], gate [T,N,k] fp32;
 * expert_idx, slot [T,N,k] int32.  w_router may be NULL only when dx is NULL;
 * logits is read only with VMOE_NO_RENORM (else it may be NULL).
 * Outputs (overwritten): dgate [T,N,k], dlogits [T,N,E], dw_router [T,d,E]
 * fp32; dbias [T,E] fp32, nullable.  dx [T,N,d] in p->dtype is read and
 * updated in place (the dX of vmoe_combine, which then holds the input
 * gradient through both the experts and the router); NULL skips it.
 * Sums run in fixed orders; no atomics. */
int vmoe_router_bwd(const vmoe_problem *p, const void *x, const float *w_router,
                    const float *logits, const int32_t *expert_idx, const float *gate,
                    const int32_t *slot, const void *dy, const void *ye, float *dgate,
                    float *dlogits, float *dw_router, float *dbias, void *dx,
                    void *cuda_stream);

/* Balance losses of the routers, with per-expert counts (they keep what an
 * uneven router would send to a full expert, Challenge #1, from being dropped).
 * Per task t, over the M tokens that take part, with p = softmax(logits):
 *   count[t,e]  = choices j of tokens n with expert_idx[t,n,j] = e, before the
 *                 capacity drops any
 *   excess[t,e] = sum_n p[n,e] - M / E, the expert's importance above an even share
 *   loss[t,0]   = E / (k M^2) sum_e count_e sum_n p[n,e]     (1 for an even load)
 *   loss[t,1]   = E / M^2 sum_e excess_e^2    (squared coefficient of variation of
 *                 the importances)
 *   loss[t,2]   = 1 / M sum_n lse_n^2, lse_n = log sum_e exp(logits[n,e])
 * A token takes part unless its token_mask is 0 or all its logits are -inf; one
 * that does not reaches no output, whatever its logits and choices hold.  A task
 * without tokens gets zeros.  Single logits of -inf are experts of probability 0.
 * An index outside [0, E) is not counted; a NaN or +inf logit of a token that
 * takes part makes its task's excess and losses NaN.
 *   logits [T,N,E] fp32, expert_idx [T,N,k] (from vmoe_route), token_mask [T,N]
 *   uint8 nullable; count [T,E] int32, tokens [T] int32 (= M), excess [T,E] fp32,
 *   loss [T,3] fp32 out (every element written).
 *   workspace: caller-owned device scratch of vmoe_balance_workspace_size(p)
 *   bytes or more (else VMOE_ERR_INVALID), 16-byte aligned, its contents clobbered.
 * p->d_model, d_ff, the capacity, the dtype and the flags are not used.  Sums in
 * fp32 and in fixed orders; the counts are whole numbers. */
int vmoe_balance(const vmoe_problem *p, const float *logits, const int32_t *expert_idx,
                 const uint8_t *token_mask, int32_t *count, int32_t *tokens, float *excess, float *loss,
                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Device bytes of scratch vmoe_balance needs for `p`, or 0 if `p` is invalid.  Host only. */
size_t vmoe_balance_workspace_size(const vmoe_problem *p);

/* Gradient of sum_t,i dloss[t,i] loss[t,i] by the logits (the counts have none):
 *   c_e = dloss[t,0] E / (k M^2) count_e + dloss[t,1] 2 E / M^2 excess_e,
 *   dlogits[t,n,e] = p_e (c_e - sum_i p_i c_i + dloss[t,2] 2 / M lse_n),
 * 0 for a token that does not take part.  logits and token_mask as given to
 * vmoe_balance; count, tokens and excess as it wrote them; dloss [T,3] fp32 on the
 * device; dlogits [T,N,E] fp32 out (every element written), which may be logits
 * itself.  Give it to vmoe_router_bwd with VMOE_DLOGITS_ADD. */
int vmoe_balance_bwd(const vmoe_problem *p, const float *logits, const uint8_t *token_mask,
                     const int32_t *count, const int32_t *tokens, const float *excess,
                     const float *dloss, float *dlogits, void *cuda_stream);

typedef enum {
    VMOE_SCORE_SOFTMAX = 0, /* s_e: the softmax of a token's logits */
    VMOE_SCORE_SIGMOID = 1  /* s_e = 1 / (1 + exp(-logit_e)) */
} vmoe_score;

/* How vmoe_gate chooses. */
typedef struct {
    int32_t score;       /* vmoe_score */
    int32_t groups;      /* divides E: experts e with the same e / (E / groups) are a group; 1: none */
    int32_t groups_kept; /* groups a token may choose from; groups_kept * (E / groups) >= k */
    int32_t group_top;   /* 1 or 2, at most E / groups */
    float scale;         /* > 0: what the gates are taken times */
} vmoe_gating;

/* Routing with scores, a bias for balance and groups of experts: vmoe_route's place
 * in a step (Section 2.1; capacity limits of Challenge #1; sequential assignment of
 * Section 3.3.1), for routers that are balanced by select_bias instead of by losses.
 *   c_e = s_e + select_bias_e;  a group's value: the sum of its group_top largest c;
 *   open: the groups_kept groups of the largest values; the choices: the k largest c
 *   in open groups, descending;  gate_j = scale s_j / sum_i s_i over the choices,
 *   scale s_j with VMOE_NO_RENORM.
 * Equal values go to the lower index, and what is larger is decided in exact
 * arithmetic (64 bits), not by fp32 roundings of s.  The bias acts on the choice
 * alone.  An expert whose logit or bias is not finite (-inf, say) is switched off: never
 * chosen; a logit that is not finite is 0 in a softmax too, a bias takes nothing from the
 * softmax, whose sum keeps the expert.  Where fewer than k experts can be chosen, the
 * rest of the token's choices have expert_idx -1, gate 0 and slot -1 and take no
 * capacity; the other entry points pass over them.  So it is for all choices of a token
 * whose token_mask is 0, whose logits may hold anything.
 *   x, w_router, logit_bias, logits, expert_idx, gate, slot, load as for vmoe_route;
 *   select_bias [T,E] fp32 nullable; token_mask [T,N] uint8 nullable;
 *   demand [T,E] int32 out, nullable: choices of each expert, dropped ones too;
 *   workspace: caller-owned device scratch of vmoe_gate_workspace_size(p) bytes or
 *   more (else VMOE_ERR_INVALID), 16-byte aligned, its contents clobbered.
 * T*N < 2^31 and N*k < 2^31 (else VMOE_ERR_UNSUPPORTED). */
int vmoe_gate(const vmoe_problem *p, const vmoe_gating *gating, const void *x, const float *w_router,
              const float *logit_bias, const float *select_bias, const uint8_t *token_mask, float *logits,
              int32_t *expert_idx, float *gate, int32_t *slot, int32_t *load, int32_t *demand, void *workspace,
              size_t workspace_bytes, void *cuda_stream);

/* Device bytes of scratch vmoe_gate needs for `p`, or 0 if `p` is invalid.  Host only. */
size_t vmoe_gate_workspace_size(const vmoe_problem *p);

/* vmoe_router_bwd for choices of vmoe_gate: the gradient of <dY, y> through the gates,
 * choices and slots held fixed, with r_j = gate_j / scale, m = sum_i r_i dgate_i:
 *   dgate_j = <dY[t,n], Ye[t, e_j, s_j]>, 0 where slot is -1
 *   sigmoid: dlogit_{e_j} = gate_j (1 - s_j) (dgate_j - m), without m with VMOE_NO_RENORM
 *   softmax: dlogit_{e_j} = gate_j (dgate_j - m); VMOE_NO_RENORM: dlogit_e =
 *   scale s_e (dgate_e - m) for every e, dgate_e 0 unless chosen
 *   dW_r = x^T dlogits, dbias = sum_n dlogits (of logit_bias), dX = dX_in + dlogits W_r^T
 * Other dlogits, and those of a token without choices, are 0.  dW_r takes 0 times such a
 * token's x, which has to be finite; its logits and dY may hold anything.  logits and
 * select_bias have no other part in it.  VMOE_DLOGITS_ADD as for vmoe_router_bwd.
 *   dx_in, dx [T,N,d] p->dtype, both or neither; dx_in may be dx.  The rest as for
 *   vmoe_router_bwd (w_router is needed with dx, logits always). */
int vmoe_gate_bwd(const vmoe_problem *p, const vmoe_gating *gating, const void *x, const float *w_router,
                  const float *logits, const int32_t *expert_idx, const float *gate, const int32_t *slot, const void *dy,
                  const void *ye, float *dgate, float *dlogits, float *dw_router, float *dbias, const void *dx_in, void *dx,
                  void *cuda_stream);

/* The balance of vmoe_gate's choices, after a step: select_bias[t,e] += rate where
 * demand[t,e] is below the task's mean, -= rate where it is above it. */
int vmoe_gate_bias(const vmoe_problem *p, const int32_t *demand, float rate, float *select_bias, void *cuda_stream);

enum {
    VMOE_HEAD_SHARED = 1u << 0 /* one head for all tasks: w, dw [V,d] instead of [T,V,d] */
};

/* A head over a vocabulary behind the blocks, and what it is trained against. */
typedef struct {
    int32_t V;         /* entries of the vocabulary */
    int32_t teacher_k; /* K: entries of a teacher's list for each token, 0: no teacher; at most 128, V <= 2^20 with one */
    float temperature; /* tau > 0 */
    uint32_t flags;    /* VMOE_HEAD_SHARED */
} vmoe_head;

/* Losses of l[t,n,:] = w[t] z[t,n], the logits never written out (Section 3.1: the
 * tasks adapt to labels and to what a larger model answers):
 *   lse = log sum_v exp(l_v),  ce = lse - l_label           of tokens with a label;
 *   tlse = log sum_v exp(l_v / tau),  logp_j = l_{i_j} / tau - tlse,
 *   kl = sum_j q_j (log q_j - logp_j),  q the softmax of teacher_logit / tau over the
 *   list's entries,                                          of tokens with a teacher.
 * A label outside [0, V) is none.  Entries of a list whose index is outside [0, V) or whose
 * logit is -inf are left out (logp 0); a list of such entries alone is no teacher.  An
 * index may be there twice: each counts.  Where a token has no label, or no teacher,
 * those outputs are 0; the z of a token that has neither is not read and costs nothing.
 *   z [T,N,d], w [T,V,d] ([V,d] with VMOE_HEAD_SHARED) p->dtype, an entry a row as in
 *   an embedding table; label [T,N] int32; teacher_idx [T,N,K] int32, teacher_logit [T,N,K]
 *   fp32; ce, lse, kl, tlse [T,N], logp [T,N,K] fp32 out.  label, ce and lse are given
 *   together or not at all; teacher_* and kl, tlse, logp exactly if teacher_k > 0; one
 *   of both is there.
 *   workspace: caller-owned device scratch, 16-byte aligned, its contents clobbered, of
 *   vmoe_head_workspace_size(p, head) bytes for this call and the backward, or of any
 *   size from vmoe_head_min_workspace_size(p, head) on (else VMOE_ERR_INVALID): the
 *   backward then takes the vocabulary in more pieces.
 * An entry may be switched off by weights of the type's lowest value, or -inf, where the
 * tokens that take part have positive values: it then adds nothing to the sums.  dz takes
 * 0 times them, so bf16 weights have to be finite in the backward.
 * Sums in fp32; fp32 operands are taken as three bf16 parts each, six products of
 * parts (2^-24).  T*N < 2^31 - 256, V <= 2^30, d_model <= 65536 (else
 * VMOE_ERR_UNSUPPORTED).  Of p only T, N, d_model, dtype and the checks matter. */
int vmoe_head_loss(const vmoe_problem *p, const vmoe_head *head, const void *z, const void *w, const int32_t *label,
                   const int32_t *teacher_idx, const float *teacher_logit, float *ce, float *lse, float *kl, float *tlse,
                   float *logp, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Gradient of sum dce ce + dlse lse + dkl kl:
 *   dl_v = (dce + dlse) exp(l_v - lse) - dce [v = label]
 *        + dkl / tau (exp(l_v / tau - tlse) - sum_{j: i_j = v} q_j)
 *   dz = dl w,  dw = dl^T z (of one head's tokens; all tokens with VMOE_HEAD_SHARED).
 * The first arguments as given to vmoe_head_loss, ce to logp as it wrote them; dce,
 * dlse, dkl [T,N] fp32, each nullable (zero; one at least is given; not looked at where
 * a token has no label, or no teacher).  dz [T,N,d], dw as w, p->dtype out, every
 * element written, either nullable.  dl, an operand of tensor cores, is rounded to
 * p->dtype: in bf16 dz and dw are then 2.3e-3 off in the mean, where rounding them alone
 * is 1.7e-3.  Of heads with N <= 128 (T*N with VMOE_HEAD_SHARED), or 256 with a small
 * vocabulary, it is kept to 2^-16.  No output may overlap an input.  Sums in fp32
 * and in fixed orders; no atomics. */
int vmoe_head_loss_bwd(const vmoe_problem *p, const vmoe_head *head, const void *z, const void *w, const int32_t *label,
                       const int32_t *teacher_idx, const float *teacher_logit, const float *ce, const float *lse,
                       const float *tlse, const float *logp, const float *dce, const float *dlse, const float *dkl, void *dz,
                       void *dw, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Device bytes of scratch for the two: what is recommended, and what will do; 0 if `p` or
 * `head` is invalid or unsupported.  Host only. */
size_t vmoe_head_workspace_size(const vmoe_problem *p, const vmoe_head *head);
size_t vmoe_head_min_workspace_size(const vmoe_problem *p, const vmoe_head *head);

enum {
    VMOE_NORM_RMS = 1u << 0,  /* root-mean-square norms (no mean); default is the layer norm */
    VMOE_NORM_POST = 1u << 1  /* a norm on the branch y */
};

/* The norms around a layer: norm(v) = (v - mean) / sqrt(var + eps) * weight + bias
 * over the d channels of a token (mean 0 with VMOE_NORM_RMS). */
typedef struct {
    float eps;            /* > 0 */
    float residual_scale; /* rho */
    uint32_t flags;
} vmoe_norm;

/* A transformer block's residual around its expert layer (Section 2.1), in one
 * pass over the tokens:
 *   w = norm(y; post_w, post_b) with VMOE_NORM_POST, else y
 *   z = rho x + gate * w             rounded to p->dtype
 *   u = norm(z; pre_w, pre_b)        of z as stored: the next layer's input
 * y NULL: no branch, u = norm(x); z, gate, post_* are NULL then.  u NULL: z alone;
 * pre_* are NULL then.  At least one of y and u is given.
 *   x, y, z, u [T,N,d] p->dtype; post_w, post_b, gate, pre_w, pre_b [T,d] fp32,
 *   each nullable (weights and gate 1, biases 0); post_stat, pre_stat [T,N,2]
 *   fp32 out, nullable: each norm's mean and 1 / sqrt(var + eps), for the backward.
 * z may be x itself; no other output may overlap an input.  d_model <= 8192 and
 * T*N < 2^31 (else VMOE_ERR_UNSUPPORTED).  Statistics and sums in fp32. */
int vmoe_block_norm(const vmoe_problem *p, const vmoe_norm *norm, const void *x, const void *y,
                    const float *post_w, const float *post_b, const float *gate, const float *pre_w,
                    const float *pre_b, void *z, void *u, float *post_stat, float *pre_stat,
                    void *cuda_stream);

/* Device bytes of scratch vmoe_block_norm_bwd needs for `p`, or 0 if `p` is
 * invalid or unsupported.  Host only. */
size_t vmoe_block_norm_bwd_workspace_size(const vmoe_problem *p);

/* Backward of vmoe_block_norm for the gradients dz of z and du of u (either may
 * be NULL: zero), with dzt = dz + (d u / d z)^T du:
 *   dx = rho dzt (dzt where y is NULL),  dy = (d w / d y)^T (gate * dzt),
 *   dpost_w = sum_n gate * dzt * yhat,  dpost_b = sum_n gate * dzt,  dgate = sum_n dzt * w,
 *   dpre_w = sum_n du * zhat,  dpre_b = sum_n du,
 * yhat and zhat the normalised y and z (yhat = y without VMOE_NORM_POST).
 *   y as given to the forward (NULL: no branch; dy, post_*, gate and their
 *   gradients are NULL then); z as it was stored, or x without a branch, needed
 *   with du; post_stat (with y and VMOE_NORM_POST) and pre_stat (with du) from the
 *   forward; the parameters as given to it.  du NULL: pre_* and their gradients
 *   are NULL.  dx, dy [T,N,d] p->dtype out; the parameters' gradients [T,d] fp32
 *   out, each nullable, NULL where its parameter is.
 *   workspace: caller-owned device scratch of
 *   vmoe_block_norm_bwd_workspace_size(p) bytes or more (else VMOE_ERR_INVALID),
 *   16-byte aligned, its contents clobbered.
 * dx may be dz itself; no other output may overlap an input.  Sums in fp32 and in
 * fixed orders; no atomics. */
int vmoe_block_norm_bwd(const vmoe_problem *p, const vmoe_norm *norm, const void *y, const void *z,
                        const float *post_stat, const float *pre_stat, const float *post_w,
                        const float *post_b, const float *gate, const float *pre_w, const void *dz,
                        const void *du, void *dx, void *dy, float *dpost_w, float *dpost_b,
                        float *dgate, float *dpre_w, float *dpre_b, void *workspace,
                        size_t workspace_bytes, void *cuda_stream);

typedef enum {
    VMOE_STATE_F32 = 0,  /* m and v in fp32 */
    VMOE_STATE_E4M3 = 1  /* m and sqrt(v) in 8 bits, a scale for each 256 elements */
} vmoe_adamw_state;

/* One tensor of vmoe_adamw; device pointers, 16-byte aligned (the scales: 4). */
typedef struct {
    void *param;       /* [numel], updated in place */
    const void *grad;  /* [numel] */
    void *m, *v;       /* moments, [numel]: fp32, or e4m3 with VMOE_STATE_E4M3 */
    float *m_scale, *v_scale; /* [ceil(numel / 256)] with VMOE_STATE_E4M3, else NULL */
    float *master;     /* [numel] fp32 copy of bf16 parameters that the update works on, nullable */
    int64_t numel;     /* 0: the tensor is passed over */
    int32_t param_dtype, grad_dtype; /* vmoe_dtype; fp32 parameters have fp32 gradients */
    int32_t state;     /* vmoe_adamw_state */
    float lr_scale, weight_decay;
} vmoe_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps; /* lr finite, betas in [0, 1), eps >= FLT_MIN */
    int32_t step;            /* t, 1 for the first update */
    uint32_t seed;           /* of the 8-bit moments' rounding */
    const int32_t *step_dev; /* device, nullable: t = step + *step_dev (at least 1) */
    const float *lr_dev;     /* device, nullable: the learning rate is lr times *lr_dev */
    const float *grad_scale; /* device, nullable: gradients are taken times it */
} vmoe_adamw_config;

/* One AdamW update of n tensors (the adaptation of Section 3.1) in one launch for
 * up to 380 of them, with r = lr lr_scale:
 *   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
 *   p = p (1 - r weight_decay) - r (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),
 * in fp32; bf16 parameters are rounded to nearest from the master copy, or from
 * their own updated value where there is none.  `tensors` and `config` are host
 * memory, read before the call returns; step, lr and seed of a captured call stay
 * what they were, so a graph that is replayed takes step_dev and lr_dev.
 * A grad_scale that is infinite or NaN leaves everything as it was.
 * VMOE_STATE_E4M3: element i is held as m = m_scale[i / 256] * m[i] and sqrt(v) =
 * v_scale[i / 256] * v[i]; a new scale is its block's largest magnitude / 448 (0
 * below 2^-100, where the block's moments become 0), and a value a = |m| / scale
 * becomes grid * floor(a / grid + (16 R + 8) / 2^20), at most 448, grid the step of
 * e4m3 at a: rounded up or down at random, a in the mean, but for a positive sqrt(v)
 * becoming 2^-9 at least, one step: at 0 the next update would be m over eps.  Elements
 * whose gradients stay 2^17 below their block's largest so move less than with fp32
 * moments.  R is the low (m) or the high (v) half of mix(0x51f6db5b i + 0x5e4087b3
 * place + 0x339cd49b t + 0xe32a5e87 seed) mod 2^32, place the tensor's index in the
 * call, with mix(h): h = (h ^ h >> 16) * 0x9e4a8af7, h = (h ^ h >> 15) * 0xa6bd2c99,
 * h ^ h >> 16.  An infinite moment makes its block's moments NaN.
 * The tensors' arrays may not overlap (not checked here; one array given twice is a
 * race).  numel < 2^38.  Asynchronous on `cuda_stream`; no workspace. */
int vmoe_adamw(int n, const vmoe_adamw_tensor *tensors, const vmoe_adamw_config *config,
               void *cuda_stream);

/* Cross-task slice planner (Section 3.2.1, fragmentation-aware expert
 * grouping; host code, no GPU).  Items (experts) i = 0..n-1 have a memory
 * footprint weight[i] >= 0 and a lifespan lifespan[i]; the value of an item is
 * v_i = weight[i] / M - eta * lifespan[i], M = budget if budget > 0, else
 * capacity.  A 0/1-knapsack DP, dp[i][j] = max(dp[i-1][j], dp[i-1][j - w_i] +
 * v_i), picks the slice of largest total value whose weight fits `capacity`;
 * the chosen items leave and the DP runs again until every item is placed.
 * Items enter the DP in shortest-job-first order (lifespan, then index) and
 * keep that order inside a slice; an item is taken only when strictly better;
 * if nothing is chosen, the first remaining item forms a slice alone;
 * zero-weight items join the first slice.
 * Output: order[n], the items slice by slice; slice_start[n + 1], where slice s
 * is order[slice_start[s] .. slice_start[s + 1]).  Returns the number of slices,
 * VMOE_ERR_INVALID (null pointers, negative weight, NaN lifespan) or
 * VMOE_ERR_UNSUPPORTED (an item heavier than capacity, or a DP table above 2^30
 * entries). */
int vmoe_plan_slices(int n, const int64_t *weight, const double *lifespan, int64_t capacity,
                     double eta, double budget, int32_t *order, int32_t *slice_start);

/* Resource shares of co-running experts (Section 3.2.2, lifespan-aware
 * aligning; host code, no GPU): the fill-clamp-refill allocation of `budget`
 * units among n experts -- each is seeded with minimum[i]; what is left is
 * shared out in proportion to work[i] among the experts below their
 * saturation[i]; an expert above its saturation is clamped to it and what it
 * gave up is shared out again, until nothing is left or every expert with work
 * is saturated.  An expert with work 0 keeps its minimum.  The real-valued
 * shares are then rounded to whole units: floored, and the units still
 * missing from their total given one each to the largest fractional parts
 * (ties to the lower index), so minimum[i] <= shares[i] <= saturation[i].
 * float64 arithmetic, sums in index order.
 * Output: shares[n].  Returns the number of units allocated (budget, or less
 * when the saturations do not reach it), VMOE_ERR_INVALID (null pointers,
 * negative or NaN work, negative minimum, saturation below minimum) or
 * VMOE_ERR_UNSUPPORTED (the minima exceed the budget). */
int vmoe_plan_shares(int n, const double *work, const int32_t *minimum, const int32_t *saturation,
                     int32_t budget, int32_t *shares);

/* Device status word of the current device: 0 when clean, otherwise a
 * vmoe_status (VMOE_ERR_DEVICE_TIMEOUT after a kernel gave up a bounded
 * wait).  Synchronises the current device.  `reset` != 0 clears the word. */
int vmoe_device_status(int reset);

/* Self-test of the failure path: launches one kernel that waits on a device
 * barrier nothing ever signals, through the same bounded wait the grouped GEMM
 * uses, and gives up after `limit_ns` nanoseconds (1 ns .. 1 s).  The wait
 * running out sets the device status word to VMOE_ERR_DEVICE_TIMEOUT (read and
 * cleared with vmoe_device_status) and the kernel returns normally, leaving the
 * context usable.  Returns VMOE_OK after the launch, VMOE_ERR_INVALID for a
 * limit out of range. */
int vmoe_selftest_bounded_wait(long long limit_ns, void *cuda_stream);

/* Kernel trace (host-side tracing aid).  While enabled on the calling host
 * thread, every kernel the library launches is bracketed by two CUDA events
 * recorded on its stream; at most `max_records` launches are kept.
 * vmoe_trace_disable stops recording and returns the number of records;
 * vmoe_trace_get synchronises on record i and returns its kernel name (static
 * storage) and duration in milliseconds.  Returns VMOE_OK or a vmoe_status. */
int vmoe_trace_enable(int max_records);
int vmoe_trace_disable(void);
int vmoe_trace_get(int i, const char **kernel_name, float *ms);

#ifdef __cplusplus
}
#endif
#endif /* VMOE_H */
