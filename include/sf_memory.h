/*
 * sf_memory -- the operators of a memory block on one MI355X (gfx950): a recurrent core with a matrix for a
 * state, and what stands around it in a residual block.  Next to sf_policy.h: same library, same conventions
 * (int status, sf_last_error(), device pointers, asynchronous on the caller's stream, nothing allocated, no
 * synchronisation, no pointer kept past the stream's work).  All functions run on the current HIP device.
 * Workspaces belong to the caller, 256-byte aligned; their contents do not matter before or after a call, but calls
 * that may run at the same time need one each.  Repeated calls give the same bits.
 *
 * Element types: SF_DTYPE_FP32 or SF_DTYPE_BF16 of the arrays marked "io"; states, decays, norm weights and
 * their gradients are fp32 always.  Sums and states are held in fp32; what a result of a bf16 call is rounded from is
 * said at each function.  Sizes of 0 in T, N, B or M are accepted and leave only what does not depend on them
 * (final states, gradients of weights).
 */
#ifndef SF_MEMORY_H
#define SF_MEMORY_H

#include "sf_policy.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear attention with a decay for each head ---------------------------------
 * For row (trajectory) n and head h, with g = exp(log_decay[h]):
 *   S_t = g (done[t][n] ? 0 : S_{t-1}) + k_t v_t^T      S_{-1} = state0,   S is [dk][dv]
 *   o_t = scale * S_t^T q_t                             state = S_{T-1}
 * done = 1 at the first step of an episode, as in sf_policy_unroll; what lies before it does not reach past
 * it, NaN and infinities included, and no step reaches an earlier one.  Key and value heads may be shared: head h
 * reads key/value head h / (H / Hk).
 * The passes over trajectories compute this in chunks of 32 steps (two matrix products inside a chunk, the
 * state between chunks), and where rows x heads are few, T is cut into pieces whose states are joined.
 *
 * Arrays are time-major: q [T][N][H][dk], k [T][N][Hk][dk], v [T][N][Hk][dv], o and its gradient [T][N][H][dv], io;
 * element (t, n, h, i) of q is q[t * q_stride[0] + n * q_stride[1] + h * q_stride[2] + i], strides in elements, so
 * that all three may lie in one projection's output.  Any strides and any alignment of the elements; a call is fast if in all its
 * arrays rows are of a multiple of eight elements, 16-byte aligned, and steps at least a row and at most 2^23 elements
 * apart.  Gradients dq, dk, dv are dense.  Results must not overlap inputs, nor one another, but for state as said below.
 * Of an infinity in an array or a state the results that it reaches are infinite or NaN.
 *   log_decay  dev [H] fp32, <= 0 (-infinity: the state is only the last step's; NaN: every result of its head is NaN
 *              that a decay enters)
 *   done       dev [T][N] bytes or NULL (no episode begins)
 *   state0     dev [N][H][dk][dv] fp32 or NULL (zero); state, dstate, dstate0 alike (NULL: not wanted / zero)
 * Errors: SF_ERR_ARG (null or misaligned pointer, struct_size, dtype), SF_ERR_SHAPE (T, N < 0; H, Hk < 1;
 * H % Hk != 0; dk or dv outside 1..128; T * N beyond 2^31 - 1, N * H beyond 2^21; scale not finite), SF_ERR_DEVICE. */
typedef struct {
  uint32_t struct_size; /* sizeof(sf_linattn_config) */
  int32_t dtype;        /* SF_DTYPE_* of q, k, v, o and their gradients */
  int32_t T, N, H, Hk, dk, dv;
  float scale;
  int64_t q_stride[3], k_stride[3], v_stride[3]; /* step, row, head */
  int64_t o_stride[3];                           /* of o, and of do in the backward pass */
} sf_linattn_config;

/* Bytes of the workspace of sf_linattn (backward = 0) or sf_linattn_backward (1); 0: none is needed, NULL may be
 * passed; -1 on a bad configuration. */
int64_t sf_linattn_workspace_bytes(const sf_linattn_config* cfg, int backward);
/* state may be state0 (the states are then updated in place), but must not overlap it otherwise (SF_ERR_ALIAS). */
int sf_linattn(const sf_linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
               const uint8_t* done, const float* state0, void* o, float* state, void* workspace, void* hip_stream);
/* Gradients with respect to q, k, v and state0, given those of o (do) and of the final state (dstate or NULL).
 * log_decay is a constant.  Nothing of the forward pass is needed but its inputs.  dstate0 must overlap neither
 * dstate nor state0 (SF_ERR_ALIAS). */
int sf_linattn_backward(const sf_linattn_config* cfg, const void* q, const void* k, const void* v,
                        const float* log_decay, const void* d_o, const uint8_t* done, const float* state0,
                        const float* dstate, void* dq, void* dk, void* dv, float* dstate0, void* workspace,
                        void* hip_stream);
/* One step for B = cfg->N rows (cfg->T must be 1, stride[0] is not used): the policy worker's side.  Row b stands for
 * environment e = env_ids[b] (b itself if env_ids is NULL), whose state is row e of
 *   state_table  dev [n_env][H][dk][dv] fp32, 16-byte aligned, read and overwritten;
 * ids must be distinct; a row whose id is outside [0, n_env) is computed from a zero state and its new state is
 * dropped.  done [B] bytes or NULL. */
int sf_linattn_step(const sf_linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                    float* state_table, int32_t n_env, const int32_t* env_ids, const uint8_t* done, void* o,
                    void* hip_stream);

/* ---- the norms behind and before a block, with its gate, residual scale and residual stream ----
 * For each of M rows of D channels, b the block's output and x the residual stream it is added to:
 *   u = N_post(b) * post_w            over each of `groups` equal groups of channels
 *   y = x + scale * act(gate) * u     the residual stream behind the block
 *   n = N_pre(y) * pre_w              what the next block is given
 *   N = SF_NORM_NONE  the row itself (post_w is not used then)
 *       SF_NORM_RMS   r / sqrt(mean r^2 + eps)
 *       SF_NORM_LAYER (r - mean r) / sqrt(mean (r - mean r)^2 + eps)
 *   act = SF_GATE_NONE: 1 (gate is not used), SF_GATE_SIGMOID, SF_GATE_SILU (g sigmoid(g))
 * groups > 1 (an attention core's norm per head) needs pre = SF_NORM_NONE.  x NULL: no residual stream, y = scale *
 * act(gate) * u.  post_w, scale, pre_w: fp32 [D] or NULL (ones).
 *   b, x, gate  dev [M] rows of D, io, row m at m * *_stride elements
 *   y, n        dev [M][D] dense, io.  y may be NULL if there is an n, n is not written without N_pre.  y may be x
 *               (dense), b or gate, n likewise if y is not it.
 * Backward: dy [M] rows (NULL: zero, with N_pre only) and dn [M] rows (with N_pre) are the gradients of y and n; dx, db,
 * dgate [M][D] dense io and dpost_w, dscale, dpre_w fp32 [D] are written where they are not NULL (zeros for a
 * weight that is not used; dgate only with a gate, SF_ERR_ARG).  Nothing of the forward pass is needed but its inputs.  dx, db, dgate may each be any one of
 * the inputs (dense).
 * workspace: sf_resnorm_workspace_bytes(cfg), NULL if no gradient of a weight is wanted.
 * Any D up to 8192 a group, any strides; rows of whole 16-byte pieces, 16-byte aligned, are read in such pieces.
 * Errors: SF_ERR_ARG, SF_ERR_SHAPE (M < 0, D or groups out of range, groups > 1024, groups with N_pre, eps < 0),
 * SF_ERR_DEVICE. */
enum { SF_NORM_NONE = 0, SF_NORM_RMS = 1, SF_NORM_LAYER = 2 };
enum { SF_GATE_NONE = 0, SF_GATE_SIGMOID = 1, SF_GATE_SILU = 2 };
typedef struct {
  uint32_t struct_size; /* sizeof(sf_resnorm_config) */
  int32_t dtype;        /* SF_DTYPE_* of the rows */
  int32_t M, D, groups, post, pre, gate_act;
  float eps;
  int64_t b_stride, x_stride, gate_stride, dy_stride, dn_stride; /* elements between rows */
} sf_resnorm_config;
int sf_resnorm(const sf_resnorm_config* cfg, const void* b, const void* x, const void* gate, const float* post_w,
               const float* scale, const float* pre_w, void* y, void* n, void* hip_stream);
int64_t sf_resnorm_workspace_bytes(const sf_resnorm_config* cfg);
int sf_resnorm_backward(const sf_resnorm_config* cfg, const void* b, const void* x, const void* gate, const float* post_w,
                        const float* scale, const float* pre_w, const void* dy, const void* dn, void* dx, void* db,
                        void* dgate, float* dpost_w, float* dscale, float* dpre_w, void* workspace, void* hip_stream);

/* ---- the gated feed-forward block --------------------------------------------------
 *   h = act(x w_gate^T) * (x w_up^T),   y = h w_down^T
 * x [M] rows of D, w_gate and w_up [F] rows of D, w_down [D] rows of F, all of one type, rows *_stride elements apart; y
 * [M][D] dense, 16-byte aligned.
 *   act = SF_ACT_SILU (g sigmoid(g)), SF_ACT_GELU (g Phi(g), by erf), SF_ACT_SIGMOID
 * bf16: products of bf16 numbers are added in fp32, h is rounded to bf16, y is rounded once more.  fp32: operands are the
 * exact sums of three bf16 numbers, of whose nine products six are added (2^-27 is left out); up to 128 rows forwards run
 * on the fp32 matrix instruction.  Infinities and NaN are only in the rows of y whose rows of x hold them; in weights they
 * reach all (of an infinity fp32 results are NaN).
 * Backward: dy [M] rows -> dx [M][D], dw_gate, dw_up [F][D], dw_down [D][F], dense, 16-byte aligned, of the same type.
 * Nothing of the forward pass is needed but its inputs.  Results must not overlap inputs.
 * Rows may have anything between them.  bf16 rows of a multiple of 64 numbers (w_down backwards: of 8), 16-byte aligned and less than 2^22
 * elements apart, are read where they are; others, and all fp32 arrays, are laid out in the workspace first.  A call of few rows forwards
 * reads all arrays where they are, in 16-byte pieces if x, w_gate and w_up (and w_down) consist of them, else number by number.
 * workspace: sf_ffn_workspace_bytes(cfg, backward), 256-byte aligned, wanted unless M is 0.
 * Errors: SF_ERR_ARG, SF_ERR_SHAPE (M outside 0 .. 2^24, D or F outside 1 .. 2^20), SF_ERR_DEVICE. */
enum { SF_ACT_SILU = 0, SF_ACT_GELU = 1, SF_ACT_SIGMOID = 2 };
typedef struct {
  uint32_t struct_size; /* sizeof(sf_ffn_config) */
  int32_t dtype;        /* SF_DTYPE_* of all arrays */
  int32_t M, D, F, act;
  int64_t x_stride, w_gate_stride, w_up_stride, w_down_stride, dy_stride; /* elements between rows */
} sf_ffn_config;
int64_t sf_ffn_workspace_bytes(const sf_ffn_config* cfg, int backward); /* -1 on a bad configuration */
int sf_ffn(const sf_ffn_config* cfg, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y,
           void* workspace, void* hip_stream);
int sf_ffn_backward(const sf_ffn_config* cfg, const void* x, const void* w_gate, const void* w_up, const void* w_down,
                    const void* dy, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                    void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
