/*
 * rc_ops.h -- C ABI of the sequence-model operators of the MI355X library:
 * the short causal convolution, the selective state space scan, the norms
 * before and after a block fused with its gate and residual scale, the gated
 * delta rule, the norms of queries and keys with their rotation by position,
 * and dropout.
 *
 * They are the nodes of a network whose recomputation rc.h plans: a segment
 * of a canonical strategy (Section 3 of Kusumoto et al.) is run forward,
 * dropped and run again with these calls, and differentiated with the
 * *_backward ones.  Single-token forms (*_step) update states in place.
 *
 * Conventions shared by every entry point:
 *  - Every pointer is device memory of the current device unless its name
 *    ends in _host; the arguments struct itself is host memory and is read
 *    before the call returns.  The library keeps no pointer.
 *  - Work is enqueued on stream (a hipStream_t, NULL: the default stream).
 *    No call synchronises, allocates or copies to the host, so every call can
 *    be captured into a graph.  Scratch is the caller's: the *_workspace
 *    calls give its size for the same arguments (its pointers are not read), and
 *    a smaller one returns RC_E_SCRATCH.  Like every 32-bit array, the scan's
 *    kept states among them, it is aligned to 4 bytes (else RC_E_ARG).
 *  - A negative return is an error (enum rc_status of rc.h); nothing is
 *    enqueued then, except after RC_E_DEVICE.  Nothing crosses the ABI as an
 *    exception.
 *  - Sizes may be zero.  A call whose outputs are empty does nothing.
 *    length and width are at most 2^30; sizes that need a launch of 2^32
 *    threads or more return RC_E_OVERFLOW.
 *  - Channels are contiguous; batch and time strides are in elements and
 *    free, with any alignment that the type has.  Outputs must not overlap
 *    inputs or each other.
 *  - Sums, states and statistics are held in 32 bits; each 16-bit output is
 *    rounded once, from its 32-bit value.  Results do not depend on the order in
 *    which workgroups run.
 *  - lengths[batch] (may be NULL: all full): tokens at and past a sequence's
 *    length are not read as numbers (they may hold NaN), their outputs and gradients are 0, and
 *    the state is the one after the last token before.  Values are clamped to [0, length].
 */
#ifndef RC_OPS_H
#define RC_OPS_H

#include "rc.h"

#ifdef __cplusplus
extern "C" {
#endif

enum rc_dtype { RC_F32 = 0, RC_BF16 = 1, RC_F16 = 2 };
enum rc_activation { RC_ACT_NONE = 0, RC_ACT_SILU = 1, RC_ACT_SIGMOID = 2 };

/* A (batch, time, channel) tensor: element (b, t, c) is
 * data[b * batch + t * time + c].  data NULL: the tensor is absent. */
typedef struct {
  void* data;
  int64_t batch, time;
} rc_view;

/*
 * Short causal convolution, each channel on its own:
 *   p[b,t,d] = bias[d] + sum_k weight[d,k] x[b, t - (taps-1) + k, d],
 *   y = p or p sigmoid(p).
 * x at negative times comes from state_in (batch, taps-1, width), oldest
 * first, or is 0.  state_out: the last taps-1 inputs before the sequence's
 * end.  All but weight and bias are of dtype; those are of param_dtype
 * (RC_F32 or dtype).  1 <= taps <= 8.
 * Backward: dy (required), dstate_out (may be absent: 0) -> dx, dstate_in
 * (may be absent), dweight and dbias (param_dtype; each may be NULL).
 */
typedef struct {
  int32_t dtype, param_dtype, activation;
  int32_t batch, length, width, taps;
  rc_view x, y, state_in, state_out;
  const void* weight;               /* [width][taps] */
  const void* bias;                 /* [width] or NULL */
  const int32_t* lengths;           /* [batch] or NULL */
  rc_view dy, dstate_out, dx, dstate_in;
  void* dweight;
  void* dbias;
  void* workspace;
  uint64_t workspace_bytes;
} rc_conv_args;

int rc_conv_forward(const rc_conv_args* args, void* stream);
int rc_conv_backward(const rc_conv_args* args, void* stream);
int rc_conv_backward_workspace(const rc_conv_args* args, uint64_t* bytes_host);
/* One token: x and y are (batch, width) (their time strides are not used),
 * state (slots, taps-1, width) is shifted by the token in place.  Row b uses
 * state slot slots[b] (slots NULL: b); a row whose slot is outside
 * [0, num_slots) is padding: y is 0 and no state is touched.  Slots of one
 * call must differ. */
typedef struct {
  int32_t dtype, param_dtype, activation;
  int32_t batch, width, taps, num_slots;
  rc_view x, y, state;
  const void* weight;
  const void* bias;
  const int32_t* slots;             /* [batch] or NULL */
} rc_conv_step_args;
int rc_conv_step(const rc_conv_step_args* args, void* stream);

/*
 * Selective state space scan.  Channel d of group g = d / (width / groups)
 * has `states` states h; with delta = softplus(dt + dt_bias) (softplus != 0)
 * or dt + dt_bias,
 *   h_t = exp(delta A[d]) h_{t-1} + delta u B[g],
 *   y_t = (h_t . C[g] + D[d] u) z sigmoid(z)        (each optional part may be absent)
 * u, dt, z, y: (batch, length, width); B, C: element (b, t, g, n) at
 * b * batch + t * time + g * group_stride + n, all of dtype.  A [width][states],
 * D, dt_bias [width] and the states [batch][width][states] are 32-bit floats, contiguous.
 * A is finite and not positive.  1 <= states <= 64; groups divides width.
 * kept: NULL, or the states that rc_scan_backward starts its recomputation
 * from (rc_scan_kept_bytes); it is written by rc_scan_forward and read by
 * rc_scan_backward of the same sizes.
 * Backward: dy (required), dstate_out (may be NULL: 0) -> du, ddt, dz (absent
 * exactly where z is), dB, dC (dtype, contiguous (batch, length, groups, states)),
 * dA, dD (if D), ddt_bias (if dt_bias), dstate_in (may be NULL), 32-bit.
 */
typedef struct {
  int32_t dtype, softplus;
  int32_t batch, length, width, states, groups;
  rc_view u, dt, z, B, C, y;
  int64_t B_group, C_group;         /* group strides of B and C */
  const float* A;
  const float* D;
  const float* dt_bias;
  const float* state_in;            /* or NULL: 0 */
  float* state_out;                 /* or NULL */
  const int32_t* lengths;
  float* kept;
  rc_view dy, du, ddt, dz;
  void* dB;
  void* dC;
  const float* dstate_out;
  float* dA;
  float* dD;
  float* ddt_bias;
  float* dstate_in;
  void* workspace;
  uint64_t workspace_bytes;
} rc_scan_args;

int rc_scan_forward(const rc_scan_args* args, void* stream);
int rc_scan_backward(const rc_scan_args* args, void* stream);
int rc_scan_kept_bytes(const rc_scan_args* args, uint64_t* bytes_host);
int rc_scan_forward_workspace(const rc_scan_args* args, uint64_t* bytes_host);
int rc_scan_backward_workspace(const rc_scan_args* args, uint64_t* bytes_host);
/* One token: u, dt, z, y are (batch, width) and B, C (batch, groups, states)
 * (time strides are not used); state (num_slots, width, states), contiguous but
 * for its slot stride, is updated in place; slots as rc_conv_step. */
typedef struct {
  int32_t dtype, softplus;
  int32_t batch, width, states, groups, num_slots;
  rc_view u, dt, z, B, C, y;
  int64_t B_group, C_group;
  const float* A;
  const float* D;
  const float* dt_bias;
  float* state;
  int64_t state_slot;               /* slot stride of state */
  const int32_t* slots;
} rc_scan_step_args;
int rc_scan_step(const rc_scan_step_args* args, void* stream);

/*
 * Norms before and after a block, with its gate and residual scale.  For
 * each of `rows` rows of `width` <= 16384 channels:
 *   v = block act(gate);  p = v / rms(v) * post_weight  (or v without post_weight);
 *   out = residual + scale p;  normed = out / rms(out) * pre_weight,
 * rms(x) = sqrt(mean(x^2) + eps).  gate, post_weight, scale and pre_weight
 * may be absent (then normed is absent too); block may be absent: out is then
 * the residual and is not written.  block, gate and normed are of dtype,
 * residual and out of residual_dtype, the weights and scale of param_dtype
 * (each RC_F32 or dtype).  Views use their batch strides as row strides.
 * stats [rows][2] (may be NULL): 1/rms of v and of out, written by forward,
 * read by backward (required there).
 * Backward: dout (residual_dtype) and dnormed (dtype), each may be absent (0)
 * -> dblock, dgate, dresidual (each absent where its input is),
 * dpost_weight, dscale, dpre_weight (param_dtype; each may be NULL).
 */
typedef struct {
  int32_t dtype, residual_dtype, param_dtype, gate_activation;
  int32_t rows, width;
  float eps;
  rc_view block, gate, residual, out, normed;
  const void* post_weight;
  const void* scale;
  const void* pre_weight;
  float* stats;
  rc_view dout, dnormed, dblock, dgate, dresidual;
  void* dpost_weight;
  void* dscale;
  void* dpre_weight;
  void* workspace;
  uint64_t workspace_bytes;
} rc_norm_args;

int rc_norm_forward(const rc_norm_args* args, void* stream);
int rc_norm_backward(const rc_norm_args* args, void* stream);
int rc_norm_backward_workspace(const rc_norm_args* args, uint64_t* bytes_host);

/* A (batch, time, head, channel) tensor: element (b, t, h, c) is
 * data[b * batch + t * time + h * head + c].  data NULL: the tensor is absent. */
typedef struct {
  void* data;
  int64_t batch, time, head;
} rc_heads;

/*
 * Gated delta rule (linear attention whose state corrects what it returns for a key).
 * Head h keeps a matrix S of key x value numbers; with k and q of key head
 * h / (heads / key_heads),
 *   S_t = exp(g) S_{t-1} + k (beta (v - exp(g) S_{t-1}^T k))^T,   o_t = scale S_t^T q.
 * q, k: (batch, length, key_heads, key); v, o: (batch, length, heads, value), all of
 * dtype.  g (absent: 0) and beta: (batch, length, heads), 32-bit floats; g is not
 * positive (-infinity forgets everything).  States (batch, heads, key, value) are
 * 32-bit floats, contiguous.  1 <= key, value <= 256; key_heads divides heads.
 * A number that is not finite makes its own token's results NaN and those that depend
 * on it (outputs after it; gradients where they go through the state), and no others.
 * kept: NULL, or what rc_delta_backward starts from (rc_delta_kept_bytes);
 * it is written by rc_delta_forward and read by rc_delta_backward of the same
 * sizes.  Both need scratch.
 * Backward: do_ (required), dstate_out (may be NULL: 0) -> dq, dk, dv (dtype),
 * dg (NULL exactly where g is absent) and dbeta (32-bit, contiguous
 * (batch, length, heads)), dstate_in (may be NULL).
 */
typedef struct {
  int32_t dtype;
  int32_t batch, length, key_heads, heads, key, value;
  float scale;
  rc_heads q, k, v, o;
  rc_view g, beta;
  const float* state_in;            /* or NULL: 0 */
  float* state_out;                 /* or NULL */
  const int32_t* lengths;
  float* kept;
  rc_heads do_, dq, dk, dv;
  float* dg;
  float* dbeta;
  const float* dstate_out;
  float* dstate_in;
  void* workspace;
  uint64_t workspace_bytes;
} rc_delta_args;

int rc_delta_forward(const rc_delta_args* args, void* stream);
int rc_delta_backward(const rc_delta_args* args, void* stream);
int rc_delta_kept_bytes(const rc_delta_args* args, uint64_t* bytes_host);
int rc_delta_forward_workspace(const rc_delta_args* args, uint64_t* bytes_host);
int rc_delta_backward_workspace(const rc_delta_args* args, uint64_t* bytes_host);
/* One token: q, k (batch, key_heads, key), v, o (batch, heads, value), g, beta
 * (batch, heads) (time strides are not used); state (num_slots, heads, key,
 * value), contiguous but for its slot stride, is updated in place; slots as
 * rc_conv_step. */
typedef struct {
  int32_t dtype;
  int32_t batch, key_heads, heads, key, value, num_slots;
  float scale;
  rc_heads q, k, v, o;
  rc_view g, beta;
  float* state;
  int64_t state_slot;               /* slot stride of state */
  const int32_t* slots;
} rc_delta_step_args;
int rc_delta_step(const rc_delta_step_args* args, void* stream);

/*
 * Norms of queries and keys, each head on its own, and their rotation by
 * position.  For x of q (heads) and k (key_heads), each `channels` <= 256 wide:
 *   y = x / sqrt(mean(x^2) + eps) * weight     (RC_QK_RMS)
 *   y = x / sqrt(sum(x^2) + eps) * weight      (RC_QK_L2)
 *   y = x weight                               (RC_QK_NONE),
 * then pair i < rotated / 2 of y is turned by the angle position * inv_freq[i]:
 *   (a, b) -> (a cos - b sin, b cos + a sin),
 * channels (i, i + rotated / 2), or (2i, 2i + 1) where interleaved.  Channels
 * from rotated on are not turned.  positions (batch, length), int32, element
 * (b, t) at b * positions_batch + t * positions_time, NULL: t.  Angles are taken in
 * 64 bits.  The weights (may be NULL: 1) are of param_dtype (RC_F32 or dtype),
 * inv_freq [rotated / 2] 32-bit (NULL where rotated is 0).
 * Backward: dq_out and dk_out, each may be absent (0) -> dq, dk, dq_weight,
 * dk_weight (param_dtype; each may be NULL).
 */
enum rc_qk_norm { RC_QK_NONE = 0, RC_QK_RMS = 1, RC_QK_L2 = 2 };
typedef struct {
  int32_t dtype, param_dtype, norm, interleaved;
  int32_t batch, length, heads, key_heads, channels, rotated;
  float eps;
  rc_heads q, k, q_out, k_out;
  const void* q_weight;
  const void* k_weight;
  const float* inv_freq;
  const int32_t* positions;
  int64_t positions_batch, positions_time;
  const int32_t* lengths;
  rc_heads dq_out, dk_out, dq, dk;
  void* dq_weight;
  void* dk_weight;
  void* workspace;
  uint64_t workspace_bytes;
} rc_qk_args;

int rc_qk_forward(const rc_qk_args* args, void* stream);
int rc_qk_backward(const rc_qk_args* args, void* stream);
int rc_qk_backward_workspace(const rc_qk_args* args, uint64_t* bytes_host);

/*
 * Dropout whose mask is never stored: element i of x (in row-major order of
 * rows x width) is kept where word i % 4 of Philox4x32-10 (Salmon, Moraes, Dror and
 * Shaw, 2011) with key seed and counter (i / 4, tag) is not below p 2^32 (rounded to a
 * whole number):
 *   out = residual + (kept ? x / (1 - p) : 0).
 * So forward, backward and a second run of either draw the same mask from the
 * same seed and tag.  0 <= p <= 1 (1 drops everything).  The seed is
 * *seed_device if that is not NULL (read when the kernel runs), else seed.
 * x is of dtype; residual (may be absent) and out of out_dtype (RC_F32 or dtype;
 * dtype without a residual).  Views use their batch strides as row strides.
 * Backward: dx = kept ? dout / (1 - p) : 0.
 */
typedef struct {
  int32_t dtype, out_dtype;
  int64_t rows, width;
  double p;
  int64_t seed, tag;
  const int64_t* seed_device;
  rc_view x, residual, out;         /* backward: dout as out, dx as x */
} rc_dropout_args;

int rc_dropout_forward(const rc_dropout_args* args, void* stream);
int rc_dropout_backward(const rc_dropout_args* args, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RC_OPS_H */
