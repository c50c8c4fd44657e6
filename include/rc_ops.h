/*
 * rc_ops.h -- C ABI of the sequence-model operators of the MI355X library:
 * the short causal convolution, the selective state space scan, and the norms
 * before and after a block fused with its gate and residual scale.
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

#ifdef __cplusplus
}
#endif

#endif /* RC_OPS_H */
