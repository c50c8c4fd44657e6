// Selective state space scan, its gradients, and its form for one token.
//
// Channel d has N states, delta = softplus(dt + bias) (or dt + bias):
//   a_n = exp(delta A_n),  h_n <- a_n h_n + delta u B_n,  y = sum_n h_n C_n + D u,
//   out = y z sigmoid(z).
// Backwards in time, with dy = dout z sigmoid(z) and g_n the gradient of the
// state after the token:
//   g_n = C_n dy + (a_n g_n of the next token),  dC_n = sum_d dy h_n,  dB_n = sum_d g_n delta u,
//   du = delta sum_n g_n B_n + D dy,  dA_n = sum g_n a_n h_n(before) delta,
//   ddelta = u sum_n g_n B_n + sum_n g_n a_n h_n(before) A_n.
//
// Four states are one lane's, Q = 1, 2, 4, 8 or 16 neighbouring lanes are a
// channel's (N <= 4 Q; missing states have A = B = C = 0), so sums over a
// channel's states are Q-lane sums and sums over channels are strided ones.
// A token past its sequence's end is a step with delta = u = dy = B = C = 0:
// the state stays, every product is 0.
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 16;           // tokens between two kept states

__device__ __forceinline__ int seq_end(const int32_t* lengths, int64_t b, int32_t length) {
  if (!lengths) return length;
  return min(max(lengths[b], 0), length);
}

// Sum over the Q lanes of a channel, in each of them.
template <int Q>
__device__ __forceinline__ float state_sum(float x) {
#pragma unroll
  for (int m = 1; m < Q; m *= 2) x += __shfl_xor(x, m);
  return x;
}
// Sum over the channels of a wave, lanes of equal q apart.
template <int Q>
__device__ __forceinline__ float channel_sum(float x) {
#pragma unroll
  for (int m = Q; m < 64; m *= 2) x += __shfl_xor(x, m);
  return x;
}

struct ScanPlan {
  int Q;
  int64_t group_width;      // channels of a group
  int64_t blocks;           // workgroups of a group's channels
  int64_t tiles;
};

struct ScanParams {
  rc_scan_args a;
  int32_t group_width, blocks, tiles, parts;
  float* part_bc;           // backward: [parts][batch][length][groups][2][4 Q]
  float* part_a;            // [batch][width][4 Q]
  float* part_d;            // [batch][width][2]: D, dt_bias
};

// A workgroup's sequence, group and channel; a wave's slot among those that
// share B and C.
template <int Q>
struct Place {
  int64_t b, g, d;
  int q, part;
  bool on;
  __device__ Place(const ScanParams& p) {
    int64_t i = blockIdx.x;
    const int64_t blk = i % p.blocks;
    i /= p.blocks;
    g = i % p.a.groups;
    b = i / p.a.groups;
    q = threadIdx.x % Q;
    const int64_t ch = blk * (kThreads / Q) + threadIdx.x / Q;
    on = ch < p.group_width;
    d = g * p.group_width + (on ? ch : 0);
    part = (int)(blk * (kThreads / 64) + threadIdx.x / 64);
  }
};

template <class T>
__device__ __forceinline__ const T* row(const rc_view& v, int64_t b, int64_t t) {
  return static_cast<const T*>(v.data) + b * v.batch + t * v.time;
}
template <class T>
__device__ __forceinline__ T* row_out(const rc_view& v, int64_t b, int64_t t) {
  return static_cast<T*>(v.data) + b * v.batch + t * v.time;
}

// The four states 4 q .. 4 q + 3 of B or C at one token.
template <class T>
__device__ __forceinline__ void load_states(const T* p, int q, int n, float (&x)[4]) {
  load_vec<4>(p + 4 * q, max(0, min(4, n - 4 * q)), x);
}

// delta of a token and its slope ddelta / ddt.
__device__ __forceinline__ float delta_of(float raw, bool soft) {
  return soft ? softplus(raw) : raw;
}

template <class T, int Q>
__global__ __launch_bounds__(kThreads) void k_scan_forward(ScanParams p) {
  const rc_scan_args& a = p.a;
  const Place<Q> w(p);
  if (!w.on) return;
  const int end = seq_end(a.lengths, w.b, a.length);
  const int ns = max(0, min(4, a.states - 4 * w.q));
  const int64_t at = (w.b * a.width + w.d) * a.states + 4 * w.q;
  float A[4], h[4];
  load_vec<4>(a.A + w.d * a.states + 4 * w.q, ns, A);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    A[i] *= kLog2e;
    h[i] = 0.f;
  }
  if (a.state_in) load_vec<4>(a.state_in + at, ns, h);
  const float D = a.D ? a.D[w.d] : 0.f, bias = a.dt_bias ? a.dt_bias[w.d] : 0.f;
  for (int t = 0; t < a.length; t++) {
    if (a.kept && t % kTile == 0)
      store_vec<4>(a.kept + ((w.b * p.tiles + t / kTile) * a.width + w.d) * (4 * Q) + 4 * w.q, 4,
                   h);
    float y = 0.f;
    if (t < end) {
      float B[4], C[4];
      load_states(row<T>(a.B, w.b, t) + w.g * a.B_group, w.q, a.states, B);
      load_states(row<T>(a.C, w.b, t) + w.g * a.C_group, w.q, a.states, C);
      const float u = (float)row<T>(a.u, w.b, t)[w.d];
      const float delta = delta_of((float)row<T>(a.dt, w.b, t)[w.d] + bias, a.softplus);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        h[i] = fmaf(fast_exp2(delta * A[i]), h[i], delta * u * B[i]);
        y = fmaf(h[i], C[i], y);
      }
      y = fmaf(D, u, state_sum<Q>(y));
      if (a.z.data) {
        const float z = (float)row<T>(a.z, w.b, t)[w.d];
        y *= z * sigmoid(z);
      }
    }
    if (w.q == 0) row_out<T>(a.y, w.b, t)[w.d] = (T)y;
  }
  if (a.state_out) store_vec<4>(a.state_out + at, ns, h);
}

template <class T, int Q>
__global__ __launch_bounds__(kThreads) void k_scan_backward(ScanParams p) {
  const rc_scan_args& a = p.a;
  const Place<Q> w(p);
  const int end = seq_end(a.lengths, w.b, a.length);
  const int ns = w.on ? max(0, min(4, a.states - 4 * w.q)) : 0;
  const int64_t at = (w.b * a.width + w.d) * a.states + 4 * w.q;
  float A[4], g[4], dA[4];          // g: gradient of the state before the later token
  load_vec<4>(a.A + w.d * a.states + 4 * w.q, ns, A);
#pragma unroll
  for (int i = 0; i < 4; i++) g[i] = dA[i] = 0.f;
  if (a.dstate_out) load_vec<4>(a.dstate_out + at, ns, g);
  const float D = a.D ? a.D[w.d] : 0.f, bias = a.dt_bias ? a.dt_bias[w.d] : 0.f;
  float dD = 0.f, dbias = 0.f;
  for (int tile = p.tiles - 1; tile >= 0; tile--) {
    const int t0 = tile * kTile;
    float h0[4], h[kTile][4];
    load_vec<4>(a.kept + ((w.b * p.tiles + tile) * a.width + w.d) * (4 * Q) + 4 * w.q, 4, h0);
#pragma unroll
    for (int j = 0; j < kTile; j++) {
      const int t = t0 + j;
      float B[4] = {0.f, 0.f, 0.f, 0.f}, u = 0.f, delta = 0.f;
      if (t < end) {
        load_states(row<T>(a.B, w.b, t) + w.g * a.B_group, w.q, a.states, B);
        u = (float)row<T>(a.u, w.b, t)[w.d];
        delta = delta_of((float)row<T>(a.dt, w.b, t)[w.d] + bias, a.softplus);
      }
#pragma unroll
      for (int i = 0; i < 4; i++)
        h[j][i] = fmaf(fast_exp2(delta * A[i] * kLog2e), j ? h[j ? j - 1 : 0][i] : h0[i],
                       delta * u * B[i]);
    }
#pragma unroll
    for (int j = kTile - 1; j >= 0; j--) {
      const int t = t0 + j;
      if (t >= a.length) continue;
      float B[4] = {0.f, 0.f, 0.f, 0.f}, C[4] = {0.f, 0.f, 0.f, 0.f};
      float u = 0.f, raw = 0.f, delta = 0.f, z = 0.f, dout = 0.f;
      const bool live = t < end && w.on;
      if (live) {
        load_states(row<T>(a.B, w.b, t) + w.g * a.B_group, w.q, a.states, B);
        load_states(row<T>(a.C, w.b, t) + w.g * a.C_group, w.q, a.states, C);
        u = (float)row<T>(a.u, w.b, t)[w.d];
        raw = (float)row<T>(a.dt, w.b, t)[w.d] + bias;
        delta = delta_of(raw, a.softplus);
        dout = (float)row<T>(a.dy, w.b, t)[w.d];
        if (a.z.data) z = (float)row<T>(a.z, w.b, t)[w.d];
      }
      const float s = sigmoid(z), dy = a.z.data ? dout * (z * s) : dout;
      float y = 0.f, through = 0.f, dd = 0.f, dB[4], dC[4];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float before = j ? h[j ? j - 1 : 0][i] : h0[i];
        y = fmaf(h[j][i], C[i], y);
        const float gi = fmaf(C[i], dy, g[i]);
        dC[i] = dy * h[j][i];
        dB[i] = gi * (delta * u);
        through = fmaf(gi, B[i], through);
        g[i] = fast_exp2(delta * A[i] * kLog2e) * gi;
        const float via = g[i] * before;
        dA[i] = fmaf(via, delta, dA[i]);
        dd = fmaf(via, A[i], dd);
      }
      y = fmaf(D, u, state_sum<Q>(y));
      through = state_sum<Q>(through);
      dd = fmaf(u, through, state_sum<Q>(dd));
      const float draw = live ? (a.softplus ? dd * sigmoid(raw) : dd) : 0.f;
      dD = fmaf(dy, u, dD);
      dbias += draw;
      if (w.on && w.q == 0) {
        row_out<T>(a.du, w.b, t)[w.d] = (T)fmaf(delta, through, D * dy);
        row_out<T>(a.ddt, w.b, t)[w.d] = (T)draw;
        if (a.z.data)
          row_out<T>(a.dz, w.b, t)[w.d] = (T)(dout * y * (s * (1.f + z * (1.f - s))));
      }
      float* out = p.part_bc +
                   (((w.part * (int64_t)a.batch + w.b) * a.length + t) * a.groups + w.g) * (8 * Q);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        dB[i] = channel_sum<Q>(dB[i]);
        dC[i] = channel_sum<Q>(dC[i]);
      }
      if (threadIdx.x % 64 < Q) {
        store_vec<4>(out + 4 * w.q, 4, dB);
        store_vec<4>(out + 4 * Q + 4 * w.q, 4, dC);
      }
    }
  }
  if (!w.on) return;
  if (a.dstate_in) store_vec<4>(a.dstate_in + at, ns, g);
  store_vec<4>(p.part_a + (w.b * a.width + w.d) * (4 * Q) + 4 * w.q, 4, dA);
  if (w.q == 0) {
    p.part_d[(w.b * a.width + w.d) * 2] = dD;
    p.part_d[(w.b * a.width + w.d) * 2 + 1] = dbias;
  }
}

// dB and dC from the waves' parts: one thread per (batch, token, group, state).
template <class T>
__global__ __launch_bounds__(256) void k_scan_sum_bc(const float* in, int64_t parts, int64_t cells,
                                                     int32_t padded, int32_t states, T* dB, T* dC) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t cell = id / (2 * padded);
  const int k = (int)(id % (2 * padded)), n = k % padded;
  if (cell >= cells || n >= states) return;
  float s = 0.f;
  for (int64_t j = 0; j < parts; j++) s += in[(j * cells + cell) * (2 * padded) + k];
  (k < padded ? dB : dC)[cell * states + n] = (T)s;
}

// dA, dD and ddt_bias from the sequences' parts.
__global__ __launch_bounds__(256) void k_scan_sum_a(const float* pa, const float* pd,
                                                    int64_t parts, int32_t width, int32_t padded,
                                                    int32_t states, float* dA, float* dD,
                                                    float* dbias) {
  __shared__ float lds[256];
  const int64_t ca = (int64_t)width * padded, cd = (int64_t)width * 2;
  const int64_t na = cdiv(ca, kSumCols);
  if (blockIdx.x < na) {
    const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x % kSumCols;
    const float s = column_sum(pa, parts, ca, c, lds);
    if (threadIdx.x < kSumCols && c < ca && c % padded < states)
      dA[c / padded * states + c % padded] = s;
  } else {
    const int64_t c = (int64_t)(blockIdx.x - na) * kSumCols + threadIdx.x % kSumCols;
    const float s = column_sum(pd, parts, cd, c, lds);
    float* out = c % 2 ? dbias : dD;
    if (threadIdx.x < kSumCols && c < cd && out) out[c / 2] = s;
  }
}

template <class T, int Q>
__global__ __launch_bounds__(kThreads) void k_scan_step(rc_scan_step_args a, int32_t blocks) {
  const int64_t b = blockIdx.x / blocks;
  const int64_t d = (int64_t)(blockIdx.x % blocks) * (kThreads / Q) + threadIdx.x / Q;
  const int q = threadIdx.x % Q;
  if (d >= a.width) return;
  const int64_t slot = a.slots ? a.slots[b] : b;
  float y = 0.f;
  if (slot >= 0 && slot < a.num_slots) {
    const int64_t g = d / (a.width / a.groups);
    const int ns = max(0, min(4, a.states - 4 * q));
    float A[4], B[4], C[4], h[4];
    float* state = a.state + slot * a.state_slot + d * a.states + 4 * q;
    load_vec<4>(state, ns, h);
    load_vec<4>(a.A + d * a.states + 4 * q, ns, A);
    load_vec<4>(row<T>(a.B, b, 0) + g * a.B_group + 4 * q, ns, B);
    load_vec<4>(row<T>(a.C, b, 0) + g * a.C_group + 4 * q, ns, C);
    const float u = (float)row<T>(a.u, b, 0)[d];
    const float z = a.z.data ? (float)row<T>(a.z, b, 0)[d] : 0.f;
    const float delta =
        delta_of((float)row<T>(a.dt, b, 0)[d] + (a.dt_bias ? a.dt_bias[d] : 0.f), a.softplus);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      h[i] = fmaf(fast_exp2(delta * A[i] * kLog2e), h[i], delta * u * B[i]);
      y = fmaf(h[i], C[i], y);
    }
    store_vec<4>(state, ns, h);
    y = fmaf(a.D ? a.D[d] : 0.f, u, state_sum<Q>(y));
    if (a.z.data) y *= z * sigmoid(z);
  }
  if (q == 0) row_out<T>(a.y, b, 0)[d] = (T)y;
}

int lanes_of(int32_t states) {
  int q = 1;
  while (4 * q < states) q *= 2;
  return q;
}

template <class F>
int by_lanes(int q, F&& f) {
  switch (q) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

bool scan_sizes_ok(int32_t dtype, int32_t batch, int32_t length, int32_t width, int32_t states,
                   int32_t groups) {
  return dtype_ok(dtype) && batch >= 0 && length >= 0 && width >= 0 && states >= 1 &&
         states <= 64 && groups >= 1 && width % groups == 0;
}
bool scan_sizes_ok(const rc_scan_args* a) {
  return a && scan_sizes_ok(a->dtype, a->batch, a->length, a->width, a->states, a->groups);
}

ScanPlan scan_plan(const rc_scan_args& a) {
  ScanPlan p;
  p.Q = lanes_of(a.states);
  p.group_width = a.width / a.groups;
  p.blocks = cdiv(p.group_width, kThreads / p.Q);
  p.tiles = cdiv(a.length, kTile);
  return p;
}

struct ScanScratch {
  uint64_t bc, a, d;
};
ScanScratch scan_scratch(const rc_scan_args& a, const ScanPlan& p) {
  const uint64_t rows = (uint64_t)a.batch * a.width;
  return {(uint64_t)p.blocks * (kThreads / 64) * a.batch * a.length * a.groups * 8 * p.Q * 4,
          rows * 4 * p.Q * 4, rows * 2 * 4};
}

int scan_check(const rc_scan_args* a, bool backward) {
  if (!scan_sizes_ok(a)) return RC_E_ARG;
  if (a->batch > 0 && a->width > 0) {
    if (!a->A) return RC_E_ARG;
    if (a->length > 0) {
      if (!a->u.data || !a->dt.data || !a->B.data || !a->C.data) return RC_E_ARG;
      if (!backward && !a->y.data) return RC_E_ARG;
      if (backward && (!a->dy.data || !a->du.data || !a->ddt.data || !a->dB || !a->dC ||
                       !a->kept || (a->z.data == nullptr) != (a->dz.data == nullptr)))
        return RC_E_ARG;
    }
  }
  if (backward && a->width > 0 &&
      (!a->dA || (a->D && !a->dD) || (a->dt_bias && !a->ddt_bias)))
    return RC_E_ARG;
  const ScanPlan p = scan_plan(*a);
  const int64_t cells = (int64_t)a->batch * a->length * a->groups;
  if (p.blocks * a->groups * a->batch >= kMaxBlocks || cdiv(cells * 8 * p.Q, 256) >= kMaxBlocks)
    return RC_E_OVERFLOW;
  return RC_OK;
}

ScanParams scan_params(const rc_scan_args& a, const ScanPlan& p) {
  ScanParams q = {};
  q.a = a;
  q.group_width = (int32_t)p.group_width;
  q.blocks = (int32_t)p.blocks;
  q.tiles = (int32_t)p.tiles;
  q.parts = (int32_t)p.blocks * (kThreads / 64);
  return q;
}

}  // namespace

extern "C" int rc_scan_kept_bytes(const rc_scan_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !scan_sizes_ok(a)) return RC_E_ARG;
  const ScanPlan p = scan_plan(*a);
  *bytes_host = (uint64_t)a->batch * p.tiles * a->width * 4 * p.Q * 4;
  return RC_OK;
}

extern "C" int rc_scan_forward_workspace(const rc_scan_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !scan_sizes_ok(a)) return RC_E_ARG;
  *bytes_host = 0;
  return RC_OK;
}

extern "C" int rc_scan_backward_workspace(const rc_scan_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !scan_sizes_ok(a)) return RC_E_ARG;
  const ScanScratch s = scan_scratch(*a, scan_plan(*a));
  *bytes_host = s.bc + s.a + s.d;
  return RC_OK;
}

extern "C" int rc_scan_forward(const rc_scan_args* args, void* stream) {
  if (const int st = scan_check(args, false)) return st;
  const rc_scan_args& a = *args;
  const ScanPlan p = scan_plan(a);
  const int64_t blocks = p.blocks * a.groups * a.batch;
  if (blocks == 0) return RC_OK;
  return by_dtype(a.dtype, [&](auto t) {
    return by_lanes(p.Q, [&](auto q) {
      k_scan_forward<decltype(t), q()><<<dim3((uint32_t)blocks), kThreads, 0,
                                         (hipStream_t)stream>>>(scan_params(a, p));
      return launched("k_scan_forward");
    });
  });
}

extern "C" int rc_scan_backward(const rc_scan_args* args, void* stream) {
  if (const int st = scan_check(args, true)) return st;
  const rc_scan_args& a = *args;
  const ScanPlan p = scan_plan(a);
  const ScanScratch need = scan_scratch(a, p);
  const uint64_t total = need.bc + need.a + need.d;
  if (total > 0 && (!a.workspace || a.workspace_bytes < total)) return RC_E_SCRATCH;
  if (a.width == 0) return RC_OK;
  ScanParams q = scan_params(a, p);
  char* ws = static_cast<char*>(a.workspace);
  q.part_bc = reinterpret_cast<float*>(ws);
  q.part_a = reinterpret_cast<float*>(ws + need.bc);
  q.part_d = reinterpret_cast<float*>(ws + need.bc + need.a);
  const hipStream_t s = (hipStream_t)stream;
  const int64_t blocks = p.blocks * a.groups * a.batch;
  const int64_t cells = (int64_t)a.batch * a.length * a.groups;
  return by_dtype(a.dtype, [&](auto t) -> int {
    using T = decltype(t);
    if (blocks > 0) {
      const int st = by_lanes(p.Q, [&](auto lanes) {
        k_scan_backward<T, lanes()><<<dim3((uint32_t)blocks), kThreads, 0, s>>>(q);
        return launched("k_scan_backward");
      });
      if (st) return st;
    }
    if (cells > 0) {
      k_scan_sum_bc<T><<<dim3((uint32_t)cdiv(cells * 8 * p.Q, 256)), 256, 0, s>>>(
          q.part_bc, q.parts, cells, 4 * p.Q, a.states, static_cast<T*>(a.dB),
          static_cast<T*>(a.dC));
      if (const int st = launched("k_scan_sum_bc")) return st;
    }
    const int64_t cols = (int64_t)a.width * 4 * p.Q;
    k_scan_sum_a<<<dim3((uint32_t)(cdiv(cols, kSumCols) + cdiv(2 * (int64_t)a.width, kSumCols))),
                   256, 0, s>>>(q.part_a, q.part_d, a.batch, a.width, 4 * p.Q, a.states, a.dA,
                                a.dD, a.ddt_bias);
    return launched("k_scan_sum_a");
  });
}

extern "C" int rc_scan_step(const rc_scan_step_args* args, void* stream) {
  if (!args) return RC_E_ARG;
  const rc_scan_step_args& a = *args;
  if (!scan_sizes_ok(a.dtype, a.batch, 1, a.width, a.states, a.groups) || a.num_slots < 0 ||
      (!a.slots && a.num_slots < a.batch))
    return RC_E_ARG;
  if (a.batch == 0 || a.width == 0) return RC_OK;
  if (!a.u.data || !a.dt.data || !a.B.data || !a.C.data || !a.y.data || !a.A || !a.state)
    return RC_E_ARG;
  const int Q = lanes_of(a.states);
  const int64_t blocks = cdiv(a.width, kThreads / Q);
  if (blocks * a.batch >= kMaxBlocks) return RC_E_OVERFLOW;
  return by_dtype(a.dtype, [&](auto t) {
    return by_lanes(Q, [&](auto q) {
      k_scan_step<decltype(t), q()><<<dim3((uint32_t)(blocks * a.batch)), kThreads, 0,
                                      (hipStream_t)stream>>>(a, (int32_t)blocks);
      return launched("k_scan_step");
    });
  });
}
