// Short causal convolution over time, every channel on its own, with bias and
// SiLU: p_t = bias + sum_k w_k x_{t-(K-1)+k}, y_t = p_t sigmoid(p_t); its
// gradients; its form for one token.
//
// Each value is used K times and each output needs ~2K + 6 operations for 4
// bytes moved (16-bit types), so the bound is memory.  A thread owns V
// neighbouring channels (one wide load per row) and a run of rows, and keeps
// the last K - 1 rows in registers: x is read once plus K - 1 rows per run
// (backward 2 K - 2, and K - 1 of dy).
// Where V does not divide the width, the last thread of a row moves back to
// the last V channels; it and its neighbour store the same values where they
// overlap.  (Odd widths with V = 1 instead: 8 x 2047 x 2049 in bfloat16
// forward 43, backward 71 us, this way 33 and 59; in 32 bits 64 and 112, this way 72 and 94.)
//
// Backward: dp_t = dy_t act'(p_t) (p_t again from x), dx_t = sum_k w_k
// dp_{t+K-1-k}, dw_k = sum_t dp_t x_{t-(K-1)+k}, dbias = sum_t dp_t.  The same walk,
// K - 1 rows past the run's end to have every dp that its dx needs; the
// weight gradients stay in registers, are summed over a workgroup's runs in
// LDS, and over workgroups by a second kernel, always in the same order.
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int kThreads = 256;

// Vector lanes of a workgroup along the channels (the rest are runs of rows).
inline int lanes_for(int64_t vecs) {
  int n = 8;
  while (n < 64 && n < vecs) n *= 2;
  return n;
}

template <class T>
struct ConvParams {
  rc_conv_args a;
  int32_t lanes;       // threads of a workgroup along the channels
  int32_t run;         // rows of a thread
  int32_t runs;        // runs of a sequence
  int32_t groups_c;    // workgroups along the channels
  float* partial;      // backward: [workgroups along time][width][K + 1]
};

__device__ __forceinline__ int seq_end(const int32_t* lengths, int32_t b, int32_t length) {
  if (!lengths) return length;
  return min(max(lengths[b], 0), length);
}

template <class T>
__device__ __forceinline__ T* at(const rc_view& v, int64_t b, int64_t t, int64_t c) {
  return static_cast<T*>(v.data) + b * v.batch + t * v.time + c;
}

// V elements at p where `ok`, else zeros.  p is readable either way: the load
// is unconditional and the choice is made on its result.  (A load in a branch whose
// result a loop hands on loses elements of 32-bit vectors: the compiler of
// ROCm 7.2 drops copies of the loaded tuple's middle registers.)
template <class T, int V>
__device__ __forceinline__ void load_if(const T* p, bool ok, float (&x)[V]) {
  load_vec<V>(p, V, x);
#pragma unroll
  for (int i = 0; i < V; i++) x[i] = ok ? x[i] : 0.f;
}

// Row t of the input before a run (t < 0: the state) of a sequence that has a
// token; 0 at and past `end`.
template <class T, int K, int V>
__device__ __forceinline__ void input_row(const rc_conv_args& a, int b, int t, int end, int c,
                                          float (&x)[V]) {
  const bool state = t < 0 && a.state_in.data;
  const T* p = state ? at<T>(a.state_in, b, t + K - 1, c)
                     : at<T>(a.x, b, max(0, min(t, end - 1)), c);
  load_if<T, V>(p, t < 0 ? state : t < end, x);
}

// Rows of a thread that are loaded together, one group ahead of their use: rows t ..,
// those from `stop` > 0 on row stop - 1 again, so that a walk reads no row past its last.
constexpr int kRows = 4;
template <class T, int V>
struct Rows {
  typedef T Raw __attribute__((ext_vector_type(V)));
  Raw x[kRows];
  __device__ __forceinline__ void load(const rc_view& v, int b, int t, int stop, int c) {
#pragma unroll
    for (int j = 0; j < kRows; j++)
      __builtin_memcpy(&x[j], at<T>(v, b, min(t + j, stop - 1), c), sizeof(Raw));
  }
};

template <class T, int K, int V>
__device__ __forceinline__ void load_weights(const rc_conv_args& a, int c,
                                             float (&w)[K][V], float (&bias)[V]) {
  // the weights of V channels lie together: wide loads
  const auto read = [&](auto type) {
    using P = decltype(type);
    const P *pw = static_cast<const P*>(a.weight) + (int64_t)c * K;
    const P* pb = static_cast<const P*>(a.bias) + c;
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
      for (int k = 0; k < K; k++) w[k][i] = (float)pw[i * K + k];
      bias[i] = a.bias ? (float)pb[i] : 0.f;
    }
  };
  if (a.param_dtype == RC_F32)
    read(float{});
  else
    read(T{});
}

// Forward: V = 8, kRows rows of loads in flight ahead of their use, no LDS.
// At 2 x 4096 x 4096, K = 4 in bfloat16 (134 MB): 27.5 us, 4.9 TB/s, a large copy's rate; in 32 bits
// (268 MB) 61 us, 4.4 TB/s; 8 taps at 8 x 2048 x 2048 42 us (3.2 TB/s), 4 taps 34: the multiply-adds
// show.
template <class T, int K, int V>
__global__ __launch_bounds__(kThreads) void k_conv_forward(ConvParams<T> p) {
  const rc_conv_args& a = p.a;
  const int lane = threadIdx.x % p.lanes, slot = threadIdx.x / p.lanes;
  const int64_t gc = blockIdx.x % p.groups_c, gt = blockIdx.x / p.groups_c;
  const int64_t cell = gt * (kThreads / p.lanes) + slot;          // (batch, run)
  const int64_t c64 = (gc * p.lanes + lane) * V;
  if (c64 >= a.width || cell >= (int64_t)a.batch * p.runs) return;
  const int c = min((int)c64, a.width - V);
  const int b = (int)(cell / p.runs), t0 = (int)(cell % p.runs) * p.run;
  const int t1 = min(t0 + p.run, a.length), end = seq_end(a.lengths, b, a.length);
  if (t0 == 0 && a.state_out.data) {
#pragma unroll
    for (int k = 0; k < K - 1; k++) {
      const int t = end - (K - 1) + k;
      float s[V];
#pragma unroll
      for (int i = 0; i < V; i++) s[i] = 0.f;
      if (t >= 0)
        load_vec<V>(at<T>(a.x, b, t, c), V, s);
      else if (a.state_in.data)
        load_vec<V>(at<T>(a.state_in, b, t + K - 1, c), V, s);
      store_vec<V>(at<T>(a.state_out, b, k, c), V, s);
    }
  }
  int t = t0;
  if (t0 < end) {
    float w[K][V], bias[V], x[K][V];
    load_weights<T, K, V>(a, c, w, bias);
#pragma unroll
    for (int k = 0; k < K - 1; k++) input_row<T, K, V>(a, b, t0 - (K - 1) + k, end, c, x[k + 1]);
    const int stop = min(t1, end);
    Rows<T, V> now, next;
    now.load(a.x, b, t, stop, c);
    for (; t < stop; t += kRows) {
      next.load(a.x, b, t + kRows, stop, c);
#pragma unroll
      for (int j = 0; j < kRows; j++) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
#pragma unroll
          for (int k = 0; k < K - 1; k++) x[k][i] = x[k + 1][i];
          x[K - 1][i] = (float)now.x[j][i];
          y[i] = bias[i];
#pragma unroll
          for (int k = 0; k < K; k++) y[i] = fmaf(w[k][i], x[k][i], y[i]);
          if (a.activation == RC_ACT_SILU) y[i] *= sigmoid(y[i]);
        }
        if (t + j < stop) store_vec<V>(at<T>(a.y, b, t + j, c), V, y);
      }
      now = next;
    }
    t = stop;
  }
  for (; t < t1; t++) {
    const float zero[V] = {};
    store_vec<V>(at<T>(a.y, b, t, c), V, zero);
  }
}

// Backward: V = 4, since a thread holds K rows of x, of dp and the weights'
// gradients of its channels.  Two waves a SIMD, as many as the registers of 8 taps in 32 bits leave;
// four for 16-bit types up to 4 taps, which spill a few registers (above, many).  8 x 2047 x 2048,
// 4 taps: bfloat16 (201 MB) 46 us, 4.4 TB/s, with two waves 49; half of it past the sequences' ends 45 us, with
// two 37; 2049 channels 59 and 57.  32 bits (402 MB) 83 us, 4.8 TB/s.  8 taps 72 and 93 us.
template <class T>
constexpr int conv_waves(int taps) {
  return taps <= 4 && sizeof(T) == 2 ? 4 : 2;
}
template <class T, int K, int V>
__global__ __launch_bounds__(kThreads, conv_waves<T>(K)) void k_conv_backward(ConvParams<T> p) {
  __shared__ float lds[kThreads * V];
  const rc_conv_args& a = p.a;
  const int lane = threadIdx.x % p.lanes, slot = threadIdx.x / p.lanes;
  const int slots = kThreads / p.lanes;
  const int64_t gc = blockIdx.x % p.groups_c, gt = blockIdx.x / p.groups_c;
  const int64_t cell = gt * slots + slot;
  const int64_t c64 = (gc * p.lanes + lane) * V;
  // channels that the load moves back by
  const int over = (int)(c64 < a.width ? max((int64_t)0, c64 + V - a.width) : 0);
  float dw[K + 1][V];                                  // the last one: bias
#pragma unroll
  for (int k = 0; k <= K; k++)
#pragma unroll
    for (int i = 0; i < V; i++) dw[k][i] = 0.f;
  if (c64 < a.width && cell < (int64_t)a.batch * p.runs) {
    const int c = min((int)c64, a.width - V);
    const int b = (int)(cell / p.runs), t0 = (int)(cell % p.runs) * p.run;
    const int t1 = min(t0 + p.run, a.length), end = seq_end(a.lengths, b, a.length);
    if (t0 >= end) {                                   // past the end: zeros, no gradients
      const float zero[V] = {};
      for (int t = t0; t < t1; t++) store_vec<V>(at<T>(a.dx, b, t, c), V, zero);
      if (t0 == 0 && a.dstate_in.data) {               // no token: the state's gradient is handed on
#pragma unroll
        for (int k = 0; k < K - 1; k++) {
          float ds[V] = {};
          if (a.dstate_out.data) load_vec<V>(at<T>(a.dstate_out, b, k, c), V, ds);
          store_vec<V>(at<T>(a.dstate_in, b, k, c), V, ds);
        }
      }
    } else {
      // row t finishes dx of row t - (K - 1); the first run also writes the
      // state's rows -(K - 1) .. -1
      const int first = t0 == 0 && a.dstate_in.data ? -(K - 1) : t0;
      float w[K][V], bias[V], x[K][V], dp[K][V];       // dp[j]: of row t - (K - 1) + j
      load_weights<T, K, V>(a, c, w, bias);
#pragma unroll
      for (int k = 0; k < K; k++)
#pragma unroll
        for (int i = 0; i < V; i++) dp[k][i] = x[k][i] = 0.f;
#pragma unroll
      for (int k = 0; k < K - 1; k++) input_row<T, K, V>(a, b, t0 - (K - 1) + k, end, c, x[k + 1]);
      Rows<T, V> now, next, dnow, dnext;
      const int stop = min(t1 + K - 1, end);
      now.load(a.x, b, t0, stop, c);
      dnow.load(a.dy, b, t0, stop, c);
      for (int g = t0; g < t1 + K - 1; g += kRows) {
        next.load(a.x, b, g + kRows, stop, c);
        dnext.load(a.dy, b, g + kRows, stop, c);
#pragma unroll
        for (int r = 0; r < kRows; r++) {
          const int t = g + r;
#pragma unroll
          for (int i = 0; i < V; i++) {
#pragma unroll
            for (int k = 0; k < K - 1; k++) {
              x[k][i] = x[k + 1][i];
              dp[k][i] = dp[k + 1][i];
            }
            x[K - 1][i] = t < end ? (float)now.x[r][i] : 0.f;
            float d = (float)dnow.x[r][i];
            if (a.activation == RC_ACT_SILU) {
              float q = bias[i];
#pragma unroll
              for (int k = 0; k < K; k++) q = fmaf(w[k][i], x[k][i], q);
              const float s = sigmoid(q);
              d *= s * (1.f + q * (1.f - s));
            }
            // chosen last: past the end q may come from tokens that are not finite
            dp[K - 1][i] = t < end ? d : 0.f;
            const float own = t < t1 ? dp[K - 1][i] : 0.f;
#pragma unroll
            for (int k = 0; k < K; k++) dw[k][i] = fmaf(own, x[k][i], dw[k][i]);
            dw[K][i] += own;
          }
          const int s = t - (K - 1);                     // the row whose dx is complete
          if (s >= first && s < t1) {
            float dx[V];
#pragma unroll
            for (int i = 0; i < V; i++) {
              dx[i] = 0.f;
#pragma unroll
              for (int k = 0; k < K; k++) dx[i] = fmaf(w[k][i], dp[K - 1 - k][i], dx[i]);
            }
            const int j = s - (end - (K - 1));           // its row in the final state
            if (a.dstate_out.data && j >= 0 && j < K - 1) {
              float ds[V];
              load_vec<V>(at<T>(a.dstate_out, b, j, c), V, ds);
#pragma unroll
              for (int i = 0; i < V; i++) dx[i] += ds[i];
            }
            if (s >= 0)
              store_vec<V>(at<T>(a.dx, b, s, c), V, dx);
            else
              store_vec<V>(at<T>(a.dstate_in, b, s + K - 1, c), V, dx);
          }
        }
        now = next;
        dnow = dnext;
      }
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int k = 0; k <= K; k++) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; i++)                        // a moved load's own channels only
      if (i >= over) lds[threadIdx.x * V + i - over] = dw[k][i];
    __syncthreads();
    for (int o = threadIdx.x; o < p.lanes * V; o += kThreads) {
      const int64_t ch = gc * p.lanes * V + o;
      float s = 0.f;
      for (int j = 0; j < slots; j++) s += lds[j * p.lanes * V + o];
      if (ch < a.width) p.partial[(gt * a.width + ch) * (K + 1) + k] = s;
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_conv_weight_sum(const float* in, int64_t parts,
                                                         int32_t width, int32_t taps, void* dw,
                                                         void* db, int32_t f32) {
  __shared__ float lds[256];
  const int64_t cols = (int64_t)width * (taps + 1);
  const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x % kSumCols;
  const float s = column_sum(in, parts, cols, c, lds);
  if (threadIdx.x >= kSumCols || c >= cols) return;
  const int64_t ch = c / (taps + 1), k = c % (taps + 1);
  if (k < taps) {
    if (dw) store_param<T>(dw, ch * taps + k, f32, s);
  } else if (db) {
    store_param<T>(db, ch, f32, s);
  }
}

// One token: y from the slot's K - 1 rows and x, the rows move up by one.  V = 2 channels
// a thread, or 1: many small threads, since a row of channels is all the work
// there is.  Bound by the launch: 48 rows of 2048 channels (1 MB) 5 us a call.
template <class T, int K, int V>
__global__ __launch_bounds__(kThreads) void k_conv_step(rc_conv_step_args a, int32_t vecs) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t b = id / vecs;
  if (b >= a.batch) return;
  const int c = (int)(id % vecs) * V;
  const int64_t slot = a.slots ? a.slots[b] : b;
  float y[V];
  if (slot < 0 || slot >= a.num_slots) {
#pragma unroll
    for (int i = 0; i < V; i++) y[i] = 0.f;
  } else {
    const bool f32 = a.param_dtype == RC_F32;
    float x[K][V];
    T* s = static_cast<T*>(a.state.data) + slot * a.state.batch + c;
#pragma unroll
    for (int k = 0; k < K - 1; k++) load_vec<V>(s + k * a.state.time, V, x[k]);
    load_vec<V>(at<T>(a.x, b, 0, c), V, x[K - 1]);
#pragma unroll
    for (int i = 0; i < V; i++) {
      y[i] = a.bias ? load_param<T>(a.bias, c + i, f32) : 0.f;
#pragma unroll
      for (int k = 0; k < K; k++)
        y[i] = fmaf(load_param<T>(a.weight, (int64_t)(c + i) * K + k, f32), x[k][i], y[i]);
      if (a.activation == RC_ACT_SILU) y[i] *= sigmoid(y[i]);
    }
#pragma unroll
    for (int k = 0; k < K - 1; k++) store_vec<V>(s + k * a.state.time, V, x[k + 1]);
  }
  store_vec<V>(at<T>(a.y, b, 0, c), V, y);
}

// Calls f(std::integral_constant<int, K>) for a checked number of taps.
template <class F>
int by_taps(int32_t k, F&& f) {
  switch (k) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
  }
}

bool conv_sizes_ok(int32_t dtype, int32_t param, int32_t act, int32_t batch, int32_t length,
                   int32_t width, int32_t taps) {
  return dtype_ok(dtype) && param_ok(param, dtype) &&
         (act == RC_ACT_NONE || act == RC_ACT_SILU) && batch >= 0 && length >= 0 && width >= 0 &&
         length <= kMaxExtent && width <= kMaxExtent && taps >= 1 && taps <= 8;
}

// The launch shape: lanes along the channels, rows of a thread, workgroups.
// Long runs read fewer rows twice and leave fewer partial sums, short ones fill the
// chip: 32 rows, halved while that gives fewer than four workgroups a compute unit.
struct ConvPlan {
  int V, lanes, run;
  int64_t runs, groups_c, groups_t;
};
ConvPlan conv_plan(const rc_conv_args& a, bool backward) {
  ConvPlan p;
  p.V = backward ? (a.width < 4 ? 1 : 4) : a.width < 8 ? 1 : 8;
  const int64_t vecs = cdiv(a.width, p.V);
  p.lanes = lanes_for(vecs);
  p.groups_c = cdiv(vecs, p.lanes);
  const int slots = kThreads / p.lanes;
  const int64_t cus4 = 4 * (int64_t)rcdp::num_cus();
  p.run = 32;
  while (p.run > 4 && p.groups_c * cdiv((int64_t)a.batch * cdiv(a.length, p.run), slots) < cus4)
    p.run /= 2;
  p.runs = a.length > 0 ? cdiv(a.length, p.run) : 1;
  p.groups_t = cdiv((int64_t)a.batch * p.runs, slots);
  return p;
}

template <class T>
ConvParams<T> conv_params(const rc_conv_args& a, const ConvPlan& p) {
  return {a, p.lanes, p.run, (int32_t)p.runs, (int32_t)p.groups_c, nullptr};
}

int64_t weight_sum_blocks(const rc_conv_args& a) {
  return cdiv((int64_t)a.width * (a.taps + 1), kSumCols);
}

int conv_check(const rc_conv_args* a, bool backward) {
  if (!a || !conv_sizes_ok(a->dtype, a->param_dtype, a->activation, a->batch, a->length, a->width,
                           a->taps) ||
      !float_aligned(a->workspace))
    return RC_E_ARG;
  const bool some = a->batch > 0 && a->width > 0;
  if (some && !a->weight) return RC_E_ARG;
  if (some && a->length > 0 && !a->x.data) return RC_E_ARG;
  if (some && a->length > 0 && (backward ? !a->dy.data || !a->dx.data : !a->y.data))
    return RC_E_ARG;
  const ConvPlan p = conv_plan(*a, backward);
  if (!launchable(p.groups_c * p.groups_t, kThreads)) return RC_E_OVERFLOW;
  if (backward && (a->dweight || a->dbias) && !launchable(weight_sum_blocks(*a), kThreads))
    return RC_E_OVERFLOW;
  return RC_OK;
}

}  // namespace

extern "C" int rc_conv_forward(const rc_conv_args* args, void* stream) {
  if (const int st = conv_check(args, false)) return st;
  const rc_conv_args& a = *args;
  const ConvPlan p = conv_plan(a, false);
  if (p.groups_c * p.groups_t == 0) return RC_OK;
  if (a.length == 0 && !a.state_out.data) return RC_OK;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_taps(a.taps, [&](auto k) {
      const dim3 grid((uint32_t)(p.groups_c * p.groups_t));
      if (p.V == 1)
        k_conv_forward<T, k(), 1><<<grid, kThreads, 0, (hipStream_t)stream>>>(conv_params<T>(a, p));
      else
        k_conv_forward<T, k(), 8><<<grid, kThreads, 0, (hipStream_t)stream>>>(conv_params<T>(a, p));
      return launched("k_conv_forward");
    });
  });
}

extern "C" int rc_conv_backward_workspace(const rc_conv_args* a, uint64_t* bytes_host) {
  if (!a || !bytes_host || !conv_sizes_ok(a->dtype, a->param_dtype, a->activation, a->batch,
                                          a->length, a->width, a->taps))
    return RC_E_ARG;
  *bytes_host = (uint64_t)conv_plan(*a, true).groups_t * a->width * (a->taps + 1) * 4;
  return RC_OK;
}

extern "C" int rc_conv_backward(const rc_conv_args* args, void* stream) {
  if (const int st = conv_check(args, true)) return st;
  const rc_conv_args& a = *args;
  const ConvPlan p = conv_plan(a, true);
  const bool weights = a.dweight || a.dbias;
  uint64_t need = 0;
  rc_conv_backward_workspace(args, &need);
  if (weights && need > 0 && (!a.workspace || a.workspace_bytes < need)) return RC_E_SCRATCH;
  if (a.width == 0) return RC_OK;
  return by_dtype(a.dtype, [&](auto t) -> int {
    using T = decltype(t);
    if (p.groups_c * p.groups_t > 0) {
      const int st = by_taps(a.taps, [&](auto k) {
        ConvParams<T> q = conv_params<T>(a, p);
        if (weights) q.partial = static_cast<float*>(a.workspace);
        const dim3 grid((uint32_t)(p.groups_c * p.groups_t));
        if (p.V == 1)
          k_conv_backward<T, k(), 1><<<grid, kThreads, 0, (hipStream_t)stream>>>(q);
        else
          k_conv_backward<T, k(), 4><<<grid, kThreads, 0, (hipStream_t)stream>>>(q);
        return launched("k_conv_backward");
      });
      if (st) return st;
    }
    if (!weights) return RC_OK;
    k_conv_weight_sum<T><<<dim3((uint32_t)weight_sum_blocks(a)), kThreads, 0,
                           (hipStream_t)stream>>>(static_cast<const float*>(a.workspace),
                                                  p.groups_t, a.width, a.taps, a.dweight, a.dbias,
                                                  a.param_dtype == RC_F32);
    return launched("k_conv_weight_sum");
  });
}

extern "C" int rc_conv_step(const rc_conv_step_args* args, void* stream) {
  if (!args) return RC_E_ARG;
  const rc_conv_step_args& a = *args;
  if (!conv_sizes_ok(a.dtype, a.param_dtype, a.activation, a.batch, 1, a.width, a.taps) ||
      a.num_slots < 0 || (!a.slots && a.num_slots < a.batch))
    return RC_E_ARG;
  if (a.batch == 0 || a.width == 0) return RC_OK;
  if (!a.x.data || !a.y.data || !a.weight || (a.taps > 1 && !a.state.data)) return RC_E_ARG;
  const int V = a.width % 2 ? 1 : 2;
  const int64_t vecs = a.width / V, blocks = cdiv(vecs * a.batch, kThreads);
  if (!launchable(blocks, kThreads)) return RC_E_OVERFLOW;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_taps(a.taps, [&](auto k) {
      if (V == 1)
        k_conv_step<T, k(), 1><<<dim3((uint32_t)blocks), kThreads, 0, (hipStream_t)stream>>>(
            a, (int32_t)vecs);
      else
        k_conv_step<T, k(), 2><<<dim3((uint32_t)blocks), kThreads, 0, (hipStream_t)stream>>>(
            a, (int32_t)vecs);
      return launched("k_conv_step");
    });
  });
}
