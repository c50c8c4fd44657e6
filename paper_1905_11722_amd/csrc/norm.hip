// Norms before and after a block, fused with the block's gate and residual
// scale, and their gradients.  For each row of D channels
//   v = u act(gate),  p = v rv w_post,  rv = 1 / sqrt(mean(v^2) + eps),
//   out = r + s p,    n = out ro w_pre, ro = 1 / sqrt(mean(out^2) + eps).
// Backward, with unit = out ro and vn = v rv:
//   dr = dout + ro (dn w_pre - unit mean(dn w_pre unit)),   dw_pre = sum dn unit,
//   ds = sum dr p,  dp = dr s,  dw_post = sum dp vn,
//   dv = rv (dp w_post - vn mean(dp w_post vn)),  du = dv act,  dgate = dv u act'.
//
// A few operations for each value moved: bound by memory.  A row stays in the
// registers of its threads from the loads to the stores, so every tensor is
// read or written once; a row needs two sums over its threads, one after the
// other.  Workgroups walk over rows with the weights' gradients (and up to
// 6144 channels the weights) in registers.  (Backward with four sums in one step,
// the second mean being linear in the first, cancels where the gradient is
// small: not kept.)
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int kVec = 8;                     // channels of a load
constexpr int kMaxWidth = 16384;

struct NormParams {
  rc_norm_args a;
  float* partial;                           // backward: [workgroups][3][width]
};

// Threads of a workgroup with TPR threads a row.
constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// Sums over the TPR threads of a row of M values.  lds has 16 M floats of its
// own for each of two calls in a row: the barrier of one call is between the
// reads of the one before and the writes of the one after.
template <int TPR, int M>
__device__ __forceinline__ void row_sums(float (&x)[M], float* lds) {
#pragma unroll
  for (int m = 0; m < M; m++) x[m] = lane_sum<TPR == 32 ? 32 : 64>(x[m]);
  if (TPR <= 64) return;
  constexpr int W = TPR / 64;
  if (threadIdx.x % 64 == 0) {
#pragma unroll
    for (int m = 0; m < M; m++) lds[threadIdx.x / 64 * M + m] = x[m];
  }
  __syncthreads();
  const int first = threadIdx.x / TPR * W;
#pragma unroll
  for (int m = 0; m < M; m++) {
    x[m] = 0.f;
#pragma unroll
    for (int i = 0; i < W; i++) x[m] += lds[(first + i) * M + m];
  }
}

// act(x) and its slope.
__device__ __forceinline__ float gate_of(float x, int32_t act, float& slope) {
  const float s = sigmoid(x);
  slope = act == RC_ACT_SILU ? s * (1.f + x * (1.f - s)) : s * (1.f - s);
  return act == RC_ACT_SILU ? x * s : s;
}

// A thread's channels of a row: NV loads of V.  Where V does not divide the width, the
// last load moves back to the last V channels: its first `over` elements are
// its neighbour's too, are left out of the sums, and are stored twice with the same
// value.  A load that begins past the width has nothing of its own.
template <int TPR, int NV, int V>
struct Columns {
  int c[NV], over[NV];
  __device__ Columns(int lane, int width) {
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int at = (k * TPR + lane) * V;
      c[k] = min(at, width - V);
      over[k] = at - c[k];
    }
  }
  __device__ bool any(int k) const { return over[k] < V; }
  __device__ float own(int k, int i, float x) const { return i >= over[k] ? x : 0.f; }
};

template <class T, int V>
__device__ __forceinline__ void load_weight(const void* w, bool f32, int c, float absent,
                                            float (&x)[V]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = absent;
  } else if (f32) {
    load_vec<V>(static_cast<const float*>(w) + c, V, x);
  } else {
    load_vec<V>(static_cast<const T*>(w) + c, V, x);
  }
}

template <class T>
__device__ __forceinline__ T* row_at(const rc_view& v, int64_t row) {
  return static_cast<T*>(v.data) + row * v.batch;
}

// Forward: several workgroups a compute unit, so that others' loads run while one sums.
// 16384 rows of 4096 channels with a gate, residual in 32 bits (940 MB): 172 us, 5.5 TB/s; in 16
// bits (671 MB) 125 us, 5.4 TB/s: a large copy's rate and more.
template <class T, class R, int TPR, int NV, int V>
__global__ __launch_bounds__(threads_of(TPR)) void k_norm_forward(NormParams p) {
  __shared__ float lds[2][16];
  const rc_norm_args& a = p.a;
  constexpr int RPW = threads_of(TPR) / TPR;
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const bool f32 = a.param_dtype == RC_F32;
  const float inv = 1.f / (float)a.width;
  const Columns<TPR, NV, V> at(lane, a.width);
  float wpost[NV][V], wpre[NV][V], scale[NV][V];
#pragma unroll
  for (int k = 0; k < NV; k++) {
    load_weight<T>(a.post_weight, f32, at.c[k], 1.f, wpost[k]);
    load_weight<T>(a.pre_weight, f32, at.c[k], 0.f, wpre[k]);
    load_weight<T>(a.scale, f32, at.c[k], 1.f, scale[k]);
  }
  for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < a.rows; r0 += (int64_t)gridDim.x * RPW) {
    const int64_t row = min(r0 + group, a.rows - 1);
    const bool on = RPW == 1 || r0 + group < a.rows;
    float out[NV][V], v[NV][V], ss[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; k++) {
      load_vec<V>(row_at<R>(a.residual, row) + at.c[k], V, out[k]);
      if (a.block.data) {
        load_vec<V>(row_at<T>(a.block, row) + at.c[k], V, v[k]);
        if (a.gate.data) {
          float g[V], slope;
          load_vec<V>(row_at<T>(a.gate, row) + at.c[k], V, g);
#pragma unroll
          for (int i = 0; i < V; i++) v[k][i] *= gate_of(g[i], a.gate_activation, slope);
        }
#pragma unroll
        for (int i = 0; i < V; i++) ss[0] += at.own(k, i, v[k][i] * v[k][i]);
      }
    }
    float rv = 1.f, ro = 0.f;
    if (a.block.data) {
      if (a.post_weight) {
        row_sums<TPR>(ss, lds[0]);
        rv = __builtin_amdgcn_rsqf(fmaf(ss[0], inv, a.eps));
      }
#pragma unroll
      for (int k = 0; k < NV; k++) {
#pragma unroll
        for (int i = 0; i < V; i++)
          out[k][i] = fmaf(scale[k][i], v[k][i] * rv * wpost[k][i], out[k][i]);
        if (on && at.any(k)) store_vec<V>(row_at<R>(a.out, row) + at.c[k], V, out[k]);
      }
    }
    if (a.pre_weight) {
      ss[0] = 0.f;
#pragma unroll
      for (int k = 0; k < NV; k++)
#pragma unroll
        for (int i = 0; i < V; i++) ss[0] += at.own(k, i, out[k][i] * out[k][i]);
      row_sums<TPR>(ss, lds[1]);
      ro = __builtin_amdgcn_rsqf(fmaf(ss[0], inv, a.eps));
#pragma unroll
      for (int k = 0; k < NV; k++) {
#pragma unroll
        for (int i = 0; i < V; i++) out[k][i] *= ro * wpre[k][i];
        if (on && at.any(k)) store_vec<V>(row_at<T>(a.normed, row) + at.c[k], V, out[k]);
      }
    }
    if (a.stats && on && lane == 0) {
      a.stats[row * 2] = rv;
      a.stats[row * 2 + 1] = ro;
    }
    // one sum a row: its buffer is read before the next row writes it
    if (TPR > 64 && !(a.pre_weight && a.block.data && a.post_weight)) __syncthreads();
  }
}

// Backward: the row's values and the weights' gradients leave registers for two waves a
// SIMD, too few to hide the loads behind others' work, so up to 4096 channels the next row's loads
// are in flight during this row's sums.  16384 rows of 4096 channels with a gate,
// residual in 32 bits (1.48 GB): 310 us without, 277 with, 5.3 TB/s; in 16 bits (1.07 GB)
// 322 and 203 us, 5.3 TB/s.  Above: 5000 channels 4.7 TB/s, 8192 4.2.  Above
// 8192, where 128 registers a thread hold neither the row nor the sums, two of
// the three weights' sums are in LDS and the gate is read and evaluated again;
// the rest still spills.  4096 rows of 16384 channels: 1.42 ms with all in
// registers or spilled, 0.63 ms (2.3 TB/s) so.
template <class T, class R, int TPR, int NV, int V>
__global__ __launch_bounds__(threads_of(TPR)) void k_norm_backward(NormParams p) {
  constexpr int RPW = threads_of(TPR) / TPR;
  constexpr bool HOLD = NV == 1;                       // the weights stay in registers
  constexpr bool AHEAD = NV == 1 && TPR <= 512;        // and the next row's loads
  constexpr bool TIGHT = TPR * NV * V > 8192;          // registers for a part only
  __shared__ float lds[2][16];
  __shared__ float4 sums[TIGHT ? 2 * NV * V / 4 : 1][TIGHT ? TPR : 1];   // dscale, dpost_weight
  __shared__ float cols[RPW > 1 ? threads_of(TPR) * V : 1];
  const rc_norm_args& a = p.a;
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const bool f32 = a.param_dtype == RC_F32;
  const float inv = 1.f / (float)a.width;
  const Columns<TPR, NV, V> at(lane, a.width);
  float held[3][V], dw[3][NV][V];
  if (HOLD) {
    load_weight<T>(a.post_weight, f32, at.c[0], 1.f, held[0]);
    load_weight<T>(a.scale, f32, at.c[0], 1.f, held[1]);
    load_weight<T>(a.pre_weight, f32, at.c[0], 0.f, held[2]);
  }
#pragma unroll
  for (int j = 0; j < 3; j++)
#pragma unroll
    for (int k = 0; k < NV; k++)
#pragma unroll
      for (int i = 0; i < V; i++) dw[j][k][i] = 0.f;
  // The thread's own slots of LDS in place of dw[1] and dw[2]: x are added to them.
  const auto add = [&](int j, int k, const float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      float4& s = sums[(j * NV + k) * (V / 4) + i / 4][threadIdx.x];
      const float4 was = s;
      s = {was.x + x[i], was.y + x[i + 1], was.z + x[i + 2], was.w + x[i + 3]};
    }
  };
  if constexpr (TIGHT) {
#pragma unroll
    for (int i = 0; i < 2 * NV * V / 4; i++) sums[i][threadIdx.x] = {0.f, 0.f, 0.f, 0.f};
  }
  typedef T TV __attribute__((ext_vector_type(V)));
  typedef R RV __attribute__((ext_vector_type(V)));
  // Loads for the next row are unconditional (elements loaded in a branch and handed on by a
  // loop: the compiler of ROCm 7.2 drops some): what is absent reads the residual's memory.
  RV in_r, in_dout;
  TV in_dn, in_v, in_g;
  float in_stats[2];
  const auto present = [&](const rc_view& v) { return v.data ? v : a.residual; };
  const rc_view from_dout = present(a.dout), from_dn = present(a.dnormed);
  const rc_view from_v = present(a.block), from_g = present(a.gate);
  const auto next = [&](int64_t r0) {                  // rows past the last: the last
    const int64_t row = min(r0 + group, a.rows - 1);
    const int c = at.c[0];
    in_stats[0] = a.stats[row * 2];
    in_stats[1] = a.stats[row * 2 + 1];
    __builtin_memcpy(&in_r, row_at<R>(a.residual, row) + c, sizeof(RV));
    __builtin_memcpy(&in_dout, row_at<R>(from_dout, row) + c, sizeof(RV));
    __builtin_memcpy(&in_dn, row_at<T>(from_dn, row) + c, sizeof(TV));
    __builtin_memcpy(&in_v, row_at<T>(from_v, row) + c, sizeof(TV));
    __builtin_memcpy(&in_g, row_at<T>(from_g, row) + c, sizeof(TV));
  };
  if (AHEAD) next((int64_t)blockIdx.x * RPW);
  for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < a.rows; r0 += (int64_t)gridDim.x * RPW) {
    const int64_t row = min(r0 + group, a.rows - 1);
    const bool on = RPW == 1 || r0 + group < a.rows;
    const float rv = AHEAD ? in_stats[0] : a.stats[row * 2];
    const float ro = AHEAD ? in_stats[1] : a.stats[row * 2 + 1];
    float dr[NV][V], dn[NV][V], vn[NV][V], act[NV][V], dact[NV][V], unit[NV][V], dot[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; k++) {
      if (AHEAD) {
#pragma unroll
        for (int i = 0; i < V; i++) {
          unit[k][i] = (float)in_r[i];
          dr[k][i] = on && a.dout.data ? (float)in_dout[i] : 0.f;
          dn[k][i] = on && a.dnormed.data ? (float)in_dn[i] : 0.f;
          vn[k][i] = a.block.data ? (float)in_v[i] : 0.f;
          if (a.gate.data) act[k][i] = (float)in_g[i];
        }
      } else {
        const int c = at.c[k];
        load_vec<V>(row_at<R>(a.residual, row) + c, V, unit[k]);
        load_vec<V>(row_at<R>(a.dout, row) + c, a.dout.data ? V : 0, dr[k]);
        load_vec<V>(row_at<T>(a.dnormed, row) + c, a.dnormed.data ? V : 0, dn[k]);
        load_vec<V>(row_at<T>(a.block, row) + c, a.block.data ? V : 0, vn[k]);
        if (a.gate.data) load_vec<V>(row_at<T>(a.gate, row) + c, V, act[k]);
      }
      float wpost[V], scale[V], wpre[V];
      if (!HOLD) {
        load_weight<T>(a.post_weight, f32, at.c[k], 1.f, wpost);
        load_weight<T>(a.scale, f32, at.c[k], 1.f, scale);
        load_weight<T>(a.pre_weight, f32, at.c[k], 0.f, wpre);
      }
#pragma unroll
      for (int i = 0; i < V; i++) {
        if (a.gate.data) {
          float slope;
          act[k][i] = gate_of(act[k][i], a.gate_activation, slope);
          dact[k][i] = vn[k][i] * slope;               // u act'
          vn[k][i] *= act[k][i];
        }
        vn[k][i] *= rv;
        const float part = vn[k][i] * (HOLD ? held[0][i] : wpost[i]);
        unit[k][i] = fmaf(HOLD ? held[1][i] : scale[i], part, unit[k][i]) * ro;
        dw[0][k][i] += on ? dn[k][i] * unit[k][i] : 0.f;
        dn[k][i] *= HOLD ? held[2][i] : wpre[i];
        dot[0] += at.own(k, i, dn[k][i] * unit[k][i]);
      }
    }
    if (AHEAD) next(r0 + (int64_t)gridDim.x * RPW);
    if (a.pre_weight) {
      row_sums<TPR>(dot, lds[0]);
      const float m = dot[0] * inv;
#pragma unroll
      for (int k = 0; k < NV; k++)
#pragma unroll
        for (int i = 0; i < V; i++)
          dr[k][i] = fmaf(ro, dn[k][i] - unit[k][i] * m, dr[k][i]);
    }
    dot[0] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++) {
      if (on && at.any(k)) store_vec<V>(row_at<R>(a.dresidual, row) + at.c[k], V, dr[k]);
      float wpost[V], scale[V];
      if (!HOLD) {
        load_weight<T>(a.post_weight, f32, at.c[k], 1.f, wpost);
        load_weight<T>(a.scale, f32, at.c[k], 1.f, scale);
      }
      float ds[V], dpost[V];
#pragma unroll
      for (int i = 0; i < V; i++) {
        const float post = HOLD ? held[0][i] : wpost[i];
        ds[i] = on ? dr[k][i] * (vn[k][i] * post) : 0.f;
        dr[k][i] *= HOLD ? held[1][i] : scale[i];      // dp
        dpost[i] = on ? dr[k][i] * vn[k][i] : 0.f;
        dr[k][i] *= post;
        dot[0] += at.own(k, i, dr[k][i] * vn[k][i]);
      }
      if constexpr (TIGHT) {
        add(0, k, ds);
        add(1, k, dpost);
      } else {
#pragma unroll
        for (int i = 0; i < V; i++) {
          dw[1][k][i] += ds[i];
          dw[2][k][i] += dpost[i];
        }
      }
    }
    if (a.block.data) {
      float m = 0.f;
      if (a.post_weight) {
        row_sums<TPR>(dot, lds[1]);
        m = dot[0] * inv;
      }
#pragma unroll
      for (int k = 0; k < NV; k++) {
        const bool store = on && at.any(k);
#pragma unroll
        for (int i = 0; i < V; i++) dr[k][i] = rv * (dr[k][i] - vn[k][i] * m);
        if (a.gate.data) {
          if (TIGHT) {
            load_vec<V>(row_at<T>(a.gate, row) + at.c[k], V, act[k]);
            load_vec<V>(row_at<T>(a.block, row) + at.c[k], V, dact[k]);
          }
#pragma unroll
          for (int i = 0; i < V; i++) {
            if (TIGHT) {
              float slope;
              act[k][i] = gate_of(act[k][i], a.gate_activation, slope);
              dact[k][i] *= slope;
            }
            dact[k][i] *= dr[k][i];
            dr[k][i] *= act[k][i];
          }
          if (store) store_vec<V>(row_at<T>(a.dgate, row) + at.c[k], V, dact[k]);
        }
        if (store) store_vec<V>(row_at<T>(a.dblock, row) + at.c[k], V, dr[k]);
      }
    }
    // one sum a row: its buffer is read before the next row writes it
    if (TPR > 64 && !(a.pre_weight && a.block.data && a.post_weight)) __syncthreads();
  }
  if (!p.partial) return;
  if constexpr (TIGHT) {
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int k = 0; k < NV; k++)
#pragma unroll
        for (int i = 0; i < V; i += 4) {
          const float4 s = sums[(j * NV + k) * (V / 4) + i / 4][threadIdx.x];
          dw[j + 1][k][i] = s.x;
          dw[j + 1][k][i + 1] = s.y;
          dw[j + 1][k][i + 2] = s.z;
          dw[j + 1][k][i + 3] = s.w;
        }
  }
#pragma unroll
  for (int j = 0; j < 3; j++) {
    float* out = p.partial + ((int64_t)blockIdx.x * 3 + j) * a.width;
    if (RPW > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; i++)
        if (i >= at.over[0]) cols[threadIdx.x * V + i - at.over[0]] = dw[j][0][i];
      __syncthreads();
      for (int o = threadIdx.x; o < TPR * V && o < a.width; o += threads_of(TPR)) {
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < RPW; g++) s += cols[g * TPR * V + o];
        out[o] = s;
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; k++)
        if (at.any(k)) store_vec<V>(out + at.c[k], V, dw[j][k]);
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_norm_weight_sum(const float* in, int64_t parts,
                                                         int32_t width, void* dpre, void* dscale,
                                                         void* dpost, int32_t f32,
                                                         int32_t second) {
  __shared__ float lds[256];
  const int64_t cols = 3 * (int64_t)width;
  const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x % kSumCols;
  const float s = column_sum(in, parts, cols, c, lds);
  if (threadIdx.x >= kSumCols || c >= cols) return;
  void* out = c < width ? dpre : c < 2 * (int64_t)width ? dscale : dpost;
  if (out) store_param<T>(out, c % width, f32, second || c >= width ? s : 0.f);
}

// Threads of a row, loads of a thread and their width: enough threads for one
// load each, up to 8192 channels forward and, by the registers, 6144 backward (5000
// channels backward: 512 threads and two loads 313 us, 768 and one 193), for two
// each above.
template <bool BACKWARD, class F>
int by_width(int32_t width, F&& f) {
  using std::integral_constant;
  const auto with = [&](auto tpr, auto nv) { return f(tpr, nv, integral_constant<int, kVec>{}); };
  if (width < kVec)
    return f(integral_constant<int, 32>{}, integral_constant<int, 1>{},
             integral_constant<int, 1>{});
  if (width <= 256) return with(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (width <= 512) return with(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (width <= 1024) return with(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (width <= 2048) return with(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (width <= 4096) return with(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (width <= 6144) return with(integral_constant<int, 768>{}, integral_constant<int, 1>{});
  if (width <= 8192)
    return with(integral_constant<int, BACKWARD ? 512 : 1024>{},
                integral_constant<int, BACKWARD ? 2 : 1>{});
  return with(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
int threads_per_row(int32_t width, bool backward) {
  const auto threads = [](auto tpr, auto, auto) { return int(tpr()); };
  return backward ? by_width<true>(width, threads) : by_width<false>(width, threads);
}

// Workgroups: as many as the chip holds at once (forward six waves a SIMD, backward two,
// by their registers), then each walks over rows.  One more than fits waits for a
// whole walk: 32768 rows of 1024 channels, eight waves asked for 103 us, six 86.
// Backward each leaves a row of partial sums, so beyond one a compute unit there are four
// rows of work for each.
int64_t norm_blocks(const rc_norm_args& a, bool backward) {
  const int tpr = threads_per_row(a.width, backward), wg = threads_of(tpr);
  const int64_t need = cdiv(a.rows, wg / tpr), cus = rcdp::num_cus();
  const int64_t most = cus * (backward ? (wg < 512 ? 512 / wg : 1) : 1536 / wg);
  if (need <= cus) return need;
  const int64_t some = backward ? (need / 4 < cus ? cus : need / 4) : need;
  return some < most ? some : most;
}

bool norm_sizes_ok(const rc_norm_args* a) {
  return a && dtype_ok(a->dtype) && param_ok(a->residual_dtype, a->dtype) &&
         param_ok(a->param_dtype, a->dtype) && a->rows >= 0 && a->width >= 0 &&
         a->width <= kMaxWidth &&
         (a->gate_activation == RC_ACT_SILU || a->gate_activation == RC_ACT_SIGMOID);
}

int norm_check(const rc_norm_args* a, bool backward) {
  if (!norm_sizes_ok(a) || !float_aligned(a->workspace)) return RC_E_ARG;
  if (a->rows > 0 && a->width > 0) {
    if (!a->residual.data) return RC_E_ARG;
    if (!a->block.data && (a->gate.data || a->post_weight || a->scale)) return RC_E_ARG;
    if (!a->block.data && !a->pre_weight) return RC_E_ARG;
    if (!backward && ((a->block.data && !a->out.data) || (a->pre_weight && !a->normed.data)))
      return RC_E_ARG;
    if (backward && (!a->stats || (a->block.data && !a->dblock.data) ||
                     (a->gate.data && !a->dgate.data) || !a->dresidual.data))
      return RC_E_ARG;
  }
  return RC_OK;
}

// Calls f(T{}, R{}) with the element types of the block and of the residual.
template <class F>
int by_dtypes(const rc_norm_args& a, F&& f) {
  return by_dtype(a.dtype, [&](auto t) {
    if (a.residual_dtype == RC_F32) return f(t, float{});
    return f(t, t);
  });
}

}  // namespace

extern "C" int rc_norm_forward(const rc_norm_args* args, void* stream) {
  if (const int st = norm_check(args, false)) return st;
  const rc_norm_args& a = *args;
  if (a.rows == 0 || a.width == 0) return RC_OK;
  return by_dtypes(a, [&](auto t, auto r) {
    return by_width<false>(a.width, [&](auto tpr, auto nv, auto v) {
      k_norm_forward<decltype(t), decltype(r), tpr(), nv(), v()>
          <<<dim3((uint32_t)norm_blocks(a, false)), threads_of(tpr()), 0, (hipStream_t)stream>>>(
              {a, nullptr});
      return launched("k_norm_forward");
    });
  });
}

extern "C" int rc_norm_backward_workspace(const rc_norm_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !norm_sizes_ok(a)) return RC_E_ARG;
  *bytes_host = a->width > 0 ? (uint64_t)norm_blocks(*a, true) * 3 * a->width * 4 : 0;
  return RC_OK;
}

extern "C" int rc_norm_backward(const rc_norm_args* args, void* stream) {
  if (const int st = norm_check(args, true)) return st;
  rc_norm_args a = *args;
  if (a.width == 0) return RC_OK;
  // Without a gradient the second norm is left out, and its weight's gradient is 0: 0 times what is
  // not finite is no 0.
  const bool second = a.dnormed.data;
  if (!second) a.pre_weight = nullptr;
  const bool weights = a.dpost_weight || a.dscale || a.dpre_weight;
  uint64_t need = 0;
  rc_norm_backward_workspace(args, &need);
  if (weights && need > 0 && (!a.workspace || a.workspace_bytes < need)) return RC_E_SCRATCH;
  const int64_t blocks = norm_blocks(a, true);
  float* partial = weights ? static_cast<float*>(a.workspace) : nullptr;
  return by_dtypes(a, [&](auto t, auto r) -> int {
    using T = decltype(t);
    if (blocks > 0) {
      const int st = by_width<true>(a.width, [&](auto tpr, auto nv, auto v) {
        k_norm_backward<T, decltype(r), tpr(), nv(), v()>
            <<<dim3((uint32_t)blocks), threads_of(tpr()), 0, (hipStream_t)stream>>>({a, partial});
        return launched("k_norm_backward");
      });
      if (st) return st;
    }
    if (!weights) return RC_OK;
    k_norm_weight_sum<T><<<dim3((uint32_t)cdiv(3 * (int64_t)a.width, kSumCols)), 256, 0,
                           (hipStream_t)stream>>>(partial, blocks, a.width, a.dpre_weight,
                                                  a.dscale, a.dpost_weight,
                                                  a.param_dtype == RC_F32, second);
    return launched("k_norm_weight_sum");
  });
}
