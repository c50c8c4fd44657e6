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
// 8192 channels the weights) in registers.  (Backward with four sums in one step,
// the second mean being linear in the first, cancels where the gradient is
// small: not kept.)
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int V = 8;                        // channels of a load
constexpr int kMaxWidth = 16384;

struct NormParams {
  rc_norm_args a;
  float* partial;                           // backward: [workgroups][3][width]
};

// Threads of a workgroup with TPR threads a row.
constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                           0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// Sum over 32 or 64 lanes, in each of them (a mirror is as good as an
// exchange once the lanes below are equal).
template <int LANES>
__device__ __forceinline__ float lane_sum(float x) {
  x = dpp_add<0xB1>(x);                                // lanes 1 apart
  x = dpp_add<0x4E>(x);                                // 2 apart
  x = dpp_add<0x141>(x);                               // half rows mirrored
  x = dpp_add<0x140>(x);                               // rows mirrored
  const unsigned a = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  if (LANES == 32) return x;
  const unsigned b = __builtin_bit_cast(unsigned, x);
  const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __builtin_bit_cast(float, (unsigned)h[0]) + __builtin_bit_cast(float, (unsigned)h[1]);
}

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

template <class T, int NV>
__device__ __forceinline__ void load_weight(const void* w, bool f32, const int (&c)[NV], int width,
                                            float absent, float (&x)[NV][V]) {
#pragma unroll
  for (int k = 0; k < NV; k++)
    if (!w) {
#pragma unroll
      for (int i = 0; i < V; i++) x[k][i] = absent;
    } else if (f32) {
      load_vec<V>(static_cast<const float*>(w) + c[k], width - c[k], x[k]);
    } else {
      load_vec<V>(static_cast<const T*>(w) + c[k], width - c[k], x[k]);
    }
}

template <class T>
__device__ __forceinline__ T* row_at(const rc_view& v, int64_t row) {
  return static_cast<T*>(v.data) + row * v.batch;
}

template <class T, class R, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void k_norm_forward(NormParams p) {
  __shared__ float lds[2][16];
  const rc_norm_args& a = p.a;
  constexpr int RPW = threads_of(TPR) / TPR;
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const bool f32 = a.param_dtype == RC_F32;
  const float inv = 1.f / (float)a.width;
  int c[NV];
#pragma unroll
  for (int k = 0; k < NV; k++) c[k] = min((k * TPR + lane) * V, a.width);
  float wpost[NV][V], wpre[NV][V], scale[NV][V];
  load_weight<T>(a.post_weight, f32, c, a.width, 1.f, wpost);
  load_weight<T>(a.pre_weight, f32, c, a.width, 0.f, wpre);
  load_weight<T>(a.scale, f32, c, a.width, 1.f, scale);
  for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < a.rows; r0 += (int64_t)gridDim.x * RPW) {
    const int64_t row = r0 + group;
    const bool on = row < a.rows;
    float out[NV][V], v[NV][V], ss[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int n = on ? a.width - c[k] : 0;
      load_vec<V>(row_at<R>(a.residual, row) + c[k], n, out[k]);
      if (a.block.data) {
        load_vec<V>(row_at<T>(a.block, row) + c[k], n, v[k]);
        if (a.gate.data) {
          float g[V], slope;
          load_vec<V>(row_at<T>(a.gate, row) + c[k], n, g);
#pragma unroll
          for (int i = 0; i < V; i++) v[k][i] *= gate_of(g[i], a.gate_activation, slope);
        }
#pragma unroll
        for (int i = 0; i < V; i++) ss[0] = fmaf(v[k][i], v[k][i], ss[0]);
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
        if (on) store_vec<V>(row_at<R>(a.out, row) + c[k], a.width - c[k], out[k]);
      }
    }
    if (a.pre_weight) {
      ss[0] = 0.f;
#pragma unroll
      for (int k = 0; k < NV; k++)
#pragma unroll
        for (int i = 0; i < V; i++) ss[0] = fmaf(out[k][i], out[k][i], ss[0]);
      row_sums<TPR>(ss, lds[1]);
      ro = __builtin_amdgcn_rsqf(fmaf(ss[0], inv, a.eps));
#pragma unroll
      for (int k = 0; k < NV; k++) {
#pragma unroll
        for (int i = 0; i < V; i++) out[k][i] *= ro * wpre[k][i];
        if (on) store_vec<V>(row_at<T>(a.normed, row) + c[k], a.width - c[k], out[k]);
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

// Backward.  (Above 8192 channels a row and its sums spill: 16384 channels run at a
// fifth of the rate of 4096.)
template <class T, class R, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void k_norm_backward(NormParams p) {
  constexpr int RPW = threads_of(TPR) / TPR;
  constexpr bool HOLD = NV == 1;                       // the weights stay in registers
  __shared__ float lds[2][16];
  __shared__ float cols[RPW > 1 ? threads_of(TPR) * V : 1];
  const rc_norm_args& a = p.a;
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const bool f32 = a.param_dtype == RC_F32;
  const float inv = 1.f / (float)a.width;
  int c[NV];
#pragma unroll
  for (int k = 0; k < NV; k++) c[k] = min((k * TPR + lane) * V, a.width);
  float held[3][V], dw[3][NV][V];
  const auto weight = [&](const void* w, int k, float absent, float (&x)[V]) {
    const int at[1] = {c[k]};
    float y[1][V];
    load_weight<T>(w, f32, at, a.width, absent, y);
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = y[0][i];
  };
  if (HOLD) {
    weight(a.post_weight, 0, 1.f, held[0]);
    weight(a.scale, 0, 1.f, held[1]);
    weight(a.pre_weight, 0, 0.f, held[2]);
  }
#pragma unroll
  for (int j = 0; j < 3; j++)
#pragma unroll
    for (int k = 0; k < NV; k++)
#pragma unroll
      for (int i = 0; i < V; i++) dw[j][k][i] = 0.f;
  for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < a.rows; r0 += (int64_t)gridDim.x * RPW) {
    const int64_t row = r0 + group;
    const bool on = row < a.rows;
    const float rv = on ? a.stats[row * 2] : 0.f, ro = on ? a.stats[row * 2 + 1] : 0.f;
    float dr[NV][V], dn[NV][V], vn[NV][V], act[NV][V], dact[NV][V], unit[NV][V], dot[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; k++) {
      const int n = on ? a.width - c[k] : 0;
      load_vec<V>(row_at<R>(a.residual, row) + c[k], n, unit[k]);
      load_vec<V>(row_at<R>(a.dout, row) + c[k], a.dout.data ? n : 0, dr[k]);
      load_vec<V>(row_at<T>(a.dnormed, row) + c[k], a.dnormed.data ? n : 0, dn[k]);
      load_vec<V>(row_at<T>(a.block, row) + c[k], a.block.data ? n : 0, vn[k]);
      if (a.gate.data) load_vec<V>(row_at<T>(a.gate, row) + c[k], n, act[k]);
      float wpost[V], scale[V], wpre[V];
      if (!HOLD) {
        weight(a.post_weight, k, 1.f, wpost);
        weight(a.scale, k, 1.f, scale);
        weight(a.pre_weight, k, 0.f, wpre);
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
        dw[0][k][i] = fmaf(dn[k][i], unit[k][i], dw[0][k][i]);
        dn[k][i] *= HOLD ? held[2][i] : wpre[i];
        dot[0] = fmaf(dn[k][i], unit[k][i], dot[0]);
      }
    }
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
      if (on)
        store_vec<V>(row_at<R>(a.dresidual, row) + c[k], a.width - c[k], dr[k]);
      float wpost[V], scale[V];
      if (!HOLD) {
        weight(a.post_weight, k, 1.f, wpost);
        weight(a.scale, k, 1.f, scale);
      }
#pragma unroll
      for (int i = 0; i < V; i++) {
        const float post = HOLD ? held[0][i] : wpost[i];
        dw[1][k][i] = fmaf(dr[k][i], vn[k][i] * post, dw[1][k][i]);
        dr[k][i] *= HOLD ? held[1][i] : scale[i];      // dp
        dw[2][k][i] = fmaf(dr[k][i], vn[k][i], dw[2][k][i]);
        dr[k][i] *= post;
        dot[0] = fmaf(dr[k][i], vn[k][i], dot[0]);
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
#pragma unroll
        for (int i = 0; i < V; i++) dr[k][i] = rv * (dr[k][i] - vn[k][i] * m);
        if (a.gate.data) {
#pragma unroll
          for (int i = 0; i < V; i++) {
            dact[k][i] *= dr[k][i];
            dr[k][i] *= act[k][i];
          }
          if (on) store_vec<V>(row_at<T>(a.dgate, row) + c[k], a.width - c[k], dact[k]);
        }
        if (on) store_vec<V>(row_at<T>(a.dblock, row) + c[k], a.width - c[k], dr[k]);
      }
    }
    // one sum a row: its buffer is read before the next row writes it
    if (TPR > 64 && !(a.pre_weight && a.block.data && a.post_weight)) __syncthreads();
  }
  if (!p.partial) return;
#pragma unroll
  for (int j = 0; j < 3; j++) {
    float* out = p.partial + ((int64_t)blockIdx.x * 3 + j) * a.width;
    if (RPW > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; i++) cols[threadIdx.x * V + i] = dw[j][0][i];
      __syncthreads();
      for (int o = threadIdx.x; o < TPR * V && o < a.width; o += threads_of(TPR)) {
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < RPW; g++) s += cols[g * TPR * V + o];
        out[o] = s;
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; k++) store_vec<V>(out + c[k], a.width - c[k], dw[j][k]);
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_norm_weight_sum(const float* in, int64_t parts,
                                                         int32_t width, void* dpre, void* dscale,
                                                         void* dpost, int32_t f32) {
  __shared__ float lds[256];
  const int64_t cols = 3 * (int64_t)width;
  const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x % kSumCols;
  const float s = column_sum(in, parts, cols, c, lds);
  if (threadIdx.x >= kSumCols || c >= cols) return;
  void* out = c < width ? dpre : c < 2 * (int64_t)width ? dscale : dpost;
  if (out) store_param<T>(out, c % width, f32, s);
}

// Threads of a row and loads of a thread: enough threads for one load each up to
// 8192 channels (backward, where two loads' registers still fit, 4096), for two
// each above.
template <bool BACKWARD, class F>
int by_width(int32_t width, F&& f) {
  using std::integral_constant;
  if (width <= 256) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (width <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (width <= 1024) return f(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (width <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (width <= 4096) return f(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (width <= 8192)
    return f(integral_constant<int, BACKWARD ? 512 : 1024>{},
             integral_constant<int, BACKWARD ? 2 : 1>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
int threads_per_row(int32_t width, bool backward) {
  const auto threads = [](auto tpr, auto) { return int(tpr()); };
  return backward ? by_width<true>(width, threads) : by_width<false>(width, threads);
}

// Workgroups: enough threads to fill the chip, then each walks over rows.
// Backward each leaves a row of partial sums, so beyond one a compute unit
// there are four rows of work for each.
int64_t norm_blocks(const rc_norm_args& a, bool backward) {
  const int tpr = threads_per_row(a.width, backward), wg = threads_of(tpr);
  const int64_t need = cdiv(a.rows, wg / tpr), cus = rcdp::num_cus();
  const int64_t most = cus * (backward ? (wg < 512 ? 512 / wg : 1) : 2048 / wg);
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
  if (!norm_sizes_ok(a)) return RC_E_ARG;
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
    return by_width<false>(a.width, [&](auto tpr, auto nv) {
      k_norm_forward<decltype(t), decltype(r), tpr(), nv()>
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
  const rc_norm_args& a = *args;
  if (a.width == 0) return RC_OK;
  const bool weights = a.dpost_weight || a.dscale || a.dpre_weight;
  uint64_t need = 0;
  rc_norm_backward_workspace(args, &need);
  if (weights && need > 0 && (!a.workspace || a.workspace_bytes < need)) return RC_E_SCRATCH;
  const int64_t blocks = norm_blocks(a, true);
  float* partial = weights ? static_cast<float*>(a.workspace) : nullptr;
  return by_dtypes(a, [&](auto t, auto r) -> int {
    using T = decltype(t);
    if (blocks > 0) {
      const int st = by_width<true>(a.width, [&](auto tpr, auto nv) {
        k_norm_backward<T, decltype(r), tpr(), nv()>
            <<<dim3((uint32_t)blocks), threads_of(tpr()), 0, (hipStream_t)stream>>>({a, partial});
        return launched("k_norm_backward");
      });
      if (st) return st;
    }
    if (!weights) return RC_OK;
    k_norm_weight_sum<T><<<dim3((uint32_t)cdiv(3 * (int64_t)a.width, kSumCols)), 256, 0,
                           (hipStream_t)stream>>>(partial, blocks, a.width, a.dpre_weight,
                                                  a.dscale, a.dpost_weight,
                                                  a.param_dtype == RC_F32);
    return launched("k_norm_weight_sum");
  });
}
