// Norms of queries and keys, each head on its own, with the rotation by position in the
// same pass.  For a row x of one head
//   y = x r w,  r = 1 / sqrt(mean(x^2) + eps)  (or the sum's, or 1),
//   pair i of y turned by position * inv_freq[i]: (a, b) -> (a cos - b sin, b cos + a sin).
// Backward: the gradient turned back gives e (of y); with u = x r,
//   dw = sum e u,   dx = r (e w - u mean(e w u))  (or the sum, or no second part).
//
// A few operations for each value moved: bound by memory.  A lane holds eight pairs of a
// row (two loads of eight channels), L lanes a row, and goes from head to head of its
// token, so that the angles are evaluated once for the heads of a thread.  32768 tokens of 32 + 8 heads
// of 128 in bf16: forward (671 MB) 154 us, 4.4 TB/s, backward (1007 MB) 240 us, 4.2 TB/s; without the
// next head's loads in flight 178 and 305.  48 single tokens: 6 us, a chain of loads, angles and stores.
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int kMaxChannels = 256, kThreads = 256, kPairs = 8;

struct QkParams {
  rc_qk_args a;
  int32_t each[2];                          // heads of a thread, of q and of k
  int32_t groups[2];                        // threads' groups of heads
  int32_t blocks;                           // workgroups over the tokens
  float* partial;                           // [blocks * (groups[0] + groups[1])][channels]
};

// A lane's channels: c[0] .. and c[1] .., n[0] and n[1] of them.
struct Unit {
  int c[2], n[2], pair;                     // pair: its first rotated pair, or -1
  __device__ Unit(const rc_qk_args& a, int u) {
    const int m = a.rotated / 2, turned = (m + kPairs - 1) / kPairs;
    pair = u < turned ? u * kPairs : -1;
    int end[2];
    if (pair < 0) {
      c[0] = a.rotated + (u - turned) * 2 * kPairs;
      c[1] = c[0] + kPairs;
      end[0] = end[1] = a.channels;
    } else if (a.interleaved) {
      c[0] = 2 * pair;
      c[1] = c[0] + kPairs;
      end[0] = end[1] = a.rotated;
    } else {
      c[0] = pair;
      c[1] = m + pair;
      end[0] = m;
      end[1] = a.rotated;
    }
#pragma unroll
    for (int i = 0; i < 2; i++) n[i] = min(max(end[i] - c[i], 0), kPairs);
  }
};

// cos and sin of position * inv_freq for a unit's pairs; the angle in turns and its fraction
// in 64 bits.  A unit that is not turned has (1, 0).
__device__ __forceinline__ void angles(const rc_qk_args& a, const Unit& u, int b, int t,
                                       float (&cos)[kPairs], float (&sin)[kPairs]) {
  const int m = a.rotated / 2;
  const double at =
      a.positions && u.pair >= 0 ? (double)a.positions[b * a.positions_batch + t * a.positions_time]
                                 : (double)t;
#pragma unroll
  for (int i = 0; i < kPairs; i++) {
    cos[i] = 1.f;
    sin[i] = 0.f;
    if (u.pair >= 0 && u.pair + i < m) {
      const double turns = at * ((double)a.inv_freq[u.pair + i] * 0.15915494309189533577);
      const float part = (float)(turns - __builtin_rint(turns));
      sincospif(2.f * part, &sin[i], &cos[i]);
    }
  }
}

// The unit's pairs turned by the angles (back: by their negatives).
__device__ __forceinline__ void turn(bool interleaved, bool back, const float (&cos)[kPairs],
                                     const float (&sin)[kPairs], float (&x)[2][kPairs]) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < kPairs; i++) {
      float &p = x[i / 4][i % 4 * 2], &q = x[i / 4][i % 4 * 2 + 1];
      const float s = back ? -sin[i] : sin[i], a = p * cos[i] - q * s;
      q = q * cos[i] + p * s;
      p = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPairs; i++) {
      const float s = back ? -sin[i] : sin[i], a = x[0][i] * cos[i] - x[1][i] * s;
      x[1][i] = x[1][i] * cos[i] + x[0][i] * s;
      x[0][i] = a;
    }
  }
}

template <class T>
__device__ __forceinline__ void load_unit(const T* row, const Unit& u, bool on, float (&x)[2][kPairs]) {
#pragma unroll
  for (int i = 0; i < 2; i++) load_vec<kPairs>(row + (u.n[i] ? u.c[i] : 0), on ? u.n[i] : 0, x[i]);
}
// The same as T, whole loads at addresses inside the row: what is past a unit's channels, or
// not `on`, is dropped by `values`.  (A row shorter than a load is loaded one by one.)
template <class T>
struct Raw {
  typedef T TV __attribute__((ext_vector_type(kPairs)));
  TV v[2];
  __device__ void load(const T* row, const Unit& u, int channels) {
#pragma unroll
    for (int i = 0; i < 2; i++) __builtin_memcpy(&v[i], row + min(u.c[i], channels - kPairs), sizeof(TV));
  }
  __device__ void values(const Unit& u, bool on, float (&x)[2][kPairs]) const {
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int e = 0; e < kPairs; e++) x[i][e] = on && e < u.n[i] ? (float)v[i][e] : 0.f;
  }
};
template <class T>
__device__ __forceinline__ void store_unit(T* row, const Unit& u, const float (&x)[2][kPairs]) {
#pragma unroll
  for (int i = 0; i < 2; i++)
    if (u.n[i]) store_vec<kPairs>(row + u.c[i], u.n[i], x[i]);
}
template <class T>
__device__ __forceinline__ void load_unit_weight(const void* w, bool f32, const Unit& u,
                                                 float (&x)[2][kPairs]) {
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int e = 0; e < kPairs; e++)
      x[i][e] = w && e < u.n[i] ? load_param<T>(w, u.c[i] + e, f32) : 1.f;
}

__device__ __forceinline__ float norm_of(const rc_qk_args& a, float square) {
  if (a.norm == RC_QK_NONE) return 1.f;
  return __builtin_amdgcn_rsqf((a.norm == RC_QK_RMS ? square / (float)a.channels : square) + a.eps);
}

// A thread's place: tensor (0 q, 1 k), heads first .. last - 1, workgroup over the tokens.
struct Place {
  int which, first, last, block;
  __device__ Place(const QkParams& p) {
    int g = blockIdx.x / p.blocks;
    block = blockIdx.x % p.blocks;
    which = g >= p.groups[0];
    if (which) g -= p.groups[0];
    first = g * p.each[which];
    last = min(first + p.each[which], which ? p.a.key_heads : p.a.heads);
  }
};

// AHEAD: every unit is whole loads, and the next head's are in flight during this one's work.
template <class T, int L, bool AHEAD>
__global__ __launch_bounds__(kThreads) void k_qk_forward(QkParams p) {
  const rc_qk_args& a = p.a;
  const Place at(p);
  const Unit u(a, threadIdx.x % L);
  const rc_heads& in = at.which ? a.k : a.q;
  const rc_heads& out = at.which ? a.k_out : a.q_out;
  float w[2][kPairs];
  load_unit_weight<T>(at.which ? a.k_weight : a.q_weight, a.param_dtype == RC_F32, u, w);
  const int64_t tokens = (int64_t)a.batch * a.length;
  for (int64_t i = (int64_t)at.block * (kThreads / L) + threadIdx.x / L; i < tokens;
       i += (int64_t)p.blocks * (kThreads / L)) {
    const int b = (int)(i / a.length), t = (int)(i % a.length);
    const bool live = !a.lengths || t < a.lengths[b];
    Raw<T> next;
    if (AHEAD) next.load(at_head<T>(in, b, t, at.first), u, a.channels);
    float cos[kPairs], sin[kPairs];
    angles(a, u, b, t, cos, sin);
    for (int h = at.first; h < at.last; h++) {
      float x[2][kPairs], s = 0.f;
      if (AHEAD) {
        next.values(u, live, x);
        next.load(at_head<T>(in, b, t, min(h + 1, at.last - 1)), u, a.channels);
      } else {
        load_unit(at_head<T>(in, b, t, h), u, live, x);
      }
#pragma unroll
      for (int j = 0; j < 2 * kPairs; j++) s = fmaf(x[j / kPairs][j % kPairs], x[j / kPairs][j % kPairs], s);
      const float r = norm_of(a, lane_sum<L>(s));
#pragma unroll
      for (int j = 0; j < 2 * kPairs; j++)
        x[j / kPairs][j % kPairs] *= r * w[j / kPairs][j % kPairs];
      turn(a.interleaved, false, cos, sin, x);
      if (!live) {
#pragma unroll
        for (int j = 0; j < 2 * kPairs; j++) x[j / kPairs][j % kPairs] = 0.f;
      }
      store_unit(at_head<T>(out, b, t, h), u, x);
    }
  }
}

template <class T, int L, bool AHEAD>
__global__ __launch_bounds__(kThreads) void k_qk_backward(QkParams p) {
  const rc_qk_args& a = p.a;
  __shared__ float sums[kThreads][2 * kPairs];
  const Place at(p);
  const Unit u(a, threadIdx.x % L);
  const rc_heads& in = at.which ? a.k : a.q;
  const rc_heads& dout = at.which ? a.dk_out : a.dq_out;
  const rc_heads& dx = at.which ? a.dk : a.dq;
  float w[2][kPairs], dw[2][kPairs];
  load_unit_weight<T>(at.which ? a.k_weight : a.q_weight, a.param_dtype == RC_F32, u, w);
#pragma unroll
  for (int j = 0; j < 2 * kPairs; j++) dw[j / kPairs][j % kPairs] = 0.f;
  const int64_t tokens = (int64_t)a.batch * a.length;
  for (int64_t i = (int64_t)at.block * (kThreads / L) + threadIdx.x / L; i < tokens;
       i += (int64_t)p.blocks * (kThreads / L)) {
    const int b = (int)(i / a.length), t = (int)(i % a.length);
    const bool live = !a.lengths || t < a.lengths[b];
    const rc_heads& given = dout.data ? dout : in;
    Raw<T> next_x, next_e;
    if (AHEAD) {
      next_x.load(at_head<T>(in, b, t, at.first), u, a.channels);
      next_e.load(at_head<T>(given, b, t, at.first), u, a.channels);
    }
    float cos[kPairs], sin[kPairs];
    angles(a, u, b, t, cos, sin);
    for (int h = at.first; h < at.last; h++) {
      float x[2][kPairs], e[2][kPairs], s = 0.f, d = 0.f;
      if (AHEAD) {
        next_x.values(u, live, x);
        next_e.values(u, live && dout.data, e);
        next_x.load(at_head<T>(in, b, t, min(h + 1, at.last - 1)), u, a.channels);
        next_e.load(at_head<T>(given, b, t, min(h + 1, at.last - 1)), u, a.channels);
      } else {
        load_unit(at_head<T>(in, b, t, h), u, live, x);
        load_unit(at_head<T>(given, b, t, h), u, live && dout.data, e);
      }
      turn(a.interleaved, true, cos, sin, e);
#pragma unroll
      for (int j = 0; j < 2 * kPairs; j++) {
        const float v = x[j / kPairs][j % kPairs];
        s = fmaf(v, v, s);
        d = fmaf(e[j / kPairs][j % kPairs] * w[j / kPairs][j % kPairs], v, d);
      }
      // (without eps a padded token's zeros would have no norm, and no share of the weights' sums)
      const float size = lane_sum<L>(s), r = live ? norm_of(a, size) : 0.f;
      d = lane_sum<L>(d) * r;                          // e w . u
      if (a.norm == RC_QK_RMS) d /= (float)a.channels;
      if (a.norm == RC_QK_NONE) d = 0.f;
#pragma unroll
      for (int j = 0; j < 2 * kPairs; j++) {
        float &v = x[j / kPairs][j % kPairs], g = e[j / kPairs][j % kPairs];
        v *= r;
        dw[j / kPairs][j % kPairs] = fmaf(g, v, dw[j / kPairs][j % kPairs]);
        v = live ? r * (g * w[j / kPairs][j % kPairs] - v * d) : 0.f;
      }
      store_unit(at_head<T>(dx, b, t, h), u, x);
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int j = 0; j < 2 * kPairs; j++) sums[threadIdx.x][j] = dw[j / kPairs][j % kPairs];
  __syncthreads();
  for (int i = threadIdx.x; i < L * 2 * kPairs; i += kThreads) {
    const int lane = i / (2 * kPairs), j = i % (2 * kPairs);
    const Unit v(a, lane);
    if (j % kPairs >= v.n[j / kPairs]) continue;
    float s = 0.f;
    for (int k = lane; k < kThreads; k += L) s += sums[k][j];
    p.partial[(int64_t)blockIdx.x * a.channels + v.c[j / kPairs] + j % kPairs] = s;
  }
}

// The weights' gradients: sums over workgroups, first those of q, then those of k.
template <class T>
__global__ __launch_bounds__(256) void k_qk_weights(QkParams p) {
  __shared__ float lds[256];
  const rc_qk_args& a = p.a;
  const int cols = (a.channels + kSumCols - 1) / kSumCols, which = blockIdx.x / cols;
  const int c = blockIdx.x % cols * kSumCols + threadIdx.x % kSumCols;
  const int64_t first = which ? (int64_t)p.blocks * p.groups[0] : 0;
  const float s = column_sum(p.partial + first * a.channels, (int64_t)p.blocks * p.groups[which],
                             a.channels, c, lds);
  void* to = which ? a.dk_weight : a.dq_weight;
  if (to && threadIdx.x < kSumCols && c < a.channels)
    store_param<T>(to, c, a.param_dtype == RC_F32, s);
}

// ------------------------------------------------------------------ host side

int units_of(const rc_qk_args& a) {
  const int m = a.rotated / 2;
  return (int)(cdiv(m, kPairs) + cdiv(a.channels - a.rotated, 2 * kPairs));
}
int lanes_of(const rc_qk_args& a) {
  int l = 1;
  while (l < units_of(a)) l *= 2;
  return l;
}

int check(const rc_qk_args* a) {
  if (!a || !dtype_ok(a->dtype) || !param_ok(a->param_dtype, a->dtype) || a->norm < RC_QK_NONE ||
      a->norm > RC_QK_L2 || a->batch < 0 || a->length < 0 || a->length > kMaxExtent || a->heads < 0 ||
      a->key_heads < 0 || a->channels < 1 || a->channels > kMaxChannels || a->rotated < 0 ||
      a->rotated > a->channels || a->rotated % 2 || (a->rotated && !a->inv_freq))
    return RC_E_ARG;
  return RC_OK;
}
bool empty(const rc_qk_args& a) { return !a.batch || !a.length || (!a.heads && !a.key_heads); }

// Heads of a thread: as many as leave 2^18 threads, four waves a SIMD.  Backward, whose
// workgroups leave sums, no more workgroups than that either.
int plan(const rc_qk_args& a, bool back, QkParams* p) {
  *p = {};
  p->a = a;
  const int L = lanes_of(a), heads[2] = {a.heads, a.key_heads};
  const int64_t rows = kThreads / L, wanted = 1024, most = (int64_t)1 << 22;
  int64_t blocks = std::min(cdiv((int64_t)a.batch * a.length, rows), most);
  for (int i = 0; i < 2; i++) {
    const int64_t each = std::min<int64_t>(
        std::max<int64_t>(blocks * ((int64_t)a.heads + a.key_heads) / wanted, 1), 16);
    p->each[i] = (int32_t)std::min<int64_t>(each, std::max(heads[i], 1));
    p->groups[i] = (int32_t)cdiv(heads[i], p->each[i]);
  }
  const int64_t groups = (int64_t)p->groups[0] + p->groups[1];
  if (groups > most) return RC_E_OVERFLOW;
  blocks = std::min(blocks, std::max<int64_t>((back ? 2 * wanted : most) / groups, 1));
  p->blocks = (int32_t)blocks;
  return RC_OK;
}
uint64_t workspace_of(const QkParams& p) {
  if (!p.a.dq_weight && !p.a.dk_weight) return 0;
  return (uint64_t)p.blocks * (p.groups[0] + p.groups[1]) * p.a.channels * sizeof(float);
}

// Whether every unit that has channels has whole loads of them.
bool whole_units(const rc_qk_args& a) {
  return a.channels >= kPairs && a.channels % kPairs == 0 &&
         a.rotated % (a.interleaved ? kPairs : 2 * kPairs) == 0;
}

template <class F>
int by_lanes(int l, F&& f) {
  if (l <= 2) return f(std::integral_constant<int, 2>{});
  if (l == 4) return f(std::integral_constant<int, 4>{});
  if (l == 8) return f(std::integral_constant<int, 8>{});
  if (l == 16) return f(std::integral_constant<int, 16>{});
  return f(std::integral_constant<int, 32>{});
}

}  // namespace

extern "C" int rc_qk_forward(const rc_qk_args* args, void* stream) {
  if (int e = check(args)) return e;
  const rc_qk_args& a = *args;
  if (empty(a)) return RC_OK;
  if ((a.heads && (!a.q.data || !a.q_out.data)) || (a.key_heads && (!a.k.data || !a.k_out.data)))
    return RC_E_ARG;
  QkParams p;
  if (int e = plan(a, false, &p)) return e;
  const unsigned grid = (unsigned)p.blocks * (p.groups[0] + p.groups[1]);
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_lanes(lanes_of(a), [&](auto l) {
      constexpr int L = decltype(l)::value;
      if (whole_units(a))
        k_qk_forward<T, L, true><<<grid, kThreads, 0, (hipStream_t)stream>>>(p);
      else
        k_qk_forward<T, L, false><<<grid, kThreads, 0, (hipStream_t)stream>>>(p);
      return launched("k_qk_forward");
    });
  });
}

extern "C" int rc_qk_backward_workspace(const rc_qk_args* args, uint64_t* bytes) {
  if (int e = check(args)) return e;
  if (!bytes) return RC_E_ARG;
  *bytes = 0;
  if (empty(*args)) return RC_OK;
  QkParams p;
  if (int e = plan(*args, true, &p)) return e;
  *bytes = workspace_of(p);
  return RC_OK;
}

extern "C" int rc_qk_backward(const rc_qk_args* args, void* stream) {
  if (int e = check(args)) return e;
  const rc_qk_args& a = *args;
  if ((a.dq_weight && !a.q_weight) || (a.dk_weight && !a.k_weight) || !float_aligned(a.workspace))
    return RC_E_ARG;
  QkParams p = {};
  if (empty(a)) {                                      // no rows: the weights' gradients are 0
    p.a = a;
    if (!a.dq_weight && !a.dk_weight) return RC_OK;
  } else {
    if ((a.heads && (!a.q.data || !a.dq.data)) || (a.key_heads && (!a.k.data || !a.dk.data)))
      return RC_E_ARG;
    if (int e = plan(a, true, &p)) return e;
    const uint64_t need = workspace_of(p);
    if (need && (!a.workspace || a.workspace_bytes < need)) return RC_E_SCRATCH;
    if (need) p.partial = static_cast<float*>(a.workspace);
  }
  const unsigned grid = (unsigned)p.blocks * (p.groups[0] + p.groups[1]);
  const hipStream_t s = (hipStream_t)stream;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (grid) {
      const int e = by_lanes(lanes_of(a), [&](auto l) {
        constexpr int L = decltype(l)::value;
        if (whole_units(a))
          k_qk_backward<T, L, true><<<grid, kThreads, 0, s>>>(p);
        else
          k_qk_backward<T, L, false><<<grid, kThreads, 0, s>>>(p);
        return launched("k_qk_backward");
      });
      if (e) return e;
    }
    if (!a.dq_weight && !a.dk_weight) return (int)RC_OK;
    k_qk_weights<T><<<(unsigned)(2 * cdiv(a.channels, kSumCols)), 256, 0, s>>>(p);
    return launched("k_qk_weights");
  });
}
