// Gated delta rule, gradients; delta.h has the formulas.
#include "delta.h"

using namespace rcdelta;

namespace {

// Backward through the states, from the last chunk to the first, as k_delta_forward goes.
template <class T, int KT, class G, bool WIDE>
__global__ __launch_bounds__(G::THREADS, (kTogether<T, KT, G>)) void k_delta_states_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, STEPS = KT / G::R, STAGES = kStages<T, KT, G>;
  __shared__ Stage<T, KT, G> stages[STAGES];
  __shared__ Parts<G, G::R == 1 ? 0 : 2> parts;
  const Walk<G> at(a);
  const int end = at.end, row = at.row, first_row = at.part * STEPS * 32, lane = threadIdx.x % 64;
  const int64_t size = (int64_t)a.key * a.value, first = (int64_t)at.bh * p.chunks;
  const bool keeps = at.col < columns_of(a.value);
  if (threadIdx.x >= G::WORKERS) {
    load_chunks<T, KT, G, WIDE, true>(p, at, a.do_, stages);
    return;
  }
  f32x4 E[2 * STEPS];
  load_state(a.dstate_out ? a.dstate_out + at.bh * size : nullptr, a, at.col, first_row, E);
  for (int i = 0; i < at.chunks; i++) {
    const int chunk = at.chunks - 1 - i, t0 = chunk * kChunk, live = min(end - t0, kChunk);
    const auto& stage = stages[i % STAGES];
    __syncthreads();
    const Chunk& c = stage.c;
    if (keeps)
      keep_state(p.dstates + (first + chunk) * (columns_of(a.value) * 32 * KT), 32 * KT, at.col, first_row, E);
    f32x4 dw[2], dr[2], g[2];
#pragma unroll
    for (int m = 0; m < 2; m++) dw[m] = dr[m] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      const Pieces<3> state = operand<3>(E[2 * s], E[2 * s + 1]);
#pragma unroll
      for (int m = 0; m < 2; m++) mul(dw[m], stage.k.rows(m, at.part * STEPS + s), state);
    }
    if constexpr (G::R > 1) {
#pragma unroll
      for (int m = 0; m < 2; m++) parts.at[m][at.part][at.wave][lane] = dw[m];
    }
    // read, and computed, before the barrier, which nothing is moved over
    f32x4 since[2], beta[2], from_o[2];
#pragma unroll
    for (int m = 0; m < 2; m++) {
      since[m] = *(const f32x4*)&c.since[16 * m + row];
      beta[m] = *(const f32x4*)&c.beta[16 * m + row];
      from_o[m] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 4; e++) g[m][e] = (float)stage.x[16 * m + row + e][at.col - at.col0];
    }
    const Pieces<N> gs = operand<N>(g[0], g[1]);
    const Pieces<3> t[2] = {pieces(c.t[0]), pieces(c.t[1])};
#pragma unroll
    for (int m = 0; m < 2; m++) mul(from_o[m], pieces(c.p[m]), gs);
    const Pieces<3> gos = operand<3>(g[0] * (a.scale * since[0]), g[1] * (a.scale * since[1]));
    const float whole = c.since[kChunk - 1];
    f32x4 left[2] = {*(const f32x4*)&c.left[row], *(const f32x4*)&c.left[16 + row]};
#pragma unroll
    for (int m = 0; m < 2 * STEPS; m++) {
      E[m] *= whole;
      mul(E[m], stage.q.columns(at.part * 2 * STEPS + m), gos);
    }
    if constexpr (G::R > 1) {
      __syncthreads();
#pragma unroll
      for (int m = 0; m < 2; m++) dw[m] = parts.sum(m, at.wave);
    }
#pragma unroll
    for (int m = 0; m < 2; m++) dw[m] = dw[m] * left[m] + from_o[m];
    const Pieces<3> dws = operand<3>(dw[0], dw[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) mul(dr[m], t[m], dws);
    const Pieces<3> drs = operand<3>(-since[0] * beta[0] * dr[0], -since[1] * beta[1] * dr[1]);
#pragma unroll
    for (int m = 0; m < 2 * STEPS; m++) mul(E[m], stage.k.columns(at.part * 2 * STEPS + m), drs);
#pragma unroll
    for (int m = 0; m < 2; m++) {
      if (G::R > 1 && at.part != m) continue;          // outputs: tile m by part m
      if (keeps)
        *(f32x4*)(p.written + ((first + chunk) * columns_of(a.value) + at.col) * kChunk + 16 * m + row) = dr[m];
      dr[m] *= beta[m];
      T* dv = at_head<T>(a.dv, at.b, t0 + 16 * m, at.h) + row * a.dv.time + at.col;
      if (at.on) {
        if (live == kChunk) {
#pragma unroll
          for (int e = 0; e < 4; e++) dv[e * a.dv.time] = (T)dr[m][e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (16 * m + row + e < live) dv[e * a.dv.time] = (T)dr[m][e];
        }
      }
    }
    if (STAGES == 1) __syncthreads();
  }
  if (a.dstate_in) store_state(a.dstate_in + at.bh * size, a, at.col, first_row, E);
  if (at.on && at.part == 0) {
    T* dv = at_head<T>(a.dv, at.b, 0, at.h) + at.col;
    for (int t = end + row / 4; t < a.length; t += 4) dv[t * a.dv.time] = (T)0.f;
  }
}

// The gradients of one chunk's inputs from the states before it and the gradients of those after
// it, head by head of those that share a key head.  Four waves; each takes some of the
// key's tiles of 16 channels, and reads its part of the states straight into operands.
template <class T, int KT>
__global__ __launch_bounds__(256) void k_delta_inputs_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, NT = (2 * KT + 3) / 4;
  __shared__ Tokens<KT, N> k, q;
  __shared__ Tokens<1, N> od;                         // rows: tokens
  __shared__ Tokens<1, 3> rd, wr;                     // rows: columns of the state
  __shared__ float M[kChunk][kChunk + 4], Q[kChunk][kChunk + 4];   // M, N of the formulas
  __shared__ double sums[kChunk];
  __shared__ float dots[4][4][kChunk], inner[4], dot_v[kChunk], beta[kChunk];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, row = lane / 16 * 4;
  const int groups = a.heads / p.each, bg = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  const int b = bg / groups, group = bg % groups, hk = group * p.each / (a.heads / a.key_heads);
  const int t0 = chunk * kChunk, live = min(length_of(a, b) - t0, kChunk), here = min(a.length - t0, kChunk);
  const int cols = columns_of(a.value);
  // dq and dk of the key head, or their parts in 32 bits where other workgroups have more
  const auto store = [&](int which, int t, int c, float x) {
    if (groups == a.key_heads)
      at_head<T>(which ? a.dk : a.dq, b, t0 + t, hk)[c] = (T)x;
    else
      p.partial[((((int64_t)which * a.batch + b) * a.length + t0 + t) * groups + group) * a.key + c] = x;
  };
  if (live <= 0) {
    for (int i = tid; i < here * a.key; i += 256) {
      store(0, i / a.key, i % a.key, 0.f);
      store(1, i / a.key, i % a.key, 0.f);
    }
    for (int i = tid; i < here * p.each; i += 256) {
      const int64_t at = ((int64_t)b * a.length + t0 + i / p.each) * a.heads + group * p.each + i % p.each;
      if (a.dg) a.dg[at] = 0.f;
      a.dbeta[at] = 0.f;
    }
    return;
  }
  k.load(at_head<T>(a.k, b, t0, hk), a.k.time, live, a.key, tid, 256);
  q.load(at_head<T>(a.q, b, t0, hk), a.q.time, live, a.key, tid, 256);
  f32x4 dq[2][NT], dk[2][NT];
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int n = 0; n < NT; n++) dq[m][n] = dk[m][n] = f32x4{0, 0, 0, 0};
  const int ti = wave > 0, tj = wave == 2;            // waves 0 to 2: tile (ti, tj) of M and N
  for (int h = group * p.each; h < (group + 1) * p.each; h++) {
    const int64_t pair = ((int64_t)b * a.heads + h) * p.chunks + chunk;
    const float* S = p.states + pair * cols * (32 * KT);
    const float* E = p.dstates + pair * cols * (32 * KT);
    const float* w_at = p.kept_written + pair * cols * kChunk;
    const float* r_at = p.written + pair * cols * kChunk;
    __syncthreads();
    if (tid < 64) {
      const double G = sum_of_g(a, b, h, t0, live);
      if (tid < kChunk) {
        sums[tid] = G;
        beta[tid] = tid < live ? at_token(a.beta, b, t0 + tid, h) : 0.f;
      }
    }
    f32x4 xq[2][NT], xr[2][NT], xw[2][NT], m_tile = {0, 0, 0, 0}, n_tile = {0, 0, 0, 0};
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int n = 0; n < NT; n++) xq[m][n] = xr[m][n] = xw[m][n] = f32x4{0, 0, 0, 0};
    float es = 0.f;
    for (int c0 = 0; c0 < cols; c0 += 32) {
      __syncthreads();
      if (tid < 128) {
        const int t = tid / 4, c = c0 + tid % 4 * 8, n = a.value - c;
        float x[8];
        load_vec<8>(at_head<T>(a.do_, b, t0 + (t < live ? t : 0), h) + (n > 0 ? c : 0), t < live ? n : 0, x);
        od.put(t, tid % 4 * 8, x);
      } else {
        const int c = (tid - 128) / 4, t = tid % 4 * 8;
        float x[8];
        load_vec<8>(w_at + (c0 + c) * kChunk + t, 8, x);
        wr.put(c, t, x);
        load_vec<8>(r_at + (c0 + c) * kChunk + t, 8, x);
        rd.put(c, t, x);
      }
      float x[NT][8], y[NT][8];
#pragma unroll
      for (int n = 0; n < NT; n++) {
        const int tile = min(wave * NT + n, 2 * KT - 1);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const int at = (c0 + e / 4 * 16 + row + e % 4) * (32 * KT) + 16 * tile + col;
          x[n][e] = S[at];
          y[n][e] = E[at];
        }
      }
      __syncthreads();
      const Pieces<N> os[2] = {od.rows(0, 0), od.rows(1, 0)};
      const Pieces<3> rs[2] = {rd.columns(0), rd.columns(1)}, ws[2] = {wr.columns(0), wr.columns(1)};
#pragma unroll
      for (int n = 0; n < NT; n++) {
        if (wave * NT + n < 2 * KT)
#pragma unroll
          for (int e = 0; e < 8; e++) es = fmaf(x[n][e], y[n][e], es);
        const Pieces<3> ss = split<3>(x[n]), ds = split<3>(y[n]);
#pragma unroll
        for (int m = 0; m < 2; m++) {
          mul(xq[m][n], os[m], ss);
          mul(xr[m][n], rs[m], ss);
          mul(xw[m][n], ws[m], ds);
        }
      }
      if (wave < 3) {
        mul(m_tile, ti ? os[1] : os[0], tj ? ws[1] : ws[0]);
        mul(n_tile, ti ? rs[1] : rs[0], tj ? ws[1] : ws[0]);
      }
    }
    // dR . v, eight threads a token
    {
      const int t = tid / 8;
      float s = 0.f;
      if (t < live) {
        const T* v = at_head<T>(a.v, b, t0 + t, h);
        for (int c = tid % 8; c < a.value; c += 8) s = fmaf(r_at[c * kChunk + t], (float)v[c], s);
      }
      s = lane_sum<8>(s);
      if (tid % 8 == 0) dot_v[t] = s;
    }
    if (wave < 3) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int i = 16 * ti + row + e, j = 16 * tj + col;
        const float d = exp_of(sums[i] - sums[j]);
        M[i][j] = j <= i ? a.scale * d * m_tile[e] : 0.f;
        Q[i][j] = j < i ? d * n_tile[e] : 0.f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; e++) M[row + e][16 + col] = Q[row + e][16 + col] = 0.f;
    }
    es = lane_sum<64>(es);
    if (lane == 0) inner[wave] = es;
    __syncthreads();
    const double last = sums[kChunk - 1];
    Pieces<3> m_rows[2], n_rows[2], m_cols[2], n_cols[2];
#pragma unroll
    for (int m = 0; m < 2; m++) {
      float x[4][8];
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int i = 16 * m + col, j = e / 4 * 16 + row + e % 4;
        x[0][e] = M[i][j];
        x[1][e] = Q[i][j];
        x[2][e] = M[j][i];
        x[3][e] = -beta[j] * Q[j][i];
      }
      m_rows[m] = split<3>(x[0]);
      n_rows[m] = split<3>(x[1]);
      m_cols[m] = split<3>(x[2]);
      n_cols[m] = split<3>(x[3]);
    }
    float dot[4][2][4];
#pragma unroll
    for (int d = 0; d < 4; d++)
#pragma unroll
      for (int m = 0; m < 2; m++)
#pragma unroll
        for (int e = 0; e < 4; e++) dot[d][m][e] = 0.f;
    float since[2][4], left[2][4];
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        since[m][e] = exp_of(sums[16 * m + row + e]);
        left[m][e] = exp_of(last - sums[16 * m + row + e]);
      }
#pragma unroll
    for (int n = 0; n < NT; n++) {
      const int tile = wave * NT + n, c = 16 * tile + col;
      if (tile >= 2 * KT) break;
      const Pieces<N> kc = k.columns(tile), qc = q.columns(tile);
#pragma unroll
      for (int m = 0; m < 2; m++) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
          xq[m][n][e] *= a.scale * since[m][e];
          xr[m][n][e] *= since[m][e];
          xw[m][n][e] *= left[m][e];
          dot[3][m][e] = fmaf(k.value(16 * m + row + e, c), xw[m][n][e], dot[3][m][e]);
        }
        mul(xq[m][n], m_rows[m], kc);
        mul(xr[m][n], n_rows[m], kc);
        mul(xw[m][n], m_cols[m], qc);
        mul(xw[m][n], n_cols[m], kc);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const int t = 16 * m + row + e;
          const float kv = k.value(t, c), qv = q.value(t, c);
          const float read = -beta[t] * xr[m][n][e];
          dot[0][m][e] = fmaf(qv, xq[m][n][e], fmaf(kv, read, dot[0][m][e]));
          dot[1][m][e] = fmaf(kv, xw[m][n][e], dot[1][m][e]);
          dot[2][m][e] = fmaf(kv, xr[m][n][e], dot[2][m][e]);
          dq[m][n][e] += xq[m][n][e];
          dk[m][n][e] += read + xw[m][n][e];
        }
      }
    }
#pragma unroll
    for (int d = 0; d < 4; d++)
#pragma unroll
      for (int m = 0; m < 2; m++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float s = lane_sum<16>(dot[d][m][e]);
          if (col == 0) dots[wave][d][16 * m + row + e] = s;
        }
    __syncthreads();
    if (tid < kChunk) {
      double s[4];
#pragma unroll
      for (int d = 0; d < 4; d++)
        s[d] = (double)dots[0][d][tid] + dots[1][d][tid] + dots[2][d][tid] + dots[3][d][tid];
      double dG = s[0] - s[1], total = s[3];
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const double after = __shfl_down(dG, d, 32);
        if (tid + d < 32) dG += after;
        total += __shfl_xor(total, d, 32);
      }
      total += (double)exp_of(last) * ((double)inner[0] + inner[1] + inner[2] + inner[3]);
      const int64_t at = ((int64_t)b * a.length + t0 + tid) * a.heads + h;
      if (tid < here) {
        if (a.dg) a.dg[at] = tid < live ? (float)(dG + total) : 0.f;
        a.dbeta[at] = tid < live ? (float)(dot_v[tid] - s[2]) : 0.f;
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; n++) {
    const int tile = wave * NT + n, c = 16 * tile + col;
    if (tile >= 2 * KT || c >= a.key) break;
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int t = 16 * m + row + e;
        if (t < here) {
          store(0, t, c, dq[m][n][e]);
          store(1, t, c, dk[m][n][e]);
        }
      }
  }
}

// dq and dk of key heads whose heads several workgroups had: the sums of their parts.
template <class T>
__global__ __launch_bounds__(256) void k_delta_shared_heads(DeltaParams p, int64_t n) {
  const rc_delta_args& a = p.a;
  const int parts = a.heads / p.each / a.key_heads;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * n) return;
  const int which = i >= n;
  const int64_t e = i - which * n;
  const int c = (int)(e % a.key);
  const int64_t row = e / a.key;                      // (b, t, key head)
  const float* from = p.partial + which * n * parts + row * parts * a.key + c;
  float s = 0.f;
  for (int j = 0; j < parts; j++) s += from[(int64_t)j * a.key];
  const int64_t token = row / a.key_heads;
  at_head<T>(which ? a.dk : a.dq, token / a.length, token % a.length, row % a.key_heads)[c] = (T)s;
}

}  // namespace

extern "C" int rc_delta_backward(const rc_delta_args* args, void* stream) {
  if (int e = check(args)) return e;
  const rc_delta_args& a = *args;
  if (empty(a)) return RC_OK;
  if (a.length && (!a.q.data || !a.k.data || !a.v.data || !a.beta.data || !a.do_.data || !a.dq.data ||
                   !a.dk.data || !a.dv.data || !a.dbeta || !a.kept || !a.dg != !a.g.data))
    return RC_E_ARG;
  if (!float_aligned(a.kept) || !float_aligned(a.workspace)) return RC_E_ARG;
  if (int e = fits(a)) return e;
  if (a.length && (!a.workspace || a.workspace_bytes < workspace_of(a, true))) return RC_E_SCRATCH;
  const hipStream_t s = (hipStream_t)stream;
  DeltaParams p = params(a);
  const int64_t pairs = pairs_of(a);
  p.each = heads_together(a);
  p.kept_written = a.kept + state_floats(a);
  p.dstates = reinterpret_cast<float*>(p.prepared + pairs);
  p.written = p.dstates + state_floats(a);
  p.partial = p.written + pairs * columns_of(a.value) * kChunk;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_key(a.key, [&](auto kt) {
      constexpr int KT = decltype(kt)::value;
      if (int e = prepare<T, KT, true>(p, s)) return e;
      const int e = by_width(a, [&](auto wide) {
        using G = ShapeOf<KT>;
        k_delta_states_back<T, KT, G, decltype(wide)::value><<<walks_of<G>(a), G::THREADS, 0, s>>>(p);
        return launched("k_delta_states_back");
      });
      if (e) return e;
      if (!p.chunks) return (int)RC_OK;
      k_delta_inputs_back<T, KT><<<(unsigned)(pairs / p.each), 256, 0, s>>>(p);
      if (int e = launched("k_delta_inputs_back")) return e;
      if (a.heads / p.each == a.key_heads) return (int)RC_OK;
      const int64_t n = (int64_t)a.batch * a.length * a.key_heads * a.key;
      k_delta_shared_heads<T><<<(unsigned)cdiv(2 * n, 256), 256, 0, s>>>(p, n);
      return launched("k_delta_shared_heads");
    });
  });
}
