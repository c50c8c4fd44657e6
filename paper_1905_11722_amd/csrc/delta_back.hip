// Gated delta rule, gradients; delta.h has the formulas.
#include "delta.h"

using namespace rcdelta;

namespace {

// Backward through the states, from the last chunk to the first, as k_delta_forward goes.
template <class T, int KT, class G, bool WIDE>
__global__ __launch_bounds__(G::THREADS, (kTogether<T, KT, G>)) void k_delta_states_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, STEPS = KT / G::R, STAGES = kStages<T, KT, G>;
  constexpr int EVERY = block_of(N, 32 * KT) / kChunk;
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
    if (keeps && (i == 0 || chunk % EVERY == EVERY - 1))
      keep_state(p.dstates + ((int64_t)at.bh * p.blocks + chunk / EVERY) * (columns_of(a.value) * 32 * KT),
                 32 * KT, at.col, first_row, E);
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

// Tile (i, j), j <= i, of a lower triangle's tiles row by row.
struct Tile {
  int i, j;
  __device__ Tile(int n) {
    i = (n >= 1) + (n >= 3) + (n >= 6);
    j = n - i * (i + 1) / 2;
  }
};

// The gradients of a block's inputs from the state before it and the gradient of the one after
// it, head by head of those that share a key head.  A wave has 16 NT of the key's channels (for narrow
// keys a part of the block's tokens too) and reads its part of both states straight into operands,
// 32 columns at a time and one time ahead; do, v, w and dR of these columns pass through LDS.  What is between tokens (M, N and dR . v)
// is tiles spread over the waves, then in LDS for all of them.
template <class T, int KT>
struct Inputs {
  static constexpr int N = kPieces<T>, BLOCK = block_of(N, 32 * KT), TILES = BLOCK / 16, STEPS = BLOCK / 32;
  static constexpr int WAVES = 8, THREADS = 64 * WAVES;
  static constexpr int NT = KT > 4 ? KT / 4 : 1, PARTS = KT < 4 ? 4 / KT : 1, MT = TILES / PARTS;
  static constexpr int TRIANGLE = TILES * (TILES + 1) / 2, TASKS = 2 * TRIANGLE + TILES;
  static constexpr int EACH = (TASKS + WAVES - 1) / WAVES;
  struct Slice {
    Tokens<1, N, BLOCK> od, vd;                        // rows: tokens
    Tokens<BLOCK / 32, 3> rd, wr;                      // rows: columns of the state
  };
  struct Between {
    Tokens<BLOCK / 32, 3, BLOCK> m, n;
  };
};

template <class T, int KT>
__global__ __launch_bounds__((Inputs<T, KT>::THREADS)) void k_delta_inputs_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  using I = Inputs<T, KT>;
  constexpr int N = I::N, BLOCK = I::BLOCK, MT = I::MT, STEPS = I::STEPS, NT = I::NT;
  constexpr int THREADS = I::THREADS, WAVES = I::WAVES, ROWS = 32 * KT;
  __shared__ Tokens<KT, N, BLOCK> k, q;
  __shared__ union Shared {
    typename I::Slice slice;
    typename I::Between between;
    __device__ Shared() {}
  } lds;
  __shared__ double sums[BLOCK];
  __shared__ float since[BLOCK], left[BLOCK], beta[BLOCK], dot_v[BLOCK], dots[WAVES][4][BLOCK], inner[WAVES];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, row = lane / 16 * 4;
  const int groups = a.heads / p.each, bg = blockIdx.x / p.blocks, block = blockIdx.x % p.blocks;
  const int b = bg / groups, group = bg % groups, hk = group * p.each / (a.heads / a.key_heads);
  const int t0 = block * BLOCK, live = min(length_of(a, b) - t0, BLOCK), here = min(a.length - t0, BLOCK);
  const int cols = columns_of(a.value);
  const bool wide = a.value % 8 == 0;
  const int first_tile = wave / I::PARTS * NT, first_m = wave % I::PARTS * MT;
  // dq and dk of the key head, or their parts in 32 bits where other workgroups have more
  const auto store = [&](int which, int t, int c, float x) {
    if (groups == a.key_heads)
      at_head<T>(which ? a.dk : a.dq, b, t0 + t, hk)[c] = (T)x;
    else
      p.partial[((((int64_t)which * a.batch + b) * a.length + t0 + t) * groups + group) * a.key + c] = x;
  };
  if (live <= 0) {
    for (int i = tid; i < here * a.key; i += THREADS) {
      store(0, i / a.key, i % a.key, 0.f);
      store(1, i / a.key, i % a.key, 0.f);
    }
    for (int i = tid; i < here * p.each; i += THREADS) {
      const int64_t at = ((int64_t)b * a.length + t0 + i / p.each) * a.heads + group * p.each + i % p.each;
      if (a.dg) a.dg[at] = 0.f;
      a.dbeta[at] = 0.f;
    }
    return;
  }
  k.load(at_head<T>(a.k, b, t0, hk), a.k.time, live, a.key, tid, THREADS);
  q.load(at_head<T>(a.q, b, t0, hk), a.q.time, live, a.key, tid, THREADS);
  f32x4 dq[NT][MT], dk[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; n++)
#pragma unroll
    for (int m = 0; m < MT; m++) dq[n][m] = dk[n][m] = f32x4{0, 0, 0, 0};
  for (int h = group * p.each; h < (group + 1) * p.each; h++) {
    const int64_t bh = (int64_t)b * a.heads + h;
    const float* S = p.states + (bh * p.blocks + block) * cols * ROWS;
    const float* E = p.dstates + (bh * p.blocks + block) * cols * ROWS;
    const int64_t chunk = bh * p.chunks + block * (BLOCK / kChunk);
    const int last_chunk = (live - 1) / kChunk;
    __syncthreads();
    if (tid < 64) {
      // sums of g from the block's first token: its chunks' one after the other
      double before = 0;
#pragma unroll
      for (int s = 0; s < STEPS; s++) {
        const double G = before + sum_of_g(a, b, h, t0 + 32 * s, live - 32 * s);
        if (tid < 32) sums[32 * s + tid] = G;
        before = __shfl(G, 31, 32);
      }
    }
    __syncthreads();
    if (tid < BLOCK) {
      since[tid] = exp_of(sums[tid]);
      left[tid] = exp_of(sums[BLOCK - 1] - sums[tid]);
      beta[tid] = tid < live ? at_token(a.beta, b, t0 + tid, h) : 0.f;
    }
    f32x4 xq[NT][MT], xr[NT][MT], xw[NT][MT], task[I::EACH];
#pragma unroll
    for (int n = 0; n < NT; n++)
#pragma unroll
      for (int m = 0; m < MT; m++) xq[n][m] = xr[n][m] = xw[n][m] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < I::EACH; i++) task[i] = f32x4{0, 0, 0, 0};
    float es = 0.f, x[NT][8], y[NT][8];
    const auto fetch = [&](int c0) {
#pragma unroll
      for (int n = 0; n < NT; n++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const int at = (c0 + e / 4 * 16 + row + e % 4) * ROWS + 16 * (first_tile + n) + col;
          x[n][e] = S[at];
          y[n][e] = E[at];
        }
    };
    // do and v by half of the threads, w and dR by the others: eight numbers of each of two, raw
    constexpr int ITEMS = BLOCK * 4;
    const int item = tid % ITEMS;
    const bool walks = tid >= ITEMS, own = tid < 2 * ITEMS;
    const int wt = item % (BLOCK / 8) * 8, xt = item / 4;
    const bool on = (walks ? wt : xt) < live;
    // an address that is always there, where one is not wide or not there
    const auto slice_at = [&](int c0, int which) -> const char* {
      if (walks)
        return (const char*)((which ? p.written : p.kept_written) +
                             ((chunk + min(wt / kChunk, last_chunk)) * cols + c0 + item / (BLOCK / 8)) * kChunk +
                             wt % kChunk);
      const int c = c0 + item % 4 * 8;
      if (!wide || c >= a.value) return (const char*)S;
      return (const char*)(at_head<T>(which ? a.v : a.do_, b, t0 + (on ? xt : 0), h) + c);
    };
    constexpr int FAR = sizeof(T) == 4 ? 16 : 0;       // the second half of eight 16-bit numbers: none
    u32x4 pre[2][2];
    const auto prefetch = [&](int c0) {
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const char* from = slice_at(c0, i);
        __builtin_memcpy(&pre[i][0], from, 16);
        __builtin_memcpy(&pre[i][1], from + (walks ? 16 : FAR), 16);
      }
    };
    fetch(0);
    prefetch(0);
    for (int c0 = 0; c0 < cols; c0 += 32) {
      __syncthreads();
      if (walks && own) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; e++) v[e] = on ? __builtin_bit_cast(float, (uint32_t)pre[i][e / 4][e % 4]) : 0.f;
          (i ? lds.slice.rd : lds.slice.wr).put(item / (BLOCK / 8), wt, v);
        }
      } else if (!walks) {
        const int c = c0 + item % 4 * 8, n = on ? a.value - c : 0;
#pragma unroll
        for (int i = 0; i < 2; i++) {
          float v[8];
          if (wide) {
            typedef T TV __attribute__((ext_vector_type(8)));
            TV r;
            __builtin_memcpy(&r, &pre[i], sizeof(r));
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = n > 0 ? (float)r[e] : 0.f;
          } else {
            load_vec<8>(at_head<T>(i ? a.v : a.do_, b, t0 + (on ? xt : 0), h) + (n > 0 ? c : 0), n, v);
          }
          (i ? lds.slice.vd : lds.slice.od).put(xt, item % 4 * 8, v);
        }
      }
      Pieces<3> ss[NT], ds[NT];
#pragma unroll
      for (int n = 0; n < NT; n++) {
#pragma unroll
        for (int e = 0; e < 8; e++) es = fmaf(x[n][e], y[n][e], es);
        ss[n] = split<3>(x[n]);
        ds[n] = split<3>(y[n]);
      }
      __syncthreads();
      fetch(min(c0 + 32, cols - 32));
      prefetch(min(c0 + 32, cols - 32));
#pragma unroll
      for (int m = 0; m < MT; m++) {
        const Pieces<N> os = lds.slice.od.rows(first_m + m, 0);
        const Pieces<3> rs = lds.slice.rd.columns(first_m + m), ws = lds.slice.wr.columns(first_m + m);
#pragma unroll
        for (int n = 0; n < NT; n++) {
          mul(xq[n][m], os, ss[n]);
          mul(xr[n][m], rs, ss[n]);
          mul(xw[n][m], ws, ds[n]);
        }
      }
#pragma unroll
      for (int i = 0; i < I::EACH; i++) {
        const int n = wave + i * WAVES;
        if (n < I::TRIANGLE) {
          const Tile at(n);
          mul(task[i], lds.slice.od.rows(at.i, 0), lds.slice.wr.columns(at.j));
        } else if (n < 2 * I::TRIANGLE) {
          const Tile at(n - I::TRIANGLE);
          mul(task[i], lds.slice.rd.columns(at.i), lds.slice.wr.columns(at.j));
        } else if (n < I::TASKS) {
          mul(task[i], lds.slice.rd.columns(n - 2 * I::TRIANGLE), lds.slice.vd.rows(n - 2 * I::TRIANGLE, 0));
        }
      }
    }
    es = lane_sum<64>(es);
    if (lane == 0) inner[wave] = first_m ? 0.f : es;   // (parts of the tokens have the same states)
    __syncthreads();
    auto& between = lds.between;
#pragma unroll
    for (int i = 0; i < I::EACH; i++) {
      const int n = wave + i * WAVES;
      if (n < 2 * I::TRIANGLE) {
        const bool of_m = n < I::TRIANGLE;
        const Tile at(of_m ? n : n - I::TRIANGLE);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const int ti = 16 * at.i + row + e, tj = 16 * at.j + col;
          const float d = exp_of(sums[ti] - sums[tj]);
          if (of_m)
            between.m.put_one(ti, tj, tj <= ti ? a.scale * d * task[i][e] : 0.f);
          else
            between.n.put_one(ti, tj, tj < ti ? d * task[i][e] : 0.f);
        }
      } else if (n < I::TASKS) {
        const int m = n - 2 * I::TRIANGLE;
#pragma unroll
        for (int e = 0; e < 4; e++)
          if (row + e == col) dot_v[16 * m + col] = task[i][e];
      }
    }
    // the tiles above the diagonal that share an operand with one below
    for (int i = tid; i < BLOCK * 8; i += THREADS) {
      const int t = i / 8 / 16 * 32 + i / 8 % 16, c = t / 32 * 32 + 16 + i % 8 * 2;
      if (t < BLOCK) {
        between.m.put_one(t, c, 0.f);
        between.m.put_one(t, c + 1, 0.f);
        between.n.put_one(t, c, 0.f);
        between.n.put_one(t, c + 1, 0.f);
      }
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; m++) {
      const int mm = first_m + m;
      float dot[4][4];
#pragma unroll
      for (int d = 0; d < 4; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) dot[d][e] = 0.f;
      const f32x4 sm = *(const f32x4*)&since[16 * mm + row], lm = *(const f32x4*)&left[16 * mm + row],
                  bm = *(const f32x4*)&beta[16 * mm + row];
#pragma unroll
      for (int n = 0; n < NT; n++) {
        const int tile = first_tile + n, c = 16 * tile + col;
        f32x4 kv, qv;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          kv[e] = k.value(16 * mm + row + e, c);
          qv[e] = q.value(16 * mm + row + e, c);
        }
        f32x4 &u = xq[n][m], &r = xr[n][m], &w = xw[n][m];
        u *= a.scale * sm;
        r *= sm;
        w *= lm;
        const f32x4 from_states = kv * w;
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
          if (s > mm / 2) continue;
          const Pieces<N> kc = k.columns(tile, s);
          mul(u, between.m.rows(mm, s), kc);
          mul(r, between.n.rows(mm, s), kc);
        }
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
          if (s < mm / 2) continue;
          mul(w, between.m.columns(mm, s), q.columns(tile, s));
          const Pieces<N> kc = k.columns(tile, s);
          float kb[8];
#pragma unroll
          for (int e = 0; e < 8; e++) {
            float v = 0.f;
#pragma unroll
            for (int i = N - 1; i >= 0; i--) v += (float)kc.p[i][e];
            kb[e] = -beta[32 * s + e / 4 * 16 + row + e % 4] * v;
          }
          mul(w, between.n.columns(mm, s), split<3>(kb));
        }
        const f32x4 read = -bm * r;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          dot[0][e] = fmaf(qv[e], u[e], fmaf(kv[e], read[e], dot[0][e]));
          dot[1][e] = fmaf(kv[e], w[e], dot[1][e]);
          dot[2][e] = fmaf(kv[e], r[e], dot[2][e]);
          dot[3][e] += from_states[e];
        }
        dq[n][m] += u;
        dk[n][m] += read + w;
      }
#pragma unroll
      for (int d = 0; d < 4; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float s = lane_sum<16>(dot[d][e]);
          if (col == 0) dots[wave][d][16 * mm + row + e] = s;
        }
    }
    __syncthreads();
    if (tid < BLOCK) {
      double s[4] = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < WAVES; w += I::PARTS)
#pragma unroll
        for (int d = 0; d < 4; d++) s[d] += (double)dots[w + tid / 16 / MT][d][tid];
      double dG = s[0] - s[1], total = s[3], ends = 0;
#pragma unroll
      for (int d = 1; d < BLOCK; d *= 2) {
        const double after = __shfl_down(dG, d, BLOCK);
        if (tid + d < BLOCK) dG += after;
        total += __shfl_xor(total, d, BLOCK);
      }
#pragma unroll
      for (int w = 0; w < WAVES; w++) ends += (double)inner[w];
      total += (double)since[BLOCK - 1] * ends;
      const int64_t at = ((int64_t)b * a.length + t0 + tid) * a.heads + h;
      if (tid < here) {
        if (a.dg) a.dg[at] = tid < live ? (float)(dG + total) : 0.f;
        a.dbeta[at] = tid < live ? (float)(dot_v[tid] - s[2]) : 0.f;
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; n++) {
    const int c = 16 * (first_tile + n) + col;
    if (c >= a.key) break;
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int t = 16 * (first_m + m) + row + e;
        if (t < here) {
          store(0, t, c, dq[n][m][e]);
          store(1, t, c, dk[n][m][e]);
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
      k_delta_inputs_back<T, KT>
          <<<(unsigned)((int64_t)a.batch * a.heads / p.each * p.blocks), Inputs<T, KT>::THREADS, 0, s>>>(p);
      if (int e = launched("k_delta_inputs_back")) return e;
      if (a.heads / p.each == a.key_heads) return (int)RC_OK;
      const int64_t n = (int64_t)a.batch * a.length * a.key_heads * a.key;
      k_delta_shared_heads<T><<<(unsigned)cdiv(2 * n, 256), 256, 0, s>>>(p, n);
      return launched("k_delta_shared_heads");
    });
  });
}
