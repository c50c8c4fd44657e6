// Gated delta rule, gradients; delta.h has the formulas.
#include "delta.h"

using namespace rcdelta;

namespace {

// Backward through the states, from the last chunk to the first, as k_delta_forward goes, and bound as
// that is: 64 chunks of 64 heads of 128 x 128 129 us.
template <class T, int KT, class G, bool WIDE, int MODE>
__global__ __launch_bounds__(G::THREADS) void k_delta_states_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, STEPS = KT / G::R, STAGES = kStages<T, KT, G>;
  constexpr int EVERY = block_of(N, 32 * KT) / kChunk;
  __shared__ Stage<T, KT, G> stages[STAGES];
  __shared__ Parts<G, G::R == 1 ? 0 : 2> parts;
  const Walk<G, MODE> at(p, 32 * KT);
  const int end = at.end, row = at.row, first_row = at.part * STEPS * 32, lane = threadIdx.x % 64;
  const int64_t first = (int64_t)at.bh * p.chunks;
  const bool keeps = MODE == kWhole && at.col < columns_of(a.value);
  const int last_chunk = (end + kChunk - 1) / kChunk - 1;
  if (MODE == kEnds && (!at.count || at.segment == 0)) return;     // no segment goes on from it
  if (threadIdx.x >= G::WORKERS) {
    load_chunks<T, KT, G, WIDE, true, MODE>(p, at, a.do_, stages);
    return;
  }
  f32x4 E[2 * STEPS];
  begin<KT, MODE>(p, at, a.dstate_out, first_row, E);
  for (int i = 0; i < at.count; i++) {
    const int chunk = at.first + at.count - 1 - i, t0 = chunk * kChunk, live = min(end - t0, kChunk);
    const auto& stage = stages[i % STAGES];
    __syncthreads();
    const Chunk& c = stage.c;
    if (keeps && (chunk == last_chunk || chunk % EVERY == EVERY - 1))
      keep_state(p.dstates + ((int64_t)at.bh * p.blocks + chunk / EVERY) * (columns_of(a.value) * 32 * KT),
                 32 * KT, at.col, first_row, E);
    f32x4 dw[2], dr[2], g[2], of_state[2];
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
    for (int m = 0; m < 2; m++) {
      of_state[m] = dw[m] * left[m];
      dw[m] = of_state[m] + from_o[m];
    }
    const Pieces<3> dws = operand<3>(dw[0], dw[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) mul(dr[m], t[m], dws);
    // do or dW of one token that is not finite has made all of its column's dR NaN: those after it again
    if (MODE == kWhole && __builtin_expect(__any(dr[0][0] != dr[0][0]), 0)) {
      asm volatile("" ::: "memory");                   // (what is in LDS is read again, and not held for this)
#pragma unroll
      for (int i = 0; i < 8; i++) g[i / 4][i % 4] = (float)stage.x[i / 4 * 16 + row + i % 4][at.col - at.col0];
      int upto = last_odd(g, row);
#pragma unroll
      for (int i = 0; i < 8; i++) g[i / 4][i % 4] = is_finite(g[i / 4][i % 4]) ? g[i / 4][i % 4] : 0.f;
      const Pieces<N> finite = operand<N>(g[0], g[1]);
#pragma unroll
      for (int m = 0; m < 2; m++) {
        if constexpr (G::R > 1) of_state[m] = parts.sum(m, at.wave) * *(const f32x4*)&c.left[16 * m + row];
        dw[m] = f32x4{0, 0, 0, 0};
        mul(dw[m], pieces(c.p[m]), finite);
        dw[m] += of_state[m];
      }
      upto = max(upto, last_odd(dw, row));
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const bool there = i / 4 * 16 + row + i % 4 > upto;
        dw[i / 4][i % 4] = there ? dw[i / 4][i % 4] : 0.f;
        dr[i / 4][i % 4] = there ? 0.f : __builtin_nanf("");
      }
      const Pieces<3> again = operand<3>(dw[0], dw[1]);
#pragma unroll
      for (int m = 0; m < 2; m++) mul(dr[m], pieces(c.t[m]), again);
    }
    const Pieces<3> drs = operand<3>(-since[0] * beta[0] * dr[0], -since[1] * beta[1] * dr[1]);
#pragma unroll
    for (int m = 0; m < 2 * STEPS; m++) mul(E[m], stage.k.columns(at.part * 2 * STEPS + m), drs);
#pragma unroll
    for (int m = 0; m < (MODE == kWhole ? 2 : 0); m++) {
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
  if constexpr (MODE == kEnds) {
    leave<KT>(p, at, first_row, E);
  } else {
    if (a.dstate_in && at.segment == 0)
      store_state(a.dstate_in + (int64_t)at.bh * a.key * a.value, a, at.col, first_row, E);
    if (at.on && at.part == 0 && at.last) {
      T* dv = at_head<T>(a.dv, at.b, 0, at.h) + at.col;
      for (int t = end + row / 4; t < a.length; t += 4) dv[t * a.dv.time] = (T)0.f;
    }
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

// Of sixteen numbers the sum of number i over a row's 16 lanes, in lane i: each exchange halves the
// numbers that a lane still has.
__device__ __forceinline__ float sixteen_sums(const f32x4 (&x)[4]) {
  const int i = threadIdx.x % 16;
  float v[16];
#pragma unroll
  for (int j = 0; j < 16; j++) v[j] = x[j / 4][j % 4];
  const auto halve = [&](auto ctrl, auto n) {
    constexpr int N = decltype(n)::value;
#pragma unroll
    for (int j = 0; j < N; j++) {
      const float keep = i & N ? v[N + j] : v[j], give = i & N ? v[j] : v[N + j];
      v[j] = keep + dpp_of<decltype(ctrl)::value>(give);
    }
  };
  halve(std::integral_constant<int, 0x140>{}, std::integral_constant<int, 8>{});  // rows mirrored
  halve(std::integral_constant<int, 0x141>{}, std::integral_constant<int, 4>{});  // half rows mirrored
  halve(std::integral_constant<int, 0x4E>{}, std::integral_constant<int, 2>{});   // 2 apart
  halve(std::integral_constant<int, 0xB1>{}, std::integral_constant<int, 1>{});   // 1 apart
  return v[0];
}

// The gradients of a block's inputs from the state before it and the gradient of the one after
// it, head by head of those that share a key head.  A wave has 16 NT of the key's channels (for narrow
// keys a part of the block's tokens too).  Both states, do, v, w and dR pass through LDS, 32 columns at a
// time and one time ahead in registers; where LDS has no room for the states a wave reads its part
// of them straight into operands, a number a load (which is what bounds it then).  What is between tokens (M, N and dR . v)
// is tiles spread over the waves, then in LDS for all of them.  Pairs of tokens (i, j) reach dg through
// Z_ij = M_ij q_i . k_j - beta_i N_ij k_i . k_j, in 32-bit sums over rows and over columns of a tile that are added to
// one another in 64 bits: what two tokens past t have with each other leaves dg_t but for those sums' roundings,
// of 16 numbers each, where dots of dq and dk left the roundings of sums over all that a token has.
// Bound by waiting for loads and LDS (47% of a wave's time), with one workgroup of eight waves a compute
// unit, which is what LDS and 256 registers allow; the matrix instructions are busy 16% of it: 64 heads of
// 128 x 128, 32 blocks each, 246 us (215 with dg from dots of dq and dk, whose roundings
// reached 2e-5 of dg over 64 tokens).  Registers spill: 100 bytes a lane for these heads, 348 for bf16 keys above 128,
// 36 and 184 for f16 of 33 to 64 and above 128, 148 and 192 for f32.  Blocks of 32 tokens, that read twice the states, took 414 where these took
// 298; states read straight into operands 284, through LDS with a head's first loads before the last one's sums end, 253.
template <class T, int KT>
struct Inputs {
  static constexpr int N = kPieces<T>, BLOCK = block_of(N, 32 * KT), TILES = BLOCK / 16, STEPS = BLOCK / 32;
  static constexpr int WAVES = 8, THREADS = 64 * WAVES;
  static constexpr int NT = KT > 4 ? KT / 4 : 1, PARTS = KT < 4 ? 4 / KT : 1, MT = TILES / PARTS;
  static constexpr int TRIANGLE = TILES * (TILES + 1) / 2, TASKS = 2 * TRIANGLE + TILES;
  static constexpr int EACH = (TASKS + WAVES - 1) / WAVES;
  static constexpr bool HELD = block_bytes(N, 32 * KT, BLOCK, true) <= kBlockBytes;
  struct Slice {
    Tokens<1, N, BLOCK> od, vd;                        // rows: tokens
    Tokens<BLOCK / 32, 3> rd, wr;                      // rows: columns of the state
    Tokens<HELD ? KT : 1, 3> s, e;                     // the same
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
  __shared__ float since[BLOCK], left[BLOCK], beta[BLOCK], dot_v[BLOCK], dots[WAVES * NT][3][BLOCK],
      inner[WAVES], of_rows[2 * I::TRIANGLE][16], of_columns[2 * I::TRIANGLE][16];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 16, row = lane / 16 * 4;
  const int groups = a.heads / p.each, bg = blockIdx.x / p.blocks, block = blockIdx.x % p.blocks;
  const int b = bg / groups, group = bg % groups, hk = group * p.each / (a.heads / a.key_heads);
  const int t0 = block * BLOCK, live = min(length_of(a, b) - t0, BLOCK), here = min(a.length - t0, BLOCK);
  const int cols = columns_of(a.value);
  const bool wide = a.value % 8 == 0;
  const int first_tile = wave / I::PARTS * NT, first_m = wave % I::PARTS * MT;
  // dq and dk of the key head, or their parts in 32 bits where other workgroups have more
  const bool whole_heads = groups == a.key_heads;
  const auto row_of = [&](int which, int t) {
    return at_head<T>(which ? a.dk : a.dq, b, t0 + t, hk);
  };
  const auto part_of = [&](int which, int t) {
    return p.partial + ((((int64_t)which * a.batch + b) * a.length + t0 + t) * groups + group) * a.key;
  };
  if (live <= 0) {
    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int vectors = (a.key + 7) / 8;
    for (int i = tid; i < 2 * here * vectors; i += THREADS) {
      const int c = i % vectors * 8, t = i / vectors % here, which = i / vectors / here;
      if (whole_heads)
        store_vec<8>(row_of(which, t) + c, a.key - c, zero);
      else
        store_vec<8>(part_of(which, t) + c, a.key - c, zero);
    }
    for (int i = tid; i < here * p.each; i += THREADS) {
      const int64_t at = ((int64_t)b * a.length + t0 + i / p.each) * a.heads + group * p.each + i % p.each;
      if (a.dg) a.dg[at] = 0.f;
      a.dbeta[at] = 0.f;
    }
    return;
  }
  // do and v by half of the threads, w and dR by the others: eight numbers of each of two, raw
  constexpr int ITEMS = BLOCK * 4;
  constexpr int FAR = sizeof(T) == 4 ? 16 : 0;         // the second half of eight 16-bit numbers: none
  const int item = tid % ITEMS, wt = item % (BLOCK / 8) * 8, xt = item / 4, xc = item % 4 * 8;
  const int last_chunk = (live - 1) / kChunk;
  const bool walks = tid >= ITEMS, own = tid < 2 * ITEMS, on = (walks ? wt : xt) < live;
  const float *S, *E;
  const char* from[2];
  float x[NT][8], y[NT][8], next_beta;
  double next_sum[3];
  u32x4 pre[2][2];
  const int held_row = min(tid / (KT * 4), 31), held_at = tid % (KT * 4) * 8;
  const bool holds = tid < KT * 128;
  const auto fetch = [&](int c0) {
    if constexpr (I::HELD) {
      __builtin_memcpy(&x[0], S + (c0 + held_row) * ROWS + held_at, 32);
      __builtin_memcpy(&y[0], E + (c0 + held_row) * ROWS + held_at, 32);
    }
#pragma unroll
    for (int n = 0; n < (I::HELD ? 0 : NT); n++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int at = (c0 + e / 4 * 16 + row + e % 4) * ROWS + 16 * (first_tile + n) + col;
        x[n][e] = S[at];
        y[n][e] = E[at];
      }
    // (an address that is always there, where one is not wide or not there)
    const bool there = walks || (wide && c0 + xc < a.value);
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const char* at = there ? from[i] + c0 * (walks ? kChunk * 4 : (int)sizeof(T)) : (const char*)S;
      __builtin_memcpy(&pre[i][0], at, 16);
      __builtin_memcpy(&pre[i][1], at + (walks ? 16 : FAR), 16);
    }
  };
  // The first loads of a head.
  const auto enter = [&](int h) {
    const int64_t bh = (int64_t)b * a.heads + h, chunk = bh * p.chunks + block * (BLOCK / kChunk);
    S = p.states + (bh * p.blocks + block) * cols * ROWS;
    E = p.dstates + (bh * p.blocks + block) * cols * ROWS;
    if (walks) {
      const int64_t at =
          ((chunk + min(wt / kChunk, last_chunk)) * cols + item / (BLOCK / 8)) * kChunk + wt % kChunk;
      from[0] = (const char*)(p.kept_written + at);
      from[1] = (const char*)(p.written + at);
    } else {
      from[0] = (const char*)(at_head<T>(a.do_, b, t0 + (on ? xt : 0), h) + xc);
      from[1] = (const char*)(at_head<T>(a.v, b, t0 + (on ? xt : 0), h) + xc);
    }
    const Chunk* c = p.prepared + chunk;
    const int t = tid % BLOCK, mine = min(t / kChunk, last_chunk);
    next_sum[0] = c[mine].sum[t % kChunk];
    next_sum[1] = c[0].sum[kChunk - 1];
    next_sum[2] = c[last_chunk].sum[kChunk - 1];
    next_beta = c[mine].beta[t % kChunk];
    fetch(0);
  };
  enter(group * p.each);
  k.load(at_head<T>(a.k, b, t0, hk), a.k.time, live, a.key, tid, THREADS);
  q.load(at_head<T>(a.q, b, t0, hk), a.q.time, live, a.key, tid, THREADS);
  f32x4 dq[NT][MT], dk[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; n++)
#pragma unroll
    for (int m = 0; m < MT; m++) dq[n][m] = dk[n][m] = f32x4{0, 0, 0, 0};
  for (int h = group * p.each; h < (group + 1) * p.each; h++) {
    if (tid < BLOCK) {
      // sums of g from the block's first token
      const double end = last_chunk ? next_sum[1] + next_sum[2] : next_sum[1];
      const double G = tid / kChunk > last_chunk ? end : tid < kChunk ? next_sum[0] : next_sum[1] + next_sum[0];
      sums[tid] = G;
      since[tid] = exp_of(G);
      left[tid] = exp_of(end - G);
      beta[tid] = tid < live ? next_beta : 0.f;
    }
    f32x4 xq[NT][MT], xr[NT][MT], xw[NT][MT], task[I::EACH];
#pragma unroll
    for (int n = 0; n < NT; n++)
#pragma unroll
      for (int m = 0; m < MT; m++) xq[n][m] = xr[n][m] = xw[n][m] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < I::EACH; i++) task[i] = f32x4{0, 0, 0, 0};
    float es = 0.f;
    for (int c0 = 0; c0 < cols; c0 += 32) {
      if (c0) __syncthreads();
      if (walks && own) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; e++) v[e] = on ? __builtin_bit_cast(float, (uint32_t)pre[i][e / 4][e % 4]) : 0.f;
          (i ? lds.slice.rd : lds.slice.wr).put(item / (BLOCK / 8), wt, v);
        }
      } else if (!walks) {
        const int n = on ? a.value - (c0 + xc) : 0;
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
            load_vec<8>((const T*)from[i] + (n > 0 ? c0 : 0), n, v);
          }
          (i ? lds.slice.vd : lds.slice.od).put(xt, xc, v);
        }
      }
      Pieces<3> ss[NT], ds[NT];
      if constexpr (I::HELD) {
        if (holds) {
#pragma unroll
          for (int e = 0; e < 8; e++) es = fmaf(x[0][e], y[0][e], es);
          lds.slice.s.put(held_row, held_at, x[0]);
          lds.slice.e.put(held_row, held_at, y[0]);
        }
      } else {
#pragma unroll
        for (int n = 0; n < NT; n++) {
#pragma unroll
          for (int e = 0; e < 8; e++) es = fmaf(x[n][e], y[n][e], es);
          ss[n] = split<3>(x[n]);
          ds[n] = split<3>(y[n]);
        }
      }
      __syncthreads();
      if constexpr (I::HELD) {
#pragma unroll
        for (int n = 0; n < NT; n++) {
          ss[n] = lds.slice.s.columns(first_tile + n);
          ds[n] = lds.slice.e.columns(first_tile + n);
        }
      }
      fetch(min(c0 + 32, cols - 32));
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
      // tiles of M and N as their transposes: four of a lane's numbers lie side by side
#pragma unroll
      for (int i = 0; i < I::EACH; i++) {
        const int n = wave + i * WAVES;
        if (n < I::TRIANGLE) {
          const Tile at(n);
          mul(task[i], lds.slice.wr.columns(at.j), lds.slice.od.rows(at.i, 0));
        } else if (n < 2 * I::TRIANGLE) {
          const Tile at(n - I::TRIANGLE);
          mul(task[i], lds.slice.wr.columns(at.j), lds.slice.rd.columns(at.i));
        } else if (n < I::TASKS) {
          mul(task[i], lds.slice.rd.columns(n - 2 * I::TRIANGLE), lds.slice.vd.rows(n - 2 * I::TRIANGLE, 0));
        }
      }
    }
    es = lane_sum<64>(es);
    if (lane == 0) inner[wave] = I::HELD || !first_m ? es : 0.f;   // (parts of the tokens have the same states)
    __syncthreads();
    auto& between = lds.between;
#pragma unroll
    for (int i = 0; i < I::EACH; i++) {
      const int n = wave + i * WAVES;
      if (n < 2 * I::TRIANGLE) {
        const bool of_m = n < I::TRIANGLE;
        const Tile at(of_m ? n : n - I::TRIANGLE);
        const int ti = 16 * at.i + col;
        const auto& reads = of_m ? q : k;
        f32x4 v, z = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KT; s++) mul(z, k.rows(at.j, s), reads.rows(at.i, s));
        const float by = of_m ? 1.f : -beta[ti];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const int tj = 16 * at.j + row + e;
          v[e] = (of_m ? tj <= ti : tj < ti) ? (of_m ? a.scale : 1.f) * decay_between(sums[ti] - sums[tj]) * task[i][e] : 0.f;
          z[e] *= by * v[e];
          z[e] = tj < ti && z[e] == z[e] ? z[e] : 0.f;
        }
        (of_m ? between.m : between.n).put_four(ti, 16 * at.j + row, v);
        const float of_row = add_32_apart(add_16_apart((z[0] + z[1]) + (z[2] + z[3])));
        float of_column = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float s = lane_sum<16>(z[e]);
          if (col == e) of_column = s;
        }
        if (row == 0) of_rows[n][col] = of_row;
        if (col < 4) of_columns[n][row + col] = of_column;
      } else if (n < I::TASKS) {
        const int m = n - 2 * I::TRIANGLE;
#pragma unroll
        for (int e = 0; e < 4; e++)
          if (row + e == col) dot_v[16 * m + col] = task[i][e];
      }
    }
    // the tiles above the diagonal that share an operand with one below
    if (tid < BLOCK * 4) {
      const int t = tid / 8 / 16 * 32 + tid / 8 % 16;  // tid / 8 of the upper halves' rows
      const f32x4 zero = {0, 0, 0, 0};
      (tid & 4 ? between.m : between.n).put_four(t, t / 32 * 32 + 16 + tid % 4 * 4, zero);
    }
    __syncthreads();
    const float whole = since[BLOCK - 1];
#pragma unroll
    for (int n = 0; n < NT; n++) {
      const int tile = first_tile + n, c = 16 * tile + col;
      Pieces<N> kc[STEPS], qc[STEPS];
      Pieces<3> kb[STEPS];                             // -beta k
#pragma unroll
      for (int s = 0; s < STEPS; s++) {
        kc[s] = k.columns(tile, s);
        qc[s] = q.columns(tile, s);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
          v[e] = 0.f;
#pragma unroll
          for (int i = N - 1; i >= 0; i--) v[e] += (float)kc[s].p[i][e];
          v[e] *= -beta[32 * s + e / 4 * 16 + row + e % 4];
        }
        kb[s] = split<3>(v);
      }
#pragma unroll
      for (int m = 0; m < MT; m++) {
        const int mm = first_m + m;
        f32x4 kv, qv;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          if (I::PARTS == 1) {                         // as a lane has them already
            kv[e] = qv[e] = 0.f;
#pragma unroll
            for (int i = N - 1; i >= 0; i--) {
              kv[e] += (float)kc[m / 2].p[i][m % 2 * 4 + e];
              qv[e] += (float)qc[m / 2].p[i][m % 2 * 4 + e];
            }
          } else {
            kv[e] = k.value(16 * mm + row + e, c);
            qv[e] = q.value(16 * mm + row + e, c);
          }
        }
        f32x4 &u = xq[n][m], &r = xr[n][m], &w = xw[n][m];
        u *= a.scale * *(const f32x4*)&since[16 * mm + row];
        r *= *(const f32x4*)&since[16 * mm + row];
        w *= *(const f32x4*)&left[16 * mm + row];
        const f32x4 minus_beta = -*(const f32x4*)&beta[16 * mm + row];
        f32x4 dot[4] = {qv * u + kv * (minus_beta * r), kv * w, {0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
          if (s <= mm / 2) {
            mul(u, between.m.rows(mm, s), kc[s]);
            mul(r, between.n.rows(mm, s), kc[s]);
          }
          if (s >= mm / 2) {
            mul(w, between.m.columns(mm, s), qc[s]);
            mul(w, between.n.columns(mm, s), kb[s]);
          }
        }
        dot[2] = kv * r;
        const float s = sixteen_sums(dot);
        if (col < 12) dots[wave * NT + n][col / 4][16 * mm + row + col % 4] = s;
        dq[n][m] += u;
        dk[n][m] += minus_beta * r + w;
      }
    }
    enter(min(h + 1, (group + 1) * p.each - 1));       // (unconditional, as every load that a loop hands on)
    __syncthreads();
    // dg and dbeta by the last wave, while the others begin the next head
    if (wave == WAVES - 1 && lane < BLOCK) {
      float s[3] = {0, 0, 0};
#pragma unroll
      for (int w = 0; w < WAVES; w += I::PARTS)
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
          for (int d = 0; d < 3; d++) s[d] += dots[(w + lane / 16 / MT) * NT + n][d][lane];
      // Where w is NaN so are s[1] and the products of pairs, which count as 0: they would leave the dg of the tokens
      // up to the first of them anyway, and those after it are NaN.  (dbeta from the first on: its g may be why.)
      const unsigned long long lost = __ballot(s[1] != s[1]);
      const int from = lost ? __builtin_ctzll(lost) : BLOCK;
      if (s[1] != s[1]) s[1] = 0.f;
      double dG = (double)s[0] - s[1], ends = 0;
      const int own = lane / 16, t = lane % 16;
      float pairs[I::TILES][4];
#pragma unroll
      for (int j = 0; j < I::TILES; j++) {
        const int lo = min(j, own), hi = max(j, own), r = own * (own + 1) / 2 + lo, c = hi * (hi + 1) / 2 + own;
        pairs[j][0] = of_rows[r][t];
        pairs[j][1] = of_rows[I::TRIANGLE + r][t];
        pairs[j][2] = of_columns[c][t];
        pairs[j][3] = of_columns[I::TRIANGLE + c][t];
      }
#pragma unroll
      for (int j = 0; j < I::TILES; j++) {
        if (j <= own) dG += (double)pairs[j][0] + pairs[j][1];
        if (j >= own) dG -= (double)pairs[j][2] + pairs[j][3];
      }
#pragma unroll
      for (int d = 1; d < BLOCK; d *= 2) {
        const double after = __shfl_down(dG, d, BLOCK);
        if (lane + d < BLOCK) dG += after;
      }
#pragma unroll
      for (int w = 0; w < WAVES; w++) ends += (double)inner[w];
      const double total = (double)lane_sum<BLOCK>(s[1]) + whole * ends;
      const int64_t at = ((int64_t)b * a.length + t0 + lane) * a.heads + h;
      if (lane < here) {
        if (a.dg) a.dg[at] = lane >= live ? 0.f : lane > from ? __builtin_nanf("") : (float)(dG + total);
        a.dbeta[at] = lane >= live ? 0.f : lane >= from ? __builtin_nanf("") : (float)(dot_v[lane] - s[2]);
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
        if (t >= here) continue;
        const float of_q = t < live ? dq[n][m][e] : 0.f, of_k = t < live ? dk[n][m][e] : 0.f;
        if (whole_heads) {
          row_of(0, t)[c] = (T)of_q;
          row_of(1, t)[c] = (T)of_k;
        } else {
          part_of(0, t)[c] = of_q;
          part_of(1, t)[c] = of_k;
        }
      }
  }
}

// dq and dk of key heads whose heads several workgroups had: the sums of their parts.
template <class T>
__global__ __launch_bounds__(256) void k_delta_shared_heads(DeltaParams p, int64_t n) {
  const rc_delta_args& a = p.a;
  const int parts = a.heads / p.each / a.key_heads;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < 2 * n; i += (int64_t)gridDim.x * 256) {
    const int which = i >= n;
    const int64_t e = i - which * n;
    const int c = (int)(e % a.key);
    const int64_t row = e / a.key;                    // (b, t, key head)
    const float* from = p.partial + which * n * parts + row * parts * a.key + c;
    float s = 0.f;
    for (int j = 0; j < parts; j++) s += from[(int64_t)j * a.key];
    const int64_t token = row / a.key_heads;
    at_head<T>(which ? a.dk : a.dq, token / a.length, token % a.length, row % a.key_heads)[c] = (T)s;
  }
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
  if (int e = fits_back(a)) return e;
  if (a.length && (!a.workspace || a.workspace_bytes < workspace_of(a, true))) return RC_E_SCRATCH;
  const hipStream_t s = (hipStream_t)stream;
  DeltaParams p = params(a);
  const int64_t pairs = pairs_of(a);
  p.each = heads_together(a);
  p.kept_written = a.kept + state_floats(a);
  p.dstates = p.between + segment_floats(a);
  p.written = p.dstates + state_floats(a);
  p.partial = p.written + pairs * columns_of(a.value) * kChunk;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_key(a.key, [&](auto kt) {
      constexpr int KT = decltype(kt)::value;
      if (int e = prepare<T, KT, true>(p, s)) return e;
      const int e = by_width(a, [&](auto wide) {
        using G = ShapeOf<KT>;
        constexpr bool WIDE = decltype(wide)::value;
        if (p.segments > 1) {
          k_delta_states_back<T, KT, G, WIDE, kEnds><<<walks_of<G, kEnds>(p, 32 * KT), G::THREADS, 0, s>>>(p);
          if (int e = launched("k_delta_states_back")) return e;
          if (int e = join<KT, true>(p, s)) return e;
        }
        k_delta_states_back<T, KT, G, WIDE, kWhole><<<walks_of<G, kWhole>(p, 0), G::THREADS, 0, s>>>(p);
        return launched("k_delta_states_back");
      });
      if (e) return e;
      if (!p.chunks) return (int)RC_OK;
      k_delta_inputs_back<T, KT>
          <<<(unsigned)((int64_t)a.batch * a.heads / p.each * p.blocks), Inputs<T, KT>::THREADS, 0, s>>>(p);
      if (int e = launched("k_delta_inputs_back")) return e;
      if (a.heads / p.each == a.key_heads) return (int)RC_OK;
      const int64_t n = (int64_t)a.batch * a.length * a.key_heads * a.key;
      k_delta_shared_heads<T><<<(unsigned)std::min<int64_t>(cdiv(2 * n, 256), 1 << 20), 256, 0, s>>>(p, n);
      return launched("k_delta_shared_heads");
    });
  });
}
