// Gated delta rule, forward and for single tokens; delta.h has the formulas.
#include "delta.h"

using namespace rcdelta;

namespace {

// Forward: a wave holds 16 columns of the state, or R waves a part each of their rows,
// in registers from the first chunk to the last.  Columns do not depend on one
// another, and what a product leaves in a lane is what the next one takes from it, so waves share
// the tokens in LDS, and the parts their sums over the key.
//
// Bound by the way through a chunk: sums over the key, their exchange, T, and the state, each after
// the other, with one or two waves a SIMD.  Waves of columns x parts of the key of 128, timed when the
// same waves loaded and computed, us a chunk: 2 x 2 2.5, 2 x 4 2.7, 4 x 1 and 4 x 2 2.9, 4 x 4 3.6; with waves that only
// load 1.75.  64 chunks of 64 heads of 128 x 128 with states kept (4 x 2048 tokens): 124 us; a prompt of
// 8192 tokens, 16 heads, in three segments: 103 us for their ends, 9 to join them, 147 for the outputs.
template <class T, int KT, class G, bool WIDE, int MODE>
__global__ __launch_bounds__(G::THREADS) void k_delta_forward(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int STEPS = KT / G::R, STAGES = kStages<T, KT, G>;
  constexpr int EVERY = block_of(kPieces<T>, 32 * KT) / kChunk;
  __shared__ Stage<T, KT, G> stages[STAGES];
  __shared__ Parts<G, G::R == 1 ? 0 : 4> parts;
  const Walk<G, MODE> at(p, 32 * KT);
  const int end = at.end, row = at.row, first_row = at.part * STEPS * 32, lane = threadIdx.x % 64;
  const int64_t first = (int64_t)at.bh * p.chunks;
  const bool keeps = MODE == kWhole && at.col < columns_of(a.value);
  if (MODE == kEnds && (!at.count || at.last)) return;             // no segment goes on from it
  if (threadIdx.x >= G::WORKERS) {
    load_chunks<T, KT, G, WIDE, false, MODE>(p, at, a.v, stages);
    return;
  }
  f32x4 S[2 * STEPS];
  begin<KT, MODE>(p, at, a.state_in, first_row, S);
  for (int i = 0; i < at.count; i++) {
    const int chunk = at.first + i, t0 = chunk * kChunk, live = min(end - t0, kChunk);
    const auto& stage = stages[i % STAGES];
    __syncthreads();
    const Chunk& c = stage.c;
    if (p.states && keeps && chunk % EVERY == 0)
      keep_state(p.states + ((int64_t)at.bh * p.blocks + chunk / EVERY) * (columns_of(a.value) * 32 * KT),
                 32 * KT, at.col, first_row, S);
    f32x4 r[2], out[2], w[2];
#pragma unroll
    for (int m = 0; m < 2; m++) r[m] = out[m] = w[m] = f32x4{0, 0, 0, 0};
    Pieces<3> state[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; s++) {
      state[s] = operand<3>(S[2 * s], S[2 * s + 1]);
#pragma unroll
      for (int m = 0; m < 2; m++) mul(r[m], stage.k.rows(m, at.part * STEPS + s), state[s]);
    }
    if constexpr (G::R > 1) {
#pragma unroll
      for (int m = 0; m < 2; m++) parts.at[m][at.part][at.wave][lane] = r[m];
    }
#pragma unroll
    for (int s = 0; s < (MODE == kWhole ? STEPS : 0); s++)
#pragma unroll
      for (int m = 0; m < 2; m++) mul(out[m], stage.q.rows(m, at.part * STEPS + s), state[s]);
    // read before the barrier, which nothing is moved over
    f32x4 since[2], beta[2], left[2], x[2];
#pragma unroll
    for (int m = 0; m < 2; m++) {
      since[m] = *(const f32x4*)&c.since[16 * m + row];
      beta[m] = *(const f32x4*)&c.beta[16 * m + row];
      left[m] = *(const f32x4*)&c.left[16 * m + row];
#pragma unroll
      for (int e = 0; e < 4; e++) x[m][e] = (float)stage.x[16 * m + row + e][at.col - at.col0];
    }
    const Pieces<3> t[2] = {pieces(c.t[0]), pieces(c.t[1])};
    if constexpr (G::R > 1) {
#pragma unroll
      for (int m = 0; m < (MODE == kWhole ? 2 : 0); m++) parts.at[2 + m][at.part][at.wave][lane] = out[m];
      __syncthreads();
#pragma unroll
      for (int m = 0; m < 2; m++) r[m] = parts.sum(m, at.wave);
    }
#pragma unroll
    for (int m = 0; m < 2; m++) r[m] = beta[m] * (x[m] - since[m] * r[m]);
    Pieces<3> rs = operand<3>(r[0], r[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) mul(w[m], t[m], rs);
    // r of one token that is not finite has made all of its column's w NaN: those before it again
    if (MODE == kWhole && __builtin_expect(__any(w[0][0] != w[0][0]), 0)) {
      asm volatile("" ::: "memory");                   // (T is read again, and not held for this)
      const int from = first_odd(r, row);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const bool there = i / 4 * 16 + row + i % 4 < from;
        r[i / 4][i % 4] = there ? r[i / 4][i % 4] : 0.f;
        w[i / 4][i % 4] = there ? 0.f : __builtin_nanf("");
        since[i / 4][i % 4] = there ? since[i / 4][i % 4] : __builtin_nanf("");      // the outputs' factor
      }
      rs = operand<3>(r[0], r[1]);
#pragma unroll
      for (int m = 0; m < 2; m++) mul(w[m], pieces(c.t[m]), rs);
    }
    const Pieces<3> us = operand<3>(w[0] * left[0], w[1] * left[1]);
    const float whole = c.since[kChunk - 1];
#pragma unroll
    for (int m = 0; m < 2 * STEPS; m++) {
      S[m] *= whole;
      mul(S[m], stage.k.columns(at.part * 2 * STEPS + m), us);
    }
    // outputs: tile m by part m
#pragma unroll
    for (int m = 0; m < (MODE == kWhole ? 2 : 0); m++) {
      if (G::R > 1 && at.part != m) continue;
      if constexpr (G::R > 1) out[m] = parts.sum(2 + m, at.wave);
      out[m] *= a.scale * since[m];
      mul(out[m], pieces(c.p[m]), rs);
      T* o = at_head<T>(a.o, at.b, t0 + 16 * m, at.h) + row * a.o.time + at.col;
      if (at.on) {
        if (live == kChunk) {
#pragma unroll
          for (int e = 0; e < 4; e++) o[e * a.o.time] = (T)out[m][e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (16 * m + row + e < live) o[e * a.o.time] = (T)out[m][e];
        }
      }
      if (p.written && keeps)
        *(f32x4*)(p.written + ((first + chunk) * columns_of(a.value) + at.col) * kChunk + 16 * m + row) = w[m];
    }
    if (STAGES == 1) __syncthreads();
  }
  if constexpr (MODE == kEnds) {
    leave<KT>(p, at, first_row, S);
  } else if (at.last) {
    if (a.state_out)
      store_state(a.state_out + (int64_t)at.bh * a.key * a.value, a, at.col, first_row, S);
    if (at.on && at.part == 0) {
      T* o = at_head<T>(a.o, at.b, 0, at.h) + at.col;
      for (int t = end + row / 4; t < a.length; t += 4) o[t * a.o.time] = (T)0.f;
    }
  }
}

// ------------------------------------------------------------- single tokens

struct StepParams {
  rc_delta_step_args a;
};

// Bound by memory: 192 x 16 states of 128 x 128, 405 MB read and written, 95 us (4.3 TB/s); of one
// sequence 5 us, the launch's.
// 32 columns of a head's state a workgroup: eight lanes of four columns by 32 groups of rows,
// each row read once, kept in registers, and written once.  Both products of the state are
// taken of the one before: o = scale (a S^T q + (q . k) w), so one exchange is enough.
template <class T, int NR>
__global__ __launch_bounds__(256) void k_delta_step(StepParams p) {
  const rc_delta_step_args& a = p.a;
  __shared__ float4 part[2][4][8];
  __shared__ float dot[4];
  const int slices = (a.value + 31) / 32, bh = blockIdx.x / slices;
  const int tid = threadIdx.x, group = tid / 8, c = blockIdx.x % slices * 32 + tid % 8 * 4;
  const int b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.key_heads);
  const int slot = a.slots ? a.slots[b] : b, n = a.value - c;
  T* o = at_head<T>(a.o, b, 0, h) + c;
  if (slot < 0 || slot >= a.num_slots) {
    const float zero[4] = {0, 0, 0, 0};
    if (group == 0 && n > 0) store_vec<4>(o, n, zero);
    return;
  }
  float* S = a.state + slot * a.state_slot + (int64_t)h * a.key * a.value + (n > 0 ? c : 0);
  const T* k = at_head<T>(a.k, b, 0, hk);
  const T* q = at_head<T>(a.q, b, 0, hk);
  float x[NR][4], kr[NR], ks[4] = {0, 0, 0, 0}, qs[4] = {0, 0, 0, 0}, qk = 0.f;
#pragma unroll
  for (int i = 0; i < NR; i++) {
    const int r = i * 32 + group, at = r < a.key ? r : 0;
    load_vec<4>(S + (int64_t)at * a.value, r < a.key ? n : 0, x[i]);
    kr[i] = r < a.key ? (float)k[at] : 0.f;
    const float qr = r < a.key ? (float)q[at] : 0.f;
    qk = fmaf(qr, kr[i], qk);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      ks[e] = fmaf(kr[i], x[i][e], ks[e]);
      qs[e] = fmaf(qr, x[i][e], qs[e]);
    }
  }
#pragma unroll
  for (int d = 8; d < 64; d *= 2) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      ks[e] += __shfl_xor(ks[e], d);
      qs[e] += __shfl_xor(qs[e], d);
    }
    qk += __shfl_xor(qk, d);
  }
  if (tid % 64 < 8) {
    part[0][tid / 64][tid % 8] = {ks[0], ks[1], ks[2], ks[3]};
    part[1][tid / 64][tid % 8] = {qs[0], qs[1], qs[2], qs[3]};
    if (tid % 64 == 0) dot[tid / 64] = qk;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 4; e++) ks[e] = qs[e] = 0.f;
  qk = 0.f;
#pragma unroll
  for (int w = 0; w < 4; w++) {
    const float4 u = part[0][w][tid % 8], y = part[1][w][tid % 8];
    ks[0] += u.x, ks[1] += u.y, ks[2] += u.z, ks[3] += u.w;
    qs[0] += y.x, qs[1] += y.y, qs[2] += y.z, qs[3] += y.w;
    qk += dot[w];
  }
  const float decay = a.g.data ? exp_of(log_decay(a.g, b, 0, h)) : 1.f;
  const float beta = at_token(a.beta, b, 0, h);
  float v[4], out[4];
  load_vec<4>(at_head<T>(a.v, b, 0, h) + (n > 0 ? c : 0), n, v);
#pragma unroll
  for (int e = 0; e < 4; e++) {
    v[e] = beta * (v[e] - decay * ks[e]);
    out[e] = a.scale * fmaf(qk, v[e], decay * qs[e]);
  }
  if (n <= 0) return;
#pragma unroll
  for (int i = 0; i < NR; i++) {
    const int r = i * 32 + group;
#pragma unroll
    for (int e = 0; e < 4; e++) x[i][e] = fmaf(kr[i], v[e], decay * x[i][e]);
    if (r < a.key) store_vec<4>(S + (int64_t)r * a.value, n, x[i]);
  }
  if (group == 0) store_vec<4>(o, n, out);
}

}  // namespace

extern "C" int rc_delta_kept_bytes(const rc_delta_args* args, uint64_t* bytes) {
  if (int e = check(args)) return e;
  if (!bytes) return RC_E_ARG;
  if (int e = fits(*args)) return e;
  *bytes = kept_bytes(*args);
  return RC_OK;
}
extern "C" int rc_delta_forward_workspace(const rc_delta_args* args, uint64_t* bytes) {
  if (int e = check(args)) return e;
  if (!bytes) return RC_E_ARG;
  if (int e = fits(*args)) return e;
  *bytes = workspace_of(*args, false);
  return RC_OK;
}
extern "C" int rc_delta_backward_workspace(const rc_delta_args* args, uint64_t* bytes) {
  if (int e = check(args)) return e;
  if (!bytes) return RC_E_ARG;
  if (int e = fits_back(*args)) return e;
  *bytes = workspace_of(*args, true);
  return RC_OK;
}

extern "C" int rc_delta_forward(const rc_delta_args* args, void* stream) {
  if (int e = check(args)) return e;
  const rc_delta_args& a = *args;
  if (empty(a)) return RC_OK;
  if (a.length && (!a.q.data || !a.k.data || !a.v.data || !a.o.data || !a.beta.data)) return RC_E_ARG;
  if (!float_aligned(a.kept) || !float_aligned(a.workspace)) return RC_E_ARG;
  if (int e = fits(a)) return e;
  if (a.length && (!a.workspace || a.workspace_bytes < workspace_of(a, false))) return RC_E_SCRATCH;
  const hipStream_t s = (hipStream_t)stream;
  DeltaParams p = params(a);
  if (a.kept) p.written = a.kept + state_floats(a);
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_key(a.key, [&](auto kt) {
      constexpr int KT = decltype(kt)::value;
      if (int e = prepare<T, KT, false>(p, s)) return e;
      return by_width(a, [&](auto wide) {
        using G = ShapeOf<KT>;
        constexpr bool WIDE = decltype(wide)::value;
        if (p.segments > 1) {
          k_delta_forward<T, KT, G, WIDE, kEnds><<<walks_of<G, kEnds>(p, 32 * KT), G::THREADS, 0, s>>>(p);
          if (int e = launched("k_delta_forward")) return e;
          if (int e = join<KT, false>(p, s)) return e;
        }
        k_delta_forward<T, KT, G, WIDE, kWhole><<<walks_of<G, kWhole>(p, 0), G::THREADS, 0, s>>>(p);
        return launched("k_delta_forward");
      });
    });
  });
}

extern "C" int rc_delta_step(const rc_delta_step_args* args, void* stream) {
  if (!args) return RC_E_ARG;
  const rc_delta_step_args& a = *args;
  if (!dtype_ok(a.dtype) || a.batch < 0 || a.num_slots < 0 || a.key < 1 || a.key > kMaxHead ||
      a.value < 1 || a.value > kMaxHead || a.heads < 0 || a.key_heads < 0 ||
      !a.heads != !a.key_heads ||
      (a.heads && a.heads % a.key_heads))
    return RC_E_ARG;
  if (!a.batch || !a.heads) return RC_OK;
  if (!a.q.data || !a.k.data || !a.v.data || !a.o.data || !a.beta.data || !a.state ||
      !float_aligned(a.state) || (!a.slots && a.num_slots < a.batch))
    return RC_E_ARG;
  const int64_t slices = cdiv(a.value, 32);
  const int64_t bh = (int64_t)a.batch * a.heads;
  if (!launchable(bh, 256) || !launchable(slices * bh, 256)) return RC_E_OVERFLOW;
  const hipStream_t s = (hipStream_t)stream;
  const unsigned grid = (unsigned)(slices * bh);
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_key(a.key, [&](auto kt) {
      k_delta_step<T, decltype(kt)::value><<<grid, 256, 0, s>>>(StepParams{a});
      return launched("k_delta_step");
    });
  });
}
