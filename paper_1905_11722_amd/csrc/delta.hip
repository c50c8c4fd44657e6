// Gated delta rule.  Each head keeps a matrix S (key x value); a token decays
// it, reads what it holds for the key k, and writes back the difference to v:
//   S_t = a_t S_{t-1} + k_t w_t^T,  w_t = beta_t (v_t - a_t S_{t-1}^T k_t),
//   o_t = scale S_t^T q_t,  a = exp(g).
//
// The walk goes by chunks of 32 tokens.  With G the sum of g from the chunk's first token,
// S the state before it, and D_ij = exp(G_i - G_j) for j <= i,
//   W = T R,   R_i = beta_i (v_i - exp(G_i) S^T k_i),
//   T = (I + A)^-1,   A_ij = beta_i D_ij k_i . k_j   for j < i,
//   O_i = scale exp(G_i) S^T q_i + sum_j P_ij w_j,   P_ij = scale D_ij q_i . k_j,
//   S' = exp(G_31) S + sum_j exp(G_31 - G_j) k_j w_j^T.
// T and P need no state: k_delta_prepare computes them for all chunks at once, T by
// forward substitution.  What is left of a chunk are five products of at most
// 32 x key x value, k_delta_forward's, one chunk after the other.
//
// Backward, with dO and the gradient E of S':
//   dW_j = sum_i P_ij do_i + exp(G_31 - G_j) E^T k_j,   dR = T^T dW,   dv = beta dR,
//   dS = exp(G_31) E + sum_i exp(G_i) (scale q_i do_i^T - beta_i k_i dR_i^T)
// again one chunk after the other, from the last (k_delta_states_back); w and dR do
// not depend on how tokens are cut into chunks.  The other gradients then need no order
// (k_delta_inputs_back).  With M_ij = D_ij scale do_i . w_j and N_ij = D_ij dR_i . w_j (j < i),
//   dq_i = scale exp(G_i) S do_i + sum_j M_ij k_j
//   x_i = exp(G_i) S dR_i + sum_j N_ij k_j,    dbeta_i = dR_i . v_i - k_i . x_i
//   dk_i = -beta_i x_i (as read) + exp(G_31 - G_i) E w_i + sum_l (M_li q_l - beta_l N_li k_l) (as written)
//   dG_i = q_i . dq_i + k_i . (dk_i as read - as written),  dG_31 += <E, S'>,
//   dg_t = sum of dG_i over i >= t.
//
// Products run on the bf16 matrix instructions with operands taken apart into
// bf16 numbers that add up to them: one for bf16, two for f16, three for 32 bits, and
// the products of pieces down to 2^-16 of the largest: 32-bit results from instructions with 16
// times the rate of the 32-bit ones.  D's exponents are differences
// of sums in 64 bits, so a token that forgets everything costs the later ones nothing.
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int kChunk = 32;
constexpr int kMaxHead = 256;

typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// bf16 numbers that hold a T exactly.
template <class T>
constexpr int kPieces = sizeof(T) == 4 ? 3 : 2;
template <>
constexpr int kPieces<bf16> = 1;

template <int N>
struct Pieces {
  bf16x8 p[N];
};

template <int N>
__device__ __forceinline__ Pieces<N> split(const float (&v)[8]) {
  Pieces<N> s;
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = v[e];
#pragma unroll
  for (int i = 0; i < N; i++)
#pragma unroll
    for (int e = 0; e < 8; e++) {
      s.p[i][e] = (bf16)x[e];
      if (i + 1 < N) x[e] -= (float)s.p[i][e];
    }
  return s;
}

// acc += A B for 16 x 32 by 32 x 16, the smallest products of pieces first.  A lane holds 8
// numbers of row (column) lane % 16; which 8 of the 32 is free as long as both sides agree.
// The result's lane holds rows 4 (lane / 16) + 0..3 of column lane % 16.
template <int NA, int NB>
__device__ __forceinline__ void mul(f32x4& acc, const Pieces<NA>& a, const Pieces<NB>& b) {
#pragma unroll
  for (int s = 2; s >= 0; s--)
#pragma unroll
    for (int i = 0; i <= s; i++)
      if (i < NA && s - i < NB)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], acc, 0, 0, 0);
}

// Two results of 16 rows each are 32 rows of an operand as they are: lane group g holds
// rows 4g + 0..3 and 16 + 4g + 0..3.  All operands below take their 32 in that order.
template <int N>
__device__ __forceinline__ Pieces<N> operand(const f32x4& lo, const f32x4& hi) {
  const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return split<N>(x);
}

// exp(x), x in 64 bits.
__device__ __forceinline__ float exp_of(double x) {
  const double e = x * 1.44269504088896340736;
  const double n = __builtin_rint(e);
  return __builtin_amdgcn_ldexpf(fast_exp2((float)(e - n)), (int)__builtin_fmax(n, -1000.0));
}

// 32 tokens of `32 KT` channels in LDS as pieces.  Within each 32 channels, groups of four
// are ordered 0 4 1 5 2 6 3 7, so that a lane's operand (above) is 16 bytes.
template <int KT, int N>
struct Tokens {
  static constexpr int STRIDE = KT * 32 + 8;
  bf16 at[N][kChunk][STRIDE];

  // From rows `row` elements apart; what is past `live` tokens or `n` channels is 0.
  template <class T>
  __device__ void load(const T* x, int64_t row, int live, int n, int thread, int threads) {
    for (int i = thread; i < kChunk * KT * 4; i += threads) {
      const int r = i / (KT * 4), c = i % (KT * 4) * 8;
      float v[8];
      load_vec<8>(x + (r < live ? r : 0) * row + (c < n ? c : 0), r < live ? n - c : 0, v);
      put(r, c, v);
    }
  }
  __device__ void put(int r, int c, const float (&v)[8]) {
    const Pieces<N> s = split<N>(v);
    bf16* to = &at[0][r][c / 32 * 32 + (c % 16 / 4) * 8 + c % 32 / 16 * 4];
#pragma unroll
    for (int i = 0; i < N; i++) {
      *(bf16x4*)(to + i * (kChunk * STRIDE)) = s.p[i].lo;
      *(bf16x4*)(to + i * (kChunk * STRIDE) + 8) = s.p[i].hi;
    }
  }
  // Row tile t (tokens 16t + ..) over channels 32s + 0..31.
  __device__ Pieces<N> rows(int t, int s) const {
    const int lane = threadIdx.x % 64;
    Pieces<N> f;
#pragma unroll
    for (int i = 0; i < N; i++)
      f.p[i] = *(const bf16x8*)&at[i][16 * t + lane % 16][32 * s + lane / 16 * 8];
    return f;
  }
  // Channels 16t + .. over the 32 tokens: reads that transpose four by four.
  __device__ Pieces<N> columns(int t) const {
    const int lane = threadIdx.x % 64;
    Pieces<N> f;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const bf16* from =
          &at[i][lane / 16 * 4 + lane % 16 / 4][t / 2 * 32 + lane % 4 * 8 + t % 2 * 4];
      typedef s16x4 __attribute__((address_space(3))) * lds;
      f.p[i].lo = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)from));
      f.p[i].hi = __builtin_bit_cast(
          bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(from + 16 * STRIDE)));
    }
    return f;
  }
  __device__ float value(int r, int c) const {
    const int at_c = c / 32 * 32 + c % 16 / 4 * 8 + c % 32 / 16 * 4 + c % 4;
    float x = (float)at[N - 1][r][at_c];
#pragma unroll
    for (int i = N - 2; i >= 0; i--) x += (float)at[i][r][at_c];
    return x;
  }
};

// What k_delta_prepare leaves for one chunk of one head: T and P (backward: their
// transposes) as operands of two row tiles, and numbers of each token.
struct Chunk {
  bf16x8 t[2][3][64], p[2][3][64];
  float since[kChunk], left[kChunk], beta[kChunk];    // exp(G_i), exp(G_31 - G_i), beta_i
};

struct DeltaParams {
  rc_delta_args a;
  int32_t chunks;
  Chunk* prepared;                                    // [batch][heads][chunks]
  float* states;                                      // [batch][heads][chunks][key][value]
  float* written;                                     // w, or dR: [batch][heads][chunks][32][value]
  const float* kept_written;
  float* dstates;
  float* partial;                                     // [2][batch][length][heads][key]
};

__device__ __forceinline__ int length_of(const rc_delta_args& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.length) : a.length;
}
__device__ __forceinline__ float at_token(const rc_view& v, int64_t b, int64_t t, int64_t h) {
  return static_cast<const float*>(v.data)[b * v.batch + t * v.time + h];
}

// g of a token.  One below -1000 counts as -1000: exp of either is 0 in 32 bits, and
// -infinity has no differences.
__device__ __forceinline__ double log_decay(const rc_view& g, int64_t b, int64_t t, int64_t h) {
  const float x = at_token(g, b, t, h);
  return x < -1000.f ? -1000.0 : (double)x;
}
// G of a chunk's 32 tokens (in every lane's token lane % 32): sums from its first token.
__device__ __forceinline__ double sum_of_g(const rc_delta_args& a, int b, int h, int t0, int live) {
  const int i = threadIdx.x % 32;
  double G = 0;
  if (a.g.data && i < live) G = log_decay(a.g, b, t0 + i, h);
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const double before = __shfl_up(G, d, 32);
    if (i >= d) G += before;
  }
  return G;
}

template <class T, int KT, bool BACK>
__global__ __launch_bounds__(64) void k_delta_prepare(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>;
  __shared__ double sums[kChunk];
  __shared__ float beta[kChunk];
  __shared__ float A[kChunk][kChunk + 4], inverse[kChunk][kChunk + 4];
  const int lane = threadIdx.x, bh = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  const int b = bh / a.heads, h = bh % a.heads;
  const int hk = h / (a.heads / a.key_heads), t0 = chunk * kChunk;
  const int live = min(length_of(a, b) - t0, kChunk);
  if (live <= 0) return;
  // tokens 16m + lane % 16 over channels 32s + 8 (lane / 16) ..
  const auto rows = [&](const rc_heads& x, int m, int s) {
    const int t = 16 * m + lane % 16, c = 32 * s + lane / 16 * 8;
    float v[8];
    load_vec<8>(at_head<T>(x, b, t0 + (t < live ? t : 0), hk) + (c < a.key ? c : 0),
                t < live ? a.key - c : 0, v);
    return split<N>(v);
  };
  Chunk& out = p.prepared[blockIdx.x];
  const double G = sum_of_g(a, b, h, t0, live);
  if (lane < kChunk) {
    const double last = __shfl(G, kChunk - 1);
    sums[lane] = G;
    beta[lane] = lane < live ? at_token(a.beta, b, t0 + lane, h) : 0.f;
    out.since[lane] = exp_of(G);
    out.left[lane] = exp_of(last - G);
    out.beta[lane] = beta[lane];
  }
  __syncthreads();
  // tiles of k_i . k_j and q_i . k_j with rows j (backward for P: rows i) and the other as columns
  f32x4 kk[2][2], qk[2][2];
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int n = 0; n < 2; n++) kk[m][n] = qk[m][n] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < KT; s++) {
    const Pieces<N> ks[2] = {rows(a.k, 0, s), rows(a.k, 1, s)};
    const Pieces<N> qs[2] = {rows(a.q, 0, s), rows(a.q, 1, s)};
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int n = 0; n < 2; n++) {
        if (m <= n) mul(kk[m][n], ks[m], ks[n]);      // rows j of tile m, columns i of tile n
        if (BACK ? m >= n : m <= n) mul(qk[m][n], BACK ? qs[m] : ks[m], BACK ? ks[n] : qs[n]);
      }
  }
  const int col = lane % 16, row = lane / 16 * 4;
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int n = 0; n < 2; n++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const int i = 16 * n + col, j = 16 * m + row + r;
        A[i][j] = j < i ? beta[i] * exp_of(sums[i] - sums[j]) * kk[m][n][r] : 0.f;
        const int pi = BACK ? j : i, pj = BACK ? i : j;
        qk[m][n][r] = pj <= pi ? a.scale * exp_of(sums[pi] - sums[pj]) * qk[m][n][r] : 0.f;
      }
#pragma unroll
  for (int n = 0; n < 2; n++) {
    const Pieces<3> f = operand<3>(qk[0][n], qk[1][n]);
#pragma unroll
    for (int i = 0; i < 3; i++) out.p[n][i][lane] = f.p[i];
  }
  __syncthreads();
  // T, a column a lane, by forward substitution
  {
    const int c = lane % 32;
    float t[kChunk];
#pragma unroll
    for (int i = 0; i < kChunk; i++) {
      float s = i == c ? 1.f : 0.f;
#pragma unroll
      for (int j = 0; j < i; j++) s = fmaf(-A[i][j], t[j], s);
      t[i] = s;
      if (lane < 32) inverse[i][c] = s;
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < 2; n++) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const int i = 16 * n + col, j = 16 * (e / 4) + row + e % 4;
      x[e] = BACK ? inverse[j][i] : inverse[i][j];
    }
    const Pieces<3> f = split<3>(x);
#pragma unroll
    for (int i = 0; i < 3; i++) out.t[n][i][lane] = f.p[i];
  }
}

// A head's state, 16 columns a wave: tile m of 16 rows, this lane's column and rows.
template <int KT>
__device__ __forceinline__ void load_state(const float* from, const rc_delta_args& a, int col,
                                           f32x4 (&S)[2 * KT]) {
  const int row = threadIdx.x % 64 / 16 * 4;
#pragma unroll
  for (int m = 0; m < 2 * KT; m++)
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = 16 * m + row + r;
      S[m][r] = from && i < a.key && col < a.value ? from[(int64_t)i * a.value + col] : 0.f;
    }
}
template <int KT>
__device__ __forceinline__ void store_state(float* to, const rc_delta_args& a, int col,
                                            const f32x4 (&S)[2 * KT]) {
  const int row = threadIdx.x % 64 / 16 * 4;
#pragma unroll
  for (int m = 0; m < 2 * KT; m++)
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = 16 * m + row + r;
      if (i < a.key && col < a.value) to[(int64_t)i * a.value + col] = S[m][r];
    }
}

// What a chunk's products need beside the state, loaded one chunk ahead: this thread's share of
// the tokens' keys and queries, T and P, and for the lane's column and its eight tokens
// (4 (lane / 16) + 0..3 and 16 more) the values or the outputs' gradients.  Loads
// are unconditional with addresses inside the chunk; what is past its end is dropped when used.
template <class T, int KT, int W, bool WIDE>
struct Feed {
  static constexpr int N = kPieces<T>, VECTORS = kChunk * KT * 4, EACH = (VECTORS + 64 * W - 1) / (64 * W);
  typedef T TV __attribute__((ext_vector_type(8)));
  TV k[EACH], q[EACH];
  bf16x8 t[2][3], p[2][3];
  T x[8];
  float4 since[2], left[2], beta[2];
  float whole;

  __device__ static int row_of(int i) { return (threadIdx.x + i * 64 * W) / (KT * 4); }
  __device__ static int channel_of(int i) { return (threadIdx.x + i * 64 * W) % (KT * 4) * 8; }

  __device__ void fetch(const rc_delta_args& a, const Chunk& c, const rc_heads& values, int b, int h, int hk,
                        int t0, int live, int col) {
#pragma unroll
    for (int i = 0; i < EACH; i++) {
      const int r = min(row_of(i), live - 1), ch = channel_of(i);
      const T* from = at_head<T>(a.k, b, t0 + r, hk);
      const T* fromq = at_head<T>(a.q, b, t0 + r, hk);
      if (WIDE) {
        const int at = ch < a.key ? ch : 0;
        __builtin_memcpy(&k[i], from + at, sizeof(TV));
        __builtin_memcpy(&q[i], fromq + at, sizeof(TV));
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) {
          k[i][e] = from[min(ch + e, a.key - 1)];
          q[i][e] = fromq[min(ch + e, a.key - 1)];
        }
      }
    }
    const int lane = threadIdx.x % 64, row = lane / 16 * 4;
#pragma unroll
    for (int m = 0; m < 2; m++) {
#pragma unroll
      for (int i = 0; i < 3; i++) {
        t[m][i] = c.t[m][i][lane];
        p[m][i] = c.p[m][i][lane];
      }
      since[m] = *(const float4*)&c.since[16 * m + row];
      left[m] = *(const float4*)&c.left[16 * m + row];
      beta[m] = *(const float4*)&c.beta[16 * m + row];
#pragma unroll
      for (int e = 0; e < 4; e++)
        x[4 * m + e] = at_head<T>(values, b, t0 + min(16 * m + row + e, live - 1), h)[min(col, a.value - 1)];
    }
    whole = c.since[kChunk - 1];
  }
  __device__ void put(Tokens<KT, N>& to_k, Tokens<KT, N>& to_q, int live, int key) const {
#pragma unroll
    for (int i = 0; i < EACH; i++) {
      const int r = row_of(i), ch = channel_of(i);
      if (VECTORS % (64 * W) && r >= kChunk) break;
      float v[8], w[8];
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const bool on = r < live && ch + e < key;
        v[e] = on ? (float)k[i][e] : 0.f;
        w[e] = on ? (float)q[i][e] : 0.f;
      }
      to_k.put(r, ch, v);
      to_q.put(r, ch, w);
    }
  }
};
__device__ __forceinline__ Pieces<3> pieces(const bf16x8 (&x)[3]) { return {{x[0], x[1], x[2]}}; }
__device__ __forceinline__ float element(const float4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// Forward: a wave holds 16 columns of the state in registers from the first chunk to the
// last; columns do not depend on one another, and what a product leaves in a lane is what the
// next one takes from it, so waves share nothing but the tokens in LDS.
template <class T, int KT, int W, bool WIDE>
__global__ __launch_bounds__(64 * W) void k_delta_forward(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, BUFFERS = sizeof(Tokens<KT, N>) * 4 <= 128 * 1024 ? 2 : 1;
  __shared__ Tokens<KT, N> tokens[BUFFERS][2];
  const int slices = (a.value + 16 * W - 1) / (16 * W);
  const int lane = threadIdx.x % 64, bh = blockIdx.x / slices, b = bh / a.heads, h = bh % a.heads;
  const int hk = h / (a.heads / a.key_heads), end = length_of(a, b);
  const int wave = blockIdx.x % slices * W + threadIdx.x / 64;
  const int col = wave * 16 + lane % 16, row = lane / 16 * 4;
  const bool on = col < a.value;
  const int64_t size = (int64_t)a.key * a.value;
  const Chunk* prepared = p.prepared + (int64_t)bh * p.chunks;
  f32x4 S[2 * KT];
  load_state<KT>(a.state_in ? a.state_in + bh * size : nullptr, a, col, S);
  T* o = at_head<T>(a.o, b, 0, h) + col;
  const int chunks = (end + kChunk - 1) / kChunk;
  Feed<T, KT, W, WIDE> next;
  if (chunks) next.fetch(a, prepared[0], a.v, b, h, hk, 0, min(end, kChunk), col);
  for (int chunk = 0; chunk < chunks; chunk++) {
    const int t0 = chunk * kChunk, live = min(end - t0, kChunk);
    Tokens<KT, N>&k = tokens[chunk % BUFFERS][0], &q = tokens[chunk % BUFFERS][1];
    if (BUFFERS == 1) __syncthreads();
    next.put(k, q, live, a.key);
    __syncthreads();
    const Feed<T, KT, W, WIDE> c = next;
    {
      const int n = min(chunk + 1, chunks - 1);
      next.fetch(a, prepared[n], a.v, b, h, hk, n * kChunk, min(end - n * kChunk, kChunk), col);
    }
    if (p.states) store_state<KT>(p.states + ((int64_t)bh * p.chunks + chunk) * size, a, col, S);
    f32x4 r[2], out[2], w[2];
#pragma unroll
    for (int m = 0; m < 2; m++) r[m] = out[m] = w[m] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < KT; s++) {
      const Pieces<3> state = operand<3>(S[2 * s], S[2 * s + 1]);
#pragma unroll
      for (int m = 0; m < 2; m++) {
        mul(r[m], k.rows(m, s), state);
        mul(out[m], q.rows(m, s), state);
      }
    }
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int t = 16 * m + row + e;
        const float x = on && t < live ? (float)c.x[4 * m + e] : 0.f, since = element(c.since[m], e);
        r[m][e] = element(c.beta[m], e) * (x - since * r[m][e]);
        out[m][e] *= a.scale * since;
      }
    const Pieces<3> rs = operand<3>(r[0], r[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) mul(w[m], pieces(c.t[m]), rs);
    const Pieces<3> ws = operand<3>(w[0], w[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) {
      mul(out[m], pieces(c.p[m]), ws);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int t = 16 * m + row + e;
        if (on && t < live) o[(t0 + t) * a.o.time] = (T)out[m][e];
        if (p.written && on)
          p.written[(((int64_t)bh * p.chunks + chunk) * kChunk + t) * a.value + col] = w[m][e];
        w[m][e] *= element(c.left[m], e);
      }
    }
    const Pieces<3> us = operand<3>(w[0], w[1]);
#pragma unroll
    for (int m = 0; m < 2 * KT; m++) {
      S[m] *= c.whole;
      mul(S[m], k.columns(m), us);
    }
  }
  if (a.state_out) store_state<KT>(a.state_out + bh * size, a, col, S);
  if (on)
    for (int t = end + lane / 16; t < a.length; t += 4) o[t * a.o.time] = (T)0.f;
}

// Backward through the states, from the last chunk to the first.
template <class T, int KT, int W, bool WIDE>
__global__ __launch_bounds__(64 * W) void k_delta_states_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, BUFFERS = sizeof(Tokens<KT, N>) * 4 <= 128 * 1024 ? 2 : 1;
  __shared__ Tokens<KT, N> tokens[BUFFERS][2];
  const int slices = (a.value + 16 * W - 1) / (16 * W);
  const int lane = threadIdx.x % 64, bh = blockIdx.x / slices, b = bh / a.heads, h = bh % a.heads;
  const int hk = h / (a.heads / a.key_heads), end = length_of(a, b);
  const int wave = blockIdx.x % slices * W + threadIdx.x / 64;
  const int col = wave * 16 + lane % 16, row = lane / 16 * 4;
  const bool on = col < a.value;
  const int64_t size = (int64_t)a.key * a.value;
  const Chunk* prepared = p.prepared + (int64_t)bh * p.chunks;
  f32x4 E[2 * KT];
  load_state<KT>(a.dstate_out ? a.dstate_out + bh * size : nullptr, a, col, E);
  T* dv = at_head<T>(a.dv, b, 0, h) + col;
  const int chunks = (end + kChunk - 1) / kChunk;
  Feed<T, KT, W, WIDE> next;
  if (chunks) {
    const int n = chunks - 1;
    next.fetch(a, prepared[n], a.do_, b, h, hk, n * kChunk, end - n * kChunk, col);
  }
  for (int chunk = chunks - 1; chunk >= 0; chunk--) {
    const int t0 = chunk * kChunk, live = min(end - t0, kChunk);
    Tokens<KT, N>&k = tokens[chunk % BUFFERS][0], &q = tokens[chunk % BUFFERS][1];
    if (BUFFERS == 1) __syncthreads();
    next.put(k, q, live, a.key);
    __syncthreads();
    const Feed<T, KT, W, WIDE> c = next;
    {
      const int n = max(chunk - 1, 0);
      next.fetch(a, prepared[n], a.do_, b, h, hk, n * kChunk, min(end - n * kChunk, kChunk), col);
    }
    store_state<KT>(p.dstates + ((int64_t)bh * p.chunks + chunk) * size, a, col, E);
    f32x4 dw[2], dr[2], g[2];
#pragma unroll
    for (int m = 0; m < 2; m++) dw[m] = dr[m] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < KT; s++) {
      const Pieces<3> state = operand<3>(E[2 * s], E[2 * s + 1]);
#pragma unroll
      for (int m = 0; m < 2; m++) mul(dw[m], k.rows(m, s), state);
    }
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        g[m][e] = on && 16 * m + row + e < live ? (float)c.x[4 * m + e] : 0.f;
        dw[m][e] *= element(c.left[m], e);
      }
    const Pieces<N> gs = operand<N>(g[0], g[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) mul(dw[m], pieces(c.p[m]), gs);
    const Pieces<3> dws = operand<3>(dw[0], dw[1]);
#pragma unroll
    for (int m = 0; m < 2; m++) {
      mul(dr[m], pieces(c.t[m]), dws);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int t = 16 * m + row + e;
        if (on) p.written[(((int64_t)bh * p.chunks + chunk) * kChunk + t) * a.value + col] = dr[m][e];
        const float x = element(c.beta[m], e) * dr[m][e], since = element(c.since[m], e);
        if (on && t < live) dv[(t0 + t) * a.dv.time] = (T)x;
        dr[m][e] = -since * x;
        g[m][e] *= a.scale * since;
      }
    }
    const Pieces<3> drs = operand<3>(dr[0], dr[1]), gos = operand<3>(g[0], g[1]);
#pragma unroll
    for (int m = 0; m < 2 * KT; m++) {
      E[m] *= c.whole;
      mul(E[m], k.columns(m), drs);
      mul(E[m], q.columns(m), gos);
    }
  }
  if (a.dstate_in) store_state<KT>(a.dstate_in + bh * size, a, col, E);
  if (on)
    for (int t = end + lane / 16; t < a.length; t += 4) dv[t * a.dv.time] = (T)0.f;
}

// The gradients of one chunk's inputs from the state before it and the gradient of
// the one after it.  Four waves; each takes some of the key's tiles of 16 channels.
template <class T, int KT>
__global__ __launch_bounds__(256) void k_delta_inputs_back(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int N = kPieces<T>, NT = (2 * KT + 3) / 4;
  __shared__ Tokens<KT, N> k, q;
  __shared__ Tokens<1, N> od;
  __shared__ Tokens<1, 3> rd, wr;
  __shared__ float M[kChunk][kChunk + 4], Q[kChunk][kChunk + 4];   // M, N of the file's head
  __shared__ double sums[kChunk];
  __shared__ float dots[4][4][kChunk], inner[4], dot_v[kChunk];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int bh = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks, b = bh / a.heads, h = bh % a.heads;
  const int per = a.heads / a.key_heads, hk = h / per, t0 = chunk * kChunk;
  const int live = min(length_of(a, b) - t0, kChunk), here = min(a.length - t0, kChunk);
  const int64_t size = (int64_t)a.key * a.value;
  // dq and dk of head h, or their parts in 32 bits where heads share a key head
  const auto store = [&](int which, int t, int c, float x) {
    if (per == 1)
      at_head<T>(which ? a.dk : a.dq, b, t0 + t, h)[c] = (T)x;
    else
      p.partial[(((int64_t)which * a.batch + b) * a.length + t0 + t) * a.heads * a.key +
                (int64_t)h * a.key + c] = x;
  };
  if (live <= 0) {
    for (int i = tid; i < here * a.key; i += 256) {
      store(0, i / a.key, i % a.key, 0.f);
      store(1, i / a.key, i % a.key, 0.f);
    }
    if (tid < here) {
      const int64_t at = ((int64_t)b * a.length + t0 + tid) * a.heads + h;
      if (a.dg) a.dg[at] = 0.f;
      a.dbeta[at] = 0.f;
    }
    return;
  }
  const float* S = p.states + ((int64_t)bh * p.chunks + chunk) * size;
  const float* E = p.dstates + ((int64_t)bh * p.chunks + chunk) * size;
  const float* w_at = p.kept_written + ((int64_t)bh * p.chunks + chunk) * kChunk * a.value;
  const float* r_at = p.written + ((int64_t)bh * p.chunks + chunk) * kChunk * a.value;
  k.load(at_head<T>(a.k, b, t0, hk), a.k.time, live, a.key, tid, 256);
  q.load(at_head<T>(a.q, b, t0, hk), a.q.time, live, a.key, tid, 256);
  if (tid < 64) {
    const double G = sum_of_g(a, b, h, t0, live);
    if (tid < kChunk) sums[tid] = G;
  }
  f32x4 xq[2][NT], xr[2][NT], xw[2][NT], m_tile = {0, 0, 0, 0}, n_tile = {0, 0, 0, 0};
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int n = 0; n < NT; n++) xq[m][n] = xr[m][n] = xw[m][n] = f32x4{0, 0, 0, 0};
  const int ti = wave > 0, tj = wave == 2;            // waves 0 to 2: tile (ti, tj) of M and N
  float es = 0.f, rv = 0.f;
  for (int c0 = 0; c0 < a.value; c0 += 32) {
    __syncthreads();
    if (tid < kChunk * 4) {
      const int t = tid / 4, c = c0 + tid % 4 * 8, n = a.value - c, at = c < a.value ? c : 0;
      const int tl = t < live ? t : 0, nl = t < live ? n : 0;
      float x[8], y[8];
      load_vec<8>(at_head<T>(a.do_, b, t0 + tl, h) + at, nl, x);
      od.put(t, tid % 4 * 8, x);
      load_vec<8>(w_at + (int64_t)t * a.value + at, n, x);
      wr.put(t, tid % 4 * 8, x);
      load_vec<8>(r_at + (int64_t)t * a.value + at, n, x);
      rd.put(t, tid % 4 * 8, x);
      load_vec<8>(at_head<T>(a.v, b, t0 + tl, h) + at, nl, y);
#pragma unroll
      for (int i = 0; i < 8; i++) rv = fmaf(x[i], y[i], rv);
    }
    __syncthreads();
    const Pieces<N> os[2] = {od.rows(0, 0), od.rows(1, 0)};
    const Pieces<3> rs[2] = {rd.rows(0, 0), rd.rows(1, 0)}, ws[2] = {wr.rows(0, 0), wr.rows(1, 0)};
#pragma unroll
    for (int n = 0; n < NT; n++) {
      const int row = 16 * (wave * NT + n) + lane % 16;
      float x[8], y[8];
      const int lo = c0 + lane / 16 * 4;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const int c = lo + e * 4, at = row < a.key && c < a.value;
        float u[4];
        load_vec<4>(S + (at ? (int64_t)row * a.value + c : 0), at ? a.value - c : 0, u);
#pragma unroll
        for (int i = 0; i < 4; i++) x[e + i] = u[i];
        load_vec<4>(E + (at ? (int64_t)row * a.value + c : 0), at ? a.value - c : 0, u);
#pragma unroll
        for (int i = 0; i < 4; i++) {
          y[e + i] = u[i];
          es = fmaf(x[e + i], u[i], es);
        }
      }
      const Pieces<3> ss = split<3>(x), ds = split<3>(y);
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
  const int col = lane % 16, row = lane / 16 * 4;
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
#pragma unroll
  for (int d = 1; d < 64; d *= 2) es += __shfl_xor(es, d);
  if (lane == 0) inner[wave] = es;
  rv += __shfl_xor(rv, 1, 4);
  rv += __shfl_xor(rv, 2, 4);
  if (tid < kChunk * 4 && tid % 4 == 0) dot_v[tid / 4] = rv;
  __syncthreads();
  const double last = sums[kChunk - 1];
  const auto beta_of = [&](int t) { return t < live ? at_token(a.beta, b, t0 + t, h) : 0.f; };
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
      x[3][e] = -beta_of(j) * Q[j][i];
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
#pragma unroll
  for (int n = 0; n < NT; n++) {
    const int tile = wave * NT + n, c = 16 * tile + col;
    if (tile >= 2 * KT) break;
    const Pieces<N> kc = k.columns(tile), qc = q.columns(tile);
#pragma unroll
    for (int m = 0; m < 2; m++) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const double G = sums[16 * m + row + e];
        xq[m][n][e] *= a.scale * exp_of(G);
        xr[m][n][e] *= exp_of(G);
        xw[m][n][e] *= exp_of(last - G);
        dot[3][m][e] = fmaf(k.value(16 * m + row + e, c), xw[m][n][e], dot[3][m][e]);
      }
      mul(xq[m][n], m_rows[m], kc);
      mul(xr[m][n], n_rows[m], kc);
      mul(xw[m][n], m_cols[m], qc);
      mul(xw[m][n], n_cols[m], kc);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int t = 16 * m + row + e;
        const float kv = k.value(t, c), qv = q.value(t, c), beta = beta_of(t);
        const float read = -beta * xr[m][n][e];
        dot[0][m][e] = fmaf(qv, xq[m][n][e], fmaf(kv, read, dot[0][m][e]));
        dot[1][m][e] = fmaf(kv, xw[m][n][e], dot[1][m][e]);
        dot[2][m][e] = fmaf(kv, xr[m][n][e], dot[2][m][e]);
        if (t < here && c < a.key) {
          store(0, t, c, xq[m][n][e]);
          store(1, t, c, read + xw[m][n][e]);
        }
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

// dq and dk of key heads that several heads share: the sums of the heads' parts.
template <class T>
__global__ __launch_bounds__(256) void k_delta_shared_heads(DeltaParams p, int64_t n) {
  const rc_delta_args& a = p.a;
  const int per = a.heads / a.key_heads;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * n) return;
  const int which = i >= n;
  const int64_t e = i - which * n;
  const int c = (int)(e % a.key);
  const int64_t row = e / a.key;                      // (b, t, key head)
  const float* from = p.partial + which * n * per + row * per * a.key + c;
  float s = 0.f;
  for (int j = 0; j < per; j++) s += from[(int64_t)j * a.key];
  const int64_t token = row / a.key_heads;
  at_head<T>(which ? a.dk : a.dq, token / a.length, token % a.length, row % a.key_heads)[c] = (T)s;
}

// ------------------------------------------------------------- single tokens

struct StepParams {
  rc_delta_step_args a;
};

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

// ------------------------------------------------------------------ host side

constexpr int kWaves = 4;

int check(const rc_delta_args* a) {
  if (!a || !dtype_ok(a->dtype) || a->batch < 0 || a->length < 0 || a->length > kMaxExtent ||
      a->key < 1 || a->key > kMaxHead || a->value < 1 || a->value > kMaxHead)
    return RC_E_ARG;
  if (a->heads < 0 || a->key_heads < 0 || (a->heads && (!a->key_heads || a->heads % a->key_heads)))
    return RC_E_ARG;
  return RC_OK;
}
bool empty(const rc_delta_args& a) { return !a.batch || !a.heads; }

int64_t chunks_of(const rc_delta_args& a) { return cdiv(a.length, kChunk); }
// Chunks of all heads.  (batch x heads is checked first: it fits a launch.)
int64_t pairs_of(const rc_delta_args& a) { return (int64_t)a.batch * a.heads * chunks_of(a); }
uint64_t kept_bytes(const rc_delta_args& a) {
  return (uint64_t)pairs_of(a) * a.value * (a.key + kChunk) * sizeof(float);
}
// Whether the sizes fit the launches.
int fits(const rc_delta_args& a) {
  const int64_t bh = (int64_t)a.batch * a.heads;
  if (!launchable(bh, 256) || !launchable(bh * cdiv(a.value, 16 * kWaves), 64 * kWaves) ||
      !launchable(pairs_of(a), 256))
    return RC_E_OVERFLOW;
  if (!launchable(cdiv(2 * (int64_t)a.batch * a.length * a.key_heads * a.key, 256), 256))
    return RC_E_OVERFLOW;
  return RC_OK;
}
uint64_t workspace_of(const rc_delta_args& a, bool back) {
  uint64_t n = (uint64_t)pairs_of(a) * sizeof(Chunk);
  if (back) {
    n += kept_bytes(a);
    if (a.heads != a.key_heads)
      n += 2 * (uint64_t)a.batch * a.length * a.heads * a.key * sizeof(float);
  }
  return n;
}

// f(whether rows of the key are whole loads of eight).
template <class F>
int by_width(int32_t key, F&& f) {
  return key % 8 ? f(std::false_type{}) : f(std::true_type{});
}
// f(integral_constant of the key's tiles of 32).
template <class F>
int by_key(int32_t key, F&& f) {
  if (key <= 32) return f(std::integral_constant<int, 1>{});
  if (key <= 64) return f(std::integral_constant<int, 2>{});
  if (key <= 128) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 8>{});
}

DeltaParams params(const rc_delta_args& a) {
  DeltaParams p = {};
  p.a = a;
  p.chunks = (int32_t)chunks_of(a);
  p.prepared = static_cast<Chunk*>(a.workspace);
  p.states = a.kept;
  return p;
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
  if (int e = fits(*args)) return e;
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
  if (a.kept) p.written = a.kept + pairs_of(a) * a.key * a.value;
  const int64_t bh = (int64_t)a.batch * a.heads;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_key(a.key, [&](auto kt) {
      constexpr int KT = decltype(kt)::value;
      if (p.chunks) {
        k_delta_prepare<T, KT, false><<<(unsigned)pairs_of(a), 64, 0, s>>>(p);
        if (int e = launched("k_delta_prepare")) return e;
      }
      return by_width(a.key, [&](auto wide) {
        k_delta_forward<T, KT, kWaves, decltype(wide)::value>
            <<<(unsigned)(bh * cdiv(a.value, 16 * kWaves)), 64 * kWaves, 0, s>>>(p);
        return launched("k_delta_forward");
      });
    });
  });
}

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
  const int64_t pairs = pairs_of(a), size = (int64_t)a.key * a.value;
  p.kept_written = a.kept + pairs * size;
  p.dstates = reinterpret_cast<float*>(p.prepared + pairs);
  p.written = p.dstates + pairs * size;
  p.partial = p.written + pairs * kChunk * a.value;
  const int64_t bh = (int64_t)a.batch * a.heads;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    return by_key(a.key, [&](auto kt) {
      constexpr int KT = decltype(kt)::value;
      if (p.chunks) {
        k_delta_prepare<T, KT, true><<<(unsigned)pairs_of(a), 64, 0, s>>>(p);
        if (int e = launched("k_delta_prepare")) return e;
      }
      const int e = by_width(a.key, [&](auto wide) {
        k_delta_states_back<T, KT, kWaves, decltype(wide)::value>
            <<<(unsigned)(bh * cdiv(a.value, 16 * kWaves)), 64 * kWaves, 0, s>>>(p);
        return launched("k_delta_states_back");
      });
      if (e) return e;
      if (!p.chunks) return (int)RC_OK;
      k_delta_inputs_back<T, KT><<<(unsigned)pairs_of(a), 256, 0, s>>>(p);
      if (int e = launched("k_delta_inputs_back")) return e;
      if (a.heads == a.key_heads) return (int)RC_OK;
      const int64_t n = (int64_t)a.batch * a.length * a.key_heads * a.key;
      k_delta_shared_heads<T><<<(unsigned)cdiv(2 * n, 256), 256, 0, s>>>(p, n);
      return launched("k_delta_shared_heads");
    });
  });
}

extern "C" int rc_delta_step(const rc_delta_step_args* args, void* stream) {
  if (!args) return RC_E_ARG;
  const rc_delta_step_args& a = *args;
  if (!dtype_ok(a.dtype) || a.batch < 0 || a.num_slots < 0 || a.key < 1 || a.key > kMaxHead ||
      a.value < 1 || a.value > kMaxHead || a.heads < 0 || a.key_heads < 0 ||
      (a.heads && (!a.key_heads || a.heads % a.key_heads)))
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
