// Shared by the gated delta rule's kernels (delta.hip, delta_back.hip).  Each head keeps a matrix S
// (key x value); a token decays it, reads what it holds for the key k, and writes back the
// difference to v:
//   S_t = a_t S_{t-1} + k_t w_t^T,  w_t = beta_t (v_t - a_t S_{t-1}^T k_t),
//   o_t = scale S_t^T q_t,  a = exp(g).
//
// The walk goes by chunks of 32 tokens.  With G the sum of g from the chunk's first token,
// S the state before it, and D_ij = exp(G_i - G_j) for j <= i,
//   W = T R,   R_i = beta_i (v_i - exp(G_i) S^T k_i),
//   T = (I + A)^-1,   A_ij = beta_i D_ij k_i . k_j   for j < i,
//   O_i = scale exp(G_i) S^T q_i + sum_j (P T)_ij R_j,   P_ij = scale D_ij q_i . k_j,
//   S' = exp(G_31) S + sum_j exp(G_31 - G_j) k_j w_j^T.
// T and P T need no state: k_delta_prepare computes them for all chunks at once, T by
// forward substitution (its diagonal tiles of 16, then the one below them from both).  What is left
// of a chunk are five products of at most 32 x key x value, k_delta_forward's, one
// chunk after the other.
//
// Backward, with dO and the gradient E of S':
//   dW_j = sum_i P_ij do_i + exp(G_31 - G_j) E^T k_j,   dR = T^T dW,   dv = beta dR,
//   dS = exp(G_31) E + sum_i exp(G_i) (scale q_i do_i^T - beta_i k_i dR_i^T)
// again one chunk after the other, from the last (k_delta_states_back); w and dR do
// not depend on how tokens are cut into chunks.  The other gradients then need no order
// (k_delta_inputs_back, by blocks of two chunks, where G and exp(G_31 - G_j) are the block's).  With
// M_ij = D_ij scale do_i . w_j and N_ij = D_ij dR_i . w_j (j < i),
//   dq_i = scale exp(G_i) S do_i + sum_j M_ij k_j
//   x_i = exp(G_i) S dR_i + sum_j N_ij k_j,    dbeta_i = dR_i . v_i - k_i . x_i
//   dk_i = -beta_i x_i (as read) + exp(G_31 - G_i) E w_i + sum_l (M_li q_l - beta_l N_li k_l) (as written)
//   dG_i = q_i . dq_i + k_i . (dk_i as read - as written)  (= the states' parts of it
//          + sum_j Z_ij - sum_l Z_li, Z_ij = M_ij q_i . k_j - beta_i N_ij k_i . k_j, j < i),
//   dG_31 += <E, S'>,
//   dg_t = sum of dG_i over i >= t.
//
// Products run on the bf16 matrix instructions with operands taken apart into bf16 numbers that
// add up to them: one for bf16, two for f16, three for 32 bits, and of the products of
// pieces those above 2^-24 of the whole: 32-bit results (3 instructions for bf16 by 32 bits, 6 for 32 by 32
// bits) where the 32-bit matrix instructions take 16 times as long each.  The states and
// the gradients of g and beta are 32-bit outputs: pieces left off (two for 32 bits) would show in them.
// D's exponents are differences of sums in 64 bits, so a token that forgets everything costs the
// later ones nothing.  (Chunks of 64 take as many matrix instructions a token and twice the registers.)
//
// A number that is not finite reaches what the formulas at the top let it reach, as NaN: its own token and
// those after it, gradients of those before it where they go through its state.  A matrix product would hand it to the
// whole chunk, for 0 times NaN is NaN: where one is found, which costs a compare and a branch a chunk (forward
// 122 to 124 us for 64 chunks, 140 to 146 for 86 of a prompt, whose states nobody writes), the product runs again
// without it and the rows that it belongs to are set to NaN.
#pragma once

#include <algorithm>
#include <cstddef>

#include "ops_internal.h"

namespace rcdelta {

using namespace rcops;

constexpr int kChunk = 32;
constexpr int kMaxHead = 256;

typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// bf16 numbers that hold a T exactly.
template <class T>
constexpr int kPieces = sizeof(T) == 4 ? 3 : 2;
template <>
inline constexpr int kPieces<bf16> = 1;

template <int N>
struct Pieces {
  bf16x8 p[N];
};

// Two at a time: one conversion, and what it left off for the next piece.
template <int N>
__device__ __forceinline__ Pieces<N> split(const float (&v)[8]) {
  u32x4 w[N];
#pragma unroll
  for (int j = 0; j < 4; j++) {
    f32x2 x = {v[2 * j], v[2 * j + 1]};
#pragma unroll
    for (int i = 0; i < N; i++) {
      const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
      w[i][j] = u;
      x[0] -= __builtin_bit_cast(float, u << 16);
      x[1] -= __builtin_bit_cast(float, u & 0xffff0000u);
    }
  }
  Pieces<N> s;
#pragma unroll
  for (int i = 0; i < N; i++) s.p[i] = __builtin_bit_cast(bf16x8, w[i]);
  return s;
}

// Whether x is a number that pieces hold: not infinity, not NaN, nor so near the largest that its first
// piece is rounded to infinity.
__device__ __forceinline__ bool is_finite(float x) { return __builtin_fabsf(x) < 0x1.ffp127f; }

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

// The same for pairs of tokens, of which there are many: off by |x| 2^-24 of itself.
__device__ __forceinline__ float decay_between(double x) {
  return fast_exp2((float)(x * 1.44269504088896340736));
}

// Elements between rows of `channels` (a multiple of 32) in LDS, 16-byte aligned.  In order: neither
// reads of 16 rows (8 bytes each) nor transposing reads of four rows (32 bytes each) meet in one of 64
// banks.  Paired: reads of eight rows (16 bytes each) do not, transposing ones hardly.  Three pieces
// leave no room for that: only reads of rows do not meet.
constexpr int stride_of(int channels, int pieces, bool paired) {
  if (paired) return channels + (channels == 32 || pieces == 3 ? 8 : 40);
  return channels + (channels == 64 || pieces == 3 ? 8 : 24);
}

// ROWS rows (tokens) of `32 KT` channels in LDS as pieces.  PAIRED: within each 32 channels groups
// of four are ordered 0 4 1 5 2 6 3 7, so that a lane's operand of a row is one read; for the
// walks, that mostly read rows (168 us for a prompt of 8192 tokens in order, 158 so).
template <int KT, int N, int ROWS = kChunk, bool PAIRED = false>
struct Tokens {
  static constexpr int STRIDE = stride_of(KT * 32, N, PAIRED);
  alignas(16) bf16 at[N][ROWS][STRIDE];

  // Where channel c of a row is.
  __device__ static int place(int c) {
    return PAIRED ? c / 32 * 32 + c % 16 / 4 * 8 + c % 32 / 16 * 4 + c % 4 : c;
  }
  // From rows `row` elements apart; what is past `live` tokens or `n` channels, or not finite, is 0.
  template <class T>
  __device__ void load(const T* x, int64_t row, int live, int n, int thread, int threads) {
    for (int i = thread; i < ROWS * KT * 4; i += threads) {
      const int r = i / (KT * 4), c = i % (KT * 4) * 8;
      float v[8];
      load_vec<8>(x + (r < live ? r : 0) * row + (c < n ? c : 0), r < live ? n - c : 0, v);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = is_finite(v[e]) ? v[e] : 0.f;
      put(r, c, v);
    }
  }
  __device__ void put(int r, int c, const float (&v)[8]) {
    const Pieces<N> s = split<N>(v);
#pragma unroll
    for (int i = 0; i < N; i++) put(i, r, c, s.p[i]);
  }
  // Eight channels of one piece, c a multiple of eight.
  __device__ void put(int i, int r, int c, const bf16x8& v) {
    if constexpr (PAIRED) {
      *(bf16x4*)&at[i][r][place(c)] = v.lo;
      *(bf16x4*)&at[i][r][place(c) + 8] = v.hi;
    } else {
      *(bf16x8*)&at[i][r][c] = v;
    }
  }
  // Four channels of one row, c a multiple of four.
  __device__ void put_four(int r, int c, const f32x4& x) {
    const float v[8] = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    const Pieces<N> s = split<N>(v);
#pragma unroll
    for (int i = 0; i < N; i++) *(bf16x4*)&at[i][r][place(c)] = s.p[i].lo;
  }
  // Row tile t (rows 16t + ..) over channels 32s + 0..31.
  __device__ Pieces<N> rows(int t, int s) const {
    const int lane = threadIdx.x % 64;
    Pieces<N> f;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const bf16* from = &at[i][16 * t + lane % 16][32 * s + lane / 16 * (PAIRED ? 8 : 4)];
      if constexpr (PAIRED) {
        f.p[i] = *(const bf16x8*)from;
      } else {
        f.p[i].lo = *(const bf16x4*)from;
        f.p[i].hi = *(const bf16x4*)(from + 16);
      }
    }
    return f;
  }
  // Channels 16t + .. over rows 32s + 0..31: reads that transpose four by four.
  __device__ Pieces<N> columns(int t, int s = 0) const {
    const int lane = threadIdx.x % 64;
    Pieces<N> f;
#pragma unroll
    for (int i = 0; i < N; i++) {
      const bf16* from = &at[i][32 * s + lane / 16 * 4 + lane % 16 / 4][place(16 * t + lane % 4 * 4)];
      typedef s16x4 __attribute__((address_space(3))) * lds;
      f.p[i].lo = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)from));
      f.p[i].hi = __builtin_bit_cast(
          bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(from + 16 * STRIDE)));
    }
    return f;
  }
  __device__ float value(int r, int c) const {
    float x = (float)at[N - 1][r][place(c)];
#pragma unroll
    for (int i = N - 2; i >= 0; i--) x += (float)at[i][r][place(c)];
    return x;
  }
};

// What k_delta_prepare leaves for one chunk of one head: T and P T (backward: the transposes of
// T and P) as operands of two row tiles, and numbers of each token.
struct Chunk {
  bf16x8 t[2][3][64], p[2][3][64];
  float since[kChunk], left[kChunk], beta[kChunk];    // exp(G_i), exp(G_31 - G_i), beta_i
  double sum[kChunk];                                 // G_i
};
constexpr int kChunkVectors = sizeof(Chunk) / 16;
static_assert(sizeof(Chunk) % 16 == 0, "copied in vectors");

// States before, and gradients of states after, every block of tokens of k_delta_inputs_back as
// a lane of the walks holds them, four rows of a column together: [batch][heads][blocks]
// [columns(value)][rows(key)] in 32 bits; w and dR likewise, four tokens of a column
// together: [batch][heads][chunks][columns(value)][32].  A block is two chunks where its keys,
// queries and products of tokens fit LDS and registers: half of the states to write, keep and read.
// Bytes of LDS with the states' slices in it too, and without them.
constexpr int block_bytes(int pieces, int rows, int block, bool held) {
  return 2 * pieces * block * (stride_of(rows, pieces, false) + stride_of(32, pieces, false)) * 2 +
         2 * 3 * 32 * stride_of(block, 3, false) * 2 + (held ? 2 * 3 * 32 * stride_of(rows, 3, false) * 2 : 0);
}
constexpr int kBlockBytes = 150 * 1024;
constexpr int block_of(int pieces, int rows) {
  return rows <= 128 && block_bytes(pieces, rows, 64, true) <= kBlockBytes ? 64 : 32;
}
__host__ __device__ inline int rows_of(int key) {
  return key <= 32 ? 32 : key <= 64 ? 64 : key <= 128 ? 128 : 256;
}
__host__ __device__ inline int columns_of(int value) { return (value + 31) / 32 * 32; }

struct DeltaParams {
  rc_delta_args a;
  int32_t chunks, blocks;
  int32_t segments, segment;                          // of the length; chunks of one
  float* between;                                     // [batch][heads][segments][rows(key)][rows(key)]
  float* ends;                                        // [batch][heads][segments][columns(value)][rows(key)]
  float* starts;
  Chunk* prepared;                                    // [batch][heads][chunks]
  float* states;
  float* written;                                     // w, or dR
  const float* kept_written;
  float* dstates;
  float* partial;                                     // [2][batch][length][heads / each][key]
  int32_t each;                                       // heads of a workgroup of k_delta_inputs_back
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
// G of a chunk's 32 tokens (in every lane's token lane % 32) from their g: sums from its first token.
__device__ __forceinline__ double sum_of_g(double G) {
  const int i = threadIdx.x % 32;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const double before = __shfl_up(G, d, 32);
    if (i >= d) G += before;
  }
  return G;
}

// One wave a chunk of a head; its loads first.  Bound by instructions that run once each: 9 us alone,
// 4096 of them (4 x 2048 tokens, 16 heads of 128) 24 us.
template <class T, int KT, bool BACK, bool WIDE>
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
  typedef T TV __attribute__((ext_vector_type(8)));
  TV raw[2][2][KT];
#pragma unroll
  for (int x = 0; x < 2; x++)
#pragma unroll
    for (int m = 0; m < 2; m++) {
      const T* from = at_head<T>(x ? a.q : a.k, b, t0 + min(16 * m + lane % 16, live - 1), hk);
#pragma unroll
      for (int s = 0; s < KT; s++) {
        const int c = 32 * s + lane / 16 * 8;
        if (WIDE) {
          __builtin_memcpy(&raw[x][m][s], from + (c < a.key ? c : 0), sizeof(TV));
        } else {
#pragma unroll
          for (int e = 0; e < 8; e++) raw[x][m][s][e] = from[min(c + e, a.key - 1)];
        }
      }
    }
  const auto rows = [&](int x, int m, int s) {
    const int c = 32 * s + lane / 16 * 8, n = 16 * m + lane % 16 < live ? a.key - c : 0;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (WIDE ? 0 : e) < n ? (float)raw[x][m][s][e] : 0.f;
    return split<N>(v);
  };
  Chunk& out = p.prepared[blockIdx.x];
  // (a g that is no number leaves the sums as they are, for those of the tokens on either side of it, and has its
  // token's beta say so)
  const double g = a.g.data && lane % 32 < live ? log_decay(a.g, b, t0 + lane % 32, h) : 0.0;
  const bool decays = g < __builtin_inf();
  const double G = sum_of_g(decays ? g : 0.0);
  if (lane < kChunk) {
    const double last = __shfl(G, kChunk - 1);
    sums[lane] = G;
    beta[lane] = lane >= live ? 0.f : decays ? at_token(a.beta, b, t0 + lane, h) : __builtin_nanf("");
    out.since[lane] = exp_of(G);
    out.left[lane] = exp_of(last - G);
    out.beta[lane] = beta[lane];
    out.sum[lane] = G;
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
    const Pieces<N> ks[2] = {rows(0, 0, s), rows(0, 1, s)};
    const Pieces<N> qs[2] = {rows(1, 0, s), rows(1, 1, s)};
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int n = 0; n < 2; n++) {
        if (m <= n) mul(kk[m][n], ks[m], ks[n]);      // rows j of tile m, columns i of tile n
        if (BACK ? m >= n : m <= n) mul(qk[m][n], BACK ? qs[m] : ks[m], BACK ? ks[n] : qs[n]);
      }
  }
  const int col = lane % 16, row = lane / 16 * 4;
  bool odd = false;                                    // a number of A is not finite
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int n = 0; n < 2; n++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const int i = 16 * n + col, j = 16 * m + row + r;
        // (the decay of the later of the two, whichever of them that is)
        const float d = m <= n || BACK ? decay_between(j <= i ? sums[i] - sums[j] : sums[j] - sums[i]) : 0.f;
        if (m <= n) {
          const float x = j < i ? beta[i] * d * kk[m][n][r] : 0.f;
          A[i][j] = x;
          odd |= !is_finite(x);
        }
        qk[m][n][r] = (BACK ? i <= j : j <= i) ? a.scale * d * qk[m][n][r] : 0.f;
      }
  __syncthreads();
  // Such numbers count as 0 here, and T_ic is set to NaN below for c up to `upto`: where on the way from token c to
  // token i there is one, whatever it is multiplied with.
  odd = __any(odd);
  int upto = -1;                                       // of row lane % 32
  if (__builtin_expect(odd, 0)) {
    for (int j = 0; j < lane % 32; j++)
      if (!is_finite(A[lane % 32][j])) upto = j;
    for (int j = 0; j <= upto; j++)
      if (!is_finite(A[lane % 32][j])) A[lane % 32][j] = 0.f;
    for (int d = 1; d < 32; d *= 2) {
      const int before = __shfl_up(upto, d, 32);
      if (lane % 32 >= d) upto = max(upto, before);
    }
    __syncthreads();
  }
  // T of the two diagonal tiles, a column a lane, by forward substitution
  {
    const int first = lane % 32 / 16 * 16;
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
      float s = i == col ? 1.f : 0.f;
#pragma unroll
      for (int j = 0; j < i; j++) s = fmaf(-A[first + i][first + j], t[j], s);
      t[i] = s;
      if (lane < 32) {
        inverse[first + i][first + col] = s;
        if (first) inverse[i][16 + col] = 0.f;
      }
    }
  }
  __syncthreads();
  // and of the one below, -T_11 A_10 T_00: four rows of a column a lane
#pragma unroll
  for (int step = 0; step < 2; step++) {
    float s[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 16; j++)
#pragma unroll
      for (int e = 0; e < 4; e++)
        s[e] = step ? fmaf(-inverse[16 + row + e][16 + j], A[16 + j][col], s[e])
                    : fmaf(A[16 + row + e][j], inverse[j][col], s[e]);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; e++) (step ? inverse : A)[16 + row + e][col] = s[e];
    __syncthreads();
  }
  if (__builtin_expect(odd, 0)) {
    for (int j = 0; lane < kChunk && j <= upto; j++) inverse[lane][j] = __builtin_nanf("");
    __syncthreads();
  }
  Pieces<3> between[2];
#pragma unroll
  for (int n = 0; n < 2; n++) between[n] = operand<3>(qk[0][n], qk[1][n]);
  f32x4 pt[2][2];
#pragma unroll
  for (int n = 0; n < 2; n++) {
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const int i = 16 * n + col, j = 16 * (e / 4) + row + e % 4;
      x[e] = inverse[i][j];
      y[e] = inverse[j][i];
    }
    const Pieces<3> f = split<3>(BACK ? y : x);
#pragma unroll
    for (int i = 0; i < 3; i++) out.t[n][i][lane] = f.p[i];
    if (!BACK) {
      // columns n of P T, transposed: rows of it are what its operand has in a lane
      if (__builtin_expect(odd, 0)) {
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = is_finite(y[e]) ? y[e] : 0.f;
      }
      const Pieces<3> columns = split<3>(y);
#pragma unroll
      for (int m = 0; m < 2; m++) {
        const float from = odd && __shfl(upto, 16 * m + col) >= 0 ? __builtin_nanf("") : 0.f;
        pt[n][m] = f32x4{from, from, from, from};
        mul(pt[n][m], columns, between[m]);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < 2; n++) {
    const Pieces<3> f = BACK ? between[n] : operand<3>(pt[0][n], pt[1][n]);
#pragma unroll
    for (int i = 0; i < 3; i++) out.p[n][i][lane] = f.p[i];
  }
}

// Column `col` of a kept state (below) from row `first` on: tile m has this lane's rows
// 16m + 4 (lane / 16) + 0..3.
template <int TILES>
__device__ __forceinline__ void load_kept(const float* from, int rows, int col, int first, f32x4 (&S)[TILES]) {
  const float* at = from + col * rows + first + threadIdx.x % 64 / 16 * 4;
#pragma unroll
  for (int m = 0; m < TILES; m++) S[m] = *(const f32x4*)(at + 16 * m);
}
// The same of a head's state as callers have it.
template <int TILES>
__device__ __forceinline__ void load_state(const float* from, const rc_delta_args& a, int col, int first,
                                           f32x4 (&S)[TILES]) {
  const int row = first + threadIdx.x % 64 / 16 * 4;
#pragma unroll
  for (int m = 0; m < TILES; m++)
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = 16 * m + row + r;
      S[m][r] = from && i < a.key && col < a.value ? from[(int64_t)i * a.value + col] : 0.f;
    }
}
template <int TILES>
__device__ __forceinline__ void store_state(float* to, const rc_delta_args& a, int col, int first,
                                            const f32x4 (&S)[TILES]) {
  const int row = first + threadIdx.x % 64 / 16 * 4;
#pragma unroll
  for (int m = 0; m < TILES; m++)
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = 16 * m + row + r;
      if (i < a.key && col < a.value) to[(int64_t)i * a.value + col] = S[m][r];
    }
}
// The same into [column][row], `rows` rows a column (col < columns_of(value)).
template <int TILES>
__device__ __forceinline__ void keep_state(float* to, int rows, int col, int first, const f32x4 (&S)[TILES]) {
  float* at = to + col * rows + first + threadIdx.x % 64 / 16 * 4;
#pragma unroll
  for (int m = 0; m < TILES; m++) *(f32x4*)(at + 16 * m) = S[m];
}

// A walk's workgroup: W waves side by side, 16 columns each, times R waves that have a part
// each of the key's channels (rows of the state) in them, and L waves that load.
template <int W_, int R_, int L_>
struct Shape {
  static constexpr int W = W_, R = R_, L = L_, COLUMNS = 16 * W;
  static constexpr int WORKERS = 64 * W * R, LOADERS = 64 * L, THREADS = WORKERS + LOADERS;
};

// What a chunk's products need beside the state, in LDS; x: the values, or the outputs'
// gradients, of the workgroup's columns.
template <class T, int KT, class G>
struct Stage {
  Tokens<KT, kPieces<T>, kChunk, true> k, q;
  union {
    Chunk c;
    u32x4 raw[kChunkVectors];
  };
  T x[kChunk][G::COLUMNS + 8];
  __device__ Stage() {}
};
template <class T, int KT, class G>
constexpr int kStages = 2 * sizeof(Stage<T, KT, G>) + 16 * 1024 <= 160 * 1024 ? 2 : 1;    // (and Parts)
// A loading wave's part of the chunks: the next one's share in registers.  Loads are
// unconditional with addresses inside the sequence; what is past its end is dropped on the way to LDS.
// WIDE: key and value are multiples of eight.  READS: q and P (P T) are needed, and not only keys and T.
template <class T, int KT, class G, bool WIDE, bool READS>
struct Feed {
  static constexpr int THREADS = G::LOADERS, VECTORS = kChunk * KT * 4, COLUMNS = G::COLUMNS;
  static constexpr int EACH = (VECTORS + THREADS - 1) / THREADS;
  // a chunk's vectors, without P's
  static constexpr int SKIP = READS ? 0 : sizeof(Chunk::p) / 16, SKIP_FROM = offsetof(Chunk, p) / 16;
  static constexpr int RAW_VECTORS = kChunkVectors - SKIP, RAW = (RAW_VECTORS + THREADS - 1) / THREADS;
  static constexpr int PER_ROW = COLUMNS / 8, VECTORS_X = kChunk * PER_ROW;
  static constexpr int EACH_X = (VECTORS_X + THREADS - 1) / THREADS;
  // Vector i of a thread is STEP (XSTEP) rows below the one before, in the same channels.
  static constexpr int STEP = THREADS / (KT * 4), XSTEP = THREADS / PER_ROW;
  static_assert(THREADS % (KT * 4) == 0 && THREADS % PER_ROW == 0, "whole rows");
  typedef T TV __attribute__((ext_vector_type(8)));
  TV k[EACH], q[EACH], x[EACH_X];
  u32x4 raw[RAW];
  int thread, row, c, xrow, xc;
  int64_t at_k, at_q, at_x;                            // the first vector's row (WIDE: and channel)

  __device__ Feed(const rc_delta_args& a, const rc_heads& values, int col0) {
    thread = threadIdx.x - G::WORKERS;
    row = thread / (KT * 4);
    c = thread % (KT * 4) * 8;
    xrow = thread / PER_ROW;
    xc = thread % PER_ROW * 8;
    at_k = row * a.k.time + first(c, a.key);
    at_q = row * a.q.time + first(c, a.key);
    at_x = xrow * values.time + first(col0 + xc, a.value);
  }
  // The channel that a wide load begins at.
  __device__ static int first(int c, int n) { return WIDE && c < n ? c : 0; }
  __device__ int raw_of(int i) const {
    const int v = min(thread + i * THREADS, RAW_VECTORS - 1);
    return v < SKIP_FROM ? v : v + SKIP;
  }
  // From row `at` + `down` rows, or from the first one (which is always there).
  __device__ static void load(TV& to, const T* from, bool there, int64_t at, int64_t down, int c, int n) {
    from += there ? at + down : first(c, n);
    if (WIDE) {
      __builtin_memcpy(&to, from, sizeof(TV));
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) to[e] = from[min(c + e, n - 1)];
    }
  }
  __device__ static void mask(TV& v, bool there, int c, int n) {
    if (WIDE) {
      if (!there || c >= n) v = TV(0);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = there && c + e < n ? v[e] : (T)0.f;
    }
  }

  __device__ void fetch(const rc_delta_args& a, const Chunk& chunk, const rc_heads& values, int b, int h, int hk,
                        int t0, int live, int col0) {
    const T* from_k = at_head<T>(a.k, b, t0, hk);
    const T* from_q = at_head<T>(a.q, b, t0, hk);
    const T* from_x = at_head<T>(values, b, t0, h);
#pragma unroll
    for (int i = 0; i < EACH; i++) {
      const bool there = row + i * STEP < live;
      load(k[i], from_k, there, at_k, i * STEP * a.k.time, c, a.key);
      if (READS) load(q[i], from_q, there, at_q, i * STEP * a.q.time, c, a.key);
    }
#pragma unroll
    for (int i = 0; i < EACH_X; i++)
      load(x[i], from_x, xrow + i * XSTEP < live, at_x, i * XSTEP * values.time, col0 + xc, a.value);
    const u32x4* from = reinterpret_cast<const u32x4*>(&chunk);
#pragma unroll
    for (int i = 0; i < RAW; i++) raw[i] = from[raw_of(i)];
  }
  // ALL: no row and no channel is past an end.
  template <bool ALL>
  __device__ void put_tokens(Stage<T, KT, G>& to, int live, int key) const {
#pragma unroll
    for (int i = 0; i < EACH; i++) {
      const int r = row + i * STEP;
      if (VECTORS % THREADS && r >= kChunk) break;
#pragma unroll
      for (int which = 0; which < (READS ? 2 : 1); which++) {
        TV u = which ? q[i] : k[i];
        auto& tokens = which ? to.q : to.k;
        if (!ALL) mask(u, r < live, c, key);
        if constexpr (kPieces<T> == 1) {
          tokens.put(0, r, c, u);
        } else {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; e++) y[e] = (float)u[e];
          tokens.put(r, c, y);
        }
      }
    }
  }
  __device__ void put(Stage<T, KT, G>& to, int live, int key, int value, int col0) const {
    if (live == kChunk && key == 32 * KT)
      put_tokens<true>(to, live, key);
    else
      put_tokens<false>(to, live, key);
#pragma unroll
    for (int i = 0; i < EACH_X; i++) {
      const int r = xrow + i * XSTEP;
      if (VECTORS_X % THREADS && r >= kChunk) break;
      TV v = x[i];
      mask(v, r < live, col0 + xc, value);
      *(TV*)&to.x[r][xc] = v;
    }
#pragma unroll
    for (int i = 0; i < RAW; i++) to.raw[raw_of(i)] = raw[i];
  }
};

// The first row of a chunk with a number that is not finite in this lane's column (kChunk: none); a lane
// has rows row + 0..3 and 16 + row + 0..3.
__device__ __forceinline__ int first_odd(const f32x4 (&x)[2], int row) {
  int at = kChunk;
#pragma unroll
  for (int i = 7; i >= 0; i--)
    if (!is_finite(x[i / 4][i % 4])) at = i / 4 * 16 + row + i % 4;
  at = min(at, __shfl_xor(at, 16));
  return min(at, __shfl_xor(at, 32));
}

// The last one (-1: none).
__device__ __forceinline__ int last_odd(const f32x4 (&x)[2], int row) {
  int at = -1;
#pragma unroll
  for (int i = 0; i < 8; i++)
    if (!is_finite(x[i / 4][i % 4])) at = i / 4 * 16 + row + i % 4;
  at = max(at, __shfl_xor(at, 16));
  return max(at, __shfl_xor(at, 32));
}

__device__ __forceinline__ Pieces<3> pieces(const bf16x8 (&x)[3][64]) {
  const int lane = threadIdx.x % 64;
  return {{x[0][lane], x[1][lane], x[2][lane]}};
}

// What a walk is for: everything, or (where the length is cut) what a segment makes of the state before
// it: ENDS from no state, with the values' columns, and from a state of ones on the diagonal, without
// values, so that S' = between S + ends.
enum { kWhole = 0, kEnds = 1 };

// A walk's place.  Workgroups of one head are as many apart as there are heads, so
// that most share one of the eight caches.
template <class G, int MODE>
struct Walk {
  int b, h, hk, bh, col0, col, row, end, wave, part;
  int segment, first, count;                           // chunks of this segment
  bool on, diagonal, last;                             // last: the segment of the sequence's end
  __device__ Walk(const DeltaParams& p, int rows) {
    const rc_delta_args& a = p.a;
    const int heads = a.batch * a.heads, lane = threadIdx.x % 64;
    const int values = (a.value + G::COLUMNS - 1) / G::COLUMNS;
    const int slices = values + (MODE == kEnds ? (rows + G::COLUMNS - 1) / G::COLUMNS : 0);
    bh = blockIdx.x % heads;
    const int slice = blockIdx.x / heads % slices;
    segment = blockIdx.x / heads / slices;
    b = bh / a.heads;
    h = bh % a.heads;
    hk = h / (a.heads / a.key_heads);
    wave = threadIdx.x / 64 % G::W;
    part = threadIdx.x / 64 / G::W;
    diagonal = slice >= values;
    col0 = (diagonal ? slice - values : slice) * G::COLUMNS;
    col = col0 + wave * 16 + lane % 16;
    row = lane / 16 * 4;
    on = col < (diagonal ? rows : a.value);
    end = length_of(a, b);
    const int chunks = (end + kChunk - 1) / kChunk;
    first = segment * p.segment;
    count = min(max(chunks - first, 0), p.segment);
    last = segment == (chunks ? (chunks - 1) / p.segment : 0);
  }
};

// The loading waves' side of a walk over the chunks, forward or (BACK) from the last: chunk
// by chunk as the working waves go, one chunk ahead of them in LDS where it holds two and
// one more in registers.  A chunk has two barriers: at its start, and between the parts'
// writes and reads of their sums over the key (Parts); with one stage a third at its end.
template <class T, int KT, class G, bool WIDE, bool BACK, int MODE>
__device__ __forceinline__ void load_chunks(const DeltaParams& p, const Walk<G, MODE>& at, const rc_heads& values,
                                            Stage<T, KT, G>* stages) {
  constexpr int STAGES = kStages<T, KT, G>;
  const rc_delta_args& a = p.a;
  if (!at.count) return;
  const Chunk* prepared = p.prepared + (int64_t)at.bh * p.chunks;
  const int columns = at.diagonal ? 0 : a.value;       // of values: a walk from the diagonal has none
  // (the gradient of the states takes both)
  Feed<T, KT, G, WIDE, BACK || MODE == kWhole> next(a, values, at.col0);
  const auto chunk_of = [&](int i) { return at.first + (BACK ? at.count - 1 - i : i); };
  const auto live_of = [&](int c) { return min(at.end - c * kChunk, kChunk); };
  const auto fetch = [&](int i) {
    const int c = chunk_of(min(i, at.count - 1));
    next.fetch(a, prepared[c], values, at.b, at.h, at.hk, c * kChunk, live_of(c), at.col0);
  };
  const auto put = [&](int i) { next.put(stages[i % STAGES], live_of(chunk_of(i)), a.key, columns, at.col0); };
  fetch(0);
  put(0);
  fetch(1);
  for (int i = 0; i < at.count; i++) {
    __syncthreads();
    if (STAGES == 2 && i + 1 < at.count) put(i + 1);
    if (STAGES == 2) fetch(i + 2);                     // (not in a branch: the loop hands it on)
    if (G::R > 1) __syncthreads();
    if (STAGES == 1) {
      __syncthreads();
      if (i + 1 < at.count) put(i + 1);
      fetch(i + 2);
    }
  }
}

// Sums over the R waves that have parts of the key, in one order for all of them, so that
// what they compute from them is the same; M results.
template <class G, int M>
struct Parts {
  f32x4 at[M][G::R][G::W][64];
  __device__ f32x4 sum(int m, int wave) const {
    const int lane = threadIdx.x % 64;
    f32x4 s = at[m][0][wave][lane];
#pragma unroll
    for (int i = 1; i < G::R; i++) s += at[m][i][wave][lane];
    return s;
  }
};
template <class G>
struct Parts<G, 0> {};

// What a walk of a segment begins with.
template <int KT, int MODE, class G, int TILES>
__device__ __forceinline__ void begin(const DeltaParams& p, const Walk<G, MODE>& at, const float* given, int first,
                                      f32x4 (&S)[TILES]) {
  const rc_delta_args& a = p.a;
  if (MODE == kEnds) {
#pragma unroll
    for (int m = 0; m < TILES; m++)
#pragma unroll
      for (int r = 0; r < 4; r++) S[m][r] = at.diagonal && first + 16 * m + at.row + r == at.col ? 1.f : 0.f;
  } else if (p.segments > 1) {
    load_kept(p.starts + ((int64_t)at.bh * p.segments + at.segment) * columns_of(a.value) * (32 * KT), 32 * KT,
              min(at.col, columns_of(a.value) - 1), first, S);
  } else {
    load_state(given ? given + (int64_t)at.bh * a.key * a.value : nullptr, a, at.col, first, S);
  }
}
// What a walk of kEnds leaves: columns of `ends` or, row by row, of `between`.
template <int KT, class G, int TILES>
__device__ __forceinline__ void leave(const DeltaParams& p, const Walk<G, kEnds>& at, int first,
                                      const f32x4 (&S)[TILES]) {
  constexpr int ROWS = 32 * KT;
  const int64_t segment = (int64_t)at.bh * p.segments + at.segment;
  if (!at.diagonal) {
    if (at.col < columns_of(p.a.value))
      keep_state(p.ends + segment * columns_of(p.a.value) * ROWS, ROWS, at.col, first, S);
  } else if (at.on) {
    float* to = p.between + segment * ROWS * ROWS + at.col;
#pragma unroll
    for (int m = 0; m < TILES; m++)
#pragma unroll
      for (int r = 0; r < 4; r++) to[(first + 16 * m + at.row + r) * ROWS] = S[m][r];
  }
}

// The states between segments, one after the other: S' = between S + ends (BACK: from the last
// to the first).  A workgroup has 16 columns of a head, each of its waves some of the
// rows; the state is between them in LDS as an operand.
template <int KT, bool BACK>
__global__ __launch_bounds__(256) void k_delta_join(DeltaParams p) {
  const rc_delta_args& a = p.a;
  constexpr int ROWS = 32 * KT, TILES = (2 * KT + 3) / 4;
  __shared__ bf16x8 state[2][KT][3][64];
  const int heads = a.batch * a.heads, bh = blockIdx.x % heads, lane = threadIdx.x % 64;
  const int cols = columns_of(a.value), col = blockIdx.x / heads * 16 + lane % 16, row = lane / 16 * 4;
  const int tile = threadIdx.x / 64 * TILES;
  const bool mine = tile < 2 * KT;
  const int chunks = (length_of(a, bh / a.heads) + kChunk - 1) / kChunk;
  const int last = chunks ? (chunks - 1) / p.segment : 0;
  const float* given = BACK ? a.dstate_out : a.state_in;
  f32x4 S[TILES];
  load_state(given ? given + (int64_t)bh * a.key * a.value : nullptr, a, col, 16 * tile, S);
  for (int i = 0; i <= last; i++) {
    const int64_t at = (int64_t)bh * p.segments + (BACK ? last - i : i);
    if (mine) keep_state(p.starts + at * cols * ROWS, ROWS, col, 16 * tile, S);
    if (i == last) break;
    if (mine) {
#pragma unroll
      for (int m = 0; m < TILES; m++) {
        const Pieces<3> s = operand<3>(S[m], S[m]);
#pragma unroll
        for (int j = 0; j < 3; j++)
          *((bf16x4*)&state[i % 2][(tile + m) / 2][j][lane] + (tile + m) % 2) = s.p[j].lo;
      }
    }
    // loads that do not wait for the state (of the widest keys there are too many to hold)
    f32x4 between[TILES][KT][2];
    const auto load = [&](int m, int s) {
      const float* from =
          p.between + (at * ROWS + 16 * min(tile + m, 2 * KT - 1) + lane % 16) * ROWS + 32 * s + row;
      between[m][s][0] = *(const f32x4*)from;
      between[m][s][1] = *(const f32x4*)(from + 16);
    };
    if (KT <= 4) {
#pragma unroll
      for (int m = 0; m < TILES; m++)
#pragma unroll
        for (int s = 0; s < KT; s++) load(m, s);
    }
    __syncthreads();
    if (mine) {
      load_kept(p.ends + at * cols * ROWS, ROWS, col, 16 * tile, S);
#pragma unroll
      for (int m = 0; m < TILES; m++)
#pragma unroll
        for (int s = 0; s < KT; s++) {
          if (KT > 4) load(m, s);
          const Pieces<3> c = {
              {state[i % 2][s][0][lane], state[i % 2][s][1][lane], state[i % 2][s][2][lane]}};
          mul(S[m], operand<3>(between[m][s][0], between[m][s][1]), c);
        }
    }
  }
}

// ------------------------------------------------------------------ host side

inline int check(const rc_delta_args* a) {
  if (!a || !dtype_ok(a->dtype) || a->batch < 0 || a->length < 0 || a->length > kMaxExtent ||
      a->key < 1 || a->key > kMaxHead || a->value < 1 || a->value > kMaxHead)
    return RC_E_ARG;
  if (a->heads < 0 || a->key_heads < 0 || !a->heads != !a->key_heads ||
      (a->heads && a->heads % a->key_heads))
    return RC_E_ARG;
  return RC_OK;
}
inline bool empty(const rc_delta_args& a) { return !a.batch || !a.heads; }

inline int64_t chunks_of(const rc_delta_args& a) { return cdiv(a.length, kChunk); }
// Chunks of all heads.  (batch x heads is checked first: it fits a launch.)
inline int64_t pairs_of(const rc_delta_args& a) { return (int64_t)a.batch * a.heads * chunks_of(a); }
inline int block_of(const rc_delta_args& a) {
  const int pieces = a.dtype == RC_BF16 ? 1 : a.dtype == RC_F16 ? 2 : 3;
  return block_of(pieces, rows_of(a.key));
}
inline int64_t blocks_of(const rc_delta_args& a) { return cdiv(a.length, block_of(a)); }
inline uint64_t state_floats(const rc_delta_args& a) {
  return (uint64_t)a.batch * a.heads * blocks_of(a) * columns_of(a.value) * rows_of(a.key);
}
inline uint64_t kept_bytes(const rc_delta_args& a) {
  return (state_floats(a) + (uint64_t)pairs_of(a) * columns_of(a.value) * kChunk) * sizeof(float);
}
// Heads of a workgroup of k_delta_inputs_back: all that share a key head, or the largest part of
// them that leaves two workgroups a compute unit.
inline int heads_together(const rc_delta_args& a) {
  const int per = a.heads / a.key_heads;
  for (int each = per; each > 1; each--)
    if (per % each == 0 && (int64_t)a.batch * a.heads * blocks_of(a) / each >= 512) return each;
  return 1;
}
// Whether the sizes fit the launches.
inline int fits(const rc_delta_args& a) {
  const int64_t bh = (int64_t)a.batch * a.heads;
  if (!launchable(bh, 256) || !launchable(bh * cdiv(a.value, 16), 512) ||
      !launchable(pairs_of(a), 256))
    return RC_E_OVERFLOW;
  return RC_OK;
}
inline int fits_back(const rc_delta_args& a) {
  if (int e = fits(a)) return e;
  if (empty(a)) return RC_OK;
  return launchable((int64_t)a.batch * a.heads / heads_together(a) * blocks_of(a), 512) ? RC_OK : RC_E_OVERFLOW;
}
// Segments of the length: more than one where the walks over the segments' ends (of values' and
// key columns, one segment fewer) and those over the segments fit the compute units at once, counted as
// slices of 32 columns, two a compute unit for keys up to 64 and one for others, and each
// segment has eight chunks (sixteen of the widest keys, whose joins take longer).  (For keys of 33 to 64 in float16 and
// float32 LDS holds one, so that as many as this gives may take two rounds: 8192 tokens of 64 x 64 in float32
// with room for 512 and for 256, 8 heads 112 and 125 us, 16 heads 215 and 199.)  Cutting costs those
// walks, and a step a segment that joins them: two segments gain from 128 chunks and keys of 65 to
// 128 on, not for others.  Forward, all kernels, bf16 heads of 128 x 128, us in one segment and in as many as
// this gives: 8192 tokens of 32, 24, 16 and 4 heads 478, 452, 441, 421 and in 2, 2, 3, 9 455, 397, 274, 127;
// 2048 tokens of 16 heads 120, in 3 90 (32 heads in one: 126, in 2 125).
inline int segments_of(const rc_delta_args& a) {
  const int rows = rows_of(a.key), room = rows <= 64 ? 512 : 256;
  const int64_t values = (int64_t)a.batch * a.heads * cdiv(a.value, 32);
  const int64_t ends = values + (int64_t)a.batch * a.heads * (rows / 32);
  const int64_t most = chunks_of(a) / (rows > 128 ? 16 : 8);
  const int64_t n = std::min<int64_t>({1 + room / ends, room / values, most, 16});
  if (n == 2 && rows == 128 && chunks_of(a) >= 128) return 2;
  return n < 3 ? 1 : (int)n;
}
inline uint64_t segment_floats(const rc_delta_args& a) {
  const int n = segments_of(a), rows = rows_of(a.key);
  return n == 1 ? 0 : (uint64_t)a.batch * a.heads * n * rows * (rows + 2 * columns_of(a.value));
}
inline uint64_t workspace_of(const rc_delta_args& a, bool back) {
  if (empty(a)) return 0;
  uint64_t n = (uint64_t)pairs_of(a) * sizeof(Chunk) + segment_floats(a) * sizeof(float);
  if (back) {
    n += kept_bytes(a);
    const int per = a.heads / a.key_heads, each = heads_together(a);
    if (per != each) n += 2 * (uint64_t)a.batch * a.length * (a.heads / each) * a.key * sizeof(float);
  }
  return n;
}

// f(whether rows of key and value are whole loads of eight).
template <class F>
inline int by_width(const rc_delta_args& a, F&& f) {
  return a.key % 8 || a.value % 8 ? f(std::false_type{}) : f(std::true_type{});
}
// f(integral_constant of the key's tiles of 32).
template <class F>
inline int by_key(int32_t key, F&& f) {
  if (key <= 32) return f(std::integral_constant<int, 1>{});
  if (key <= 64) return f(std::integral_constant<int, 2>{});
  if (key <= 128) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 8>{});
}

inline DeltaParams params(const rc_delta_args& a) {
  DeltaParams p = {};
  p.a = a;
  p.chunks = (int32_t)chunks_of(a);
  p.blocks = (int32_t)blocks_of(a);
  p.prepared = static_cast<Chunk*>(a.workspace);
  p.states = a.kept;
  p.segment = (int32_t)cdiv(p.chunks, segments_of(a));
  p.segments = p.chunks ? (int32_t)cdiv(p.chunks, p.segment) : 1;
  p.segment = std::max(p.segment, 1);
  const int64_t n = (int64_t)a.batch * a.heads * p.segments * rows_of(a.key);
  p.between = reinterpret_cast<float*>(p.prepared + pairs_of(a));
  p.ends = p.between + n * rows_of(a.key);
  p.starts = p.ends + n * columns_of(a.value);
  return p;
}

template <class T, int KT, bool BACK>
inline int prepare(const DeltaParams& p, hipStream_t s) {
  if (!p.chunks) return RC_OK;
  if (p.a.key % 8)
    k_delta_prepare<T, KT, BACK, false><<<(unsigned)pairs_of(p.a), 64, 0, s>>>(p);
  else
    k_delta_prepare<T, KT, BACK, true><<<(unsigned)pairs_of(p.a), 64, 0, s>>>(p);
  return launched("k_delta_prepare");
}
// Workgroups of a walk.
template <class G, int MODE>
inline unsigned walks_of(const DeltaParams& p, int rows) {
  const int64_t slices = cdiv(p.a.value, G::COLUMNS) + (MODE == kEnds ? cdiv(rows, G::COLUMNS) : 0);
  return (unsigned)((int64_t)p.a.batch * p.a.heads * slices * p.segments);
}
template <int KT, bool BACK>
inline int join(const DeltaParams& p, hipStream_t s) {
  k_delta_join<KT, BACK>
      <<<(unsigned)((int64_t)p.a.batch * p.a.heads * (columns_of(p.a.value) / 16)), 256, 0, s>>>(p);
  return launched("k_delta_join");
}
// The shape of a walk's workgroups.
template <int KT>
using ShapeOf = Shape<KT >= 2 ? 2 : 4, KT >= 2 ? 2 : 1, 4>;

}  // namespace rcdelta
