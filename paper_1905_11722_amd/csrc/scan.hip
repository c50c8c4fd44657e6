// Selective state space scan, its gradients, and its form for one token.
//
// Channel d has N states, delta = softplus(dt + bias) (or dt + bias):
//   a_n = exp(delta A_n),  h_n <- a_n h_n + delta u B_n,  y = sum_n h_n C_n + D u,
//   out = y z sigmoid(z).
// Backwards in time, with dy = dout z sigmoid(z) and g_n the gradient of the
// state after the token:
//   g_n = C_n dy + (a_n g_n of the next token),  dC_n = sum_d dy h_n,  dB_n = sum_d g_n delta u,
//   du = delta sum_n g_n B_n + D dy,  dA_n = sum g_n a_n h_n(before) delta,
//   ddelta = u sum_n g_n B_n + sum_n g_n a_n h_n(before) A_n.
//
// S = 1, 2 or 4 states are one lane's, Q = 4, 8 or 16 neighbouring lanes are a
// channel's (N <= S Q; missing states have A = B = C = 0), so sums over a
// channel's states are Q-lane sums and sums over channels are strided ones.
// A token past its sequence's end is a step with delta = u = dy = B = C = 0:
// the state stays, every product is 0.
#include "ops_internal.h"

using namespace rcops;

namespace {

constexpr int kFwdTile = 32;        // tokens staged together, forward
constexpr int kSumThreads = 256;

constexpr int kKeep = 16;           // tokens between two kept states, a backward tile:
                                    // its states stay in registers

// Channels of a workgroup.
constexpr int channels_of(int Q) { return Q > 8 ? 32 : 64; }

__device__ __forceinline__ int seq_end(const int32_t* lengths, int64_t b, int32_t length) {
  if (!lengths) return length;
  return min(max(lengths[b], 0), length);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL,
                                                               0xf, 0xf, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

// x of lane J of the quad, in each of its lanes.
template <int J>
__device__ __forceinline__ float quad_lane(float x) {
  return dpp<J * 0x55>(x);
}

// Sums over the Q lanes of a channel of four values at once: lane q gets that
// of v[q & 3].  (Mirrors first: the quads then hold the whole sums.)
template <int Q>
__device__ __forceinline__ float state_sums(float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; j++) {
    if (Q > 4) v[j] += dpp<kHalfMirror>(v[j]);
    if (Q > 8) v[j] += dpp<kMirror>(v[j]);
  }
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
  const float a = (odd ? v[1] : v[0]) + dpp<kXor1>(odd ? v[0] : v[1]);
  const float b = (odd ? v[3] : v[2]) + dpp<kXor1>(odd ? v[2] : v[3]);
  return (high ? b : a) + dpp<kXor2>(high ? a : b);
}

// One step of a sum over the lanes of a row of 16 that hold the same states
// of different channels, for pairs of values at once: half of the lanes go on
// with v[2 i], half with v[2 i + 1].  BANKS = 8: lanes 8 apart, lane bit 3
// chooses; 4: lanes 4 apart, bit 2 chooses.  The bank masks write each
// half in place of a select; two wait states before a DPP read and after the
// block cover what the compiler does not see inside.
template <int BANKS, int M>
__device__ __forceinline__ void bank_sums(const float* v, float* r) {
#pragma unroll
  for (int i = 0; i < M; i += 2) {
    if (BANKS == 8)
      asm("s_nop 1\n\t"
          "v_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
          "v_add_f32_dpp %1, %4, %4 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
          "v_add_f32_dpp %0, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
          "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
          "s_nop 1"
          : "=&v"(r[i]), "=&v"(r[i + 1])
          : "v"(v[2 * i]), "v"(v[2 * i + 1]), "v"(v[2 * i + 2]), "v"(v[2 * i + 3]));
    else
      asm("s_nop 1\n\t"
          "v_add_f32_dpp %0, %2, %2 row_ror:12 row_mask:0xf bank_mask:0x5\n\t"
          "v_add_f32_dpp %1, %4, %4 row_ror:12 row_mask:0xf bank_mask:0x5\n\t"
          "v_add_f32_dpp %0, %3, %3 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
          "v_add_f32_dpp %1, %5, %5 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
          "s_nop 1"
          : "=&v"(r[i]), "=&v"(r[i + 1])
          : "v"(v[2 * i]), "v"(v[2 * i + 1]), "v"(v[2 * i + 2]), "v"(v[2 * i + 3]));
  }
}
// The same over rows: even rows go on with x, odd ones with y; and over halves.
__device__ __forceinline__ float row_sums(float x, float y) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x),
                                                  __builtin_bit_cast(unsigned, y), false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float half_sums(float x, float y) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x),
                                                  __builtin_bit_cast(unsigned, y), false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// Sums over the 64 / Q channels of a wave of 64 / Q values at once; the lane
// gets that of v[channel_value<Q>(lane)].
template <int Q>
__device__ __forceinline__ float channel_sums(const float* v) {
  if (Q == 4) {
    float a[8], b[4];
    bank_sums<8, 8>(v, a);
    bank_sums<4, 4>(a, b);
    return half_sums(row_sums(b[0], b[1]), row_sums(b[2], b[3]));
  } else if (Q == 8) {
    float a[4];
    bank_sums<8, 4>(v, a);
    return half_sums(row_sums(a[0], a[1]), row_sums(a[2], a[3]));
  } else {
    return half_sums(row_sums(v[0], v[1]), row_sums(v[2], v[3]));
  }
}
template <int Q>
__device__ __forceinline__ int channel_value(int lane) {
  const int rows = lane >> 4;                          // row bits 0 and 1
  if (Q == 4) return (lane >> 3 & 1) | (lane >> 2 & 1) << 1 | rows << 2;
  if (Q == 8) return (lane >> 3 & 1) | rows << 1;
  return rows;
}

struct ScanParams {
  rc_scan_args a;
  int32_t group_width, blocks;      // channels of a group, workgroups for them
  int32_t chunks, chunk;            // pieces of the length, tokens of one (a multiple of the tile)
  int32_t keeps;                    // kept states of a sequence
  float* ends;                      // [batch][chunks][width][N]: a chunk's own end state (forward)
                                    // or gradient before it (backward), from nothing
  float* steps;                     // [batch][chunks][width]: sum of delta over the chunk
  float* part_bc;                   // backward: [blocks][batch][length][groups][2][N]
  float* part_a;                    // [batch][chunks][width][N]
  float* part_d;                    // [batch][chunks][width][2]: D, dt_bias
};

template <class T>
__device__ __forceinline__ const T* row(const rc_view& v, int64_t b, int64_t t) {
  return static_cast<const T*>(v.data) + b * v.batch + t * v.time;
}
template <class T>
__device__ __forceinline__ T* row_out(const rc_view& v, int64_t b, int64_t t) {
  return static_cast<T*>(v.data) + b * v.batch + t * v.time;
}

__device__ __forceinline__ float delta_of(float raw, bool soft) {
  const float s = softplus(raw);    // chosen, not branched to: elements overlap
  return soft ? s : raw;
}

// First channel (of the group) of a block: blocks of equal sizes but for one
// channel, or for four where four divide the group, so that no block has less than a
// load.
__device__ __forceinline__ int block_start(const ScanParams& p, int blk) {
  const int unit = p.group_width % 4 ? 1 : 4;
  return (int)((int64_t)blk * (p.group_width / unit) / p.blocks) * unit;
}

// What a workgroup works on.  Workgroup i runs on XCD i % 8: neighbours in
// (batch, group, chunk, block) go to one XCD, whose L2 then holds the B and C that they share.
template <int Q, int S>
struct Place {
  static constexpr int N = Q * S, CW = channels_of(Q);
  int64_t b, g;
  int blk, piece;                   // block of channels, chunk
  int base, have;                   // the block's first channel (of the group) and channels
  int q, ch;                        // the lane's states and channel (in the block)
  int64_t d;                        // its channel, clamped to the group
  bool on;
  __device__ Place(const ScanParams& p) {
    const uint32_t per = gridDim.x / 8, rem = gridDim.x % 8, xcd = blockIdx.x % 8;
    uint32_t i = xcd * per + min(xcd, rem) + blockIdx.x / 8;
    blk = (int)(i % (uint32_t)p.blocks);
    i /= (uint32_t)p.blocks;
    piece = (int)(i % (uint32_t)p.chunks);
    i /= (uint32_t)p.chunks;
    g = i % (uint32_t)p.a.groups;
    b = i / (uint32_t)p.a.groups;
    q = threadIdx.x % Q;
    ch = threadIdx.x / Q;
    base = block_start(p, blk);
    have = block_start(p, blk + 1) - base;
    on = ch < have;
    d = g * p.group_width + base + min(ch, have - 1);
  }
  // The lane's S values of an array [.][width][states] (0 for missing states).
  __device__ void load(const float* x, int64_t before, const ScanParams& p, float (&v)[S]) const {
    const float* at = x + (before * p.a.width + d) * p.a.states;
#pragma unroll
    for (int i = 0; i < S; i++) v[i] = q * S + i < p.a.states ? at[q * S + i] : 0.f;
  }
  __device__ void store(float* x, int64_t before, const ScanParams& p, const float (&v)[S]) const {
    float* at = x + (before * p.a.width + d) * p.a.states;
#pragma unroll
    for (int i = 0; i < S; i++)
      if (on && q * S + i < p.a.states) at[q * S + i] = v[i];
  }
  // The same of a padded array [.][width][N].
  __device__ float* padded(float* x, int64_t before, const ScanParams& p) const {
    return x + (before * p.a.width + d) * N + q * S;
  }
};

// A thread's share of a tile: NV vectors of VEC channels of one column.  Where VEC
// does not divide the block's channels, the last column moves back by the
// difference: its first elements are its neighbour's too, whose thread is a
// lane of the same wave, reads and writes the same values in the same order,
// and sums them once (see `put`).
template <class T, int Q, int VEC, int TILE>
struct Tile {
  static constexpr int CW = channels_of(Q);
  static constexpr int threads = CW * Q;
  static constexpr int columns = CW / VEC;
  static constexpr int rows = threads / columns > TILE ? TILE : threads / columns;
  static constexpr int NV = TILE / rows;
  typedef T Raw __attribute__((ext_vector_type(VEC)));
  int64_t d;                        // first channel of the column, clamped
  int c, r;                         // its place in the block, first row
  int over;                         // elements past the block's last channel, to be zeros
  // Every thread has a row of its own in a tile (else: `lead`).
  static constexpr bool all = threads / columns <= TILE;
  bool lead;
  bool on;                          // and its channel exists
  template <class P>
  __device__ Tile(const ScanParams& p, const P& place) {
    const int have = place.have;
    c = threadIdx.x % columns * VEC;
    lead = all || threadIdx.x / columns < rows;
    r = min((int)threadIdx.x / columns, rows - 1);
    on = lead && c < have;
    over = on ? max(0, c + VEC - have) : 0;
    c -= over;
    d = place.g * p.group_width + place.base + min(c, have - VEC);
  }
  // Row r of the column to LDS.
  template <class E, int ROW>
  __device__ void put(E* lds, int row, const E (&x)[VEC]) const {
    if (!all && !lead) return;
#pragma unroll
    for (int i = 0; i < VEC; i++) lds[row * ROW + c + i] = x[i];
    if (VEC > 1)
      for (int i = 0; i < over; i++) lds[row * ROW + c + VEC + i] = E{};
  }
  // The thread's place in row `t` + its first row.
  __device__ T* start(const rc_view& v, int64_t b, int t) const {
    return static_cast<T*>(v.data) + b * v.batch + (int64_t)(t + r) * v.time + d;
  }
  // The tile of tokens t0 .. from the thread's place p in it.  Loads are
  // unconditional, rows past the sequence clamped to its last: what is past an
  // end is dropped where it is used.
  __device__ void load(const T* p, int64_t time, int t0, int length, Raw (&x)[NV]) const {
#pragma unroll
    for (int k = 0; k < NV; k++) {
      int64_t at = (int64_t)(k * rows) * time;
      if (t0 + TILE > length) at -= max(0, t0 + k * rows + r - (length - 1)) * time;
      __builtin_memcpy(&x[k], p + at, sizeof(Raw));
    }
  }
  __device__ void vector(const float* w, float (&x)[VEC]) const {
#pragma unroll
    for (int i = 0; i < VEC; i++) x[i] = w ? w[d + i] : 0.f;
  }
};

// A tile of B or C to LDS in 32 bits: [TILE][N], zeros past the end and for missing states.
template <class T, int N, int TILE, int THREADS>
struct StateTile {
  static constexpr int ROWS = THREADS / N;
  static constexpr int NE = TILE > ROWS ? TILE / ROWS : 1;
  const T* p;                       // the thread's place in the tile to load next
  T x[NE];
  __device__ void start(const rc_view& v, int64_t group, int64_t b, int t, int states) {
    p = static_cast<const T*>(v.data) + b * v.batch + (int64_t)(t + threadIdx.x / N) * v.time +
        group + min((int)threadIdx.x % N, states - 1);
  }
  __device__ void load(int64_t time, int t0, int length) {
#pragma unroll
    for (int k = 0; k < NE; k++) {
      int64_t at = (int64_t)(k * ROWS) * time;
      if (t0 + (TILE > ROWS ? TILE : ROWS) > length)
        at -= max(0, t0 + k * ROWS + (int)(threadIdx.x / N) - (length - 1)) * time;
      x[k] = p[at];
    }
  }
  __device__ void put(float* lds, int t0, int end, int states) const {
#pragma unroll
    for (int k = 0; k < NE; k++) {
      const int r = k * ROWS + threadIdx.x / N;
      const float v = (float)x[k];
      if (TILE >= ROWS || r < TILE)
        lds[r * N + threadIdx.x % N] = t0 + r < end && (int)threadIdx.x % N < states ? v : 0.f;
    }
  }
};

// S states of LDS, where they are aligned to their size.  (kept and the workspace are aligned to a
// float only: load_vec and store_vec.)
template <int S>
__device__ __forceinline__ void read_states(const float* lds, float (&x)[S]) {
  typedef float FV __attribute__((ext_vector_type(S)));
  const FV v = *reinterpret_cast<const FV*>(lds);
#pragma unroll
  for (int i = 0; i < S; i++) x[i] = v[i];
}
// The state that enters chunk `piece`, from the chunks before it (or, REVERSE, the
// gradient of the state that leaves it, from the chunks after it).
template <int Q, int S, bool REVERSE>
__device__ __forceinline__ void enter(const ScanParams& p, const Place<Q, S>& w,
                                      const float (&A)[S], float (&h)[S]) {
  constexpr int AHEAD = 8;          // chunks whose loads are in flight together
  const int count = REVERSE ? p.chunks - 1 - w.piece : w.piece;
  const int first = REVERSE ? p.chunks - 1 : 0, step = REVERSE ? -1 : 1;
  for (int k0 = 0; k0 < count; k0 += AHEAD) {
    float own[AHEAD][S], sum[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; k++) {
      const int64_t at = w.b * p.chunks + first + step * min(k0 + k, count - 1);
      load_vec<S>(w.padded(p.ends, at, p), S, own[k]);
      sum[k] = p.steps[at * p.a.width + w.d];
    }
#pragma unroll
    for (int k = 0; k < AHEAD; k++)
#pragma unroll
      for (int i = 0; i < S; i++) {
        const float next = fmaf(fast_exp2(sum[k] * A[i]), h[i], own[k][i]);
        h[i] = k0 + k < count ? next : h[i];
      }
  }
}

// Forward.  A tile of tokens is staged to LDS in 32 bits (delta and delta u of
// each channel, B, C), each element converted once by one thread; then the
// lanes walk over it, four tokens at a time: each lane of a quad reads one
// token's delta and delta u of its channel and the quad shares them, and each
// ends with one token's y, which takes their place.  Rows of LDS are padded so
// that the four rows that a quad reads lie in different banks.
// ENDS: only the end state of the chunk from nothing, and its sum of delta.
// Bound by VALU issue (89% busy): 33 instructions for a step of a wave over a token
// with 4 states a lane, 20 of them the recurrence's.  16 x 2048 x 4096, 16 states in bfloat16: 605 us, 3.5e12 state
// steps/s, in 32 bits 615; one prompt of 16384 x 2048 264 us.
template <class T, int Q, int S, int VEC, bool ENDS>
__global__ __launch_bounds__(channels_of(Q) * Q) void k_scan_forward(ScanParams p) {
  constexpr int TILE = kFwdTile, N = Q * S, CW = channels_of(Q), ROW = CW + 8;
  __shared__ float2 lds_d[TILE * ROW];
  __shared__ __align__(16) float lds_b[TILE * N], lds_c[ENDS ? 4 : TILE * N];
  const rc_scan_args& a = p.a;
  const Place<Q, S> w(p);
  const Tile<T, Q, VEC, TILE> tile(p, w);
  using TileT = Tile<T, Q, VEC, TILE>;
  const int end = seq_end(a.lengths, w.b, a.length);
  const int t_first = w.piece * p.chunk, t_last = min(t_first + p.chunk, a.length);
  if (ENDS && w.piece == p.chunks - 1) return;         // nothing follows it
  float A[S], h[S], total = 0.f;
  w.load(a.A, 0, p, A);
#pragma unroll
  for (int i = 0; i < S; i++) {
    A[i] *= kLog2e;
    h[i] = 0.f;
  }
  if (!ENDS) {
    if (a.state_in) w.load(a.state_in, w.b, p, h);
    if (p.chunks > 1) enter<Q, S, false>(p, w, A, h);
  }
  float D[VEC], bias[VEC];
  tile.vector(a.D, D);
  tile.vector(a.dt_bias, bias);
  typename TileT::Raw u[TileT::NV], dt[TileT::NV], z[TileT::NV] = {};
  StateTile<T, N, TILE, CW * Q> B, C;
  const T *at_u = tile.start(a.u, w.b, t_first), *at_dt = tile.start(a.dt, w.b, t_first);
  // Loads are not in branches whose results the loop hands on (the compiler of ROCm 7.2 drops some
  // of their elements): without a gate dt is read twice.
  const bool gated = a.z.data;
  const rc_view from_z = gated ? a.z : a.dt;
  const T* at_z = tile.start(from_z, w.b, t_first);
  T* at_y = tile.start(a.y, w.b, t_first);
  B.start(a.B, w.g * a.B_group, w.b, t_first, a.states);
  C.start(a.C, w.g * a.C_group, w.b, t_first, a.states);
  const auto fetch = [&](int t0) {                     // and on to the next tile
    tile.load(at_u, a.u.time, t0, a.length, u);
    tile.load(at_dt, a.dt.time, t0, a.length, dt);
    at_u += TILE * a.u.time;
    at_dt += TILE * a.dt.time;
    B.load(a.B.time, t0, a.length);
    B.p += TILE * a.B.time;
    if (ENDS) return;
    tile.load(at_z, from_z.time, t0, a.length, z);
    at_z += TILE * from_z.time;
    C.load(a.C.time, t0, a.length);
    C.p += TILE * a.C.time;
  };
  const int live = min(t_last, end);                   // tiles from here on are zeros
  int t0 = t_first;
  if (t0 < live) fetch(t0);
  for (; t0 < live; t0 += TILE, at_y += TILE * a.y.time) {
#pragma unroll
    for (int k = 0; k < TileT::NV; k++) {
      const int r = k * TileT::rows + tile.r;
      const bool ok = tile.on && t0 + r < end;
      float2 d[VEC];
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        const float delta = delta_of((float)dt[k][i] + bias[i], a.softplus);
        const float du = delta * (float)u[k][i];
        d[i] = {ok ? delta : 0.f, ok ? du : 0.f};
      }
      tile.template put<float2, ROW>(lds_d, r, d);
    }
    B.put(lds_b, t0, end, a.states);
    if (!ENDS) C.put(lds_c, t0, end, a.states);
    __syncthreads();
    typename TileT::Raw u0[TileT::NV], z0[TileT::NV];  // of this tile, for its outputs
#pragma unroll
    for (int k = 0; k < TileT::NV; k++) {
      u0[k] = u[k];
      z0[k] = z[k];
    }
    fetch(t0 + TILE);
#pragma unroll 2
    for (int i4 = 0; i4 < TILE / 4; i4++) {
      if (!ENDS && a.kept && i4 % (kKeep / 4) == 0 && w.on && t0 + 4 * i4 < a.length)
        store_vec<S>(w.padded(a.kept, w.b * p.keeps + (t0 + 4 * i4) / kKeep, p), S, h);
      const int at = (4 * i4 + (w.q & 3)) * ROW + w.ch;
      const float2 d = lds_d[at];
      float y[4];
      const auto token = [&](auto J) {
        const float delta = quad_lane<J()>(d.x), du = quad_lane<J()>(d.y);
        float b[S], c[S];
        read_states<S>(lds_b + (4 * i4 + J()) * N + w.q * S, b);
        if (!ENDS) read_states<S>(lds_c + (4 * i4 + J()) * N + w.q * S, c);
        y[J()] = 0.f;
#pragma unroll
        for (int i = 0; i < S; i++) {
          h[i] = fmaf(fast_exp2(delta * A[i]), h[i], du * b[i]);
          if (!ENDS) y[J()] = fmaf(h[i], c[i], y[J()]);
        }
      };
      token(std::integral_constant<int, 0>{});
      token(std::integral_constant<int, 1>{});
      token(std::integral_constant<int, 2>{});
      token(std::integral_constant<int, 3>{});
      if (ENDS)
        total += d.x;                                  // of the lane's token of four
      else
        lds_d[at].x = state_sums<Q>(y);
    }
    __syncthreads();
    if (!ENDS && tile.on) {
#pragma unroll
      for (int k = 0; k < TileT::NV; k++) {
        const int r = k * TileT::rows + tile.r, t = t0 + r;
        float y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; i++) {
          const float zi = (float)z0[k][i], act = zi * sigmoid(zi);
          y[i] = fmaf(D[i], (float)u0[k][i], lds_d[r * ROW + tile.c + i].x);
          y[i] *= gated ? act : 1.f;
          y[i] = t < end ? y[i] : 0.f;
        }
        if (t < t_last) store_vec<VEC>(at_y + k * TileT::rows * a.y.time, VEC, y);
      }
    }
    // a wave stages the elements whose outputs it has just read
  }
  for (; !ENDS && t0 < t_last; t0 += TILE, at_y += TILE * a.y.time) {
    const float zero[VEC] = {};
#pragma unroll
    for (int k = 0; k < TileT::NV; k++)
      if (tile.on && t0 + k * TileT::rows + tile.r < t_last)
        store_vec<VEC>(at_y + k * TileT::rows * a.y.time, VEC, zero);
  }
  if (ENDS) {
    total += dpp<kXor1>(total);
    total += dpp<kXor2>(total);
    if (w.on) {
      store_vec<S>(w.padded(p.ends, w.b * p.chunks + w.piece, p), S, h);
      if (w.q == 0) p.steps[(w.b * p.chunks + w.piece) * a.width + w.d] = total;
    }
  } else if (a.state_out && w.piece == p.chunks - 1) {
    w.store(a.state_out, w.b, p, h);
  }
}

// Backward.  Tiles from the last to the first: staged as forward (with dy =
// dout z sigmoid(z)), then the lanes compute the tile's states again from the
// kept one, with the decays, into registers, and walk back over them.  The
// sums over a channel's states take the staged inputs' places in LDS (a
// channel is read and written by one wave), where the staging threads pick
// them up for du, ddt and dz.  With four states a lane the decays are computed again on the
// way back, since keeping them spills; with fewer they stay (8 x 1024 x 2048 with
// 8 states 232 -> 221 us).  ENDS: only the gradient of the state before the chunk,
// from nothing after it, and its sum of delta.
// Bound by VALU issue (87% busy): 105 instructions for a step of a wave, 60 of them
// the recurrence's.  16 x 2048 x 4096, 16 states in bfloat16: 1.86 ms, 1.15e12 state steps/s, in 32 bits 1.83.
template <class T, int Q, int S, int VEC, bool ENDS>
__global__ __launch_bounds__(channels_of(Q) * Q, 2) void k_scan_backward(ScanParams p) {
  constexpr int TILE = kKeep, N = Q * S, CW = channels_of(Q), ROW = CW + 4;
  constexpr int THREADS = CW * Q, WAVES = THREADS / 64;
  constexpr int VALUES = 64 / Q;                       // of a sum over a wave's channels
  constexpr int STEPS = VALUES > 2 * S ? VALUES / (2 * S) : 1;   // tokens of one such sum
  __shared__ float4 lds_d[TILE * ROW];                 // delta, delta u, dy
  __shared__ __align__(16) float lds_c[TILE * N], lds_b[ENDS ? 4 : TILE * N];
  __shared__ float lds_bc[ENDS ? 1 : WAVES * TILE * 2 * N];
  const rc_scan_args& a = p.a;
  const Place<Q, S> w(p);
  const Tile<T, Q, VEC, TILE> tile(p, w);
  using TileT = Tile<T, Q, VEC, TILE>;
  const int end = seq_end(a.lengths, w.b, a.length);
  const int t_first = w.piece * p.chunk, t_last = min(t_first + p.chunk, a.length);
  if (ENDS && w.piece == 0) return;                    // nothing precedes it
  const int wave = threadIdx.x / 64, mine = channel_value<Q>(threadIdx.x % 64);
  float A[S], g[S], dA[S], total = 0.f;                // g: of the state before the later token
  w.load(a.A, 0, p, A);
#pragma unroll
  for (int i = 0; i < S; i++) {
    A[i] *= kLog2e;
    g[i] = dA[i] = 0.f;
  }
  if (!ENDS) {
    if (a.dstate_out) w.load(a.dstate_out, w.b, p, g);
    if (p.chunks > 1) enter<Q, S, true>(p, w, A, g);
  }
  float D[VEC], bias[VEC], dD[VEC], dbias[VEC];
  tile.vector(a.D, D);
  tile.vector(a.dt_bias, bias);
#pragma unroll
  for (int i = 0; i < VEC; i++) dD[i] = dbias[i] = 0.f;
  typename TileT::Raw u[TileT::NV] = {}, dt[TileT::NV], z[TileT::NV] = {}, dout[TileT::NV];
  StateTile<T, N, TILE, THREADS> B, C;
  float h0[S];
  const bool gated = a.z.data;
  const rc_view from_z = gated ? a.z : a.dt;           // as forward
  // tiles past the end: zeros
  const int live = t_first + (int)cdiv(max(0, min(t_last, end) - t_first), TILE) * TILE;
  if (!ENDS) {
    const float zero[VEC] = {};
    for (int t = live + threadIdx.x / TileT::columns; t < t_last; t += THREADS / TileT::columns)
      if (tile.on || tile.c < w.have) {
        store_vec<VEC>(row_out<T>(a.du, w.b, t) + tile.d, VEC, zero);
        store_vec<VEC>(row_out<T>(a.ddt, w.b, t) + tile.d, VEC, zero);
        if (a.z.data) store_vec<VEC>(row_out<T>(a.dz, w.b, t) + tile.d, VEC, zero);
      }
    const int64_t cell = ((w.blk * (int64_t)a.batch + w.b) * a.length) * a.groups + w.g;
    for (int t = live + threadIdx.x / (2 * N); t < t_last; t += THREADS / (2 * N))
      p.part_bc[(cell + (int64_t)t * a.groups) * (2 * N) + threadIdx.x % (2 * N)] = 0.f;
  }
  // from the last live tile back; the first one is fetched twice
  const int t_top = max(live - TILE, t_first);
  const T *at_u = tile.start(a.u, w.b, t_top), *at_dt = tile.start(a.dt, w.b, t_top);
  const T *at_z = tile.start(from_z, w.b, t_top), *at_dy = tile.start(a.dy, w.b, t_top);
  T *at_du = tile.start(a.du, w.b, t_top), *at_ddt = tile.start(a.ddt, w.b, t_top);
  T* at_dz = tile.start(a.dz, w.b, t_top);
  const float* at_kept = w.padded(a.kept, w.b * p.keeps + t_top / TILE, p);
  B.start(a.B, w.g * a.B_group, w.b, t_top, a.states);
  C.start(a.C, w.g * a.C_group, w.b, t_top, a.states);
  const auto fetch = [&](int t0) {                     // and back to the tile before
    const int64_t back = t0 > t_first ? TILE : 0;
    tile.load(at_dt, a.dt.time, t0, a.length, dt);
    at_dt -= back * a.dt.time;
    tile.load(at_z, from_z.time, t0, a.length, z);
    at_z -= back * from_z.time;
    tile.load(at_dy, a.dy.time, t0, a.length, dout);
    at_dy -= back * a.dy.time;
    C.load(a.C.time, t0, a.length);
    C.p -= back * a.C.time;
    if (ENDS) return;
    tile.load(at_u, a.u.time, t0, a.length, u);
    at_u -= back * a.u.time;
    B.load(a.B.time, t0, a.length);
    B.p -= back * a.B.time;
    load_vec<S>(at_kept, S, h0);
    at_kept -= back / TILE * a.width * N;
  };
  int t0 = live - TILE;
  if (t0 >= t_first) fetch(t0);
  for (; t0 >= t_first; t0 -= TILE) {
    float step[TileT::NV][VEC];                        // delta of the thread's elements
#pragma unroll
    for (int k = 0; k < TileT::NV; k++) {
      const int r = k * TileT::rows + tile.r;
      const bool ok = tile.on && t0 + r < end;
      float4 d[VEC];
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        const float delta = delta_of((float)dt[k][i] + bias[i], a.softplus);
        const float zi = (float)z[k][i], act = zi * sigmoid(zi), o = (float)dout[k][i];
        const float du = delta * (float)u[k][i], dy = o * (gated ? act : 1.f);
        step[k][i] = ok ? delta : 0.f;
        d[i] = {step[k][i], ok ? du : 0.f, ok ? dy : 0.f, 0.f};
      }
      tile.template put<float4, ROW>(lds_d, r, d);
    }
    C.put(lds_c, t0, end, a.states);
    if (!ENDS) B.put(lds_b, t0, end, a.states);
    float h[ENDS ? 1 : TILE + 1][S];
    if (!ENDS) {
#pragma unroll
      for (int i = 0; i < S; i++) h[0][i] = h0[i];
    }
    __syncthreads();
    typename TileT::Raw u0[TileT::NV], dt0[TileT::NV], z0[TileT::NV], dout0[TileT::NV];
#pragma unroll
    for (int k = 0; k < TileT::NV; k++) {
      u0[k] = u[k];
      dt0[k] = dt[k];
      z0[k] = z[k];
      dout0[k] = dout[k];
    }
    fetch(max(t0 - TILE, t_first));
    if (ENDS) {
#pragma unroll 2
      for (int i4 = TILE / 4 - 1; i4 >= 0; i4--) {
        const float4 d = lds_d[(4 * i4 + (w.q & 3)) * ROW + w.ch];
        const auto token = [&](auto J) {
          const float delta = quad_lane<J()>(d.x), dy = quad_lane<J()>(d.z);
          float c[S];
          read_states<S>(lds_c + (4 * i4 + J()) * N + w.q * S, c);
#pragma unroll
          for (int i = 0; i < S; i++) g[i] = fast_exp2(delta * A[i]) * fmaf(c[i], dy, g[i]);
        };
        token(std::integral_constant<int, 3>{});
        token(std::integral_constant<int, 2>{});
        token(std::integral_constant<int, 1>{});
        token(std::integral_constant<int, 0>{});
        total += d.x;
      }
    } else {
      float4 d[TILE / 4];
#pragma unroll
      for (int i4 = 0; i4 < TILE / 4; i4++) {
        d[i4] = lds_d[(4 * i4 + (w.q & 3)) * ROW + w.ch];
        const auto token = [&](auto J) {
          const int j = 4 * i4 + J();
          const float delta = quad_lane<J()>(d[i4].x), du = quad_lane<J()>(d[i4].y);
          float b[S];
          read_states<S>(lds_b + j * N + w.q * S, b);
#pragma unroll
          for (int i = 0; i < S; i++) {
            h[j + 1][i] = fmaf(fast_exp2(delta * A[i]), h[j][i], du * b[i]);
          }
        };
        token(std::integral_constant<int, 0>{});
        token(std::integral_constant<int, 1>{});
        token(std::integral_constant<int, 2>{});
        token(std::integral_constant<int, 3>{});
      }
      float v[STEPS * 2 * S];                          // dB, dC of STEPS tokens
#pragma unroll
      for (int i4 = TILE / 4 - 1; i4 >= 0; i4--) {
        float y[4], through[4], dd[4];
        const auto token = [&](auto J) {
          const int j = 4 * i4 + J();
          float delta = quad_lane<J()>(d[i4].x);
          if (S == 4) asm("" : "+v"(delta));           // decays again, not kept: registers
          const float du = quad_lane<J()>(d[i4].y), dy = quad_lane<J()>(d[i4].z);
          float b[S], c[S], *bc = v + j % STEPS * 2 * S;
          read_states<S>(lds_b + j * N + w.q * S, b);
          read_states<S>(lds_c + j * N + w.q * S, c);
          y[J()] = through[J()] = dd[J()] = 0.f;
#pragma unroll
          for (int i = 0; i < S; i++) {
            y[J()] = fmaf(h[j + 1][i], c[i], y[J()]);
            const float gi = fmaf(c[i], dy, g[i]);
            bc[i] = gi * du;
            bc[S + i] = dy * h[j + 1][i];
            through[J()] = fmaf(gi, b[i], through[J()]);
            g[i] = fast_exp2(delta * A[i]) * gi;
            const float via = g[i] * h[j][i];
            dA[i] = fmaf(via, delta, dA[i]);
            dd[J()] = fmaf(via, A[i], dd[J()]);
          }
          if (j % STEPS == 0) {
#pragma unroll
            for (int m = 0; m < STEPS * 2 * S; m += VALUES) {
              const int e = m + mine;                  // value of token j + e / 2S
              lds_bc[(wave * TILE + j + e / (2 * S)) * 2 * N + e / S % 2 * N + w.q * S + e % S] =
                  channel_sums<Q>(v + m);
            }
          }
        };
        token(std::integral_constant<int, 3>{});
        token(std::integral_constant<int, 2>{});
        token(std::integral_constant<int, 1>{});
        token(std::integral_constant<int, 0>{});
        lds_d[(4 * i4 + (w.q & 3)) * ROW + w.ch] = {state_sums<Q>(through), state_sums<Q>(dd),
                                                    state_sums<Q>(y), 0.f};
      }
    }
    __syncthreads();
    if (!ENDS) {
      const int64_t cell = ((w.blk * (int64_t)a.batch + w.b) * a.length + t0) * a.groups + w.g;
      for (int e = threadIdx.x; e < TILE * 2 * N; e += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < WAVES; k++) s += lds_bc[k * TILE * 2 * N + e];
        const int r = e / (2 * N);                     // past the end h may not be finite: chosen
        if (t0 + r < t_last)
          p.part_bc[(cell + (int64_t)r * a.groups) * (2 * N) + e % (2 * N)] = t0 + r < end ? s : 0.f;
      }
#pragma unroll
      for (int k = 0; k < TileT::NV; k++) {
        const int r = k * TileT::rows + tile.r, t = t0 + r;
        const bool ok = t < end;
        float du[VEC], ddt[VEC], dz[VEC];
#pragma unroll
        for (int i = 0; i < VEC; i++) {
          const float4 sums = lds_d[r * ROW + tile.c + i];
          const float ui = (float)u0[k][i], zi = (float)z0[k][i], o = (float)dout0[k][i];
          const float s = sigmoid(zi), dy = o * (gated ? zi * s : 1.f);
          const float slope = sigmoid((float)dt0[k][i] + bias[i]);
          const float y = fmaf(D[i], ui, sums.z), dd = fmaf(ui, sums.x, sums.y * kLn2);
          const float own = dy * ui, raw = dd * (a.softplus ? slope : 1.f);
          const float through = fmaf(step[k][i], sums.x, D[i] * dy);
          const float gate = o * y * (s * (1.f + zi * (1.f - s)));
          du[i] = ok ? through : 0.f;
          ddt[i] = ok ? raw : 0.f;
          dz[i] = ok ? gate : 0.f;
          dD[i] += ok ? own : 0.f;
          dbias[i] += ddt[i];
        }
        if (tile.on && t < t_last) {
          store_vec<VEC>(at_du + k * TileT::rows * a.du.time, VEC, du);
          store_vec<VEC>(at_ddt + k * TileT::rows * a.ddt.time, VEC, ddt);
          if (gated) store_vec<VEC>(at_dz + k * TileT::rows * a.dz.time, VEC, dz);
        }
      }
      at_du -= TILE * a.du.time;
      at_ddt -= TILE * a.ddt.time;
      at_dz -= TILE * a.dz.time;
    }
    __syncthreads();                                   // the next tile takes the same LDS
  }
  const int64_t before = w.b * p.chunks + w.piece;
  if (ENDS) {
    total += dpp<kXor1>(total);
    total += dpp<kXor2>(total);
    if (w.on) {
      store_vec<S>(w.padded(p.ends, before, p), S, g);
      if (w.q == 0) p.steps[before * a.width + w.d] = total;
    }
    return;
  }
  if (w.on) store_vec<S>(w.padded(p.part_a, before, p), S, dA);
  if (a.dstate_in && w.piece == 0) w.store(a.dstate_in, w.b, p, g);
  // D and dt_bias: the threads of a column, then one sum for each channel
  float* sums = reinterpret_cast<float*>(lds_d);       // [rows][channels] of (dD, dbias)
  if (tile.lead) {
#pragma unroll
    for (int i = 0; i < VEC; i++) {
      sums[(tile.r * CW + tile.c + i) * 2] = dD[i];
      sums[(tile.r * CW + tile.c + i) * 2 + 1] = dbias[i];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * CW; e += THREADS) {
    if (e / 2 >= w.have) continue;
    float s = 0.f;
    for (int r = 0; r < TileT::rows; r++) s += sums[r * 2 * CW + e];
    p.part_d[(before * a.width + w.g * p.group_width + w.base + e / 2) * 2 + e % 2] = s;
  }
}

// The sums over workgroups, in one launch: the first `cell_blocks` workgroups
// take dB and dC (one thread for each (batch, token, group, state), eight
// blocks' parts in flight), the next dA, the last dD and ddt_bias (columns of the
// parts of sequences and chunks).  Memory bound and short: 8 x 2048 x 2048 reads 71 MB in
// 15 us.
template <class T>
__global__ __launch_bounds__(kSumThreads) void k_scan_sums(ScanParams p, int64_t cells, int32_t N,
                                                           int64_t cell_blocks,
                                                           int64_t a_blocks) {
  __shared__ float lds[kSumThreads];
  const int32_t states = p.a.states;
  const int64_t blk = blockIdx.x;
  if (blk < cell_blocks) {
    const int64_t id = blk * kSumThreads + threadIdx.x;
    const int64_t cell = id / (2 * N), stride = cells * 2 * N;
    const int k = (int)(id % (2 * N)), n = k % N;
    if (cell >= cells || n >= states) return;
    const float* in = p.part_bc + cell * (2 * N) + k;
    float s = 0.f;
    int j = 0;
    for (; j + 8 <= p.blocks; j += 8) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = in[(j + i) * stride];
      s += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    for (; j < p.blocks; j++) s += in[j * stride];
    static_cast<T*>(k < N ? p.a.dB : p.a.dC)[cell * states + n] = (T)s;
    return;
  }
  const bool decay = blk < cell_blocks + a_blocks;
  const int64_t cols = (int64_t)p.a.width * (decay ? N : 2);
  const int64_t c = (blk - cell_blocks - (decay ? 0 : a_blocks)) * kSumCols +
                    threadIdx.x % kSumCols;
  const float s = column_sum(decay ? p.part_a : p.part_d, (int64_t)p.a.batch * p.chunks, cols, c,
                             lds);
  if (threadIdx.x >= kSumCols || c >= cols) return;
  if (decay) {
    if (c % N < states) p.a.dA[c / N * states + c % N] = s;
  } else {
    float* out = c % 2 ? p.a.ddt_bias : p.a.dD;
    if (out) out[c / 2] = s;
  }
}

constexpr int kStepThreads = 256, kStepRows = 2;

// Sum over the Q lanes of a channel, in each of them.
template <int Q>
__device__ __forceinline__ float state_sum(float x) {
  if (Q > 1) x += dpp<kXor1>(x);
  if (Q > 2) x += dpp<kXor2>(x);
  if (Q > 4) x += dpp<kHalfMirror>(x);
  if (Q > 8) x += dpp<kMirror>(x);
  return x;
}

template <class F>
int by_lanes(int q, F&& f) {
  switch (q) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

// A thread takes the same states of R channels, all loads before the first use: on a full
// chip the time is that of a slot's index and then the states behind it.  Memory
// bound; 256 rows of 4096 channels, 16 states (134 MB of states moved): R = 1 35 us,
// R = 2 28 us (4.8 TB/s, a large copy's rate), R = 4 36 us.
template <class T, int Q, int R>
__global__ __launch_bounds__(kStepThreads) void k_scan_step(rc_scan_step_args a, int32_t blocks) {
  constexpr int STRIDE = kStepThreads / Q;             // channels between a thread's
  const uint32_t b = blockIdx.x / (uint32_t)blocks;
  const int d0 = (int)(blockIdx.x % (uint32_t)blocks) * STRIDE * R + threadIdx.x / Q;
  const int q = threadIdx.x % Q, ns = max(0, min(4, a.states - 4 * q));
  const int64_t slot = a.slots ? a.slots[b] : b;
  const bool live = slot >= 0 && slot < a.num_slots;
  float h[R][4], A[R][4], B[R][4], C[R][4], u[R], z[R], raw[R], D[R], bias[R];
  float* state = a.state + (live ? slot : 0) * a.state_slot + 4 * q;
#pragma unroll
  for (int r = 0; r < R; r++) {
    const int d = d0 + r * STRIDE;
    if (!live || d >= a.width) continue;
    const int64_t g = d / (a.width / a.groups);
    load_vec<4>(state + (int64_t)d * a.states, ns, h[r]);
    load_vec<4>(a.A + (int64_t)d * a.states + 4 * q, ns, A[r]);
    load_vec<4>(row<T>(a.B, b, 0) + g * a.B_group + 4 * q, ns, B[r]);
    load_vec<4>(row<T>(a.C, b, 0) + g * a.C_group + 4 * q, ns, C[r]);
    u[r] = (float)row<T>(a.u, b, 0)[d];
    z[r] = a.z.data ? (float)row<T>(a.z, b, 0)[d] : 0.f;
    raw[r] = (float)row<T>(a.dt, b, 0)[d];
    D[r] = a.D ? a.D[d] : 0.f;
    bias[r] = a.dt_bias ? a.dt_bias[d] : 0.f;
  }
#pragma unroll
  for (int r = 0; r < R; r++) {
    const int d = d0 + r * STRIDE;
    if (d >= a.width) continue;
    float y = 0.f;
    if (live) {
      const float delta = delta_of(raw[r] + bias[r], a.softplus);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        h[r][i] = fmaf(fast_exp2(delta * A[r][i] * kLog2e), h[r][i], delta * u[r] * B[r][i]);
        y = fmaf(h[r][i], C[r][i], y);
      }
      store_vec<4>(state + (int64_t)d * a.states, ns, h[r]);
      y = fmaf(D[r], u[r], state_sum<Q>(y));
      if (a.z.data) y *= z[r] * sigmoid(z[r]);
    }
    if (q == 0) row_out<T>(a.y, b, 0)[d] = (T)y;
  }
}

bool scan_sizes_ok(int32_t dtype, int32_t batch, int32_t length, int32_t width, int32_t states,
                   int32_t groups) {
  return dtype_ok(dtype) && batch >= 0 && length >= 0 && width >= 0 && length <= kMaxExtent &&
         width <= kMaxExtent && states >= 1 && states <= 64 && groups >= 1 && width % groups == 0;
}
bool scan_sizes_ok(const rc_scan_args* a) {
  return a && scan_sizes_ok(a->dtype, a->batch, a->length, a->width, a->states, a->groups);
}

// How a scan is cut up.  A channel takes a quad of lanes (more above 16
// states).  The kernels are bound by instruction issue, which wants waves on
// every SIMD, and evenly: where batch and channels give few, or just more than a
// whole number for each, the length is cut into chunks, which costs a pass
// over all but one of them for their end states.  bfloat16, 16 states, 2048 tokens and
// channels (a batch of 8 is one wave a SIMD), whole or best cut, us:
//   batch     2        4        6        8       10       12       16       20
//   forward  198/75   199/131  199/185  202/233  335/289  335/340  338/409  458/520
//   backward 655/175  658/317  664/460  672/590  957/729  964/865  977/1110 1482/1390
// With v waves a SIMD on average and k on the fullest, a whole pass costs 95 +
// 130 k forward (one wave: 202, see scan_plan), a cut one 1.7 times 130 v; backward 490
// k (one wave: 665) and 1.18 times 490 v.  The factors are this table's; what they choose was then timed
// in bfloat16 and float32 with 4, 16, 32 and 64 states, batches 1 to 16: the faster of the two or
// within 6% of it but for 4 states forward at one wave a SIMD (bfloat16, whole 147, cut 128).
bool scan_cut(double v, double k, bool backward) {
  return backward ? k == 1. || 1.18 * v < k : 1.7 * v < (k == 1. ? 1.36 : .5 + k);
}
struct ScanPlan {
  int S, Q, VEC;
  int64_t group_width, blocks;
  int64_t chunks, chunk, keeps;
};
ScanPlan scan_plan(const rc_scan_args& a, bool backward) {
  ScanPlan p;
  p.group_width = a.width / a.groups;
  p.S = a.states > 8 ? 4 : a.states > 4 ? 2 : 1;
  p.Q = a.states > 32 ? 16 : a.states > 16 ? 8 : 4;
  p.VEC = p.group_width < 4 ? 1 : 4;                   // channels of a load
  p.blocks = cdiv(p.group_width, channels_of(p.Q));
  // Chunks: sixteen waves a compute unit at least, up to twice as many where
  // that spreads them more evenly (batch 12 above: 3 chunks 4.5 workgroups a compute unit, 959 us;
  // 4 chunks 6 workgroups, 865).  They have 64 tokens at least (32: 2048 tokens of 1024
  // channels forward 40 for 37) and number 128 at most, whose joining is a
  // loop (16384 tokens of 64 channels forward and backward, 32 chunks 324, 128 chunks 117).
  const int64_t groups = (int64_t)a.batch * a.groups * p.blocks, cus = rcdp::num_cus();
  const int64_t group_waves = channels_of(p.Q) * p.Q / 64;
  const int64_t most = cdiv(a.length, 64) < 128 ? cdiv(a.length, 64) : 128;
  p.chunks = 1;
  if (groups > 0 && scan_cut((double)(groups * group_waves) / (4 * cus),
                             (double)(cdiv(groups, cus) * group_waves / 4), backward)) {
    const int64_t least = cdiv(16 * cus, groups * group_waves);
    double best = 0.;
    for (int64_t n = least; n <= 2 * least && n <= most; n++) {
      const double even = (double)(groups * n) / cdiv(groups * n, cus);
      if (even <= best) continue;
      best = even;
      p.chunks = n;
    }
    if (least > most) p.chunks = most;
  }
  if (p.chunks < 1) p.chunks = 1;
  p.chunk = cdiv(cdiv(a.length, p.chunks), kFwdTile) * kFwdTile;
  if (p.chunk < kFwdTile) p.chunk = kFwdTile;
  p.chunks = a.length > 0 ? cdiv(a.length, p.chunk) : 1;
  p.keeps = cdiv(a.length, kKeep);
  // One wave a SIMD, uncut: eight lanes of two states halve what a wave has to issue for
  // a token (8 x 2048 x 2048 forward 236 us with four lanes, 199 with eight, where the kept states
  // are written 232 and 210; lengths of 1 to 64 tokens, which are never cut, 7.0 to 11.0 and 6.5 to 10.2;
  // with more waves equal, and cut 133 for 137).  The kept states lie alike.
  if (!backward && p.chunks == 1 && groups <= cus && p.Q == 4 && p.S == 4) {
    p.Q = 8;
    p.S = 2;
  }
  return p;
}

struct ScanScratch {
  uint64_t ends, steps, bc, a, d;
  uint64_t total() const { return ends + steps + bc + a + d; }
};
ScanScratch scan_scratch(const rc_scan_args& a, const ScanPlan& p, bool backward) {
  const uint64_t rows = (uint64_t)a.batch * p.chunks * a.width, N = p.Q * p.S;
  ScanScratch s = {};
  if (p.chunks > 1) {
    s.ends = rows * N * 4;
    s.steps = (rows * 4 + 255) & ~255ull;
  }
  if (backward) {
    s.bc = (uint64_t)p.blocks * a.batch * a.length * a.groups * 2 * N * 4;
    s.a = rows * N * 4;
    s.d = rows * 2 * 4;
  }
  return s;
}

// Workgroups of k_scan_sums: for dB and dC, for dA, for dD and ddt_bias.
struct SumBlocks {
  int64_t cells, a, d;
  int64_t total() const { return cells + a + d; }
};
SumBlocks sum_blocks(const rc_scan_args& a, const ScanPlan& p) {
  const int N = p.Q * p.S;
  return {cdiv((int64_t)a.batch * a.length * a.groups * (2 * N), kSumThreads),
          cdiv((int64_t)a.width * N, kSumCols), cdiv((int64_t)a.width * 2, kSumCols)};
}

int scan_check(const rc_scan_args* a, bool backward) {
  if (!scan_sizes_ok(a) || !float_aligned(a->kept) || !float_aligned(a->workspace)) return RC_E_ARG;
  if (a->batch > 0 && a->width > 0) {
    if (!a->A) return RC_E_ARG;
    if (a->length > 0) {
      if (!a->u.data || !a->dt.data || !a->B.data || !a->C.data) return RC_E_ARG;
      if (!backward && !a->y.data) return RC_E_ARG;
      if (backward && (!a->dy.data || !a->du.data || !a->ddt.data || !a->kept ||
                       (a->z.data == nullptr) != (a->dz.data == nullptr)))
        return RC_E_ARG;
    }
  }
  if (backward && a->batch > 0 && a->length > 0 && (!a->dB || !a->dC)) return RC_E_ARG;
  if (backward && a->width > 0 &&
      (!a->dA || (a->D && !a->dD) || (a->dt_bias && !a->ddt_bias)))
    return RC_E_ARG;
  const ScanPlan p = scan_plan(*a, backward);
  if (!launchable(p.blocks * a->groups * a->batch * p.chunks, channels_of(p.Q) * p.Q))
    return RC_E_OVERFLOW;
  if (backward && !launchable(sum_blocks(*a, p).total(), kSumThreads)) return RC_E_OVERFLOW;
  return RC_OK;
}

ScanParams scan_params(const rc_scan_args& a, const ScanPlan& p, const ScanScratch& s) {
  ScanParams q = {};
  q.a = a;
  q.group_width = (int32_t)p.group_width;
  q.blocks = (int32_t)p.blocks;
  q.chunks = (int32_t)p.chunks;
  q.chunk = (int32_t)p.chunk;
  q.keeps = (int32_t)p.keeps;
  char* ws = static_cast<char*>(a.workspace);
  q.ends = reinterpret_cast<float*>(ws);
  q.steps = reinterpret_cast<float*>(ws + s.ends);
  q.part_bc = reinterpret_cast<float*>(ws + s.ends + s.steps);
  q.part_a = reinterpret_cast<float*>(ws + s.ends + s.steps + s.bc);
  q.part_d = reinterpret_cast<float*>(ws + s.ends + s.steps + s.bc + s.a);
  return q;
}

// Calls f(Q, S, VEC) with the plan's constants.
template <bool BACKWARD, class F>
int by_plan(const ScanPlan& p, F&& f) {
  using std::integral_constant;
  const auto with = [&](auto Q, auto S) {
    if (p.VEC == 1) return f(Q, S, integral_constant<int, 1>{});
    return f(Q, S, integral_constant<int, 4>{});
  };
  if constexpr (!BACKWARD)
    if (p.Q == 8 && p.S == 2) return with(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  if (p.Q == 16) return with(integral_constant<int, 16>{}, integral_constant<int, 4>{});
  if (p.Q == 8) return with(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  if (p.S == 4) return with(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  if (p.S == 2) return with(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  return with(integral_constant<int, 4>{}, integral_constant<int, 1>{});
}

}  // namespace

extern "C" int rc_scan_kept_bytes(const rc_scan_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !scan_sizes_ok(a)) return RC_E_ARG;
  const ScanPlan p = scan_plan(*a, false);
  *bytes_host = (uint64_t)a->batch * p.keeps * a->width * p.Q * p.S * 4;
  return RC_OK;
}

extern "C" int rc_scan_forward_workspace(const rc_scan_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !scan_sizes_ok(a)) return RC_E_ARG;
  *bytes_host = scan_scratch(*a, scan_plan(*a, false), false).total();
  return RC_OK;
}

extern "C" int rc_scan_backward_workspace(const rc_scan_args* a, uint64_t* bytes_host) {
  if (!bytes_host || !scan_sizes_ok(a)) return RC_E_ARG;
  *bytes_host = scan_scratch(*a, scan_plan(*a, true), true).total();
  return RC_OK;
}

extern "C" int rc_scan_forward(const rc_scan_args* args, void* stream) {
  if (const int st = scan_check(args, false)) return st;
  const rc_scan_args& a = *args;
  const ScanPlan p = scan_plan(a, false);
  const ScanScratch need = scan_scratch(a, p, false);
  if (need.total() > 0 && (!a.workspace || a.workspace_bytes < need.total())) return RC_E_SCRATCH;
  const int64_t blocks = p.blocks * a.groups * a.batch * p.chunks;
  if (blocks == 0) return RC_OK;
  const ScanParams q = scan_params(a, p, need);
  const hipStream_t s = (hipStream_t)stream;
  return by_dtype(a.dtype, [&](auto t) {
    return by_plan<false>(p, [&](auto Q, auto S, auto VEC) -> int {
      using T = decltype(t);
      const dim3 grid((uint32_t)blocks), threads(channels_of(Q()) * Q());
      if constexpr (Q() != 8 || S() != 2)              // (that one is never cut)
        if (p.chunks > 1) {
          k_scan_forward<T, Q(), S(), VEC(), true><<<grid, threads, 0, s>>>(q);
          if (const int st = launched("k_scan_forward ends")) return st;
        }
      k_scan_forward<T, Q(), S(), VEC(), false><<<grid, threads, 0, s>>>(q);
      return launched("k_scan_forward");
    });
  });
}

extern "C" int rc_scan_backward(const rc_scan_args* args, void* stream) {
  if (const int st = scan_check(args, true)) return st;
  const rc_scan_args& a = *args;
  const ScanPlan p = scan_plan(a, true);
  const ScanScratch need = scan_scratch(a, p, true);
  if (need.total() > 0 && (!a.workspace || a.workspace_bytes < need.total())) return RC_E_SCRATCH;
  const ScanParams q = scan_params(a, p, need);
  const hipStream_t s = (hipStream_t)stream;
  const int64_t blocks = p.blocks * a.groups * a.batch * p.chunks;
  return by_dtype(a.dtype, [&](auto t) -> int {
    using T = decltype(t);
    if (blocks > 0) {
      const int st = by_plan<true>(p, [&](auto Q, auto S, auto VEC) -> int {
        const dim3 grid((uint32_t)blocks), threads(channels_of(Q()) * Q());
        if (p.chunks > 1) {
          k_scan_backward<T, Q(), S(), VEC(), true><<<grid, threads, 0, s>>>(q);
          if (const int e = launched("k_scan_backward ends")) return e;
        }
        k_scan_backward<T, Q(), S(), VEC(), false><<<grid, threads, 0, s>>>(q);
        return launched("k_scan_backward");
      });
      if (st) return st;
    }
    const SumBlocks n = sum_blocks(a, p);
    if (n.total() == 0) return RC_OK;                  // (without channels: zeros to dB and dC)
    k_scan_sums<T><<<dim3((uint32_t)n.total()), kSumThreads, 0, s>>>(
        q, (int64_t)a.batch * a.length * a.groups, p.Q * p.S, n.cells, n.a);
    return launched("k_scan_sums");
  });
}

extern "C" int rc_scan_step(const rc_scan_step_args* args, void* stream) {
  if (!args) return RC_E_ARG;
  const rc_scan_step_args& a = *args;
  if (!scan_sizes_ok(a.dtype, a.batch, 1, a.width, a.states, a.groups) || a.num_slots < 0 ||
      (!a.slots && a.num_slots < a.batch))
    return RC_E_ARG;
  if (a.batch == 0 || a.width == 0) return RC_OK;
  if (!a.u.data || !a.dt.data || !a.B.data || !a.C.data || !a.y.data || !a.A || !a.state)
    return RC_E_ARG;
  const int Q = a.states > 32 ? 16 : a.states > 16 ? 8 : a.states > 8 ? 4 : a.states > 4 ? 2 : 1;
  // R channels a thread where that still gives eight workgroups a compute unit
  const int64_t wide = cdiv(a.width, kStepThreads / Q * kStepRows);
  const bool many = wide * a.batch >= 8 * (int64_t)rcdp::num_cus();
  const int64_t blocks = many ? wide : cdiv(a.width, kStepThreads / Q);
  if (!launchable(blocks * a.batch, kStepThreads)) return RC_E_OVERFLOW;
  return by_dtype(a.dtype, [&](auto t) {
    return by_lanes(Q, [&](auto q) {
      using T = decltype(t);
      const dim3 grid((uint32_t)(blocks * a.batch));
      if (many)
        k_scan_step<T, q(), kStepRows><<<grid, kStepThreads, 0, (hipStream_t)stream>>>(
            a, (int32_t)blocks);
      else
        k_scan_step<T, q(), 1><<<grid, kStepThreads, 0, (hipStream_t)stream>>>(a, (int32_t)blocks);
      return launched("k_scan_step");
    });
  });
}
