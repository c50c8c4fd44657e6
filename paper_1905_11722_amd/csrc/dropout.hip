// Dropout whose mask is never stored: word i % 4 of Philox4x32-10 (Salmon, Moraes, Dror and
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with counter (i / 4, tag) and key
// seed decides about element i, so whoever knows seed and tag draws the mask again.
//
// A thread has eight elements, 40 products of 32 by 32 bits for their two calls, about 195 vector
// instructions in all.  16384 x 4096 from bf16 onto a 32-bit residual stream: 671 MB in 116 us, 5.8 TB/s, its
// gradient 403 MB in 76 us, 5.3 TB/s: a large copy's rate and more, memory bounds both.  From bf16 to bf16 without a
// residual they take 52 us, and in the cache no less for each (4096 rows 15.3 us, 8192 26.8): there the instructions do.
#include "ops_internal.h"

using namespace rcops;

namespace {

struct DropoutParams {
  rc_dropout_args a;
  int64_t units;                            // of eight elements
  uint32_t below;                           // words below it are dropped
  bool all;                                 // or all of them
  float gain;
};
// Elements of a unit: one after the other in every tensor; in one row of each; anywhere.
enum { kFlat = 0, kWhole = 1, kSingle = 2 };

struct Words {
  uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint64_t counter, uint64_t tag, uint64_t seed) {
  uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)tag,
           c3 = (uint32_t)(tag >> 32), k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; i++) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

// Forward: T x -> R out with residual; backward: R x (the gradient) -> T out.
template <class I, class O, int WALK>
__global__ __launch_bounds__(256) void k_dropout(DropoutParams p, rc_view in, rc_view add, rc_view out) {
  const rc_dropout_args& a = p.a;
  const uint64_t seed = (uint64_t)(a.seed_device ? *a.seed_device : a.seed);
  const int64_t total = a.rows * a.width;
  const I* x = static_cast<const I*>(in.data);
  const O* r = static_cast<const O*>(add.data);
  O* y = static_cast<O*>(out.data);
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < p.units; u += (int64_t)gridDim.x * 256) {
    const int64_t first = u * 8;
    const int n = (int)min(total - first, (int64_t)8);
    float v[8], s[8];
    int64_t row = 0, col = first;
    if (WALK != kFlat) {
      row = first / a.width;
      col = first - row * a.width;
    }
    if (WALK == kSingle) {
      int64_t i = row, c = col;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        v[e] = e < n ? (float)x[i * in.batch + c] : 0.f;
        s[e] = e < n && r ? (float)r[i * add.batch + c] : 0.f;
        if (++c == a.width) c = 0, i++;
      }
    } else {
      load_vec<8>(x + row * in.batch + col, n, v);
      if (r) load_vec<8>(r + row * add.batch + col, n, s);
    }
    const Words w[2] = {philox((uint64_t)u * 2, (uint64_t)a.tag, seed),
                        philox((uint64_t)u * 2 + 1, (uint64_t)a.tag, seed)};
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float z = !p.all && w[e / 4].w[e % 4] >= p.below ? v[e] * p.gain : 0.f;
      v[e] = r ? s[e] + z : z;
    }
    if (WALK == kSingle) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        if (e < n) y[row * out.batch + col] = (O)v[e];
        if (++col == a.width) col = 0, row++;
      }
    } else {
      store_vec<8>(y + row * out.batch + col, n, v);
    }
  }
}

int check(const rc_dropout_args* a) {
  if (!a || !dtype_ok(a->dtype) || !param_ok(a->out_dtype, a->dtype) || a->rows < 0 || a->width < 0 ||
      !(a->p >= 0 && a->p <= 1))
    return RC_E_ARG;
  if (a->rows && a->width > ((int64_t)1 << 62) / a->rows) return RC_E_OVERFLOW;
  return RC_OK;
}

template <class I, class O>
int launch(const rc_dropout_args& a, rc_view in, rc_view add, rc_view out, void* stream) {
  DropoutParams p = {};
  p.a = a;
  p.units = cdiv(a.rows * a.width, 8);
  const double below = __builtin_nearbyint(a.p * 4294967296.0);
  p.all = below >= 4294967296.0;
  p.below = p.all ? 0 : (uint32_t)below;
  p.gain = p.all ? 0.f : (float)(1.0 / (1.0 - a.p));
  const auto flat = [&](const rc_view& v) { return !v.data || v.batch == a.width || a.rows == 1; };
  const unsigned grid = (unsigned)std::min<int64_t>(cdiv(p.units, 256), 1 << 20);
  const hipStream_t s = (hipStream_t)stream;
  if (flat(in) && flat(add) && flat(out))
    k_dropout<I, O, kFlat><<<grid, 256, 0, s>>>(p, in, add, out);
  else if (a.width % 8 == 0)
    k_dropout<I, O, kWhole><<<grid, 256, 0, s>>>(p, in, add, out);
  else
    k_dropout<I, O, kSingle><<<grid, 256, 0, s>>>(p, in, add, out);
  return launched("k_dropout");
}

}  // namespace

extern "C" int rc_dropout_forward(const rc_dropout_args* args, void* stream) {
  if (int e = check(args)) return e;
  const rc_dropout_args& a = *args;
  if (!a.residual.data && a.out_dtype != a.dtype) return RC_E_ARG;
  if (!a.rows || !a.width) return RC_OK;
  if (!a.x.data || !a.out.data) return RC_E_ARG;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (a.out_dtype == RC_F32) return launch<T, float>(a, a.x, a.residual, a.out, stream);
    return launch<T, T>(a, a.x, a.residual, a.out, stream);
  });
}

extern "C" int rc_dropout_backward(const rc_dropout_args* args, void* stream) {
  if (int e = check(args)) return e;
  const rc_dropout_args& a = *args;
  if (!a.rows || !a.width) return RC_OK;
  if (!a.x.data || !a.out.data) return RC_E_ARG;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (a.out_dtype == RC_F32) return launch<float, T>(a, a.out, rc_view{}, a.x, stream);
    return launch<T, T>(a, a.out, rc_view{}, a.x, stream);
  });
}
