// Shared by the sequence-model operators (conv.hip, scan.hip, norm.hip, delta.hip, qk.hip,
// dropout.hip): element types, wide loads and stores, activations, argument checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rc_internal.h"
#include "rc_ops.h"

namespace rcops {

using bf16 = __bf16;
using f16 = _Float16;

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;

// V consecutive elements at p as floats; those from n on are 0.  A whole
// vector is one wide load whatever p's alignment (the hardware takes unaligned
// addresses), a ragged end goes element by element.
template <int V, class T>
__device__ __forceinline__ void load_vec(const T* p, int n, float (&x)[V]) {
  typedef T TV __attribute__((ext_vector_type(V)));
  if (n >= V) {
    TV r;
    __builtin_memcpy(&r, p, sizeof(r));
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = (float)r[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = i < n ? (float)p[i] : 0.f;
  }
}

template <int V, class T>
__device__ __forceinline__ void store_vec(T* p, int n, const float (&x)[V]) {
  typedef T TV __attribute__((ext_vector_type(V)));
  if (n >= V) {
    TV r;
#pragma unroll
    for (int i = 0; i < V; i++) r[i] = (T)x[i];
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < V; i++)
      if (i < n) p[i] = (T)x[i];
  }
}

// Parameters come in 32 bits or in the activations' type T.
template <class T>
__device__ __forceinline__ float load_param(const void* p, int64_t i, bool f32) {
  return f32 ? static_cast<const float*>(p)[i] : (float)static_cast<const T*>(p)[i];
}
template <class T>
__device__ __forceinline__ void store_param(void* p, int64_t i, bool f32, float x) {
  if (f32)
    static_cast<float*>(p)[i] = x;
  else
    static_cast<T*>(p)[i] = (T)x;
}

// exp2 of the hardware: at most 1 ulp off, results below 2^-126 are 0.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// 1 / (1 + e^-x): e^-x overflows to infinity for x below -88 and the quotient to 0.
__device__ __forceinline__ float sigmoid(float x) {
  return fast_rcp(1.f + fast_exp2(-kLog2e * x));
}

// log(1 + e^x) = max(x, 0) + log1p(w), w = e^-|x| in (0, 1].  log1p(w) is
// log(s) w / (s - 1) with s = 1 + w rounded: log(s) / (s - 1) hardly changes over the rounding.
__device__ __forceinline__ float softplus(float x) {
  const float w = fast_exp2(-kLog2e * __builtin_fabsf(x));
  const float s = 1.f + w;
  const float r = s - 1.f;
  const float l = r == 0.f ? w : kLn2 * __builtin_amdgcn_logf(s) * (w * fast_rcp(r));
  return __builtin_fmaxf(x, 0.f) + l;                  // a NaN comes through w
}

template <int CTRL>
__device__ __forceinline__ float dpp_of(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + dpp_of<CTRL>(x);
}
// Sum of each lane's with that of the lane 16 (32) away.
__device__ __forceinline__ float add_16_apart(float x) {
  const unsigned a = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float add_32_apart(float x) {
  const unsigned a = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
// Sum over groups of 1, 2, 4 .. 64 lanes, in each of them (a mirror is as good as an
// exchange once the lanes below are equal).
template <int LANES>
__device__ __forceinline__ float lane_sum(float x) {
  if (LANES == 1) return x;
  x = dpp_add<0xB1>(x);                                // lanes 1 apart
  if (LANES == 2) return x;
  x = dpp_add<0x4E>(x);                                // 2 apart
  if (LANES == 4) return x;
  x = dpp_add<0x141>(x);                               // half rows mirrored
  if (LANES == 8) return x;
  x = dpp_add<0x140>(x);                               // rows mirrored
  if (LANES == 16) return x;
  x = add_16_apart(x);
  return LANES == 32 ? x : add_32_apart(x);
}

// An element of a (batch, time, head, channel) tensor.
template <class T>
__device__ __forceinline__ T* at_head(const rc_heads& v, int64_t b, int64_t t, int64_t h) {
  return static_cast<T*>(v.data) + b * v.batch + t * v.time + h * v.head;
}

__host__ __device__ inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- host side
inline int dtype_size(int32_t d) { return d == RC_F32 ? 4 : 2; }
inline bool dtype_ok(int32_t d) { return d >= RC_F32 && d <= RC_F16; }
inline bool float_aligned(const void* p) { return (uintptr_t)p % sizeof(float) == 0; }
inline bool param_ok(int32_t p, int32_t d) { return p == RC_F32 || p == d; }

// The launch's own error, if any, as a status (by_dtype, before the first launch of a
// call, drops what another library's calls left).
inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return RC_OK;
  rcdp::set_last_error(what, e);
  return RC_E_DEVICE;
}

// Calls f(T{}) with the element type of a (checked) dtype.
template <class F>
inline int by_dtype(int32_t d, F&& f) {
  (void)hipGetLastError();
  if (d == RC_F32) return f(float{});
  if (d == RC_BF16) return f(bf16{});
  return f(f16{});
}

// Whether a launch holds that many workgroups: its threads are fewer than 2^32.
inline bool launchable(int64_t blocks, int threads) {
  return blocks <= (((int64_t)1 << 32) - 1) / threads;
}
// Tokens and channels: indexes a few tiles past the last stay in 32 bits.
constexpr int32_t kMaxExtent = 1 << 30;

// Column sums of a partial buffer, a column reduction's last step:
// sum over p < parts of in[p * cols + c] for the workgroup's column of this
// thread.  256 threads take 16 columns, sixteen slices of the parts each,
// eight loads in flight; always the same slices in the same order.  The
// threads of slice 0 return the sums.  (512 parts of 12288 columns: 64 columns a
// workgroup with one load in flight took 18 us, this way 6.)
constexpr int kSumCols = 16;
__device__ __forceinline__ float column_sum(const float* in, int64_t parts, int64_t cols,
                                            int64_t c, float* lds /* [256] */) {
  constexpr int SLICES = 256 / kSumCols;
  const int slice = threadIdx.x / kSumCols;
  float s = 0.f;
  if (c < cols) {
    int64_t p = slice;
    for (; p + 7 * SLICES < parts; p += 8 * SLICES) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = in[(p + i * SLICES) * cols + c];
      s += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    for (; p < parts; p += SLICES) s += in[p * cols + c];
  }
  lds[threadIdx.x] = s;
  __syncthreads();
  if (slice) return 0.f;
#pragma unroll
  for (int i = 1; i < SLICES; i++) s += lds[threadIdx.x + i * kSumCols];
  return s;
}

}  // namespace rcops
