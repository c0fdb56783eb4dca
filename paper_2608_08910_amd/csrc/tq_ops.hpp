// Building blocks of the operators around the frozen integer passes (router, block norms,
// low-rank adapters): element types, unaligned vector access, wave reductions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "tq_device.hpp"
#include "tq_internal.hpp"

namespace tq {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T, int N>
struct VecOf {
  // (rows of odd width start anywhere: the vector asks for its element's alignment only)
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// N consecutive elements as fp32. Global memory takes vector accesses at any element boundary.
template <int N, typename T>
__device__ __forceinline__ void load_n(const T* p, float (&v)[N]) {
  const auto w = *reinterpret_cast<const typename VecOf<T, N>::type*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)w[i];
}

// fp32 values rounded to T (nearest even), N consecutive elements.
template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, const float (&v)[N]) {
  typename VecOf<T, N>::type w;
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = (T)v[i];
  *reinterpret_cast<typename VecOf<T, N>::type*>(p) = w;
}

// Element e of a row that starts at a wave-uniform address: a 32-bit byte offset, so that the address
// takes one vector register (rows are below 4 GB).
template <typename T>
__device__ __forceinline__ T* at_element(T* row, uint32_t e) {
  typedef typename std::conditional<std::is_const<T>::value, const char, char>::type C;
  return reinterpret_cast<T*>(reinterpret_cast<C*>(row) + e * (uint32_t)sizeof(T));
}

// How the vectors of N elements lie in a row of n: N divides n; the last one may be a part, n >= N; n < N.
constexpr int kRowWhole = 0, kRowTail = 1, kRowShort = 2;

// v[i] = v[(i + d) mod N]
template <int N>
__device__ __forceinline__ void rotate(float (&v)[N], uint32_t d) {
#pragma unroll
  for (int s = 1; s < N; s <<= 1) {
    float u[N];
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = v[(i + s) % N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = d & s ? u[i] : v[i];
  }
}

// The elements e .. e+N-1 of a row of n > 0, those past its end as `fill`; nothing past it is read. Without
// branches, since the compiler waits for a load where two paths to its value meet. A part of a vector is taken from the last
// N elements of the row, by one load and a rotation instead of N loads (so in the router: it and its gradients, 4000 tokens of
// 1001 experts in fp32, 48 us against 66).
template <int ROW, int N, typename T>
__device__ __forceinline__ void load_row(const T* row, uint32_t e, uint32_t n, float (&v)[N], float fill = 0.0f) {
  if constexpr (ROW == kRowShort) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)*at_element(row, min(e + i, n - 1));
  } else {
    const uint32_t s = min(e, n - N);
    load_n<N>(at_element(row, s), v);
    if constexpr (ROW == kRowTail) rotate(v, e - s);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = e + (ROW == kRowWhole ? 0 : i) < n ? v[i] : fill;
}

template <int ROW, int N, typename T>
__device__ __forceinline__ void store_row(T* row, uint32_t e, uint32_t n, const float (&v)[N]) {
  if (ROW == kRowWhole ? e < n : ROW == kRowTail && e + N <= n) {
    store_n<N>(at_element(row, e), v);
  } else if (ROW != kRowWhole) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e + i < n) *at_element(row, e + i) = (T)v[i];
  }
}

// Calls f with how vectors of N lie in a row of n, as a constant.
template <int N = 4, typename F>
inline void with_row(int n, F f) {
  if (n % N == 0) f(std::integral_constant<int, kRowWhole>{});
  else if (n >= N) f(std::integral_constant<int, kRowTail>{});
  else f(std::integral_constant<int, kRowShort>{});
}

__device__ __forceinline__ int readlane_i(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float readlane_f(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// The lanes of a mask below one's own.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

template <int CTRL>
__device__ __forceinline__ int dpp_i(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false); }
template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) { return __int_as_float(dpp_i<CTRL>(__float_as_int(v))); }

// Sum over the 16 lanes of a row; every lane receives it.
__device__ __forceinline__ float row_sum_f32(float v) {
  v += dpp_f<kDppXor1>(v);
  v += dpp_f<kDppXor2>(v);
  v += dpp_f<kDppHalfMirror>(v);
  v += dpp_f<kDppRowRor8>(v);
  return v;
}

// Sum and maximum over a wave (the four 16-lane rows through scalar registers); wave-uniform.
__device__ __forceinline__ float wave_sum_f32(float v) {
  v = row_sum_f32(v);
  return (readlane_f(v, 0) + readlane_f(v, 16)) + (readlane_f(v, 32) + readlane_f(v, 48));
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t u) {
  u = max(u, (uint32_t)dpp_i<kDppXor1>((int)u));
  u = max(u, (uint32_t)dpp_i<kDppXor2>((int)u));
  u = max(u, (uint32_t)dpp_i<kDppHalfMirror>((int)u));
  u = max(u, (uint32_t)dpp_i<kDppRowRor8>((int)u));
  return max(max((uint32_t)readlane_i((int)u, 0), (uint32_t)readlane_i((int)u, 16)),
             max((uint32_t)readlane_i((int)u, 32), (uint32_t)readlane_i((int)u, 48)));
}

// Calls f with a value of the element type that `type` names; `type` has been checked.
template <typename F>
inline void with_type(int32_t type, F f) {
  if (type == TQ_F32) f(float{});
  else if (type == TQ_BF16) f(bf16_t{});
  else f(f16_t{});
}

// Items of `threads` threads each that one launch takes: its threads are counted in 32 bits.
inline int64_t items_per_launch(int threads) { return (int64_t{1} << 31) / threads; }

inline bool known_type(int32_t type) { return type == TQ_F32 || type == TQ_BF16 || type == TQ_F16; }
inline size_t type_bytes(int32_t type) { return type == TQ_F32 ? 4 : 2; }

}  // namespace tq
