// Row-wise access to fp32, bf16 and fp16 arrays, shared by the operators around an expert block.
#pragma once

#include <climits>

#include "common.h"

namespace janus {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// N consecutive values as fp32, in pieces of at most 16 bytes, at any multiple of their size (the memory
// takes runs at any address; ones that cross a line cost a second access).  Stores round to nearest, ties to
// even.
template <typename T, int N>
__device__ __forceinline__ void load_run(const T* __restrict__ p, float* v) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  if constexpr (N == 1) {
    v[0] = (float)p[0];
  } else if constexpr (sizeof(T) * N <= 16) {
    const vec u = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = (float)u[j];
  } else {
    load_run<T, N / 2>(p, v);
    load_run<T, N / 2>(p + N / 2, v + N / 2);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_run(T* __restrict__ p, const float* v) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  if constexpr (N == 1) {
    p[0] = (T)v[0];
  } else if constexpr (sizeof(T) * N <= 16) {
    vec u;
#pragma unroll
    for (int j = 0; j < N; ++j) u[j] = (T)v[j];
    *reinterpret_cast<vec*>(p) = u;
  } else {
    store_run<T, N / 2>(p, v);
    store_run<T, N / 2>(p + N / 2, v + N / 2);
  }
}

// Sum over the 16 lanes of a DPP row, in every lane of it.
__device__ __forceinline__ float row16_sum(float v) {
  v = dpp_step<0xB1>(v);    // quad_perm(1, 0, 3, 2)
  v = dpp_step<0x4E>(v);    // quad_perm(2, 3, 0, 1)
  v = dpp_step<0x141>(v);   // row_half_mirror
  return dpp_step<0x140>(v);   // row_mirror
}

// s = 1 / (1 + exp(-a)) and c = 1 - s, the larger of them to 2.2 units of 2^-24 of itself and the smaller to 5.6, at any
// a, down into fp32's subnormal range.  exp(-|a|) = 2^n 2^f, where f is formed from the whole product |a| log2(e) in two
// fused steps (the plain product would be rounded to |a| 2^-24, and so would the result); the reciprocal of 1 + e takes
// one step of Newton's with what the sum lost; and the smaller one is e / (1 + e), without a difference.  (With the
// hardware's reciprocal of the rounded sum alone, SiLU of a value next to the middle of two bf16 went to the wrong one.)
struct Sigmoid {
  float s, c;
};
__device__ __forceinline__ Sigmoid sigmoid(float a) {
  constexpr float kLog2e = 1.44269502f, kRest = 1.92596299e-8f;     // log2(e) = their sum to 2^-50
  const float x = __builtin_amdgcn_fmed3f(fabsf(a), 0.f, 150.0f);   // exp(-150) is zero in fp32
  const float n = rintf(-kLog2e * x);
  const float f = fmaf(-kRest, x, fmaf(-kLog2e, x, -n));
  const float e = ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
  const float t = 1.0f + e, lost = e - (t - 1.0f), r = __builtin_amdgcn_rcpf(t);
  const float large = fmaf(r, fmaf(-lost, r, fmaf(-t, r, 1.0f)), r), small = e * large;
  return a < 0.f ? Sigmoid{small, large} : Sigmoid{large, small};
}

// An fp32 value's first eight bits, which bf16 holds, and two values' as a pair, a first.
__device__ __forceinline__ float high_part(float a) { return __uint_as_float(__float_as_uint(a) & 0xFFFF0000u); }
__device__ __forceinline__ unsigned pack_high(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

inline bool type_known(int t) { return t == JANUS_F32 || t == JANUS_BF16 || t == JANUS_F16; }
inline int type_bytes(int t) { return t == JANUS_F32 ? 4 : 2; }

// Runs f with a value of the element type that `type` names.
template <typename F>
inline void with_type(int type, F f) {
  if (type == JANUS_F32) f(float{});
  else if (type == JANUS_BF16) f(__bf16{});
  else f(_Float16{});
}

// Whether every row of `ld` elements starts on a multiple of `align` bytes (null arrays do).
inline bool rows_aligned(const void* p, int64_t ld, int elem, int align = 16) {
  return !p || ((reinterpret_cast<uintptr_t>(p) % align) == 0 && (ld * elem) % align == 0);
}

// The last launch's error, as a return code.
inline int launched() {
  JANUS_HIP_TRY(hipGetLastError());
  return JANUS_OK;
}

}  // namespace janus
