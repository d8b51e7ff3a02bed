// Activations held in 8 bits, and the backward pass that reads them.
//
// A row's columns are cut into blocks of 32.  A block holds int8 values q and one code byte c, and
// stands for q 2^(c - 127): the power of two is the smallest with max|x| <= 127 2^(c - 127), but at least
// 2^-126, so the rounding (to nearest, ties to even) is off by at most half of it, max|x| / 127.  Code 255
// stands for a block that held an infinity or NaN: all of it is NaN when read.
// A power of two and seven bits fit bf16 exactly, so a product with a bf16 value is exact in fp32.
#include "rows.h"

namespace janus {

constexpr int kPackBlock = 32;

__device__ __forceinline__ int pack_code(float top) {
  const int bits = __float_as_int(top);
  if (bits >= 0x7F800000) return 255;
  return max((bits >> 23) - 6 + ((bits & 0x7FFFFF) > 0x7E0000), 1);
}
// 2^(c - 127), NaN for 255
__device__ __forceinline__ float code_scale(int c) { return __int_as_float(c == 255 ? 0x7FC00000 : c << 23); }

// Eight columns of a row from column c, zero past d.  `wide`: the row's addresses allow whole runs.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ row, int c, int d, bool wide, float (&v)[8]) {
  if (wide && c + 8 <= d) {
    load_run<T, 8>(row + c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < d ? (float)row[c + j] : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* __restrict__ row, int c, int d, bool wide, const float (&v)[8]) {
  if (wide && c + 8 <= d) {
    store_run<T, 8>(row + c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < d) row[c + j] = (T)v[j];
  }
}
__device__ __forceinline__ void load8q(const int8_t* __restrict__ row, int c, int d, bool wide, float (&v)[8]) {
  if (wide && c + 8 <= d) {
    const uint2 u = *reinterpret_cast<const uint2*>(row + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = (float)(int8_t)(u.x >> (8 * j));
      v[4 + j] = (float)(int8_t)(u.y >> (8 * j));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < d ? (float)row[c + j] : 0.f;
  }
}

// Rows are shared out over `tpr` threads (a power of two, at most 256) of eight columns each; four
// neighbouring threads hold a block.
struct PackShape {
  long long rows;
  int d, tpr;
  bool wide_x, wide_q, wide_g, wide_v;
};

template <typename T>
__global__ __launch_bounds__(256) void pack_rows_kernel(PackShape s, const T* __restrict__ x, long long ldx,
                                                        int8_t* __restrict__ q, long long ldq,
                                                        uint8_t* __restrict__ code, long long ldc) {
  const int per = 256 / s.tpr, t = threadIdx.x % s.tpr;
  const int cols = (s.d + kPackBlock - 1) / kPackBlock * kPackBlock;
  for (long long m = (long long)blockIdx.x * per + threadIdx.x / s.tpr; m < s.rows; m += (long long)gridDim.x * per) {
    for (int c = t * 8; c < cols; c += s.tpr * 8) {
      float v[8], top = 0.f;
      load8(x + m * ldx, c, s.d, s.wide_x, v);
      int bad = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        top = fmaxf(top, fabsf(v[j]));
        bad |= !(fabsf(v[j]) < INFINITY);
      }
      if (bad) top = INFINITY;
      top = fmaxf(top, __shfl_xor(top, 1, 64));
      top = fmaxf(top, __shfl_xor(top, 2, 64));
      const int k = pack_code(top);
      const float inv = __int_as_float(k == 255 ? 0 : (254 - k) << 23);   // 2^(127 - k)
      unsigned w[2] = {0u, 0u};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int n = k == 255 ? 0 : (int)rintf(v[j] * inv);
        w[j >> 2] |= (unsigned)(n & 255) << (8 * (j & 3));
      }
      int8_t* out = q + m * ldq + c;
      if (s.wide_q && c + 8 <= s.d) {
        *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < s.d) out[j] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
      }
      if ((t & 3) == 0) code[m * ldc + c / kPackBlock] = (uint8_t)k;
    }
  }
}

// value = x, or SiLU(x) and out = grad SiLU'(x), of the stored x.
template <typename T, bool kSilu>
__global__ __launch_bounds__(256) void unpack_rows_kernel(PackShape s, const int8_t* __restrict__ q, long long ldq,
                                                          const uint8_t* __restrict__ code, long long ldc,
                                                          const T* grad, long long ldg, T* out, long long ldo, T* value,
                                                          long long ldv) {
  const int per = 256 / s.tpr, t = threadIdx.x % s.tpr;
  for (long long m = (long long)blockIdx.x * per + threadIdx.x / s.tpr; m < s.rows; m += (long long)gridDim.x * per) {
    for (int c = t * 8; c < s.d; c += s.tpr * 8) {
      float v[8];
      load8q(q + m * ldq, c, s.d, s.wide_q, v);
      const float scale = code_scale(code[m * ldc + c / kPackBlock]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= scale;
      if constexpr (kSilu) {
        if (out) {
          float g[8];
          load8(grad + m * ldg, c, s.d, s.wide_g, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] *= silu_d1(v[j]);
          store8(out + m * ldo, c, s.d, s.wide_x, g);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = silu(v[j]);
      }
      if (value) store8(value + m * ldv, c, s.d, s.wide_v, v);
    }
  }
}

// G_g[p, q] = sum over the rows m of group g of X[m, p] B[m, q]: 64 x 64 tiles, 16 rows at a time.
template <typename T>
__global__ __launch_bounds__(256) void packed_wgrad_kernel(const int8_t* __restrict__ q, long long ldq,
                                                           const uint8_t* __restrict__ code, long long ldc,
                                                           const T* __restrict__ b, long long ldb, int P, int Q,
                                                           const int* __restrict__ off, long long rows,
                                                           float* __restrict__ G) {
  __shared__ float A[16][64], B[16][64];
  const int p0 = blockIdx.x * 64, q0 = blockIdx.y * 64, g = blockIdx.z;
  const long long m0 = max(off[g], 0), m1 = min((long long)off[g + 1], rows);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  float acc[4][4] = {};
  for (long long m = m0; m < m1; m += 16) {
    for (int e = threadIdx.x; e < 1024; e += 256) {
      const int r = e >> 6, c = e & 63;
      const long long row = m + r;
      A[r][c] = row < m1 && p0 + c < P
                    ? (float)q[row * ldq + p0 + c] * code_scale(code[row * ldc + (p0 + c) / kPackBlock]) : 0.f;
      B[r][c] = row < m1 && q0 + c < Q ? (float)b[row * ldb + q0 + c] : 0.f;
    }
    __syncthreads();
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += A[r][ty * 4 + i] * B[r][tx * 4 + j];
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + ty * 4 + i, c = q0 + tx * 4 + j;
      if (p < P && c < Q) G[((long long)g * P + p) * Q + c] = acc[i][j];
    }
}

static PackShape pack_shape(long long rows, int d) {
  int tpr = 4;
  while (tpr < 256 && tpr * 8 < d) tpr <<= 1;
  return PackShape{rows, d, tpr, false, false, false, false};
}
static unsigned pack_grid(const PackShape& s) {
  const long long need = (s.rows + 256 / s.tpr - 1) / (256 / s.tpr);
  return (unsigned)(need < 8192 ? need : 8192);
}

static int check_packed(const void* q, int64_t ldq, const void* code, int64_t ldc, int64_t rows, int32_t d, int type) {
  if (rows < 0 || rows > INT_MAX || d < 1 || !type_known(type)) return JANUS_EINVAL;
  if (rows > 0 && (!q || !code || ldq < d || ldc < (d + kPackBlock - 1) / kPackBlock)) return JANUS_EINVAL;
  return JANUS_OK;
}

}  // namespace janus

using namespace janus;

extern "C" int janus_pack_rows(const void* x, int64_t ldx, int32_t type, int64_t rows, int32_t d, int8_t* q,
                               int64_t ldq, uint8_t* code, int64_t ldc, void* stream) {
  int rc = check_packed(q, ldq, code, ldc, rows, d, type);
  if (rc) return rc;
  if (rows > 0 && (!x || ldx < d)) return JANUS_EINVAL;
  if (rows == 0) return JANUS_OK;
  PackShape s = pack_shape(rows, d);
  s.wide_x = rows_aligned(x, ldx, type_bytes(type));
  s.wide_q = rows_aligned(q, ldq, 1, 8);
  with_type(type, [&](auto zero) {
    using T = decltype(zero);
    hipLaunchKernelGGL(pack_rows_kernel<T>, dim3(pack_grid(s)), dim3(256), 0, static_cast<hipStream_t>(stream), s,
                       static_cast<const T*>(x), ldx, q, ldq, code, ldc);
  });
  return launched();
}

extern "C" int janus_unpack_rows(const int8_t* q, int64_t ldq, const uint8_t* code, int64_t ldc, int64_t rows,
                                 int32_t d, int32_t type, int32_t act, const void* grad, int64_t ldg, void* out,
                                 int64_t ldo, void* value, int64_t ldv, void* stream) {
  int rc = check_packed(q, ldq, code, ldc, rows, d, type);
  if (rc) return rc;
  if (act != JANUS_ACT_NONE && act != JANUS_ACT_SILU) return JANUS_EINVAL;
  if (rows == 0) return JANUS_OK;
  if ((!grad) != (!out) || (act == JANUS_ACT_NONE && grad) || (!out && !value) || (grad && (ldg < d || ldo < d)) ||
      (value && ldv < d))
    return JANUS_EINVAL;
  const int e = type_bytes(type);
  PackShape s = pack_shape(rows, d);
  s.wide_q = rows_aligned(q, ldq, 1, 8);
  s.wide_g = rows_aligned(grad, ldg, e);
  s.wide_x = rows_aligned(out, ldo, e);
  s.wide_v = rows_aligned(value, ldv, e);
  with_type(type, [&](auto zero) {
    using T = decltype(zero);
    auto go = [&](auto silu) {
      hipLaunchKernelGGL((unpack_rows_kernel<T, decltype(silu)::value>), dim3(pack_grid(s)), dim3(256), 0,
                         static_cast<hipStream_t>(stream), s, q, ldq, code, ldc, static_cast<const T*>(grad), ldg,
                         static_cast<T*>(out), ldo, static_cast<T*>(value), ldv);
    };
    if (act == JANUS_ACT_SILU) go(std::true_type{});
    else go(std::false_type{});
  });
  return launched();
}

static int check_packed_wgrad(int64_t rows, int32_t n_groups, int32_t P, int32_t Q, int32_t type) {
  if (rows < 0 || rows > INT_MAX || n_groups < 1 || n_groups > 1024 || P < 1 || Q < 1 || !type_known(type))
    return JANUS_EINVAL;
  return JANUS_OK;
}

extern "C" int64_t janus_packed_wgrad_workspace(int64_t rows, int32_t n_groups, int32_t P, int32_t Q, int32_t type) {
  int rc = check_packed_wgrad(rows, n_groups, P, Q, type);
  if (rc) return rc;
  return 16;
}

extern "C" int janus_packed_wgrad(const int8_t* q, int64_t ldq, const uint8_t* code, int64_t ldc, const void* B,
                                  int64_t ldb, int32_t type, float* G, const int32_t* row_off, int32_t n_groups,
                                  int64_t rows, int32_t P, int32_t Q, void* work, int64_t work_bytes, void* stream) {
  int rc = check_packed_wgrad(rows, n_groups, P, Q, type);
  if (!rc) rc = check_packed(q, ldq, code, ldc, rows, P, type);
  if (rc) return rc;
  if (!G || !row_off || (rows > 0 && (!B || ldb < Q)) || !work || !rows_aligned(work, 0, 1) ||
      work_bytes < janus_packed_wgrad_workspace(rows, n_groups, P, Q, type))
    return JANUS_EINVAL;
  with_type(type, [&](auto zero) {
    using T = decltype(zero);
    hipLaunchKernelGGL(packed_wgrad_kernel<T>, dim3(cdiv(P, 64), cdiv(Q, 64), n_groups), dim3(256), 0,
                       static_cast<hipStream_t>(stream), q, ldq, code, ldc, static_cast<const T*>(B), ldb, P, Q,
                       row_off, rows, G);
  });
  return launched();
}
