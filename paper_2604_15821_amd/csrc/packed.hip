// Activations held in 8 bits, and the backward pass that reads them.
//
// A row's columns are cut into blocks of 32.  A block holds int8 values q and one code byte c, and
// stands for q 2^(c - 127): the power of two is the smallest with max|x| <= 127 2^(c - 127), but at least
// 2^-126, so the rounding (to nearest, ties to even) is off by at most half of it: max|x| / 127, or 2^-127 where
// that is more.  Code 255 stands for a block that held an infinity or NaN: all of it is NaN when read.
// A power of two and seven bits fit bf16 exactly, so a product with a bf16 value is exact in fp32.
// Packing and unpacking are bound by memory: 150 001 x 2048 fp32 to 8 bits 317 us (4.9 TB/s); SiLU and the gradient
// through it in bf16 385 us (5.6 TB/s).
#include <algorithm>
#include <type_traits>

#include "chunk_cut.h"
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

// Eight columns of a row from column c, and their values later, so that several arrays can be asked for before the
// first is waited for.  Columns past d read the last one; WHOLE: d is a multiple of eight, there are none.
template <typename T, bool WHOLE>
struct Raw8 {
  typedef unsigned words __attribute__((ext_vector_type(sizeof(T) < 2 ? 2 : 4), aligned(sizeof(T))));
  static constexpr int kWords = sizeof(T) * 8 / sizeof(words);
  words w[kWords];
  __device__ __forceinline__ void load(const T* __restrict__ row, int c, int d) {
    if (WHOLE || c + 8 <= d) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const words*>(row + c)[i];
    } else {
      T v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = row[min(c + j, d - 1)];
      __builtin_memcpy(w, v, sizeof v);
    }
  }
  __device__ __forceinline__ void values(float (&o)[8]) const {
    if constexpr (sizeof(T) == 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = (float)((int)(w[0][j / 4] << (24 - 8 * (j % 4))) >> 24);   // one instruction each
    } else {
      T v[8];
      __builtin_memcpy(v, w, sizeof v);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = (float)v[j];
    }
  }
};
template <bool WHOLE, typename T>
__device__ __forceinline__ void store8(T* __restrict__ row, int c, int d, const float (&v)[8]) {
  if (WHOLE || c + 8 <= d) {
    store_run<T, 8>(row + c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < d) row[c + j] = (T)v[j];
  }
}
typedef unsigned bytes8 __attribute__((ext_vector_type(2), aligned(1)));

// Rows are shared out over `tpr` threads (a power of two, at most 256) of eight columns each; four
// neighbouring threads hold a block.
struct PackShape {
  long long rows;
  int d, tpr;
};

template <typename T>
__global__ __launch_bounds__(256) void pack_rows_kernel(PackShape s, const T* __restrict__ x, long long ldx,
                                                        int8_t* __restrict__ q, long long ldq,
                                                        uint8_t* __restrict__ code, long long ldc) {
  const int per = 256 / s.tpr, t = threadIdx.x % s.tpr;
  const int cols = (s.d + kPackBlock - 1) / kPackBlock * kPackBlock;
  for (long long m = (long long)blockIdx.x * per + threadIdx.x / s.tpr; m < s.rows; m += (long long)gridDim.x * per) {
    for (int c = t * 8; c < cols; c += s.tpr * 8) {
      Raw8<T, false> raw;
      raw.load(x + m * ldx, c, s.d);
      float v[8], top = 0.f;
      raw.values(v);
      if (c + 8 > s.d) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < s.d ? v[j] : 0.f;
      }
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
      if (c + 8 <= s.d) {
        *reinterpret_cast<bytes8*>(out) = bytes8{w[0], w[1]};
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < s.d) out[j] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
      }
      if ((t & 3) == 0) code[m * ldc + c / kPackBlock] = (uint8_t)k;
    }
  }
}

// The largest finite values of a type are rounded up to 64 steps of the largest code that they get, which is beyond the
// type: such a value reads as the largest finite one, which is nearer to them than the half step that rounding may cost.
template <typename T>
struct Top {
  static constexpr int kCode = 249;
  static constexpr float kOver = INFINITY, kMost = std::is_same_v<T, float> ? 0x1.fffffep127f : 0x1.fep127f;
};
template <>
struct Top<_Float16> {
  static constexpr int kCode = 137;
  static constexpr float kOver = 65536.0f, kMost = 65504.0f;
};

// value = x, or SiLU(x) and out = grad SiLU'(x), of the stored x.  Widths that are multiples of eight have no code for a
// row's end, so that all loads of a thread are in flight together.
template <typename T, bool kSilu, bool WHOLE>
__global__ __launch_bounds__(256) void unpack_rows_kernel(PackShape s, const int8_t* __restrict__ q, long long ldq,
                                                          const uint8_t* __restrict__ code, long long ldc,
                                                          const T* grad, long long ldg, T* out, long long ldo, T* value,
                                                          long long ldv) {
  const int per = 256 / s.tpr, t = threadIdx.x % s.tpr;
  for (long long m = (long long)blockIdx.x * per + threadIdx.x / s.tpr; m < s.rows; m += (long long)gridDim.x * per) {
    for (int c = t * 8; c < s.d; c += s.tpr * 8) {
      Raw8<int8_t, WHOLE> raw;
      Raw8<T, WHOLE> raw_g;
      raw.load(q + m * ldq, c, s.d);
      const int power = code[m * ldc + c / kPackBlock];
      if (kSilu && out) raw_g.load(grad + m * ldg, c, s.d);
      float v[8];
      raw.values(v);
      const float scale = code_scale(power);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= scale;
      if (power == Top<T>::kCode) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (fabsf(v[j]) == Top<T>::kOver) v[j] = copysignf(Top<T>::kMost, v[j]);
      }
      if constexpr (kSilu) {
        Sigmoid f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = sigmoid(v[j]);
        if (out) {
          float g[8];
          raw_g.values(g);
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] *= f[j].s * fmaf(v[j], f[j].c, 1.0f);
          store8<WHOLE>(out + m * ldo, c, s.d, g);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= f[j].s;
      }
      if (value) store8<WHOLE>(value + m * ldv, c, s.d, v);
    }
  }
}

// ------------------------------------------------------------------ the weight gradient
// G_g[p, c] = sum over the rows m of group g of X[m, p] B[m, c] on the bf16 matrix instructions
// (v_mfma_f32_32x32x16_bf16).  X is exact in bf16; B is taken as it is (bf16), as two bf16 terms (fp16: eight and three of its
// eleven bits) or three (fp32: eight bits each, by truncation), which sum to it exactly, so every product is exact.
//
// A workgroup of four waves (2 x 2) owns 128 rows p and COLS columns of a group's chunk of rows m (COLS = 256
// with one term, else 128).  Both operands arrive with p and c, not m, along memory rows.  They are put into LDS as they
// come, [32 m][p or c] in bf16, and read with the transposing ds_read_b64_tr_b16: 16 lanes give the addresses of
// four rows of 16 values and receive four m of one column each, two reads an operand of the 32 x 32 x 16
// instruction.  The 32-byte units of a row are stored at unit ^ 2 (m % 4), so that the four rows and two units that 32
// lanes read fall on different banks.  Stages of 32 rows alternate between two LDS buffers, and a stage's registers are
// loaded two stages before it is multiplied.
//
// Rows are cut into chunks, a group's longest first and given to the dies in turn, so that the tiles of a chunk
// share its die's L2 and none runs long at the end.  A group's only chunk writes the gradient itself; else
// each writes a partial and a second kernel adds them in order.
// Measured, 150 001 rows in 64 ragged groups, 512 x 2048, a whole call: bf16 0.39 ms (800 TFLOP/s; the product 0.36 at the
// clock of an idle card, 0.42 once calls follow each other, its matrix units busy 48 % of the time in which a CU has
// work), fp16 0.71 ms, fp32 1.06 ms (297 TFLOP/s, 890 of bf16 products).
struct PackedChunk {
  int group, r0, r1, alone;
};

constexpr int kWgP = 128, kWgRows = 32;

template <typename T>
struct Terms;
template <>
struct Terms<__bf16> {
  static constexpr int kPlanes = 1, kCols = 256;
};
template <>
struct Terms<_Float16> {
  static constexpr int kPlanes = 2, kCols = 128;
};
template <>
struct Terms<float> {
  static constexpr int kPlanes = 3, kCols = 128;
};

// Where the rows of both operands start on four bytes (WORDS: always for fp32), a chunk's rows are a buffer: words
// behind the one that holds its last value are zero, so its ragged end needs no code.  Past a row's end a run goes on
// into the next one; those columns are not stored.  Other rows are read by runs at any address in the same way, but
// at the very end of the array value by value, and rows behind the chunk are read as its last one and cleared
// before they are used.
typedef __amdgpu_buffer_rsrc_t buffer;
__device__ __forceinline__ buffer rows_buffer(const void* p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// What plane q leaves of a value.  Not inf - inf: an infinity leaves zero, in fp16, whose second plane is the last, itself (by
// one instruction in place of two: 2.5 % of the call against 5; fp32, 3 %).
template <typename T>
__device__ __forceinline__ float rest(float a, int q) {
  const float high = high_part(a);
  if constexpr (std::is_same_v<T, _Float16>) return a - __builtin_amdgcn_fmed3f(high, -65504.0f, 65504.0f);
  return q == 0 && a == high ? 0.f : a - high;
}

// Eight values of a row of B, and their planes.
template <typename T>
struct Octet {
  T v[8];
  __device__ __forceinline__ void load(buffer b, unsigned at) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
    for (int j = 0; j < 8; j += V) {
      const vec u = __builtin_bit_cast(vec, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(b, at + j * sizeof(T), 0, 0));
#pragma unroll
      for (int i = 0; i < V; ++i) v[j + i] = u[i];
    }
  }
  __device__ __forceinline__ void load(const T* __restrict__ b, long long at, long long end) {
    if (at + 8 <= end) {
      __builtin_memcpy(v, b + at, sizeof v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = b[min(at + j, end - 1)];
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (T)0.f;
  }
  __device__ __forceinline__ void planes(uint4 (&o)[Terms<T>::kPlanes]) const {
    if constexpr (Terms<T>::kPlanes == 1) {
      __builtin_memcpy(&o[0], v, 16);
    } else {
      unsigned w[Terms<T>::kPlanes][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a = (float)v[2 * i], b = (float)v[2 * i + 1];
#pragma unroll
        for (int q = 0; q < Terms<T>::kPlanes; ++q) {
          w[q][i] = pack_high(a, b);
          a = rest<T>(a, q);
          b = rest<T>(b, q);
        }
      }
#pragma unroll
      for (int q = 0; q < Terms<T>::kPlanes; ++q) o[q] = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
    }
  }
};

// Sixteen packed values of a row and their code, as bf16.  (Behind the end both are zero: a scale of zero.)
struct Sixteen {
  u32x4 q;
  int code;
  __device__ __forceinline__ void load(buffer b, unsigned at, buffer codes, unsigned at_code) {
    q = (u32x4)__builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0);
    code = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(codes, at_code, 0, 0);
  }
  __device__ __forceinline__ void load(const int8_t* __restrict__ x, long long at, long long end, int c) {
    if (at + 16 <= end) {
      __builtin_memcpy(&q, x + at, 16);
    } else {
      int8_t v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = x[min(at + j, end - 1)];
      __builtin_memcpy(&q, v, 16);
    }
    code = c;
  }
  // the half `first` of them, then the other
  __device__ __forceinline__ void values(int first, uint4 (&o)[2]) const {
    const float s = code_scale(code);
    const unsigned in[4] = {first ? q.z : q.x, first ? q.w : q.y, first ? q.x : q.z, first ? q.y : q.w};
    unsigned w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned u = in[i >> 1] >> (16 * (i & 1));
      w[i] = pack_high((float)(int8_t)u * s, (float)(int8_t)(u >> 8) * s);
    }
    o[0] = make_uint4(w[0], w[1], w[2], w[3]);
    o[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ bf16x8 read_columns(const char* lo, const char* hi) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lo);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)hi);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Where a row's 32-byte unit lies.
__device__ __forceinline__ int place(int unit, int m) { return unit ^ (2 * (m & 3)); }

// Bytes of `rows` rows up to the last one's last value, in units of what one read takes.
__device__ __forceinline__ unsigned last_byte(int rows, long long ld, int width, int size, unsigned unit) {
  const unsigned n = rows ? (unsigned)(((rows - 1) * ld + width) * size) : 0u;
  return (n + unit - 1) & ~(unit - 1);
}

template <typename T, bool WORDS>
__global__ __launch_bounds__(256, 2) void packed_wgrad_kernel(const int8_t* __restrict__ q, long long ldq,
                                                              const uint8_t* __restrict__ code, long long ldc,
                                                              const T* __restrict__ b, long long ldb, long long n_rows,
                                                              int P, int Q, const PackedChunk* __restrict__ chunks,
                                                              const int* __restrict__ n_chunks, int tiles_p,
                                                              int tiles_q, float* __restrict__ partial,
                                                              float* __restrict__ G) {
  constexpr int NP = Terms<T>::kPlanes, COLS = Terms<T>::kCols;
  constexpr int kPass = COLS / 64, kFrag = COLS / 64;   // octets of B per thread and stage; 32-column blocks per wave
  constexpr int kRowA = kWgP * 2, kRowB = COLS * 2, kBytesA = kWgRows * kRowA, kBytesB = kWgRows * kRowB;
  constexpr int kStage = kBytesA + NP * kBytesB;
  __shared__ __align__(16) char lds[2 * kStage];
  // block -> die block % 8 -> chunk, tile: the tiles of a chunk are consecutive blocks of one die; fewer chunks than
  // dies are cut into eight equal runs of tiles
  const int tiles = tiles_p * tiles_q, slot = blockIdx.x >> 3, die = blockIdx.x & 7, all = *n_chunks;
  int at = slot / tiles * 8 + die, tile = slot % tiles;
  if (all < 8) {
    const int per = (all * tiles + 7) / 8, i = die * per + slot;
    at = slot < per ? i / tiles : all;
    tile = i % tiles;
  }
  if (at >= all) return;
  const PackedChunk ch = chunks[at];
  const int p0 = tile / tiles_q * kWgP, c0 = tile % tiles_q * COLS;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;

  // staging: thread t holds 16 values of X's row t / 8 and, per pass, 8 values of a row of B
  const int rows = ch.r1 - ch.r0;
  const buffer bufA = rows_buffer(q + ch.r0 * ldq, last_byte(rows, ldq, P, 1, 4));
  const buffer bufC = rows_buffer(code + ch.r0 * ldc, last_byte(rows, ldc, (P + kPackBlock - 1) / kPackBlock, 1, 1));
  const buffer bufB = rows_buffer(b + ch.r0 * ldb, last_byte(rows, ldb, Q, sizeof(T), 4));
  const int ma = t >> 3, ua = t & 7, half = ma & 1;
  const int wa = ma * kRowA + (place(ua, ma) << 5);
  constexpr int kPerRow = COLS / 8, kRowsPass = 256 / kPerRow;
  const int mb = t / kPerRow, ob = t % kPerRow;
  unsigned atA = ma * (unsigned)ldq + p0 + 16 * ua, atC = ma * (unsigned)ldc + (p0 + 16 * ua) / kPackBlock;
  unsigned atB = (mb * (unsigned)ldb + c0 + 8 * ob) * (unsigned)sizeof(T);
  const unsigned stepB = kWgRows * (unsigned)ldb * (unsigned)sizeof(T), passB = stepB / (32 / kRowsPass);
  struct Regs {
    Sixteen a;
    Octet<T> b[kPass];
  };
  int ahead = ch.r0;   // the next stage's first row
  auto load = [&](Regs& r) {
    if constexpr (WORDS) {
      r.a.load(bufA, atA, bufC, atC);
#pragma unroll
      for (int i = 0; i < kPass; ++i) r.b[i].load(bufB, atB + i * passB);
      atA += kWgRows * (unsigned)ldq;
      atC += kWgRows * (unsigned)ldc;
      atB += stepB;
    } else {
      const long long ra = min(ahead + ma, ch.r1 - 1);
      const int cA = p0 + 16 * ua;
      r.a.load(q, ra * ldq + cA, (n_rows - 1) * ldq + P, code[ra * ldc + min(cA, P - 1) / kPackBlock]);
#pragma unroll
      for (int i = 0; i < kPass; ++i)
        r.b[i].load(b, min(ahead + mb + i * kRowsPass, ch.r1 - 1) * ldb + c0 + 8 * ob, (n_rows - 1) * ldb + Q);
      ahead += kWgRows;
    }
  };
  int staged = ch.r0;
  auto stage = [&](Regs& r, char* to) {
    if constexpr (!WORDS) {
      if (staged + kWgRows > ch.r1) {
        if (staged + ma >= ch.r1) r.a.code = 0;   // a scale of zero
#pragma unroll
        for (int i = 0; i < kPass; ++i)
          if (staged + mb + i * kRowsPass >= ch.r1) r.b[i].clear();
      }
      staged += kWgRows;
    }
    uint4 o[2];   // odd rows write their second half first: two rows then fill all banks
    r.a.values(half, o);
    *reinterpret_cast<uint4*>(to + wa + 16 * half) = o[0];
    *reinterpret_cast<uint4*>(to + wa + 16 - 16 * half) = o[1];
#pragma unroll
    for (int i = 0; i < kPass; ++i) {
      const int m = mb + i * kRowsPass;
      uint4 w[NP];
      r.b[i].planes(w);
      char* at_b = to + kBytesA + m * kRowB + (place(ob >> 1, m) << 5) + ((ob & 1) << 4);
#pragma unroll
      for (int n = 0; n < NP; ++n) *reinterpret_cast<uint4*>(at_b + n * kBytesB) = w[n];
    }
  };

  // operand addresses: 16-lane group g reads columns 16 (g % 2) .. + 15 and rows 8 (g / 2) + 4 h + r
  const int g = lane >> 4, r = (lane >> 2) & 3, sub = (lane & 3) * 8;
  int fa[2][2], fb[kFrag][2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int m = 8 * (g >> 1) + 4 * h + r;
#pragma unroll
    for (int f = 0; f < 2; ++f) fa[f][h] = m * kRowA + (place((wave >> 1) * 4 + 2 * f + (g & 1), m) << 5) + sub;
#pragma unroll
    for (int f = 0; f < kFrag; ++f)
      fb[f][h] = kBytesA + m * kRowB + (place((wave & 1) * (COLS / 32) + 2 * f + (g & 1), m) << 5) + sub;
  }
  f32x16 acc[2][kFrag];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < kFrag; ++j) acc[i][j] = f32x16{};
  auto multiply = [&](const char* from) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      bf16x8 x[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) x[f] = read_columns(from + fa[f][0] + kb * 16 * kRowA, from + fa[f][1] + kb * 16 * kRowA);
#pragma unroll
      for (int n = NP - 1; n >= 0; --n)   // small terms first
#pragma unroll
        for (int f = 0; f < kFrag; ++f) {
          const int o = n * kBytesB + kb * 16 * kRowB;
          const bf16x8 y = read_columns(from + fb[f][0] + o, from + fb[f][1] + o);
#pragma unroll
          for (int i = 0; i < 2; ++i) acc[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y, acc[i][f], 0, 0, 0);
        }
    }
  };

  Regs r0, r1;
  const int steps = (rows + kWgRows - 1) / kWgRows;
  // multiplies the stage in `from` while `next` holds the one after it and `after` is loaded with the next but one
  auto step = [&](const char* from, char* to, Regs& next, Regs& after) {
    load(after);
    multiply(from);
    stage(next, to);
    __syncthreads();
  };
  if (steps > 0) {
    load(r0);
    load(r1);
    stage(r0, lds);
    __syncthreads();
  }
  for (int s = 0; s < steps; s += 2) {
    step(lds, lds + kStage, r1, r0);
    if (s + 1 < steps) step(lds + kStage, lds, r0, r1);
  }

  float* out = ch.alone ? G + (long long)ch.group * P * Q : partial + (long long)at * P * Q;
  // row 8 (k / 4) + 4 (lane / 32) + k % 4 of a block, column lane % 32
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int f = 0; f < kFrag; ++f) {
      const int c = c0 + (wave & 1) * (COLS / 2) + 32 * f + (lane & 31);
      const int p = p0 + (wave >> 1) * 64 + 32 * i + 4 * (lane >> 5);
      if (c < Q) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const int row = p + 8 * (k >> 2) + (k & 3);
          if (row < P) out[(long long)row * Q + c] = acc[i][f][k];
        }
      }
    }
}

// Chunks of at most kc rows, equally long within a group, groups with the longest chunks first.  first[g]: a
// group's first chunk, count[g]: how many.  Offsets are held to [0, rows], so chunks always lie inside.
__global__ __launch_bounds__(1024) void packed_chunks_kernel(const int* __restrict__ off, int groups, long long rows,
                                                             int kc, PackedChunk* __restrict__ chunks, int most,
                                                             int* __restrict__ n_chunks, int* __restrict__ first,
                                                             int* __restrict__ count) {
  __shared__ int2 size_n[1024];   // rows per chunk, chunks
  const int g = threadIdx.x;
  int a = 0, size = 0;
  if (g < groups) {
    a = min(max(off[g], 0), (int)rows);
    size = max(min(max(off[g + 1], 0), (int)rows) - a, 0);
  }
  const ChunkCut cut = chunk_cut(size, kc, kWgRows);
  const int each = cut.each, n = g < groups ? cut.count : 0;
  size_n[g] = make_int2(each, n);
  __syncthreads();
  int at = 0, all = 0;
  if (g < groups) {
#pragma unroll 8
    for (int o = 0; o < groups; ++o) {
      const int2 v = size_n[o];
      at += v.x > each || (v.x == each && o < g) ? v.y : 0;
      all += v.y;
    }
  }
  if (g < groups) {
    first[g] = at;
    const int held = min(n, max(most - at, 0));   // fewer only where offsets overlap
    count[g] = held;
    for (int i = 0; i < held; ++i)
      chunks[at + i] = PackedChunk{g, a + i * each, a + (int)min((i + 1ll) * each, (long long)size), n == 1};
  }
  if (g == 0) *n_chunks = min(all, most);
}

// The sum of partials [k0, k1) at p, in order, FLIGHT in flight.
template <int FLIGHT, typename vec>
__device__ __forceinline__ vec sum_partials(const float* __restrict__ p, long long PQ, int k0, int k1) {
  vec v = {};
  for (int k = k0; k < k1; k += FLIGHT) {
    vec u[FLIGHT];
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) u[j] = *reinterpret_cast<const vec*>(p + min(k + j, k1 - 1) * PQ);
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j)
      if (k + j < k1) v += u[j];
  }
  return v;
}

// Adds the partials of groups with several chunks.  A thread owns V neighbouring values; from eight chunks on, the
// workgroup's four waves take a quarter of the chunks each for the same values, added in order.
template <int V>
__global__ __launch_bounds__(256) void packed_reduce_kernel(const float* __restrict__ partial,
                                                            const int* __restrict__ first,
                                                            const int* __restrict__ count, long long PQ,
                                                            float* __restrict__ G) {
  typedef float vec __attribute__((ext_vector_type(V)));
  __shared__ vec red[3][64];
  const int g = blockIdx.y, n = count[g];
  if (n < 2) return;
  const float* p = partial + first[g] * PQ;
  float* out = G + g * PQ;
  if (n < 8) {
    for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * V; i < PQ; i += (long long)gridDim.x * 256 * V)
      *reinterpret_cast<vec*>(out + i) = sum_partials<4, vec>(p + i, PQ, 0, n);
    return;
  }
  const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, each = (n + 3) / 4;
  for (long long i0 = (long long)blockIdx.x * (64 * V); i0 < PQ; i0 += (long long)gridDim.x * (64 * V)) {
    const long long i = i0 + lane * V;
    vec v = {};
    if (i < PQ) v = sum_partials<8, vec>(p + i, PQ, slice * each, min((slice + 1) * each, n));
    if (slice) red[slice - 1][lane] = v;
    __syncthreads();
    if (slice == 0 && i < PQ) {
#pragma unroll
      for (int q = 0; q < 3; ++q) v += red[q][lane];
      *reinterpret_cast<vec*>(out + i) = v;
    }
    __syncthreads();
  }
}

struct WgradPlan {
  int tiles_p, tiles_q, kc, most;
  int64_t chunks, first, count, partial, total;   // offsets in bytes
};
// The chunk length.  Where at least half of the 512 resident workgroups are left after one more chunk per group (whose
// last chunks are ragged), chunks that fill them in one round; else half of what each would get of all rows, so
// that the last ones end together.  (One group of 65 536 rows, 512 x 2048, bf16: 227 us by the second rule, 185 by the first.)
// Not below 512 rows, where partials cost more than they save (100 000 rows, 4 groups, 128 x 128, bf16: 29 us at 512,
// 36 at 256), nor above 16 224, so that the bytes of a chunk and of the 128 rows that reads may run ahead stay within the
// 32-bit offsets of a buffer for rows of up to 256 KB.
constexpr int kMostChunkRows = 16224, kReadAhead = 4 * kWgRows, kWgSlots = 512;
static_assert((kMostChunkRows + kReadAhead) * 262144ll <= UINT_MAX && kMostChunkRows % kWgRows == 0);
static WgradPlan wgrad_plan(int64_t rows, int groups, int P, int Q, int type) {
  WgradPlan w;
  w.tiles_p = (int)cdiv(P, kWgP);
  w.tiles_q = (int)cdiv(Q, type == JANUS_BF16 ? Terms<__bf16>::kCols : Terms<float>::kCols);
  const double work = (double)rows * w.tiles_p * w.tiles_q;   // rows of all tiles
  const double room = kWgSlots - (double)(groups - 1) * w.tiles_p * w.tiles_q;
  const double share = room >= kWgSlots / 2 ? work / room : work / (2 * kWgSlots);
  const double kc = share < 512 ? 512 : share > kMostChunkRows ? kMostChunkRows : share;
  w.kc = (int)((kc + kWgRows - 1) / kWgRows) * kWgRows;
  w.most = (int)(groups + rows / w.kc);
  w.chunks = 16;
  w.first = w.chunks + (int64_t)w.most * sizeof(PackedChunk);
  w.count = w.first + 4 * (int64_t)groups;
  w.partial = (w.count + 4 * (int64_t)groups + 15) / 16 * 16;
  w.total = w.partial + (int64_t)(4ull * w.most * P * Q);   // sizes beyond a launch, which overflow it, are refused
  return w;
}
// Workgroups of the product: every die's share of the chunks, rounded up.
static double wgrad_blocks(const WgradPlan& w) { return (w.most + 7) / 8 * 8.0 * w.tiles_p * w.tiles_q; }

static PackShape pack_shape(long long rows, int d) {
  int tpr = 4;
  while (tpr < 256 && tpr * 8 < d) tpr <<= 1;
  return PackShape{rows, d, tpr};
}
static unsigned pack_grid(const PackShape& s) {
  const long long need = (s.rows + 256 / s.tpr - 1) / (256 / s.tpr);
  return (unsigned)(need < 8192 ? need : 8192);
}
// Unpacking: workgroups that take several rows each spare a short call the set-up per row (200 000 x 200 bf16, SiLU and
// gradient, 52 us with 8192 workgroups, 60 with as many as rows allow); in a long call they drift apart over the memory
// (150 001 x 2048: 439 us with 8192, 401 with 32 768, 386 with 65 536).
static unsigned unpack_grid(const PackShape& s) {
  const long long need = (s.rows + 256 / s.tpr - 1) / (256 / s.tpr), most = need < 32768 ? 8192 : 65536;
  return (unsigned)(need < most ? need : most);
}

// Columns are counted in 32 bits, a step of the widest rows' threads (2048) behind the last one included.
constexpr int kWidest = INT_MAX - 4096;
static int check_packed(const void* q, int64_t ldq, const void* code, int64_t ldc, int64_t rows, int32_t d, int type) {
  if (rows < 0 || rows > INT_MAX || d < 1 || !type_known(type)) return JANUS_EINVAL;
  if (d > kWidest) return JANUS_EUNSUPPORTED;
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
  const PackShape s = pack_shape(rows, d);
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
  const PackShape s = pack_shape(rows, d);
  with_type(type, [&](auto zero) {
    using T = decltype(zero);
    auto go = [&](auto silu, auto whole) {
      hipLaunchKernelGGL((unpack_rows_kernel<T, decltype(silu)::value, decltype(whole)::value>), dim3(unpack_grid(s)),
                         dim3(256), 0, static_cast<hipStream_t>(stream), s, q, ldq, code, ldc,
                         static_cast<const T*>(grad), ldg, static_cast<T*>(out), ldo, static_cast<T*>(value), ldv);
    };
    auto by_width = [&](auto silu) {
      if (d % 8 == 0) go(silu, std::true_type{});
      else go(silu, std::false_type{});
    };
    if (act == JANUS_ACT_SILU) by_width(std::true_type{});
    else by_width(std::false_type{});
  });
  return launched();
}

static int check_packed_wgrad(int64_t rows, int32_t n_groups, int32_t P, int32_t Q, int32_t type) {
  if (rows < 0 || rows > INT_MAX - 4096 || n_groups < 1 || n_groups > 1024 || P < 1 || Q < 1 || !type_known(type))
    return JANUS_EINVAL;
  // a launch holds fewer than 2^32 threads
  const WgradPlan w = wgrad_plan(rows, n_groups, P, Q, type);
  return wgrad_blocks(w) < (1 << 24) ? JANUS_OK : JANUS_EUNSUPPORTED;
}

extern "C" int64_t janus_packed_wgrad_workspace(int64_t rows, int32_t n_groups, int32_t P, int32_t Q, int32_t type) {
  int rc = check_packed_wgrad(rows, n_groups, P, Q, type);
  if (rc) return rc;
  return wgrad_plan(rows, n_groups, P, Q, type).total;
}

extern "C" int janus_packed_wgrad(const int8_t* q, int64_t ldq, const uint8_t* code, int64_t ldc, const void* B,
                                  int64_t ldb, int32_t type, float* G, const int32_t* row_off, int32_t n_groups,
                                  int64_t rows, int32_t P, int32_t Q, void* work, int64_t work_bytes, void* stream) {
  int rc = check_packed_wgrad(rows, n_groups, P, Q, type);
  if (!rc) rc = check_packed(q, ldq, code, ldc, rows, P, type);
  if (rc) return rc;
  const WgradPlan w = wgrad_plan(rows, n_groups, P, Q, type);
  if (rows > 0 && (ldb > UINT_MAX || std::max({ldq, ldc, ldb * type_bytes(type)}) > UINT_MAX / (w.kc + kReadAhead)))
    return JANUS_EUNSUPPORTED;
  if (!G || !row_off || (rows > 0 && (!B || ldb < Q)) || !work || !rows_aligned(work, 0, 1) ||
      work_bytes < janus_packed_wgrad_workspace(rows, n_groups, P, Q, type))
    return JANUS_EINVAL;
  const int64_t blocks = (int64_t)wgrad_blocks(w);
  char* base = static_cast<char*>(work);
  int* n_chunks = reinterpret_cast<int*>(base);
  PackedChunk* chunks = reinterpret_cast<PackedChunk*>(base + w.chunks);
  int* first = reinterpret_cast<int*>(base + w.first);
  int* count = reinterpret_cast<int*>(base + w.count);
  float* partial = reinterpret_cast<float*>(base + w.partial);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(packed_chunks_kernel, dim3(1), dim3((n_groups + 63) / 64 * 64), 0, st, row_off, n_groups, rows, w.kc, chunks, w.most,
                     n_chunks, first, count);
  const bool words = rows_aligned(q, ldq, 1, 4) && rows_aligned(B, ldb, type_bytes(type), 4);
  with_type(type, [&](auto zero) {
    using T = decltype(zero);
    auto go = [&](auto in_words) {
      hipLaunchKernelGGL((packed_wgrad_kernel<T, decltype(in_words)::value>), dim3((unsigned)blocks), dim3(256), 0, st, q,
                         ldq, code, ldc, static_cast<const T*>(B), ldb, rows, P, Q, chunks, n_chunks, w.tiles_p, w.tiles_q,
                         partial, G);
    };
    if (words) go(std::true_type{});
    else go(std::false_type{});
  });
  const int64_t PQ = (int64_t)P * Q;
  if (rows > w.kc) {   // else no group has several chunks
    auto reduce = [&](auto v) {
      const unsigned bx = cdiv(PQ, 64 * v.value);
      hipLaunchKernelGGL(packed_reduce_kernel<v.value>, dim3(bx < 1024 ? bx : 1024, n_groups), dim3(256), 0, st, partial,
                         first, count, PQ, G);
    };
    if (PQ % 4 == 0 && rows_aligned(G, 0, 4)) reduce(std::integral_constant<int, 4>{});
    else reduce(std::integral_constant<int, 1>{});
  }
  return launched();
}
