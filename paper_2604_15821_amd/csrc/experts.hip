// A whole expert layer for a few tokens: router, top-k, experts and their weighted sum.
//
//   l = x Wr + beta;  the top_k largest of a token, lower index first on ties
//   g = softmax(l) of the chosen (normalize: divided by their sum)
//   y = sum_c g_c W2_c^T SiLU(W1_c^T x)
//
// Bound by the chosen experts' weights, which are read once: 48 tokens, 32 experts of 1024 x 4096 bf16, 114 to 136 us for 537 MB,
// by where the weights lie in memory (the products 4.3 to 5.2 and 3.3 to 5.2 TB/s), and for a token or two by the chain of
// launches: 19 us for 17 MB (512 x 2048 fp32).
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace janus {

constexpr int kExpertTokens = 64;   // tokens of a call, at most
constexpr int kMaxExperts = 256;
constexpr int kMaxTopK = 8;
constexpr int kMostShares = 16;     // of a large router's rows

struct ExpertArgs {
  int tokens, d, h, n, k, normalize;
  const float* router;
  const float* beta;
};

// Router of one token by a workgroup of W waves.  Lanes take V neighbouring experts each (four, of which the last
// lane's may be its neighbour's too; one where there are fewer), the rest of a wave and the waves take rows, up to
// sixteen in flight; rows are added over the lanes (to four sums per wave) and then over the waves.  Every expert then counts
// those that come before it: its rank is its place among the chosen, without a round for each of them.
// NaN ranks like -inf and makes the token's gates NaN; a token without any finite or +inf logit
// (all experts masked) has gates of zero.
template <int W>
struct RouteArea {
  float red[W][kMaxExperts];   // of a wave: one sum per expert, or up to four one behind the other
  __align__(16) float key[kMaxExperts];
  float sum[4], top[kMaxTopK], gate[kMaxTopK];
  int eid[kMaxTopK], nan;
};
// logit parts of rows [begin, end): red[wave]
template <typename T, int V, int W>
__device__ __forceinline__ void route_sums(const ExpertArgs& a, const T* __restrict__ x, int begin, int end,
                                           RouteArea<W>& s) {
  typedef float vec __attribute__((ext_vector_type(V), aligned(4)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int units = (a.n + V - 1) / V;
  int wide = 1;
  while (wide < units && wide < 64) wide <<= 1;
  const int per = 64 / wide, rows = per * W, row0 = wave * per + lane / wide;
  for (int u0 = 0; u0 < units; u0 += 64) {
    const int u = u0 + (lane & (wide - 1)), c0 = max(min(V * u, a.n - V), 0);
    vec sum = {};
    const float* w = a.router + c0;
    auto add = [&](auto flight, int i) {   // rows i, i + rows, ..; past the end the last one is read and not added
      vec r[flight.value];
      float v[flight.value];
#pragma unroll
      for (int j = 0; j < flight.value; ++j) {
        const int q = min(i + j * rows, end - 1);
        r[j] = *reinterpret_cast<const vec*>(w + (long long)q * a.n);
        v[j] = (float)x[q];
      }
#pragma unroll
      for (int j = 0; j < flight.value; ++j)
        if (i + j * rows < end) sum += r[j] * v[j];
    };
    for (int i = begin; i < end;) {
      if (i + 8 * rows < end) {
        add(std::integral_constant<int, 16>{}, i + row0);
        i += 16 * rows;
      } else {
        add(std::integral_constant<int, 8>{}, i + row0);
        i += 8 * rows;
      }
    }
    const int left = max(wide, 16);   // lanes of one sum: four, two or one sums per wave
#pragma unroll
    for (int c = 0; c < V; ++c) {
      for (int o = wide; o < left; o <<= 1) sum[c] += __shfl_xor(sum[c], o, 64);
      if ((lane & (left - 1)) < wide && u < units) s.red[wave][lane / left * (V * left) + c0 + c] = sum[c];
    }
  }
  __syncthreads();
}
template <int V, int W>
__device__ __forceinline__ float route_sum(const RouteArea<W>& s, int n, int e) {
  const int left = n <= 16 * V ? 16 : n <= 32 * V ? 32 : 64;
  float l = 0.f;
  for (int i = 0; i < 64 / left; ++i) {
#pragma unroll
    for (int p = 0; p < W; ++p) l += s.red[p][i * (V * left) + e];
  }
  return l;
}

// beta of expert threadIdx.x, asked for before the sums so that it is there after them
__device__ __forceinline__ float route_beta(const ExpertArgs& a) {
  return a.beta && (int)threadIdx.x < a.n ? a.beta[threadIdx.x] : 0.f;
}

// The chosen experts (eid) and their logits (top) from the logit l of expert threadIdx.x.
template <int W>
__device__ __forceinline__ void route_rank(const ExpertArgs& a, float l, RouteArea<W>& s) {
  const int e = threadIdx.x;
  if (e == 0) s.nan = 0;
  const float key = e < a.n && l == l ? l : -INFINITY;
  if (e < kMaxExperts) s.key[e] = key;
  __syncthreads();
  if (e < a.n) {
    if (l != l) s.nan = 1;
    int rank = 0;
    for (int q = 0; q < a.n; q += 32) {   // keys past the last expert are -inf and of a higher index
      f32x4 o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = *reinterpret_cast<const f32x4*>(s.key + q + 4 * i);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) rank += q + 4 * i + j < e ? o[i][j] >= key : o[i][j] > key;
    }
    if (rank < a.k) s.top[rank] = key, s.eid[rank] = e;
  }
  __syncthreads();
}

// The gates of the choice.
template <int W>
__device__ __forceinline__ void route_gates(const ExpertArgs& a, float l, RouteArea<W>& s) {
  const int e = threadIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float top = s.top[0];
  if (e < kMaxExperts) {
    const float p = wave_sum(top == -INFINITY || e >= a.n ? 0.f : expf(l - top));
    if (lane == 0) s.sum[wave] = p;
  }
  __syncthreads();
  if (e < a.k) {
    auto p = [&](int c) { return top == -INFINITY ? 0.f : expf(s.top[c] - top); };
    float over = 0.f;
    if (a.normalize)
      for (int c = 0; c < a.k; ++c) over += p(c);
    else
      over = (s.sum[0] + s.sum[1]) + (s.sum[2] + s.sum[3]);
    s.gate[e] = s.nan ? NAN : over > 0.f || over != over ? p(e) / over : 0.f;
  }
  __syncthreads();
}

constexpr int kRouteWaves = 16;
template <typename T, int V>
__global__ __launch_bounds__(64 * kRouteWaves) void expert_route_kernel(ExpertArgs a, const T* __restrict__ x,
                                                                        long long ldx, int* __restrict__ eid,
                                                                        float* __restrict__ gate,
                                                                        int* __restrict__ arrived, int n_arrived) {
  __shared__ RouteArea<kRouteWaves> s;
  const int t = blockIdx.x;
  if (t == 0)   // the counts of the second product's workgroups
    for (int i = threadIdx.x; i < n_arrived; i += 64 * kRouteWaves) arrived[i] = 0;
  const float beta = route_beta(a);
  route_sums<T, V, kRouteWaves>(a, x + t * ldx, 0, a.d, s);
  const float l = (int)threadIdx.x < a.n ? route_sum<V>(s, a.n, threadIdx.x) + beta : 0.f;
  route_rank(a, l, s);
  route_gates(a, l, s);
  if ((int)threadIdx.x < a.k) {
    eid[t * a.k + threadIdx.x] = s.eid[threadIdx.x];
    gate[t * a.k + threadIdx.x] = s.gate[threadIdx.x];
  }
}

// The same for a large router, of which one workgroup would read too much: blockIdx.x takes a share of the rows,
// and a second kernel adds the shares in order and chooses.
template <typename T, int V>
__global__ __launch_bounds__(64 * kRouteWaves) void expert_logits_kernel(ExpertArgs a, const T* __restrict__ x,
                                                                         long long ldx, int rows,
                                                                         float* __restrict__ share) {
  __shared__ RouteArea<kRouteWaves> s;
  const int t = blockIdx.y, begin = blockIdx.x * rows;
  route_sums<T, V, kRouteWaves>(a, x + t * ldx, begin, min(begin + rows, a.d), s);
  const int e = threadIdx.x;
  if (e < a.n) share[((long long)t * gridDim.x + blockIdx.x) * a.n + e] = route_sum<V>(s, a.n, e);
}
__global__ __launch_bounds__(kMaxExperts) void expert_choose_kernel(ExpertArgs a, const float* __restrict__ share,
                                                                    int shares, int* __restrict__ eid,
                                                                    float* __restrict__ gate, int* __restrict__ arrived,
                                                                    int n_arrived) {
  __shared__ RouteArea<1> s;
  const int t = blockIdx.x, e = threadIdx.x;
  if (t == 0)
    for (int i = e; i < n_arrived; i += kMaxExperts) arrived[i] = 0;
  float l = 0.f;
  const float beta = route_beta(a);
  if (e < a.n) {
    const float* p = share + (long long)t * shares * a.n + e;
    float v[kMostShares];
#pragma unroll
    for (int z = 0; z < kMostShares; ++z) v[z] = p[min(z, shares - 1) * a.n];
#pragma unroll
    for (int z = 0; z < kMostShares; ++z)
      if (z < shares) l += v[z];
    l += beta;
  }
  route_rank(a, l, s);
  route_gates(a, l, s);
  if (e < a.k) eid[t * a.k + e] = s.eid[e], gate[t * a.k + e] = s.gate[e];
}

// ------------------------------------------------------------------ the experts' products
// A wave multiplies up to 16 MT tokens (rows of the 16 x 16 matrix instructions) with 32 rows of a weight matrix
// at a time, 16 COLS columns of it.  Lane l holds rows 8 (l / 16) .. + 7 of those, COLS neighbouring columns
// from COLS (l % 16) on, read by eight loads of up to 16 bytes that stay in flight while the
// stage before is multiplied.  The order of k within an instruction is free as long as both operands
// agree, so no value has to change its lane: fp32 takes one instruction of four k per row and column
// (lane's row j is k = j of its group), 16-bit types one of 32 k per column after packing pairs of
// rows, one byte permutation per two values.
template <typename T, int COLS>
struct Panel {
  typedef T vec __attribute__((ext_vector_type(COLS)));
  vec row[8];
  // rows k0 + 8 (lane / 16) + j below K of w [K, n] at the lane's columns; the lane's rows lie all below K or
  // all behind it (K is a multiple of 8), where they read the last ones
  __device__ __forceinline__ void load(const T* __restrict__ w, long long n, int k, int K) {
    const T* p = w + (long long)min(k, K - 8) * n;
#pragma unroll
    for (int j = 0; j < 8; ++j) row[j] = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p + j * n));
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int c = 0; c < COLS; ++c) row[j][c] = (T)0.f;
  }
};

// Eight consecutive k of one token: as they are, or an fp32 value as the sum of three bf16 of eight bits each (by
// truncation, so the sum is exact), for products with 16-bit weights.
template <typename T>
struct Eight {
  typedef T vec __attribute__((ext_vector_type(8)));
  vec v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void clear() { v = vec{}; }
};
struct EightSplit {
  bf16x8 term[3];
  __device__ __forceinline__ void load(const float* p) {
    const f32x8 v = *reinterpret_cast<const f32x8*>(p);
    unsigned w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const float ah = high_part(a), bh = high_part(b);
        w[q][i] = pack_high(a, b);
        a = a == ah ? 0.f : a - ah;   // not inf - inf
        b = b == bh ? 0.f : b - bh;
      }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) term[q] = __builtin_bit_cast(bf16x8, make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]));
  }
  __device__ __forceinline__ void clear() { term[0] = term[1] = term[2] = bf16x8{}; }
};

// column c of a panel of 16-bit values: eight k in order
template <typename T, int COLS>
__device__ __forceinline__ uint4 panel_column(const Panel<T, COLS>& p, int c) {
  unsigned o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned a, b;
    __builtin_memcpy(&a, reinterpret_cast<const char*>(&p.row[2 * i]) + 4 * (c / 2), 4);
    __builtin_memcpy(&b, reinterpret_cast<const char*>(&p.row[2 * i + 1]) + 4 * (c / 2), 4);
    o[i] = __builtin_amdgcn_perm(b, a, c % 2 ? 0x07060302u : 0x05040100u);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

template <bool EXACT, int COLS>
__device__ __forceinline__ void multiply(const Eight<float>& a, const Panel<float, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], w.row[j][c], acc[c], 0, 0, 0);
}
template <bool EXACT, int COLS>
__device__ __forceinline__ void multiply(const Eight<__bf16>& a, const Panel<__bf16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c)
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, __builtin_bit_cast(bf16x8, panel_column(w, c)), acc[c], 0, 0, 0);
}
template <bool EXACT, int COLS>
__device__ __forceinline__ void multiply(const Eight<_Float16>& a, const Panel<_Float16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c)
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, __builtin_bit_cast(f16x8, panel_column(w, c)), acc[c], 0, 0, 0);
}
// The smaller terms of a sum meet an infinity of the other operand as well, and zero times infinity is NaN.  Where a
// product holds a NaN it is formed again (EXACT): they take that operand with its infinities and NaN as zeros, the largest
// term has them.  (All terms of a value have its sign, so nothing else can go wrong.  Looking at every operand on the way
// costs 8 % of a call.)  Two bf16 of a word: the sign bits of those that are not finite, and the word without them.
__device__ __forceinline__ unsigned beyond(unsigned u) { return ((u & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ unsigned finite_only(unsigned u) {
  const unsigned m = beyond(u);
  return u & ~(m | (m - (m >> 15)));
}
__device__ __forceinline__ uint4 finite_only(uint4 u) {
  return make_uint4(finite_only(u.x), finite_only(u.y), finite_only(u.z), finite_only(u.w));
}

template <bool EXACT, int COLS>
__device__ __forceinline__ void multiply(const EightSplit& a, const Panel<__bf16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    const uint4 b = panel_column(w, c);
    uint4 f = b;
    if (EXACT) f = finite_only(b);
#pragma unroll
    for (int q = 2; q >= 0; --q)   // small terms first
      acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.term[q], __builtin_bit_cast(bf16x8, q ? f : b), acc[c], 0, 0, 0);
  }
}
// An fp16 weight is exactly the sum of two bf16 (eight and three bits of it), whose range the hidden values
// fit, while fp16 would cut them off at 65504 and 2^-24.
template <bool EXACT, int COLS>
__device__ __forceinline__ void multiply(const EightSplit& a, const Panel<_Float16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    unsigned hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = (float)w.row[2 * i][c], y = (float)w.row[2 * i + 1][c];
      const float xh = high_part(x), yh = high_part(y);
      hi[i] = pack_high(x, y);
      lo[i] = pack_high(x == xh ? 0.f : x - xh, y == yh ? 0.f : y - yh);   // not inf - inf
    }
    const uint4 h = make_uint4(hi[0], hi[1], hi[2], hi[3]), top = __builtin_bit_cast(uint4, a.term[0]);
    const bf16x8 bl = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    uint4 f = h, t = top;
    if (EXACT) f = finite_only(h), t = finite_only(top);
#pragma unroll
    for (int q = 2; q >= 0; --q) {   // small terms first
      const bf16x8 low = q ? a.term[q] : __builtin_bit_cast(bf16x8, t);
      acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(low, bl, acc[c], 0, 0, 0);
      acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.term[q], __builtin_bit_cast(bf16x8, q ? f : h), acc[c], 0, 0, 0);
    }
  }
}

constexpr int kExpertWaves = 8;

// The slots (token * top_k + choice) that chose this workgroup's expert, in order.  With at most as many slots as
// experts, blockIdx.y is a slot and stands for its expert if no earlier slot chose the same; else it is the
// expert.  Returns their number.
struct ExpertSlots {
  int slot[kExpertTokens];
  int count, expert;
};
__device__ __forceinline__ int find_slots(const ExpertArgs& a, const int* __restrict__ eid, ExpertSlots& s) {
  if (threadIdx.x < 64) {
    const int slots = a.tokens * a.k;
    const int e = slots <= a.n ? eid[blockIdx.y] : blockIdx.y;
    int n = 0;
    bool first = true;
    for (int base = 0; base < slots; base += 64) {
      const int q = base + threadIdx.x;
      const bool hit = q < slots && eid[q] == e;
      const unsigned long long all = __ballot(hit);
      if (slots <= a.n && all && n == 0) first = base + __ffsll(all) - 1 == (int)blockIdx.y;
      const int at = n + __popcll(all & ((1ull << threadIdx.x) - 1));
      if (hit && at < kExpertTokens) s.slot[at] = q;
      n += __popcll(all);
    }
    if (threadIdx.x == 0) s.count = first ? min(n, kExpertTokens) : 0, s.expert = e;
  }
  __syncthreads();
  return s.count;
}

// One expert's slots base .. base + 16 MT - 1 times columns of its weight, over the rows [k0, k1) of it.  `deep` waves
// (a power of two) share COLS * 16 columns: they take stages of 32 rows in turn and are added in order; the
// workgroup owns kExpertWaves / deep such blocks of columns.  done(t, c, v): value of the t-th slot in column c.
// `A` is the operand of a token's values S, row ld apart, slot q reading row q / per.
template <typename T, typename S, typename A, int COLS, int MT, typename F>
__device__ __forceinline__ void expert_product(const ExpertSlots& s, int base, const S* __restrict__ x, long long ldx, int per,
                                               const T* __restrict__ w, int n, int k0, int k1, int K, int deep,
                                               float* __restrict__ lds, F done) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = 8 * (lane >> 4);
  const int across = kExpertWaves / deep, level = wave & (deep - 1);
  const int first = blockIdx.x * across * (16 * COLS), c0 = first + wave / deep * (16 * COLS);
  // columns past the end (n is a multiple of 16, so of COLS) read the last ones and are not stored
  const T* wl = w + min(c0 + COLS * (lane & 15), n - COLS);
  const int count = min(s.count - base, 16 * MT), tiles = (count + 15) >> 4;
  const S* xr[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) xr[m] = x + s.slot[base + min(16 * m + (lane & 15), count - 1)] / per * ldx;
  f32x4 acc[MT][COLS];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[m][c] = f32x4{};
  Panel<T, COLS> now, next;
  auto product = [&](auto exact, int k) {
    const bool behind = k + sub >= k1;
    if (behind) now.clear();
#pragma unroll
    for (int m = 0; m < MT; ++m)
      if (m < tiles) {
        A v;
        v.load(xr[m] + min(k + sub, K - 8));
        if (behind) v.clear();
        multiply<exact.value, COLS>(v, now, acc[m]);
      }
  };
  const int first_k = k0 + 32 * level;
  if (first_k < k1) now.load(wl, n, first_k + sub, K);
  for (int k = first_k; k < k1; k += 32 * deep) {
    const bool more = k + 32 * deep < k1;
    if (more) next.load(wl, n, k + 32 * deep + sub, K);
    product(std::false_type{}, k);
    if (more) now = next;
  }
  if constexpr (std::is_same_v<A, EightSplit>) {
    bool nan = false;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int c = 0; c < COLS; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) nan |= acc[m][c][i] != acc[m][c][i];
    if (__any(nan)) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int c = 0; c < COLS; ++c) acc[m][c] = f32x4{};
      for (int k = first_k; k < k1; k += 32 * deep) {
        now.load(wl, n, k + sub, K);
        product(std::true_type{}, k);
      }
    }
  }
  // row 4 (lane / 16) + i of the result, column COLS (lane % 16) + c
  for (int m = 0; m < tiles; ++m) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* o = lds + (wave * 16 + 4 * (lane >> 4) + i) * (16 * COLS) + COLS * (lane & 15);
#pragma unroll
      for (int q = 0; q < MT; ++q)
        if (q == m) {
#pragma unroll
          for (int c = 0; c < COLS; ++c) o[c] = acc[q][c][i];
        }
    }
    __syncthreads();
    const int rows = min(16, count - 16 * m);
    const int part = rows * 16 * COLS;
    for (int e = threadIdx.x; e < across * part; e += 64 * kExpertWaves) {
      float v = 0.f;
      int block = 0, i = e;
      if (deep == kExpertWaves) {
#pragma unroll
        for (int q = 0; q < kExpertWaves; ++q) v += lds[q * (256 * COLS) + i];
      } else {
        block = e / part;
        i = e - block * part;
        for (int q = 0; q < deep; ++q) v += lds[(block * deep + q) * (256 * COLS) + i];
      }
      const int c = first + block * (16 * COLS) + i % (16 * COLS);
      if (c < n) done(base + 16 * m + i / (16 * COLS), c, v);
    }
  }
}

// Waves that share a block of columns of a product over `rows` rows: one per stage, at most all.
__host__ __device__ inline int deep_waves(int rows) {
  int deep = 1;
  while (deep < kExpertWaves && 32 * deep < rows) deep <<= 1;
  return deep;
}

// hidden[slot, j] = SiLU(sum_i x[i] W1[e, i, j])
// kRoute (one token): every workgroup routes the token itself, with V experts per lane, and the first one
// writes the choice.
template <typename T, int COLS, int MT, int V, bool kRoute>
__global__ __launch_bounds__(64 * kExpertWaves) void expert_up_kernel(ExpertArgs a, const T* __restrict__ x,
                                                                      long long ldx, const T* __restrict__ w1,
                                                                      int* __restrict__ eid, float* __restrict__ gate,
                                                                      int* __restrict__ arrived, int n_arrived,
                                                                      float* __restrict__ hidden) {
  __shared__ ExpertSlots s;
  __shared__ float lds[kExpertWaves * 256 * COLS];
  __shared__ std::conditional_t<kRoute, RouteArea<kExpertWaves>, int> r;
  float l = 0.f;
  if constexpr (kRoute) {
    const float beta = route_beta(a);
    route_sums<T, V, kExpertWaves>(a, x, 0, a.d, r);
    if ((int)threadIdx.x < a.n) l = route_sum<V>(r, a.n, threadIdx.x) + beta;
    route_rank(a, l, r);
    if (threadIdx.x == 0) s.count = 1, s.slot[0] = blockIdx.y, s.expert = r.eid[blockIdx.y];
    __syncthreads();
  } else {
    if (find_slots(a, eid, s) == 0) return;
  }
  for (int base = 0; base < s.count; base += 16 * MT)
    expert_product<T, T, Eight<T>, COLS, MT>(s, base, x, ldx, a.k, w1 + (long long)s.expert * a.d * a.h, a.h, 0, a.d,
                                             a.d, deep_waves(a.d), lds, [&](int t, int c, float v) {
                                               hidden[(long long)s.slot[t] * a.h + c] = v * sigmoid(v).s;
                                             });
  if constexpr (kRoute) {   // the gates are not needed before
    if (blockIdx.x == 0 && blockIdx.y == 0) {
      route_gates(a, l, r);
      for (int i = threadIdx.x; i < n_arrived; i += 64 * kExpertWaves) arrived[i] = 0;
      if ((int)threadIdx.x < a.k) eid[threadIdx.x] = r.eid[threadIdx.x], gate[threadIdx.x] = r.gate[threadIdx.x];
    }
  }
}

// y[t, c] = sum_q gate[t, q] sum_z part[t k + q, z, c] in that order, eight parts in flight.  A gate of zero leaves its
// expert out, whatever that one's weights hold.
template <typename F>
__device__ __forceinline__ float expert_sum(const ExpertArgs& a, const float* __restrict__ gate, float* part, int splits,
                                            int t, int c, F load) {
  const int n = a.k * splits;
  const float* g = gate + t * a.k;
  float* p = part + (long long)t * n * a.d + c;
  float out = 0.f, v = 0.f;
  for (int i = 0; i < n; i += 8) {
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = load(p + (long long)min(i + j, n - 1) * a.d);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < n) {
        v += u[j];
        if ((i + j + 1) % splits == 0) {
          const float w = g[(i + j) / splits];
          out += w == 0.f ? 0.f : w * v;
          v = 0.f;
        }
      }
  }
  return out;
}

// part[slot, split, i] = sum over the split's rows j of hidden[slot, j] W2[e, j, i].
// kJoin: the last workgroup of a column block to finish adds the parts (expert_sum); else expert_join_kernel does.
// The parts then cross the dies' L2 caches, so they are written and read as relaxed atomics of device scope,
// which pass those caches by; a wave waits for its own to be done before the workgroup's arrival is counted.
// (A device-scope fence in their place writes back a whole L2 per wave: 36 against 11 us for one token.)
template <typename T, int COLS, int MT, bool kJoin>
__global__ __launch_bounds__(64 * kExpertWaves) void expert_down_kernel(ExpertArgs a, const float* __restrict__ hidden,
                                                                        const T* __restrict__ w2,
                                                                        const int* __restrict__ eid,
                                                                        const float* __restrict__ gate, float* part,
                                                                        int* __restrict__ arrived, int rows_per_split,
                                                                        T* __restrict__ y, long long ldy) {
  using A = std::conditional_t<std::is_same_v<T, float>, Eight<float>, EightSplit>;
  __shared__ ExpertSlots s;
  __shared__ float lds[kExpertWaves * 256 * COLS];
  __shared__ int last;
  const int splits = gridDim.z, k0 = blockIdx.z * rows_per_split;
  const int count = find_slots(a, eid, s), deep = deep_waves(rows_per_split);
  for (int base = 0; base < count; base += 16 * MT)
    expert_product<T, float, A, COLS, MT>(s, base, hidden, a.h, 1, w2 + (long long)s.expert * a.h * a.d, a.d, k0,
                                          min(k0 + rows_per_split, a.h), a.h, deep, lds, [&](int t, int c, float v) {
                                            float* o = part + ((long long)s.slot[t] * splits + blockIdx.z) * a.d + c;
                                            if constexpr (kJoin)
                                              __hip_atomic_store(o, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                                            else
                                              *o = v;
                                          });
  if constexpr (kJoin) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(arrived + blockIdx.x, 1) == (int)(gridDim.y * gridDim.z) - 1;
    __syncthreads();
    if (!last) return;
    const int width = kExpertWaves / deep * (16 * COLS);
    for (int e = threadIdx.x; e < a.tokens * width; e += 64 * kExpertWaves) {
      const int t = e / width, c = blockIdx.x * width + e % width;
      if (c < a.d)
        y[t * ldy + c] = (T)expert_sum(a, gate, part, splits, t, c, [](float* p) {
          return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        });
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void expert_join_kernel(ExpertArgs a, const float* __restrict__ gate, float* part,
                                                          int splits, T* __restrict__ y, long long ldy) {
  const int c = blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
  if (c < a.d) y[t * ldy + c] = (T)expert_sum(a, gate, part, splits, t, c, [](float* p) { return *p; });
}

// How a call is shared out.  A panel of weights is multiplied by as many tiles of 16 tokens as most experts will
// have (an even share and half as much again); an expert with more reads its weights again.  Fewer tiles leave registers for
// more workgroups per CU.  A wave takes 64 (16-bit types: 128) columns of an expert, where that leaves fewer than 256
// workgroups half as many; all eight waves of a workgroup the same ones if there are stages for them, else more
// columns (d = 64, h = 3536, 128 experts, 44 tokens, bf16: 44 us with idle waves, 37 without).  The second product is also cut along its
// rows, into at most one stage of 32 rows per wave, until there are 512 workgroups.  Its parts are joined by the last
// workgroup of each column block where that has one value per thread or less, else (a few workgroups would
// join for long while the others idle) by a kernel of their own.  One token is routed by every workgroup of the
// first product where the router is small (up to 256 KB, read from L2 in little more than the time of the
// launch that this saves); a larger router is shared out, 128 KB to a workgroup.
constexpr int kRouterWhole = 65536;
struct ExpertPlan {
  int experts, cols_up, cols_down, blocks_up, blocks_down, splits, rows_per_split, tiles, shares, rows_per_share;
  bool join, route_inside;
};
static ExpertPlan expert_plan(const janus_experts* p, int tokens) {
  ExpertPlan q;
  const int slots = tokens * p->top_k, wide = p->type == JANUS_F32 ? 4 : 8;
  q.experts = slots < p->n_experts ? slots : p->n_experts;
  auto blocks = [&](int n, int cols, int rows) { return (int)cdiv(n, 16 * cols * (kExpertWaves / deep_waves(rows))); };
  auto columns = [&](int n, int rows) {
    return (long long)q.experts * blocks(n, wide, rows) < 256 ? wide / 2 : wide;
  };
  q.cols_up = columns(p->d_hidden, p->d);
  q.cols_down = columns(p->d, p->d_hidden);
  q.blocks_up = blocks(p->d_hidden, q.cols_up, p->d);
  const int stage = 32 * kExpertWaves, most = (int)cdiv(p->d_hidden, stage);
  const int want = (int)cdiv(512, (long long)q.experts * blocks(p->d, q.cols_down, p->d_hidden));
  q.splits = want < most ? want : most;
  q.rows_per_split = (int)cdiv(cdiv(p->d_hidden, q.splits), 32) * 32;
  q.splits = (int)cdiv(p->d_hidden, q.rows_per_split);
  q.blocks_down = blocks(p->d, q.cols_down, q.rows_per_split);
  const int share = cdiv(3ll * slots, 2ll * p->n_experts), all = tokens < share ? tokens : share;
  q.tiles = all <= 16 ? 1 : all <= 32 ? 2 : 4;
  q.join = (long long)tokens * cdiv(p->d, q.blocks_down) <= 64 * kExpertWaves;
  const long long router = (long long)p->d * p->n_experts;
  q.route_inside = tokens == 1 && router <= kRouterWhole;
  const int shares = router <= kRouterWhole ? 1 : (int)std::min<long long>(cdiv(router, kRouterWhole / 2), kMostShares);
  q.rows_per_share = (int)cdiv(p->d, shares);
  q.shares = (int)cdiv(p->d, q.rows_per_share);
  return q;
}
struct ExpertWork {
  int64_t hidden, part, arrived, total;   // offsets in bytes
};
static ExpertWork expert_work(const janus_experts* p, int tokens, const ExpertPlan& q) {
  const int64_t slots = (int64_t)tokens * p->top_k;
  ExpertWork w;
  w.hidden = 0;
  w.part = w.hidden + 4 * slots * p->d_hidden;
  // the router's shares are read before the parts are written
  const int64_t parts = slots * q.splits * p->d, shares = q.shares > 1 ? (int64_t)tokens * q.shares * p->n_experts : 0;
  w.arrived = w.part + (4 * std::max(parts, shares) + 15) / 16 * 16;
  w.total = w.arrived + 4 * ((q.blocks_down + 3) / 4 * 4);
  return w;
}

static int check_experts(const janus_experts* p, int tokens) {
  if (!p || tokens < 0 || p->d < 1 || p->d_hidden < 1 || p->n_experts < 1 || p->top_k < 1 ||
      p->top_k > p->n_experts || !type_known(p->type) || (p->normalize != 0 && p->normalize != 1))
    return JANUS_EINVAL;
  if (tokens > kExpertTokens || p->n_experts > kMaxExperts || p->top_k > kMaxTopK || p->d % 16 || p->d_hidden % 16 ||
      p->d > 16384 || p->d_hidden > 65536)
    return JANUS_EUNSUPPORTED;
  return JANUS_OK;
}

}  // namespace janus

using namespace janus;

extern "C" int64_t janus_expert_layer_workspace(const janus_experts* p, int32_t tokens) {
  int rc = check_experts(p, tokens);
  if (rc) return rc;
  return tokens ? expert_work(p, tokens, expert_plan(p, tokens)).total : 16;
}

extern "C" int janus_expert_layer(const janus_experts* p, const void* x, int64_t ldx, int32_t tokens, void* y,
                                  int64_t ldy, int32_t* eid, float* gate, void* work, int64_t work_bytes,
                                  void* stream) {
  int rc = check_experts(p, tokens);
  if (rc) return rc;
  if (tokens == 0) return JANUS_OK;
  if (!p->router || !p->w_up || !p->w_down || !x || !y || !eid || !gate || ldx < p->d || ldy < p->d || !work ||
      work_bytes < janus_expert_layer_workspace(p, tokens))
    return JANUS_EINVAL;
  const int e = type_bytes(p->type);
  if (!rows_aligned(x, ldx, e) || !rows_aligned(y, ldy, e) || !rows_aligned(p->w_up, 0, e) ||
      !rows_aligned(p->w_down, 0, e) || !rows_aligned(work, 0, 1))
    return JANUS_EINVAL;
  const ExpertArgs a{tokens, p->d, p->d_hidden, p->n_experts, p->top_k, p->normalize, p->router, p->beta};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const ExpertPlan plan = expert_plan(p, tokens);
  const ExpertWork at = expert_work(p, tokens, plan);
  char* base = static_cast<char*>(work);
  float* hidden = reinterpret_cast<float*>(base + at.hidden);
  float* part = reinterpret_cast<float*>(base + at.part);
  int* arrived = reinterpret_cast<int*>(base + at.arrived);
  with_type(p->type, [&](auto zero) {
    using T = decltype(zero);
    const int counts = plan.blocks_down;
    const T* xt = static_cast<const T*>(x);
    const T* up = static_cast<const T*>(p->w_up);
    auto by_columns = [&](int cols, auto f) {
      constexpr int kWide = sizeof(T) == 4 ? 4 : 8;
      if (cols == kWide) f(std::integral_constant<int, kWide>{});
      else f(std::integral_constant<int, kWide / 2>{});
    };
    auto by_tiles = [&](auto f) {
      if (plan.tiles == 1) f(std::integral_constant<int, 1>{});
      else if (plan.tiles == 2) f(std::integral_constant<int, 2>{});
      else f(std::integral_constant<int, 4>{});
    };
    auto by_router = [&](auto f) {
      if (a.n >= 4) f(std::integral_constant<int, 4>{});
      else f(std::integral_constant<int, 1>{});
    };
    auto launch_up = [&](auto cols, auto mt, auto v, auto routes) {
      hipLaunchKernelGGL((expert_up_kernel<T, cols.value, mt.value, v.value, routes.value>),
                         dim3(plan.blocks_up, plan.experts), dim3(64 * kExpertWaves), 0, st, a, xt, ldx, up,
                         eid, gate, arrived, counts, hidden);
    };
    auto launch_down = [&](auto cols, auto mt, auto join) {
      hipLaunchKernelGGL((expert_down_kernel<T, cols.value, mt.value, join.value>),
                         dim3(plan.blocks_down, plan.experts, plan.splits), dim3(64 * kExpertWaves), 0, st, a,
                         hidden, static_cast<const T*>(p->w_down), eid, gate, part, arrived, plan.rows_per_split,
                         static_cast<T*>(y), ldy);
    };
    const std::integral_constant<int, 1> one;
    if (plan.route_inside) {
      by_columns(plan.cols_up, [&](auto cols) { by_router([&](auto v) { launch_up(cols, one, v, std::true_type{}); }); });
    } else {
      by_router([&](auto v) {
        if (plan.shares == 1)
          hipLaunchKernelGGL((expert_route_kernel<T, v.value>), dim3(tokens), dim3(64 * kRouteWaves), 0, st, a, xt, ldx,
                             eid, gate, arrived, counts);
        else
          hipLaunchKernelGGL((expert_logits_kernel<T, v.value>), dim3(plan.shares, tokens), dim3(64 * kRouteWaves), 0, st,
                             a, xt, ldx, plan.rows_per_share, part);
      });
      if (plan.shares > 1)
        hipLaunchKernelGGL(expert_choose_kernel, dim3(tokens), dim3(kMaxExperts), 0, st, a, part, plan.shares, eid, gate,
                           arrived, counts);
      by_columns(plan.cols_up,
                 [&](auto cols) { by_tiles([&](auto mt) { launch_up(cols, mt, one, std::false_type{}); }); });
    }
    by_columns(plan.cols_down, [&](auto cols) {
      if (plan.join) launch_down(cols, one, std::true_type{});
      else by_tiles([&](auto mt) { launch_down(cols, mt, std::false_type{}); });
    });
    if (!plan.join)
      hipLaunchKernelGGL(expert_join_kernel<T>, dim3(cdiv(a.d, 256), tokens), dim3(256), 0, st, a, gate, part,
                         plan.splits, static_cast<T*>(y), ldy);
  });
  return launched();
}
