// A whole expert layer for a few tokens: router, top-k, experts and their weighted sum.
//
//   l = x Wr + beta;  the top_k largest of a token, lower index first on ties
//   g = softmax(l) of the chosen (normalize: divided by their sum)
//   y = sum_c g_c W2_c^T SiLU(W1_c^T x)
#include <type_traits>

#include "rows.h"

namespace janus {

constexpr int kExpertTokens = 64;   // tokens of a call, at most
constexpr int kMaxExperts = 256;
constexpr int kMaxTopK = 8;

struct ExpertArgs {
  int tokens, d, h, n, k, normalize;
  const float* router;
  const float* beta;
};

// Router of one token per workgroup: logits summed by 256 / 2^ceil(log2 n) threads per expert, then the
// choice by one wave that holds four experts per lane.
template <typename T>
__global__ __launch_bounds__(256) void expert_route_kernel(ExpertArgs a, const T* __restrict__ x, long long ldx,
                                                           int* __restrict__ eid, float* __restrict__ gate,
                                                           int* __restrict__ arrived, int n_arrived) {
  __shared__ float red[256], logit[kMaxExperts];
  const int t = blockIdx.x;
  if (t == 0)   // the counts of the second product's workgroups
    for (int i = threadIdx.x; i < n_arrived; i += 256) arrived[i] = 0;
  int wide = 1;
  while (wide < a.n) wide <<= 1;
  const int e = threadIdx.x & (wide - 1), part = threadIdx.x / wide, parts = 256 / wide;
  float s = 0.f;
  if (e < a.n)
    for (int i = part; i < a.d; i += parts) s += (float)x[t * ldx + i] * a.router[(long long)i * a.n + e];
  red[threadIdx.x] = s;
  __syncthreads();
  if ((int)threadIdx.x < a.n) {
    float v = 0.f;
    for (int p = 0; p < parts; ++p) v += red[p * wide + threadIdx.x];
    logit[threadIdx.x] = v + (a.beta ? a.beta[threadIdx.x] : 0.f);
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  // NaN ranks like -inf and makes the token's gates NaN; a token without any finite or +inf logit
  // (all experts masked) has gates of zero
  float l[4], key[4], top = -INFINITY;
  bool taken[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int q = threadIdx.x + 64 * j;
    l[j] = q < a.n ? logit[q] : -INFINITY;
    taken[j] = q >= a.n;
    key[j] = l[j] == l[j] ? l[j] : -INFINITY;
    top = fmaxf(top, key[j]);
  }
  bool nan = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) nan |= l[j] != l[j];
  nan = __any(nan);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  float p[4], sum = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    p[j] = top == -INFINITY ? 0.f : expf(l[j] - top);
    if ((int)threadIdx.x + 64 * j >= a.n) p[j] = 0.f;
    sum += p[j];
  }
  sum = wave_sum(sum);
  float chosen = 0.f, mine = 0.f;
  int mine_e = 0;
  for (int c = 0; c < a.k; ++c) {
    float best = -INFINITY, bp = 0.f;
    int at = INT_MAX;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (!taken[j] && (at == INT_MAX || key[j] > best)) best = key[j], bp = p[j], at = threadIdx.x + 64 * j;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float v = __shfl_xor(best, o, 64), vp = __shfl_xor(bp, o, 64);
      const int va = __shfl_xor(at, o, 64);
      if (va != INT_MAX && (at == INT_MAX || v > best || (v == best && va < at))) best = v, bp = vp, at = va;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((int)threadIdx.x + 64 * j == at) taken[j] = true;
    chosen += bp;
    if ((int)threadIdx.x == c) mine = bp, mine_e = at;
  }
  const float over = a.normalize ? chosen : sum;
  if ((int)threadIdx.x < a.k) {
    eid[t * a.k + threadIdx.x] = mine_e;
    gate[t * a.k + threadIdx.x] = nan ? NAN : over > 0.f || over != over ? mine / over : 0.f;
  }
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

// Eight consecutive k of one token: as they are, or an fp32 value as the sum of two bf16 (hi rounded to
// nearest, lo the rounded rest: together 2^-16 of the value), for products with 16-bit weights.
template <typename T>
struct Eight {
  typedef T vec __attribute__((ext_vector_type(8)));
  vec v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void clear() { v = vec{}; }
};
struct EightSplit {
  bf16x8 hi, lo;
  __device__ __forceinline__ void load(const float* p) {
    const f32x8 v = *reinterpret_cast<const f32x8*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi[j] = (__bf16)v[j];
      const float h = (float)hi[j];
      lo[j] = h - h == 0.f ? (__bf16)(v[j] - h) : (__bf16)0.f;
    }
  }
  __device__ __forceinline__ void clear() { hi = bf16x8{}, lo = bf16x8{}; }
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

template <int COLS>
__device__ __forceinline__ void multiply(const Eight<float>& a, const Panel<float, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], w.row[j][c], acc[c], 0, 0, 0);
}
template <int COLS>
__device__ __forceinline__ void multiply(const Eight<__bf16>& a, const Panel<__bf16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c)
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, __builtin_bit_cast(bf16x8, panel_column(w, c)), acc[c], 0, 0, 0);
}
template <int COLS>
__device__ __forceinline__ void multiply(const Eight<_Float16>& a, const Panel<_Float16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c)
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, __builtin_bit_cast(f16x8, panel_column(w, c)), acc[c], 0, 0, 0);
}
template <int COLS>
__device__ __forceinline__ void multiply(const EightSplit& a, const Panel<__bf16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    const bf16x8 b = __builtin_bit_cast(bf16x8, panel_column(w, c));
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.lo, b, acc[c], 0, 0, 0);
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.hi, b, acc[c], 0, 0, 0);
  }
}
// An fp16 weight is exactly the sum of two bf16 (eight and three bits of it), whose range the hidden values
// fit, while fp16 would cut them off at 65504 and 2^-24.
template <int COLS>
__device__ __forceinline__ void multiply(const EightSplit& a, const Panel<_Float16, COLS>& w, f32x4 (&acc)[COLS]) {
#pragma unroll
  for (int c = 0; c < COLS; ++c) {
    unsigned hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = (float)w.row[2 * i][c], y = (float)w.row[2 * i + 1][c];
      const unsigned xb = __float_as_uint(x), yb = __float_as_uint(y);
      hi[i] = __builtin_amdgcn_perm(yb, xb, 0x07060302u);
      const float xh = __uint_as_float(xb & 0xFFFF0000u), yh = __uint_as_float(yb & 0xFFFF0000u);
      const float xl = x == xh ? 0.f : x - xh, yl = y == yh ? 0.f : y - yh;   // not inf - inf
      lo[i] = __builtin_amdgcn_perm(__float_as_uint(yl), __float_as_uint(xl), 0x07060302u);
    }
    const bf16x8 bh = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    const bf16x8 bl = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.lo, bl, acc[c], 0, 0, 0);
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.lo, bh, acc[c], 0, 0, 0);
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.hi, bl, acc[c], 0, 0, 0);
    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.hi, bh, acc[c], 0, 0, 0);
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

// One expert's tokens times COLS * 16 columns of its weight, over the rows [k0, k1) of it; the waves take stages
// of 32 rows in turn and are added in order.  done(t, c, v): value of the t-th slot in column c.
// `A` is the operand of a token's values S, row ld apart, slot q reading row q / per.
template <typename T, typename S, typename A, int COLS, int MT, typename F>
__device__ __forceinline__ void expert_product(const ExpertSlots& s, const S* __restrict__ x, long long ldx, int per,
                                               const T* __restrict__ w, int n, int k0, int k1, int K,
                                               float* __restrict__ lds, F done) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = 8 * (lane >> 4);
  const int c0 = blockIdx.x * (16 * COLS);
  // columns past the end (n is a multiple of 16, so of COLS) read the last ones and are not stored
  const T* wl = w + min(c0 + COLS * (lane & 15), n - COLS);
  const int tiles = (s.count + 15) >> 4;
  const S* xr[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) xr[m] = x + s.slot[min(16 * m + (lane & 15), s.count - 1)] / per * ldx;
  f32x4 acc[MT][COLS];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[m][c] = f32x4{};
  Panel<T, COLS> now, next;
  int k = k0 + 32 * wave;
  if (k < k1) now.load(wl, n, k + sub, K);
  for (; k < k1; k += 32 * kExpertWaves) {
    const bool more = k + 32 * kExpertWaves < k1;
    if (more) next.load(wl, n, k + 32 * kExpertWaves + sub, K);
    const bool behind = k + sub >= k1;
    if (behind) now.clear();
#pragma unroll
    for (int m = 0; m < MT; ++m)
      if (m < tiles) {
        A v;
        v.load(xr[m] + min(k + sub, K - 8));
        if (behind) v.clear();
        multiply<COLS>(v, now, acc[m]);
      }
    if (more) now = next;
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
    const int rows = min(16, s.count - 16 * m);
    for (int e = threadIdx.x; e < rows * 16 * COLS; e += 64 * kExpertWaves) {
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < kExpertWaves; ++q) v += lds[q * (256 * COLS) + e];
      const int c = c0 + e % (16 * COLS);
      if (c < n) done(16 * m + e / (16 * COLS), c, v);
    }
  }
}

// hidden[slot, j] = SiLU(sum_i x[i] W1[e, i, j])
template <typename T, int COLS, int MT>
__global__ __launch_bounds__(64 * kExpertWaves) void expert_up_kernel(ExpertArgs a, const T* __restrict__ x,
                                                                      long long ldx, const T* __restrict__ w1,
                                                                      const int* __restrict__ eid,
                                                                      float* __restrict__ hidden) {
  __shared__ ExpertSlots s;
  __shared__ float lds[kExpertWaves * 256 * COLS];
  if (find_slots(a, eid, s) == 0) return;
  expert_product<T, T, Eight<T>, COLS, MT>(s, x, ldx, a.k, w1 + (long long)s.expert * a.d * a.h, a.h, 0, a.d, a.d, lds,
                                           [&](int t, int c, float v) {
                                             hidden[(long long)s.slot[t] * a.h + c] = silu(v);
                                           });
}

// part[slot, split, i] = sum over the split's rows j of hidden[slot, j] W2[e, j, i]; the last workgroup of a
// column block to finish adds the parts of every token: y = sum_c gate sum_split part, in that order.
template <typename T, int COLS, int MT>
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
  if (find_slots(a, eid, s) > 0)
    expert_product<T, float, A, COLS, MT>(s, hidden, a.h, 1, w2 + (long long)s.expert * a.h * a.d, a.d, k0,
                                          min(k0 + rows_per_split, a.h), a.h, lds, [&](int t, int c, float v) {
                                            part[((long long)s.slot[t] * splits + blockIdx.z) * a.d + c] = v;
                                          });
  __threadfence();   // this thread's parts before the workgroup's arrival
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(arrived + blockIdx.x, 1) == (int)(gridDim.y * gridDim.z) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();   // the others' parts after their arrival
  const int c0 = blockIdx.x * (16 * COLS);
  for (int e = threadIdx.x; e < a.tokens * 16 * COLS; e += 64 * kExpertWaves) {
    const int t = e / (16 * COLS), c = c0 + e % (16 * COLS);
    if (c >= a.d) continue;
    float out = 0.f;
    for (int q = 0; q < a.k; ++q) {
      const float* p = part + (long long)(t * a.k + q) * splits * a.d + c;
      float v = 0.f;
      for (int z = 0; z < splits; ++z) v += p[(long long)z * a.d];
      out += gate[t * a.k + q] * v;
    }
    y[t * ldy + c] = (T)out;
  }
}

// How a call is shared out.  A workgroup takes one expert and 64 (16-bit types: 128) columns; where that leaves
// fewer than 256 workgroups, half as many columns.  The second product is also cut along its
// rows, into at most one stage of 32 rows per wave, until there are 512 workgroups.
struct ExpertPlan {
  int experts, cols_up, cols_down, splits, rows_per_split;
};
static ExpertPlan expert_plan(const janus_experts* p, int tokens) {
  ExpertPlan q;
  const int slots = tokens * p->top_k, wide = p->type == JANUS_F32 ? 4 : 8;
  q.experts = slots < p->n_experts ? slots : p->n_experts;
  auto cols = [&](int n) { return (long long)q.experts * cdiv(n, 16 * wide) < 256 ? wide / 2 : wide; };
  q.cols_up = cols(p->d_hidden);
  q.cols_down = cols(p->d);
  const long long blocks = (long long)q.experts * cdiv(p->d, 16 * q.cols_down);
  const int stage = 32 * kExpertWaves, most = (int)cdiv(p->d_hidden, stage);
  const int want = (int)cdiv(512, blocks);
  q.splits = want < most ? want : most;
  q.rows_per_split = (int)cdiv(cdiv(p->d_hidden, q.splits), 32) * 32;
  q.splits = (int)cdiv(p->d_hidden, q.rows_per_split);
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
  w.arrived = w.part + 4 * slots * q.splits * p->d;
  w.total = w.arrived + 4 * ((cdiv(p->d, 16 * q.cols_down) + 3) / 4 * 4);
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
    hipLaunchKernelGGL(expert_route_kernel<T>, dim3(tokens), dim3(256), 0, st, a, static_cast<const T*>(x), ldx, eid,
                       gate, arrived, (int)cdiv(a.d, 16 * plan.cols_down));
    auto product = [&](auto cols, auto mt, bool up) {
      constexpr int kCols = decltype(cols)::value, kTiles = decltype(mt)::value;
      const unsigned bx = cdiv(up ? a.h : a.d, 16 * kCols);
      if (up)
        hipLaunchKernelGGL((expert_up_kernel<T, kCols, kTiles>), dim3(bx, plan.experts), dim3(64 * kExpertWaves), 0, st,
                           a, static_cast<const T*>(x), ldx, static_cast<const T*>(p->w_up), eid, hidden);
      else
        hipLaunchKernelGGL((expert_down_kernel<T, kCols, kTiles>), dim3(bx, plan.experts, plan.splits),
                           dim3(64 * kExpertWaves), 0, st, a, hidden, static_cast<const T*>(p->w_down), eid, gate, part,
                           arrived, plan.rows_per_split, static_cast<T*>(y), ldy);
    };
    auto with_tiles = [&](auto cols, bool up) {
      if (tokens <= 16) product(cols, std::integral_constant<int, 1>{}, up);
      else if (tokens <= 32) product(cols, std::integral_constant<int, 2>{}, up);
      else product(cols, std::integral_constant<int, 4>{}, up);
    };
    constexpr int kWide = sizeof(T) == 4 ? 4 : 8;
    for (const bool up : {true, false}) {
      if ((up ? plan.cols_up : plan.cols_down) == kWide) with_tiles(std::integral_constant<int, kWide>{}, up);
      else with_tiles(std::integral_constant<int, kWide / 2>{}, up);
    }
  });
  return launched();
}
