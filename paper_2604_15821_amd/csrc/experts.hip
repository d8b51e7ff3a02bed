// A whole expert layer for a few tokens: router, top-k, experts and their weighted sum.
//
//   l = x Wr + beta;  the top_k largest of a token, lower index first on ties
//   g = softmax(l) of the chosen (normalize: divided by their sum)
//   y = sum_c g_c W2_c^T SiLU(W1_c^T x)
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
                                                           int* __restrict__ eid, float* __restrict__ gate) {
  __shared__ float red[256], logit[kMaxExperts];
  const int t = blockIdx.x;
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

// hidden[slot, j] = SiLU(sum_i x[i] W1[e, i, j])
template <typename T>
__global__ __launch_bounds__(256) void expert_up_kernel(ExpertArgs a, const T* __restrict__ x, long long ldx,
                                                        const T* __restrict__ w1, const int* __restrict__ eid,
                                                        float* __restrict__ hidden) {
  const int slot = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= a.h) return;
  const T* w = w1 + (long long)eid[slot] * a.d * a.h + j;
  const T* v = x + slot / a.k * ldx;
  float s = 0.f;
  for (int i = 0; i < a.d; ++i) s += (float)v[i] * (float)w[(long long)i * a.h];
  hidden[(long long)slot * a.h + j] = silu(s);
}

// y[t, i] = sum_c gate sum_j hidden[slot, j] W2[e, j, i]
template <typename T>
__global__ __launch_bounds__(256) void expert_down_kernel(ExpertArgs a, const float* __restrict__ hidden,
                                                          const T* __restrict__ w2, const int* __restrict__ eid,
                                                          const float* __restrict__ gate, T* __restrict__ y,
                                                          long long ldy) {
  const int t = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.d) return;
  float out = 0.f;
  for (int c = 0; c < a.k; ++c) {
    const int slot = t * a.k + c;
    const T* w = w2 + (long long)eid[slot] * a.h * a.d + i;
    const float* v = hidden + (long long)slot * a.h;
    float s = 0.f;
    for (int j = 0; j < a.h; ++j) s += v[j] * (float)w[(long long)j * a.d];
    out += gate[slot] * s;
  }
  y[t * ldy + i] = (T)out;
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
  return (int64_t)tokens * p->top_k * p->d_hidden * 4 + 16;
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
  with_type(p->type, [&](auto zero) {
    using T = decltype(zero);
    float* hidden = static_cast<float*>(work);
    hipLaunchKernelGGL(expert_route_kernel<T>, dim3(tokens), dim3(256), 0, st, a, static_cast<const T*>(x), ldx, eid,
                       gate);
    hipLaunchKernelGGL(expert_up_kernel<T>, dim3(cdiv(a.h, 256), tokens * a.k), dim3(256), 0, st, a,
                       static_cast<const T*>(x), ldx, static_cast<const T*>(p->w_up), eid, hidden);
    hipLaunchKernelGGL(expert_down_kernel<T>, dim3(cdiv(a.d, 256), tokens), dim3(256), 0, st, a, hidden,
                       static_cast<const T*>(p->w_down), eid, gate, static_cast<T*>(y), ldy);
  });
  return launched();
}
