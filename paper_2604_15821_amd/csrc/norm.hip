// Norms after and before a block, fused with its gate and residual scale, and their gradients.
//
//   u = w_post b beta,  beta = 1 / sqrt(mean(b^2) + eps)
//   r = x + scale gate u
//   n = w_pre r rho,    rho = 1 / sqrt(mean(r^2) + eps)
//
// and backwards, from the gradients dr and dn at the stored r and b:
//
//   D  = dr + rho w_pre dn - r rho^3 <w_pre dn, r> / d          (dx = D)
//   v  = D scale gate w_post
//   db = beta v - b beta^3 <v, b> / d
//   dw_pre[c] = sum_m dn r rho
//   with T = D b beta:  dgate = scale w_post T (summed over a sequence's rows),
//   Q[c] = sum_m gate T,  dscale = w_post Q,  dw_post = scale Q
//
// so one column sum serves scale and w_post, and the statistics are taken again from r and b, which
// are read anyway: nothing but r and b need be kept for the backward pass.  All of it is bound by
// memory: 2 rows in and 2 out, backwards 4 in and 2 out.  Measured: 59 186 x 512 fp32, 512 sequences, 100 us
// forward (4.9 TB/s, where a copy reaches 5.2), 157 us backward (4.7 TB/s) and 10 us for its sums; 16 384 x 4096 bf16
// 170 and 8 us.
//
// Work: a group of L lanes owns a row and C of its columns per lane; groups take runs of
// consecutive rows, so that the parameters, a sequence's gate and the column sums stay in
// registers.  The sums of a workgroup's groups are added through LDS and written as one partial;
// a second kernel adds the partials in their order.  A sequence that lies within one group's run is
// finished there; of others each group writes its part, which the second kernel adds in order.  No
// atomics, so results are the same on every run.
#include "rows.h"

namespace janus {

struct NormArgs {
  long long rows, ldg;
  const float* w_post;
  const float* scale;
  const float* w_pre;
  const void* gate;
  const int* gate_off;
  int d, n_seq;
  float eps, inv_d;
};

struct NormGradOut {
  float* partial;   // [workgroups][2][d]: dw_pre and Q
  float* part_seq;  // [groups][2][d]: T of the sequence that enters a run, and of the one that leaves it
  void* dgate;
  long long lddg;
};

// The columns of a lane: C in runs of 16 bytes and, where d is no multiple of a run (ODD), one of the rest.
template <typename T, int L, int C, bool ODD>
struct Row {
  static constexpr int V = 16 / (int)sizeof(T), N = C + ODD;
  static constexpr int kThreads = L < 256 ? 256 : L;
  static constexpr int kGroups = kThreads / L;
  static __device__ __forceinline__ int col(int i, int lane) { return (i * L + lane) * V; }
  static __device__ __forceinline__ int whole(int d) { return ODD ? d / V * V : d; }   // columns in runs
  // Runs and rests past the end read the last ones and become zero, so that no load is behind a branch of a lane.
  template <typename S>
  static __device__ __forceinline__ void load(const S* p, float (&v)[N], int lane, int d) {
    const int w = whole(d);
    if (!ODD || w > 0) {
#pragma unroll
      for (int i = 0; i < C / V; ++i) load_run<S, V>(p + min(col(i, lane), w - V), v + i * V);
    }
    if (ODD) v[C] = (float)p[min(w + lane, d - 1)];
    trim(v, lane, d);
  }
  static __device__ __forceinline__ void trim(float (&v)[N], int lane, int d) {
    const int w = whole(d);
#pragma unroll
    for (int i = 0; i < C / V; ++i)
      if (col(i, lane) >= w) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[i * V + j] = 0.f;
      }
    if (ODD && w + lane >= d) v[C] = 0.f;
  }
  // a row's values as they are stored, to be taken apart later
  struct Raw {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    vec v[C / V];
    T rest;
    __device__ __forceinline__ void load(const T* p, int lane, int d) {
      const int w = whole(d);
      if (!ODD || w > 0) {
#pragma unroll
        for (int i = 0; i < C / V; ++i) v[i] = *reinterpret_cast<const vec*>(p + min(col(i, lane), w - V));
      }
      if (ODD) rest = p[min(w + lane, d - 1)];
    }
    __device__ __forceinline__ void values(float (&o)[N], int lane, int d) const {
#pragma unroll
      for (int i = 0; i < C / V; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) o[i * V + j] = (float)v[i][j];
      if (ODD) o[C] = (float)rest;
      trim(o, lane, d);
    }
  };
  template <typename S>
  static __device__ __forceinline__ void store(S* p, const float (&v)[N], int lane, int d) {
    const int w = whole(d);
#pragma unroll
    for (int i = 0; i < C / V; ++i) {
      const int c = col(i, lane);
      if (c < w) store_run<S, V>(p + c, v + i * V);
    }
    if (ODD && w + lane < d) p[w + lane] = (S)v[C];
  }
};

// Sums of N values over the L lanes of a group, in every lane.  Groups of several waves meet in LDS,
// in two areas used in turn: a wave that is back here has passed a barrier since every read of
// the area it writes.
template <int L, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* lds, int& turn) {
  if constexpr (L == 16) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = row16_sum(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = wave_sum(v[j]);
    if constexpr (L > 64) {
      constexpr int W = L / 64;
      float* area = lds + turn * (W * 4);
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) area[(threadIdx.x >> 6) * 4 + j] = v[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[j] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v[j] += area[w * 4 + j];
      }
    }
  }
}

// Rows that take part: all of them, or those of a sequence.
__device__ __forceinline__ long long norm_limit(const NormArgs& a) {
  if (!a.gate_off) return a.rows;
  const long long e = a.n_seq > 0 ? a.gate_off[a.n_seq] : 0;
  return min(max(e, 0ll), a.rows);
}

// The sequence that row m (below norm_limit) belongs to: the last one that begins at or before it.
__device__ __forceinline__ int seq_of(const int* off, int n, long long m) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= m) lo = mid; else hi = mid;
  }
  return lo;
}

template <typename T, int L, int C, bool ODD>
__global__ __launch_bounds__((L < 256 ? 256 : L)) void residual_norm_kernel(
    NormArgs a, const T* x, long long ldx, const T* b, long long ldb, T* r, long long ldr, T* n, long long ldn,
    long long run) {
  using R = Row<T, L, C, ODD>;
  __shared__ float lds[L > 64 ? L / 64 * 8 : 1];
  int turn = 0;
  const int lane = threadIdx.x % L;
  const long long r0 = ((long long)blockIdx.x * R::kGroups + threadIdx.x / L) * run;
  const long long r1 = min(r0 + run, norm_limit(a));
  float sw[R::N], wp[R::N], g[R::N];
#pragma unroll
  for (int j = 0; j < R::N; ++j) sw[j] = 1.f, wp[j] = 0.f, g[j] = 1.f;
  if (a.scale) R::load(a.scale, sw, lane, a.d);
  if (a.w_post) {
    float w[R::N];
    R::load(a.w_post, w, lane, a.d);
#pragma unroll
    for (int j = 0; j < R::N; ++j) sw[j] *= w[j];
  }
  if (a.w_pre) R::load(a.w_pre, wp, lane, a.d);
  long long seq_end = -1;
  for (long long m = r0; m < r1; ++m) {
    float xv[R::N], bv[R::N];
    R::load(x + m * ldx, xv, lane, a.d);
    R::load(b + m * ldb, bv, lane, a.d);
    if (a.gate) {
      const T* gate = static_cast<const T*>(a.gate);
      if (!a.gate_off) {
        R::load(gate + m * a.ldg, g, lane, a.d);
      } else if (m >= seq_end) {
        const int s = seq_of(a.gate_off, a.n_seq, m);
        seq_end = a.gate_off[s + 1];
        R::load(gate + s * a.ldg, g, lane, a.d);
      }
    }
    float beta = 1.f, s[1];
    if (a.w_post) {
      s[0] = 0.f;
#pragma unroll
      for (int j = 0; j < R::N; ++j) s[0] += bv[j] * bv[j];
      group_sum<L, 1>(s, lds, turn);
      beta = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
    }
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < R::N; ++j) {
      xv[j] += bv[j] * beta * sw[j] * g[j];
      s[0] += xv[j] * xv[j];
    }
    R::store(r + m * ldr, xv, lane, a.d);
    if (a.w_pre) {
      group_sum<L, 1>(s, lds, turn);
      const float rho = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
#pragma unroll
      for (int j = 0; j < R::N; ++j) xv[j] *= rho * wp[j];
      R::store(n + m * ldn, xv, lane, a.d);
    }
  }
}

template <typename T, int L, int C, bool ODD>
__global__ __launch_bounds__((L < 256 ? 256 : L), (C == 8 ? 3 : 2)) void residual_norm_grad_kernel(
    NormArgs a, const T* dr, long long lddr, const T* dn, long long lddn, const T* r, long long ldr, const T* b,
    long long ldb, T* dx, long long lddx, T* db, long long lddb, NormGradOut o, long long run) {
  using R = Row<T, L, C, ODD>;
  constexpr int kSum = R::kGroups > 1 ? R::kThreads * R::N : 1;
  __shared__ float lds[L > 64 ? L / 64 * 8 : 1];
  __shared__ float sums[kSum];
  int turn = 0;
  const int lane = threadIdx.x % L;
  const long long group = (long long)blockIdx.x * R::kGroups + threadIdx.x / L;
  const long long r0 = group * run;
  const long long r1 = min(r0 + run, norm_limit(a));
  float sw[R::N], wp[R::N], g[R::N], P[R::N], Q[R::N], t[R::N];
#pragma unroll
  for (int j = 0; j < R::N; ++j) sw[j] = 1.f, wp[j] = 0.f, g[j] = 1.f, P[j] = Q[j] = t[j] = 0.f;
  if (a.scale) R::load(a.scale, sw, lane, a.d);
  if (a.w_post) {
    float w[R::N];
    R::load(a.w_post, w, lane, a.d);
#pragma unroll
    for (int j = 0; j < R::N; ++j) sw[j] *= w[j];
  }
  if (a.w_pre) R::load(a.w_pre, wp, lane, a.d);
  const T* gate = static_cast<const T*>(a.gate);
  T* dgate = static_cast<T*>(o.dgate);
  int seq = -1;
  long long seq_begin = 0, seq_end = -1;
  // the sequence's sum so far: whole, or the part that this run holds
  auto finish = [&](long long upto) {
#pragma unroll
    for (int j = 0; j < R::N; ++j) Q[j] += g[j] * t[j];
    if (dgate) {
      if (seq_begin >= r0 && seq_end <= upto) {
#pragma unroll
        for (int j = 0; j < R::N; ++j) t[j] *= sw[j];
        R::store(dgate + seq * o.lddg, t, lane, a.d);
      } else {
        R::store(o.part_seq + (2 * group + (seq_begin >= r0)) * a.d, t, lane, a.d);
      }
    }
#pragma unroll
    for (int j = 0; j < R::N; ++j) t[j] = 0.f;
  };
  // the next row, where there are registers for it
  constexpr bool kAhead = !ODD && (C == 8 || sizeof(T) == 2);
  typename R::Raw ahead_b, ahead_dr, ahead_r, ahead_dn;
  auto fetch = [&](long long m) {
    ahead_b.load(b + m * ldb, lane, a.d);
    if (dr) ahead_dr.load(dr + m * lddr, lane, a.d);
    if (a.w_pre) {
      ahead_r.load(r + m * ldr, lane, a.d);
      ahead_dn.load(dn + m * lddn, lane, a.d);
    }
  };
  if (kAhead && r0 < r1) fetch(r0);
  for (long long m = r0; m < r1; ++m) {
    float D[R::N], bv[R::N], rv[R::N], nv[R::N];
#pragma unroll
    for (int j = 0; j < R::N; ++j) D[j] = 0.f;
    if constexpr (kAhead) {
      ahead_b.values(bv, lane, a.d);
      if (dr) ahead_dr.values(D, lane, a.d);
      if (a.w_pre) {
        ahead_r.values(rv, lane, a.d);
        ahead_dn.values(nv, lane, a.d);
      }
      if (m + 1 < r1) fetch(m + 1);
    } else {
      R::load(b + m * ldb, bv, lane, a.d);
      if (dr) R::load(dr + m * lddr, D, lane, a.d);
      if (a.w_pre) {
        R::load(r + m * ldr, rv, lane, a.d);
        R::load(dn + m * lddn, nv, lane, a.d);
      }
    }
    if (a.gate) {
      if (!a.gate_off) {
        R::load(gate + m * a.ldg, g, lane, a.d);
      } else if (m >= seq_end) {
        if (seq >= 0) finish(m);
        seq = seq_of(a.gate_off, a.n_seq, m);
        seq_begin = a.gate_off[seq];
        seq_end = a.gate_off[seq + 1];
        R::load(gate + seq * a.ldg, g, lane, a.d);
      }
    }
    float s[3] = {0.f, 0.f, 0.f};
    if (a.w_pre) {
#pragma unroll
      for (int j = 0; j < R::N; ++j) s[0] += rv[j] * rv[j], s[1] += wp[j] * nv[j] * rv[j];
    }
    if (a.w_post) {
#pragma unroll
      for (int j = 0; j < R::N; ++j) s[2] += bv[j] * bv[j];
    }
    if (a.w_pre || a.w_post) group_sum<L, 3>(s, lds, turn);
    if (a.w_pre) {
      const float rho = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
      const float k = rho * rho * (s[1] * a.inv_d);
#pragma unroll
      for (int j = 0; j < R::N; ++j) {
        const float rh = rv[j] * rho;
        D[j] += rho * wp[j] * nv[j] - rh * k;
        P[j] += nv[j] * rh;
      }
    }
    R::store(dx + m * lddx, D, lane, a.d);
    float beta = 1.f, k = 0.f;
    if (a.w_post) {
      beta = 1.0f / sqrtf(s[2] * a.inv_d + a.eps);
      float q[1] = {0.f};
#pragma unroll
      for (int j = 0; j < R::N; ++j) q[0] += D[j] * sw[j] * g[j] * bv[j];
      group_sum<L, 1>(q, lds, turn);
      k = beta * beta * (q[0] * a.inv_d);
    }
    float e[R::N];
#pragma unroll
    for (int j = 0; j < R::N; ++j) {
      const float bh = bv[j] * beta, Tj = D[j] * bh;
      e[j] = beta * (D[j] * sw[j] * g[j]) - bh * k;
      if (a.gate_off) {
        t[j] += Tj;
      } else {
        Q[j] += g[j] * Tj;
        t[j] = Tj * sw[j];
      }
    }
    R::store(db + m * lddb, e, lane, a.d);
    if (dgate && !a.gate_off) R::store(dgate + m * o.lddg, t, lane, a.d);
  }
  if (seq >= 0) finish(r1);
  // the workgroup's groups, added in order
  auto join = [&](float (&v)[R::N], float* out) {
    if constexpr (R::kGroups == 1) {
      R::store(out, v, lane, a.d);
    } else {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < R::N; ++j) sums[j * R::kThreads + threadIdx.x] = v[j];
      __syncthreads();
      if (threadIdx.x < L) {
        for (int q = 1; q < R::kGroups; ++q) {
#pragma unroll
          for (int j = 0; j < R::N; ++j) v[j] += sums[j * R::kThreads + q * L + lane];
        }
        R::store(out, v, lane, a.d);
      }
    }
  };
  float* out = o.partial + (long long)blockIdx.x * 2 * a.d;
  if (a.w_pre) join(P, out);
  if (a.w_post || a.scale) join(Q, out + a.d);
}

// Adds n values `stride` floats apart in order, eight in flight.
__device__ __forceinline__ float sum_apart(const float* p, long long stride, int n) {
  float s = 0.f;
  for (int i = 0; i < n; i += 8) {
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = p[min(i + j, n - 1) * stride];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < n) s += u[j];
  }
  return s;
}

// Adds the partials.  Workgroups with blockIdx.y = 0 (dw_pre) and 1 (Q) own 16 columns; 32 slices of consecutive
// partials are added in order.  The others own SCOLS columns of sequences whose rows lie in several runs (in
// slices, like those), and clear the gradients of sequences without rows.
constexpr int kFinishSlices = 32;
template <typename T, int SCOLS>
__global__ __launch_bounds__(16 * kFinishSlices) void residual_norm_finish_kernel(NormArgs a, NormGradOut o, int parts,
                                                                                  long long run, float* dw_post,
                                                                                  float* dscale, float* dw_pre) {
  if (blockIdx.y < 2) {
    __shared__ float red[kFinishSlices][16];
    const bool pre = blockIdx.y == 0;
    if (pre ? !dw_pre : !dw_post && !dscale) return;
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), sl = threadIdx.x >> 4;
    const int each = (parts + kFinishSlices - 1) / kFinishSlices, p0 = sl * each;
    float s = 0.f;
    if (c < a.d && p0 < parts)
      s = sum_apart(o.partial + ((long long)p0 * 2 + !pre) * a.d + c, 2ll * a.d, min(each, parts - p0));
    red[sl][threadIdx.x & 15] = s;
    __syncthreads();
    if (sl == 0 && c < a.d) {
      s = 0.f;
#pragma unroll
      for (int q = 0; q < kFinishSlices; ++q) s += red[q][threadIdx.x];
      if (pre) {
        dw_pre[c] = s;
      } else {
        if (dw_post) dw_post[c] = s * (a.scale ? a.scale[c] : 1.f);
        if (dscale) dscale[c] = s * (a.w_post ? a.w_post[c] : 1.f);
      }
    }
    return;
  }
  T* dgate = static_cast<T*>(o.dgate);
  const long long limit = norm_limit(a);
  constexpr int kSlices = 16 * kFinishSlices / SCOLS;
  __shared__ float red[kSlices][SCOLS];
  const int cl = threadIdx.x % SCOLS, sl = threadIdx.x / SCOLS, tiles = (a.d + SCOLS - 1) / SCOLS;
  const long long blocks = (long long)gridDim.x * (gridDim.y - 2);
  for (long long i = blockIdx.x + (long long)gridDim.x * (blockIdx.y - 2); i < (long long)a.n_seq * tiles; i += blocks) {
    const long long s = i / tiles;
    const int c = (int)(i % tiles) * SCOLS + cl;
    const long long m0 = max((long long)a.gate_off[s], 0ll), m1 = min((long long)a.gate_off[s + 1], limit);
    const bool empty = m1 <= m0;
    const long long w0 = empty ? 0 : m0 / run, w1 = empty ? 0 : (m1 - 1) / run;
    if (!empty && w0 == w1) continue;   // its run has written it
    const long long each = (w1 - w0 + kSlices - 1) / kSlices, q0 = sl * each;   // of the parts behind the first
    float v = 0.f;
    if (c < a.d && q0 < w1 - w0)
      v = sum_apart(o.part_seq + 2 * (w0 + 1 + q0) * a.d + c, 2ll * a.d, (int)min(each, w1 - w0 - q0));
    red[sl][cl] = v;
    __syncthreads();
    if (sl == 0 && c < a.d) {
      v = empty ? 0.f : o.part_seq[(2 * w0 + 1) * a.d + c];
#pragma unroll
      for (int q = 0; q < kSlices; ++q) v += red[q][cl];
      if (a.scale) v *= a.scale[c];
      if (a.w_post) v *= a.w_post[c];
      dgate[s * o.lddg + c] = (T)v;
    }
    __syncthreads();
  }
}

// Lanes per row of a width (with 8 or 16 columns per lane, the first that hold it), and the workgroups that the
// backward kernel's registers let a CU hold, as which it is launched at most: more would run as a
// second, shorter round and write more partials.
struct NormShape {
  int lanes, resident;
};
static NormShape norm_shape(int d) {
  if (d <= 128) return {16, 3};
  if (d <= 512) return {64, 3};
  if (d <= 1024) return {64, 2};
  if (d <= 2048) return {256, 3};
  if (d <= 4096) return {256, 2};
  return {512, 1};
}

template <typename F>
static void with_shape(int d, F f) {
  if (d <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
  else if (d <= 512) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
  else if (d <= 1024) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
  else if (d <= 2048) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{});
  else if (d <= 4096) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, 512>{}, std::integral_constant<int, 16>{});
}

// Rows per group and workgroups of a launch that aims at `target` workgroups.
struct NormPlan {
  long long run;
  int blocks, groups_per_block;
};
static NormPlan norm_plan(long long rows, int d, int target) {
  const int lanes = norm_shape(d).lanes;
  const int per = lanes < 256 ? 256 / lanes : 1;
  const long long run = rows > 0 ? (rows + (long long)target * per - 1) / ((long long)target * per) : 1;
  const long long groups = (rows + run - 1) / run;
  return {run, (int)((groups + per - 1) / per), per};
}
constexpr int kForwardBlocks = 4096;
static int grad_blocks(int d) { return 256 * norm_shape(d).resident; }

static int check_norm(const janus_norm* p) {
  if (!p || p->rows < 0 || p->rows > INT_MAX || p->d < 1 || !type_known(p->type) || !(p->eps >= 0.f) ||
      !(p->eps <= 3.0e38f) || (p->gate_off && !p->gate) || (p->gate && p->ldg < p->d) || (p->gate_off && p->n_seq < 0))
    return JANUS_EINVAL;
  if (p->d > 8192) return JANUS_EUNSUPPORTED;
  return JANUS_OK;
}

static NormArgs norm_args(const janus_norm* p) {
  return NormArgs{p->rows, p->ldg, p->w_post, p->scale, p->w_pre, p->gate, p->gate_off,
                  p->d, p->gate_off ? p->n_seq : 0, p->eps, 1.0f / (float)p->d};
}

}  // namespace janus

using namespace janus;

extern "C" int janus_residual_norm(const janus_norm* p, const void* x, int64_t ldx, const void* b, int64_t ldb,
                                   void* r, int64_t ldr, void* n, int64_t ldn, void* stream) {
  int rc = check_norm(p);
  if (rc) return rc;
  if (p->rows > 0 && (!x || !b || !r || ldx < p->d || ldb < p->d || ldr < p->d)) return JANUS_EINVAL;
  if (p->rows > 0 && ((p->w_pre && (!n || ldn < p->d)) || (!p->w_pre && n))) return JANUS_EINVAL;
  if (p->rows == 0) return JANUS_OK;
  const bool odd = p->d % (16 / type_bytes(p->type)) != 0;
  const NormArgs a = norm_args(p);
  const NormPlan plan = norm_plan(p->rows, p->d, kForwardBlocks);
  with_type(p->type, [&](auto zero) {
    using T = decltype(zero);
    with_shape(p->d, [&](auto L, auto C) {
      auto go = [&](auto rest) {
        constexpr bool kOdd = decltype(rest)::value;
        using R = Row<T, L.value, C.value, kOdd>;
        hipLaunchKernelGGL((residual_norm_kernel<T, L.value, C.value, kOdd>), dim3(plan.blocks), dim3(R::kThreads), 0,
                           static_cast<hipStream_t>(stream), a, static_cast<const T*>(x), ldx,
                           static_cast<const T*>(b), ldb, static_cast<T*>(r), ldr, static_cast<T*>(n), ldn, plan.run);
      };
      if (odd) go(std::true_type{});
      else go(std::false_type{});
    });
  });
  return launched();
}

extern "C" int64_t janus_residual_norm_grad_workspace(const janus_norm* p) {
  int rc = check_norm(p);
  if (rc) return rc;
  const NormPlan plan = norm_plan(p->rows, p->d, grad_blocks(p->d));
  int64_t floats = (int64_t)plan.blocks * 2 * p->d;
  if (p->gate_off) floats += (int64_t)plan.blocks * plan.groups_per_block * 2 * p->d;
  return 4 * floats + 16;
}

extern "C" int janus_residual_norm_grad(const janus_norm* p, const void* dr, int64_t lddr, const void* dn,
                                        int64_t lddn, const void* r, int64_t ldr, const void* b, int64_t ldb,
                                        void* dx, int64_t lddx, void* db, int64_t lddb, float* dw_post, float* dscale,
                                        float* dw_pre, void* dgate, int64_t lddg, void* work, int64_t work_bytes,
                                        void* stream) {
  int rc = check_norm(p);
  if (rc) return rc;
  if (p->rows > 0 && (!b || !dx || !db || ldb < p->d || lddx < p->d || lddb < p->d || (dr && lddr < p->d)))
    return JANUS_EINVAL;
  if (p->rows > 0 && ((p->w_pre && (!dn || !r || lddn < p->d || ldr < p->d)) || (!p->w_pre && dn))) return JANUS_EINVAL;
  if ((dw_post && !p->w_post) || (dscale && !p->scale) || (dw_pre && !p->w_pre) || (dgate && (!p->gate || lddg < p->d)))
    return JANUS_EINVAL;
  if (!work || reinterpret_cast<uintptr_t>(work) % 16 || work_bytes < janus_residual_norm_grad_workspace(p))
    return JANUS_EINVAL;
  const bool odd = p->d % (16 / type_bytes(p->type)) != 0;
  const NormArgs a = norm_args(p);
  const NormPlan plan = norm_plan(p->rows, p->d, grad_blocks(p->d));
  NormGradOut o{static_cast<float*>(work), nullptr, dgate, lddg};
  o.part_seq = o.partial + (int64_t)plan.blocks * 2 * p->d;
  hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(p->type, [&](auto zero) {
    using T = decltype(zero);
    if (plan.blocks > 0)
      with_shape(p->d, [&](auto L, auto C) {
        auto go = [&](auto rest) {
          constexpr bool kOdd = decltype(rest)::value;
          using R = Row<T, L.value, C.value, kOdd>;
          hipLaunchKernelGGL((residual_norm_grad_kernel<T, L.value, C.value, kOdd>), dim3(plan.blocks),
                             dim3(R::kThreads), 0, st, a, static_cast<const T*>(dr), lddr, static_cast<const T*>(dn),
                             lddn, static_cast<const T*>(r), ldr, static_cast<const T*>(b), ldb, static_cast<T*>(dx),
                             lddx, static_cast<T*>(db), lddb, o, plan.run);
        };
        if (odd) go(std::true_type{});
        else go(std::false_type{});
      });
    const bool sums = dw_post || dscale || dw_pre, seqs = dgate && a.gate_off && a.n_seq > 0;
    if (sums || seqs) {
      const unsigned bx = cdiv(p->d, 16);
      auto finish = [&](auto cols) {
        const long long blocks = seqs ? (long long)a.n_seq * cdiv(p->d, cols.value) : 0;
        hipLaunchKernelGGL((residual_norm_finish_kernel<T, cols.value>),
                           dim3(bx, 2 + cdiv(blocks < 8192 ? blocks : 8192, bx)), dim3(16 * kFinishSlices), 0, st, a, o,
                           plan.blocks, plan.run, dw_post, dscale, dw_pre);
      };
      // many short sequences: few slices of many columns; few long ones: the other way round
      const long long runs = (long long)plan.blocks * plan.groups_per_block;
      if (runs <= 16ll * a.n_seq) finish(std::integral_constant<int, 128>{});
      else finish(std::integral_constant<int, 16>{});
    }
  });
  return launched();
}
