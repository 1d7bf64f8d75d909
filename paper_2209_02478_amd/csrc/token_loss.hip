// Losses on the log-probabilities of given tokens, over rows of logits: the log-probabilities alone, a preference
// loss on pairs of sequences, a clipped policy loss with a KL term; the losses with their gradient on the logits.
//
// With x a row's logits, y its label and p = softmax(x):  logp = x_y - log sum_v exp(x_v),  and for a loss that is a
// function of the log-probabilities  dloss/dx_v = (dloss/dlogp) (1[v = y] - p_v).  A row is not scored when its
// label lies outside [0, V): its logits are not read, its log-probability counts as 0, its gradient is written as zeros.
// Maxima, sums of exponentials and everything behind them are fp32, sums over the rows of a sequence fp64; the one
// rounding to bf16 is the gradient's, when it is stored.
#include "device_common.h"

#include <algorithm>

namespace mk {

constexpr int kRowThreads = 256;

// sum (maximum) over the block, in every thread; a fixed order
template <int NW>
__device__ __forceinline__ float block_max(float v, float* s) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v = fmaxf(v, s[w]);
  return v;
}
template <int NW>
__device__ __forceinline__ float block_sum(float v, float* s) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += s[w];
  return v;
}

__device__ __forceinline__ bool is_scored(int label, int V) { return (unsigned)label < (unsigned)V; }

// what the policy loss makes of one token: d loss / d logp, and the four numbers that are kept of its row
__device__ __forceinline__ float policy_token(const PolicyArgs& a, int row, float logp, float4* kept) {
  const float w = a.scale * (a.weight ? a.weight[row] : 1.f);
  *kept = make_float4(logp, 0.f, 0.f, 0.f);
  if (w == 0.f) return 0.f;                             // left out, whatever its other numbers are
  const float A = a.advantage[row], ratio = expf(logp - a.old_logp[row]);
  const float gain = ratio * A, bound = fminf(fmaxf(ratio, a.ratio_low), a.ratio_high) * A;
  const bool clipped = gain > bound;                    // the bound holds the gain back: it has no gradient
  float loss = clipped ? -bound : -gain, d = clipped ? 0.f : -gain;
  if (a.ref_logp) {
    const float r = a.ref_logp[row] - logp, e = expm1f(r), kl = e - r;
    kept->z = w * kl;
    if (a.kl_weight != 0.f) { loss += a.kl_weight * kl; d -= a.kl_weight * e; }
  }
  kept->y = w * loss;
  kept->w = clipped ? w : 0.f;
  return w * d;
}

template <typename T>
__device__ __forceinline__ void zero_row(T* g, int64_t ldl) {
  for (int64_t c = threadIdx.x; c < ldl; c += blockDim.x) st<T>(g + c, 0.f);
}

// One block for a row, whatever its length and alignment.
// MODE 0: logp[row], and where stat is given the row's maximum and the reciprocal of its sum of exponentials.
// MODE 1: the policy loss's numbers of the row, and its gradient where dlogits is given (it may be logits).
template <typename T, int MODE>
__global__ __launch_bounds__(kRowThreads) void token_rows_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                 float* __restrict__ logp, float2* __restrict__ stat, T* dlogits,
                                                                 PolicyArgs pa, int V) {
  constexpr int NW = kRowThreads / 64;
  __shared__ float sm[NW], ss[NW];
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* x = logits + (int64_t)row * ldl;
  T* g = dlogits ? dlogits + (int64_t)row * ldl : nullptr;
  const int label = labels[row];
  if (!is_scored(label, V)) {
    if (MODE == 0) {
      if (tid == 0) logp[row] = 0.f;
    } else {
      if (tid == 0) ((float4*)pa.rows)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (g) zero_row(g, ldl);
    }
    return;
  }
  float m = -INFINITY;
  for (int c = tid; c < V; c += kRowThreads) m = fmaxf(m, ld<T>(x + c));
  m = block_max<NW>(m, sm);
  float s = 0.f;
  for (int c = tid; c < V; c += kRowThreads) s += __expf(ld<T>(x + c) - m);
  s = block_sum<NW>(s, ss);
  const float lp = (ld<T>(x + label) - m) - logf(s);
  if (MODE == 0) {
    if (tid == 0) {
      logp[row] = lp;
      if (stat) stat[row] = make_float2(m, 1.f / s);
    }
    return;
  }
  float4 kept;
  const float d = policy_token(pa, row, lp, &kept);
  if (tid == 0) ((float4*)pa.rows)[row] = kept;
  if (!g) return;
  const float k = -d / s;
  __syncthreads();                                      // (in place: every thread has read the label's logit)
  for (int64_t c = tid; c < ldl; c += kRowThreads)
    st<T>(g + c, c < V ? __expf(ld<T>(x + c) - m) * k + (c == label ? d : 0.f) : 0.f);
}

// first row and end of sequence s, inside [0, T] whatever ends holds
__device__ __forceinline__ int2 sequence_rows(const int32_t* ends, int s, int L, int T) {
  const int64_t a = ends ? (s ? ends[s - 1] : 0) : (int64_t)s * L, b = ends ? ends[s] : (int64_t)(s + 1) * L;
  const int first = (int)min(max(a, (int64_t)0), (int64_t)T);
  return make_int2(first, (int)min(max(b, (int64_t)first), (int64_t)T));
}

// sequence that a row belongs to; `sequences` for a row behind the last one
__device__ __forceinline__ int sequence_of(const int32_t* ends, int row, int L, int sequences) {
  if (!ends) return row / L;
  int lo = 0, hi = sequences;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > row) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__device__ __forceinline__ float softplus(float z) { return fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))); }

// loss of a pair with margin z; 0 times an infinite term is left out
__device__ __forceinline__ float pair_loss(float z, float smoothing) {
  float l = 0.f;
  if (smoothing < 1.f) l += (1.f - smoothing) * softplus(-z);
  if (smoothing > 0.f) l += smoothing * softplus(z);
  return l;
}
// d loss / d (log-probability of the pair's chosen sequence); the rejected one's is its negative
__device__ __forceinline__ float pair_slope(float z, const PreferenceArgs& a) {
  return -a.beta / (float)a.pairs * ((1.f - a.smoothing) / (1.f + expf(z)) - a.smoothing / (1.f + expf(-z)));
}

// One block for a pair: the sums of both sequences, in fp64 because the margin is the small difference of
// four sums over a thousand rows, and the margin.
__global__ __launch_bounds__(256) void pair_sums_kernel(PreferenceArgs a, const float* __restrict__ logp, int T) {
  __shared__ double red[256];
  const int p = blockIdx.x, tid = threadIdx.x;
  double h = 0.0;
  for (int k = 0; k < 2; ++k) {
    const int2 r = sequence_rows(a.ends, 2 * p + k, a.L, T);
    double s = 0.0;
    for (int i = r.x + tid; i < r.y; i += 256) s += (double)logp[i];
    red[tid] = s;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
      if (tid < o) red[tid] += red[tid + o];
      __syncthreads();
    }
    s = red[0];
    __syncthreads();
    if (tid == 0) a.seq_logp[2 * p + k] = (float)s;
    s -= (double)a.ref_logp[2 * p + k];
    h = k ? h - s : s;
  }
  if (tid == 0) a.margin[p] = (float)((double)a.beta * h);
}

__global__ __launch_bounds__(256) void pair_loss_kernel(PreferenceArgs a) {
  __shared__ double red[256];
  const int tid = threadIdx.x;
  double s = 0.0;
  for (int p = tid; p < a.pairs; p += 256) s += (double)pair_loss(a.margin[p], a.smoothing);
  red[tid] = s;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (tid < o) red[tid] += red[tid + o];
    __syncthreads();
  }
  if (tid == 0) *a.loss = (float)(red[0] / (double)a.pairs);
}

// gradient of the preference loss, one block for a row
template <typename T>
__global__ __launch_bounds__(kRowThreads) void pair_grad_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                const float2* __restrict__ stat, T* dlogits, PreferenceArgs a, int V) {
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* x = logits + (int64_t)row * ldl;
  T* g = dlogits + (int64_t)row * ldl;
  const int label = labels[row], s = sequence_of(a.ends, row, a.L, 2 * a.pairs);
  if (!is_scored(label, V) || s >= 2 * a.pairs) {
    zero_row(g, ldl);
    return;
  }
  const float slope = pair_slope(a.margin[s >> 1], a), d = s & 1 ? -slope : slope;
  const float2 ms = stat[row];
  const float k = -d * ms.y;
  for (int64_t c = tid; c < ldl; c += kRowThreads)
    st<T>(g + c, c < V ? __expf(ld<T>(x + c) - ms.x) * k + (c == label ? d : 0.f) : 0.f);
}

// loss, KL term and clipped share over all rows
__global__ __launch_bounds__(1024) void policy_stats_kernel(const float4* __restrict__ rows, int T, float* __restrict__ stats) {
  __shared__ double red[3][1024];
  const int tid = threadIdx.x;
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = tid; i < T; i += 1024) {
    const float4 r = rows[i];
    s[0] += (double)r.y; s[1] += (double)r.z; s[2] += (double)r.w;
  }
  for (int k = 0; k < 3; ++k) red[k][tid] = s[k];
  __syncthreads();
  for (int o = 512; o > 0; o >>= 1) {
    if (tid < o) for (int k = 0; k < 3; ++k) red[k][tid] += red[k][tid + o];
    __syncthreads();
  }
  if (tid < 3) stats[tid] = (float)red[tid][0];
}

// ---------------------------------------------------------------- launchers
// rows of one launch: the threads of a grid are counted in 32 bits
constexpr int kRowsPerLaunch = 1 << 20;

size_t token_loss_workspace_bytes(int T) { return (size_t)(T > 0 ? T : 0) * sizeof(float2); }

template <typename T, int MODE>
static void rows_t(const void* logits, int64_t ldl, const int32_t* labels, float* logp, float2* stat, void* dlogits, const PolicyArgs& pa,
                   int rows, int V, hipStream_t st) {
  for (int r = 0; r < rows; r += kRowsPerLaunch) {
    PolicyArgs a = pa;
    if (MODE == 1) {
      a.old_logp += r; a.advantage += r; a.rows += 4 * (int64_t)r;
      if (a.ref_logp) a.ref_logp += r;
      if (a.weight) a.weight += r;
    }
    hipLaunchKernelGGL((token_rows_kernel<T, MODE>), dim3(std::min(rows - r, kRowsPerLaunch)), dim3(kRowThreads), 0, st,
                       (const T*)logits + r * ldl, ldl, labels + r, logp ? logp + r : nullptr, stat ? stat + r : nullptr,
                       dlogits ? (T*)dlogits + r * ldl : nullptr, a, V);
  }
}

void token_logprob(int dtype, const void* logits, int64_t ldl, const int32_t* labels, float* logp, int T, int V, void* workspace, hipStream_t st) {
  (void)workspace;
  if (dtype == BF16) rows_t<bf16_t, 0>(logits, ldl, labels, logp, nullptr, nullptr, PolicyArgs(), T, V, st);
  else rows_t<float, 0>(logits, ldl, labels, logp, nullptr, nullptr, PolicyArgs(), T, V, st);
}

template <typename T>
static void preference_t(const void* logits, int64_t ldl, const int32_t* labels, const PreferenceArgs& a, void* dlogits, float* logp, int rows,
                         int V, void* workspace, hipStream_t st) {
  float2* stat = (float2*)workspace;
  rows_t<T, 0>(logits, ldl, labels, logp, stat, nullptr, PolicyArgs(), rows, V, st);
  hipLaunchKernelGGL(pair_sums_kernel, dim3(a.pairs), dim3(256), 0, st, a, logp, rows);
  hipLaunchKernelGGL(pair_loss_kernel, dim3(1), dim3(256), 0, st, a);
  if (dlogits && rows > 0)
    hipLaunchKernelGGL(pair_grad_kernel<T>, dim3(rows), dim3(kRowThreads), 0, st, (const T*)logits, ldl, labels, stat, (T*)dlogits, a, V);
}

void preference_loss(int dtype, const void* logits, int64_t ldl, const int32_t* labels, const PreferenceArgs& a, void* dlogits, float* logp,
                     int T, int V, void* workspace, hipStream_t st) {
  if (dtype == BF16) preference_t<bf16_t>(logits, ldl, labels, a, dlogits, logp, T, V, workspace, st);
  else preference_t<float>(logits, ldl, labels, a, dlogits, logp, T, V, workspace, st);
}

void policy_loss(int dtype, const void* logits, int64_t ldl, const int32_t* labels, const PolicyArgs& a, void* dlogits, int T, int V,
                 void* workspace, hipStream_t st) {
  (void)workspace;
  if (dtype == BF16) rows_t<bf16_t, 1>(logits, ldl, labels, nullptr, nullptr, dlogits, a, T, V, st);
  else rows_t<float, 1>(logits, ldl, labels, nullptr, nullptr, dlogits, a, T, V, st);
  hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(1024), 0, st, (const float4*)a.rows, T, a.stats);
}

}  // namespace mk
