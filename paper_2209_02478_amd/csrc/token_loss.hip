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

// 16 bytes of a row, as they are stored
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xFF80FF80u;        // -inf
  static __device__ __forceinline__ void values(u32x4 u, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ u32x4 bits(const float (&v)[8]) {
    return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
  // element e on: -inf
  static __device__ __forceinline__ u32x4 cut(u32x4 u, int e) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (2 * i >= e) u[i] = kNone;
      else if (2 * i + 1 >= e) u[i] = (u[i] & 0xFFFFu) | (kNone & 0xFFFF0000u);
    }
    return u;
  }
};
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xFF800000u;
  static __device__ __forceinline__ void values(u32x4 u, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
  }
  static __device__ __forceinline__ u32x4 bits(const float (&v)[4]) {
    return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
  static __device__ __forceinline__ u32x4 cut(u32x4 u, int e) {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i >= e) u[i] = kNone;
    return u;
  }
};

constexpr float kLog2e = 1.44269504088896340736f;

// Rows of whole 16-byte chunks on 16-byte addresses, held in registers as they are stored: read once, and with their
// gradient written once.  WAVES waves share a row (one: a block has four rows and no barrier), NCH chunks a lane.
template <typename T, int WAVES, int NCH, int MODE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, WAVES == 16 && NCH <= 8 ? 8 : 4)
void token_rows_held_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels, float* __restrict__ logp,
                            float2* __restrict__ stat, float* __restrict__ slope, T* dlogits, PolicyArgs pa, int rows, int V) {
  constexpr int N = Chunk<T>::N, TPR = 64 * WAVES;
  __shared__ float sm[WAVES], ss[WAVES];
  const int row = WAVES == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  if (row >= rows) return;                              // (a wave with a row to itself)
  const T* x = logits + (int64_t)row * ldl;
  u32x4* g = dlogits ? (u32x4*)(dlogits + (int64_t)row * ldl) : nullptr;
  const int label = labels[row], chunks = (V + N - 1) / N;
  const int64_t wide = ldl / N;
  const u32x4 zero = {0u, 0u, 0u, 0u};
  if (MODE == 0 && slope && tid == 0) slope[row] = 0.f;
  if (!is_scored(label, V)) {
    if (MODE == 0) {
      if (tid == 0) logp[row] = 0.f;
    } else {
      if (tid == 0) ((float4*)pa.rows)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (g) for (int64_t c = tid; c < wide; c += TPR) g[c] = zero;
    }
    return;
  }
  const float picked = ld<T>(x + label);
  u32x4 raw[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = tid + TPR * i;
    raw[i] = u32x4{Chunk<T>::kNone, Chunk<T>::kNone, Chunk<T>::kNone, Chunk<T>::kNone};
    if (c < chunks) raw[i] = ((const u32x4*)x)[c];
  }
  if (V % N) {
#pragma unroll
    for (int i = 0; i < NCH; ++i)
      if (tid + TPR * i == chunks - 1) raw[i] = Chunk<T>::cut(raw[i], V % N);
  }
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    float v[N];
    Chunk<T>::values(raw[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, v[e]);
  }
  m = WAVES == 1 ? wave_max(m) : block_max<WAVES>(m, sm);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    float v[N];
    Chunk<T>::values(raw[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
  }
  s = WAVES == 1 ? wave_sum(s) : block_sum<WAVES>(s, ss);
  const float lp = (picked - m) - logf(s);
  if (MODE == 0) {
    if (tid == 0) {
      logp[row] = lp;
      if (stat) stat[row] = make_float2(m, 1.f / s);
    }
    return;
  }
  float4 kept;
  const float d = policy_token(pa, row, lp, &kept), k = -d / s;
  if (tid == 0) ((float4*)pa.rows)[row] = kept;
  if (!g) return;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = tid + TPR * i;
    if (c >= chunks) break;
    float v[N];
    Chunk<T>::values(raw[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - m) * kLog2e) * k;
    if (label / N == c) {
#pragma unroll
      for (int e = 0; e < N; ++e) if (label % N == e) v[e] += d;
    }
    g[c] = Chunk<T>::bits(v);
  }
  for (int64_t c = chunks + tid; c < wide; c += TPR) g[c] = zero;
}

// chunks a lane and waves a row that hold a row of `chunks`, or none
#define HELD_ROWS(CHUNKS, M)                     \
  if ((CHUNKS) <= 64) { M(1, 1); }               \
  else if ((CHUNKS) <= 128) { M(1, 2); }         \
  else if ((CHUNKS) <= 256) { M(1, 4); }         \
  else if ((CHUNKS) <= 512) { M(4, 2); }         \
  else if ((CHUNKS) <= 1024) { M(4, 4); }        \
  else if ((CHUNKS) <= 2048) { M(8, 4); }        \
  else if ((CHUNKS) <= 4096) { M(16, 4); }       \
  else if ((CHUNKS) <= 7168) { M(16, 7); }       \
  else if ((CHUNKS) <= 8192) { M(16, 8); }       \
  else if ((CHUNKS) <= 16384) { M(16, 16); }

// One block for a row, whatever its length and alignment.
// MODE 0: logp[row]; stat[row] (optional), the row's maximum and the reciprocal of its sum of exponentials; slope[row]
// (optional) = 0, until pair_sums_kernel writes the rows of a pair.
// MODE 1: the policy loss's numbers of the row, and its gradient where dlogits is given (it may be logits).
template <typename T, int MODE>
__global__ __launch_bounds__(kRowThreads) void token_rows_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                 float* __restrict__ logp, float2* __restrict__ stat,
                                                                 float* __restrict__ slope, T* dlogits, PolicyArgs pa, int V) {
  constexpr int NW = kRowThreads / 64;
  __shared__ float sm[NW], ss[NW];
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* x = logits + (int64_t)row * ldl;
  T* g = dlogits ? dlogits + (int64_t)row * ldl : nullptr;
  const int label = labels[row];
  if (MODE == 0 && slope && tid == 0) slope[row] = 0.f;
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

// One block for a pair: the sums of both sequences, in fp64 because the margin is the small difference of four sums
// over a thousand rows; the margin; and d loss / d logp of each of the pair's rows.
constexpr int kPairThreads = 512;
__global__ __launch_bounds__(kPairThreads) void pair_sums_kernel(PreferenceArgs a, const float* __restrict__ logp, float* __restrict__ slope,
                                                                 int first, int T) {
  __shared__ double red[kPairThreads];
  const int p = first + blockIdx.x, tid = threadIdx.x;
  const int2 r[2] = {sequence_rows(a.ends, 2 * p, a.L, T), sequence_rows(a.ends, 2 * p + 1, a.L, T)};
  double h = 0.0;
  for (int k = 0; k < 2; ++k) {
    double s = 0.0;
    for (int i = r[k].x + tid; i < r[k].y; i += kPairThreads) s += (double)logp[i];
    red[tid] = s;
    __syncthreads();
    for (int o = kPairThreads / 2; o > 0; o >>= 1) {
      if (tid < o) red[tid] += red[tid + o];
      __syncthreads();
    }
    s = red[0];
    __syncthreads();
    if (tid == 0) a.seq_logp[2 * p + k] = (float)s;
    s -= (double)a.ref_logp[2 * p + k];
    h = k ? h - s : s;
  }
  const float z = (float)((double)a.beta * h);
  if (tid == 0) a.margin[p] = z;
  if (!slope) return;
  const float d = pair_slope(z, a);
  for (int k = 0; k < 2; ++k)
    for (int i = r[k].x + tid; i < r[k].y; i += kPairThreads) slope[i] = k ? -d : d;
}

// mean loss of the pairs, by one block
__device__ __forceinline__ void mean_pair_loss(const PreferenceArgs& a) {
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
__global__ __launch_bounds__(256) void pair_loss_kernel(PreferenceArgs a) { mean_pair_loss(a); }

// Gradient from what the pass before left of each row, any alignment: one block for a row, and one more, of 256 threads
// like the others, for the mean loss (with_loss).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void pair_grad_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                const float2* __restrict__ stat, const float* __restrict__ slope,
                                                                T* dlogits, PreferenceArgs a, int rows, int V) {
  const int row = rows - 1 - (int)blockIdx.x, tid = threadIdx.x;
  if (row < 0) { mean_pair_loss(a); return; }
  const T* x = logits + (int64_t)row * ldl;
  T* g = dlogits + (int64_t)row * ldl;
  const int label = labels[row];
  const float d = slope[row];
  if (!is_scored(label, V) || d == 0.f) {
    zero_row(g, ldl);
    return;
  }
  const float2 ms = stat[row];
  const float k = -d * ms.y;
  for (int64_t c = tid; c < ldl; c += kRowThreads)
    st<T>(g + c, c < V ? __expf(ld<T>(x + c) - ms.x) * k + (c == label ? d : 0.f) : 0.f);
}

// The same for rows of whole 16-byte chunks: kGradChunks chunks a thread, `parts` blocks a row, the last row first, which
// the pass before has read last.
constexpr int kGradChunks = 4;
template <typename T>
__global__ __launch_bounds__(kRowThreads) void pair_grad_chunk_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                      const float2* __restrict__ stat, const float* __restrict__ slope,
                                                                      T* dlogits, PreferenceArgs a, int rows, int V, int parts) {
  constexpr int N = Chunk<T>::N;
  const int row = rows - 1 - (int)(blockIdx.x / (unsigned)parts);
  if (row < 0) { mean_pair_loss(a); return; }
  const int c0 = (int)(blockIdx.x % (unsigned)parts) * (kRowThreads * kGradChunks) + threadIdx.x, chunks = (V + N - 1) / N, wide = (int)(ldl / N);
  const u32x4* x = (const u32x4*)(logits + (int64_t)row * ldl);
  u32x4* g = (u32x4*)(dlogits + (int64_t)row * ldl);
  const int label = labels[row];
  const float d = slope[row];
  const u32x4 zero = {0u, 0u, 0u, 0u};
  if (!is_scored(label, V) || d == 0.f) {
#pragma unroll
    for (int i = 0; i < kGradChunks; ++i)
      if (c0 + kRowThreads * i < wide) g[c0 + kRowThreads * i] = zero;
    return;
  }
  u32x4 raw[kGradChunks];
#pragma unroll
  for (int i = 0; i < kGradChunks; ++i)
    if (c0 + kRowThreads * i < chunks) raw[i] = x[c0 + kRowThreads * i];
  const float2 ms = stat[row];
  const float k = -d * ms.y;
#pragma unroll
  for (int i = 0; i < kGradChunks; ++i) {
    const int c = c0 + kRowThreads * i;
    if (c < chunks) {
      if (c == chunks - 1 && V % N) raw[i] = Chunk<T>::cut(raw[i], V % N);
      float v[N];
      Chunk<T>::values(raw[i], v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - ms.x) * kLog2e) * k;
      if (label / N == c) {
#pragma unroll
        for (int e = 0; e < N; ++e) if (label % N == e) v[e] += d;
      }
      g[c] = Chunk<T>::bits(v);
    } else if (c < wide) {
      g[c] = zero;
    }
  }
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

// of each row its maximum and the reciprocal of its sum of exponentials, and d loss / d logp
size_t token_loss_workspace_bytes(int T) { return (size_t)(T > 0 ? T : 0) * (sizeof(float2) + sizeof(float)); }

template <typename T>
static bool whole_chunks(const void* a, const void* b, int64_t ldl) {
  return ldl % Chunk<T>::N == 0 && ldl / Chunk<T>::N <= INT32_MAX && (((uintptr_t)a | (uintptr_t)b) & 15) == 0;
}

template <typename T, int MODE>
static void rows_t(const void* logits, int64_t ldl, const int32_t* labels, float* logp, float2* stat, float* slope, void* dlogits,
                   const PolicyArgs& pa, int rows, int V, hipStream_t st) {
  const int chunks = (V + Chunk<T>::N - 1) / Chunk<T>::N;
  const bool held = whole_chunks<T>(logits, dlogits, ldl) && chunks <= 16384;
  for (int r = 0; r < rows; r += kRowsPerLaunch) {
    const int n = std::min(rows - r, kRowsPerLaunch);
    PolicyArgs a = pa;
    if (MODE == 1) {
      a.old_logp += r; a.advantage += r; a.rows += 4 * (int64_t)r;
      if (a.ref_logp) a.ref_logp += r;
      if (a.weight) a.weight += r;
    }
    const T* x = (const T*)logits + r * ldl;
    T* g = dlogits ? (T*)dlogits + r * ldl : nullptr;
    float *lp = logp ? logp + r : nullptr, *sl = slope ? slope + r : nullptr;
    float2* sta = stat ? stat + r : nullptr;
    if (held) {
#define H_(WAVES, NCH)                                                                                                               \
  hipLaunchKernelGGL((token_rows_held_kernel<T, WAVES, NCH, MODE>), dim3(WAVES == 1 ? (n + 3) / 4 : n), dim3(WAVES == 1 ? 256 : 64 * WAVES), \
                     0, st, x, ldl, labels + r, lp, sta, sl, g, a, n, V)
      HELD_ROWS(chunks, H_)
#undef H_
    } else {
      hipLaunchKernelGGL((token_rows_kernel<T, MODE>), dim3(n), dim3(kRowThreads), 0, st, x, ldl, labels + r, lp, sta, sl, g, a, V);
    }
  }
}

void token_logprob(int dtype, const void* logits, int64_t ldl, const int32_t* labels, float* logp, int T, int V, void* workspace, hipStream_t st) {
  (void)workspace;
  if (dtype == BF16) rows_t<bf16_t, 0>(logits, ldl, labels, logp, nullptr, nullptr, nullptr, PolicyArgs(), T, V, st);
  else rows_t<float, 0>(logits, ldl, labels, logp, nullptr, nullptr, nullptr, PolicyArgs(), T, V, st);
}

template <typename T>
static void preference_t(const void* logits, int64_t ldl, const int32_t* labels, const PreferenceArgs& a, void* dlogits, float* logp, int rows,
                         int V, void* workspace, hipStream_t st) {
  float2* stat = (float2*)workspace;
  float* slope = dlogits ? (float*)(stat + rows) : nullptr;
  rows_t<T, 0>(logits, ldl, labels, logp, stat, slope, nullptr, PolicyArgs(), rows, V, st);
  hipLaunchKernelGGL(pair_sums_kernel, dim3(a.pairs), dim3(kPairThreads), 0, st, a, logp, slope, 0, rows);
  if (!dlogits || rows <= 0) {
    hipLaunchKernelGGL(pair_loss_kernel, dim3(1), dim3(256), 0, st, a);
    return;
  }
  const bool vec = whole_chunks<T>(logits, dlogits, ldl);
  const int64_t per_block = (int64_t)kRowThreads * kGradChunks, parts = vec ? (ldl / Chunk<T>::N + per_block - 1) / per_block : 1;
  const int most = (int)std::max<int64_t>(1, ((int64_t)kRowsPerLaunch * 8) / parts);
  for (int r = 0; r < rows; r += most) {
    const int n = std::min(rows - r, most);
    const int extra = r + n == rows;                    // the mean loss, once
    const T* x = (const T*)logits + r * ldl;
    T* g = (T*)dlogits + r * ldl;
    if (vec)
      hipLaunchKernelGGL(pair_grad_chunk_kernel<T>, dim3((unsigned)(n * parts + extra)), dim3(kRowThreads), 0, st, x, ldl, labels + r, stat + r,
                         slope + r, g, a, n, V, (int)parts);
    else
      hipLaunchKernelGGL(pair_grad_kernel<T>, dim3(n + extra), dim3(kRowThreads), 0, st, x, ldl, labels + r, stat + r, slope + r, g, a, n, V);
  }
}

void preference_loss(int dtype, const void* logits, int64_t ldl, const int32_t* labels, const PreferenceArgs& a, void* dlogits, float* logp,
                     int T, int V, void* workspace, hipStream_t st) {
  if (dtype == BF16) preference_t<bf16_t>(logits, ldl, labels, a, dlogits, logp, T, V, workspace, st);
  else preference_t<float>(logits, ldl, labels, a, dlogits, logp, T, V, workspace, st);
}

void policy_loss(int dtype, const void* logits, int64_t ldl, const int32_t* labels, const PolicyArgs& a, void* dlogits, int T, int V,
                 void* workspace, hipStream_t st) {
  (void)workspace;
  if (dtype == BF16) rows_t<bf16_t, 1>(logits, ldl, labels, nullptr, nullptr, nullptr, dlogits, a, T, V, st);
  else rows_t<float, 1>(logits, ldl, labels, nullptr, nullptr, nullptr, dlogits, a, T, V, st);
  hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(1024), 0, st, (const float4*)a.rows, T, a.stats);
}

}  // namespace mk
