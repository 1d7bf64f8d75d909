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

// sum of 64 * WAVES threads' numbers, in the first wave's lanes, by one barrier; red: WAVES * 64 places
template <int WAVES>
__device__ __forceinline__ double first_wave_sum(double v, double* red, int tid) {
  red[tid] = v;
  __syncthreads();
  v = 0.0;
  if (tid < 64) {
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += red[64 * w + tid];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  }
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

// 16 bytes of a row, as they are stored
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct Packed;
template <> struct Packed<bf16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t kNone = 0xFF80FF80u;        // -inf
  static __device__ __forceinline__ void values(u32x4 u, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ u32x4 bits(const float (&v)[8]) {
    return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};
template <> struct Packed<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kNone = 0xFF800000u;
  static __device__ __forceinline__ void values(u32x4 u, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
  }
  static __device__ __forceinline__ u32x4 bits(const float (&v)[4]) {
    return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
constexpr float kLog2e = 1.44269504088896340736f;

// elements from e on are -inf
template <typename T>
__device__ __forceinline__ u32x4 cut_chunk(u32x4 u, int e) {
  constexpr int per = 4 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (per * i >= e) u[i] = Packed<T>::kNone;
    else if (per == 2 && 2 * i + 1 == e) u[i] = (u[i] & 0xFFFFu) | (Packed<T>::kNone & 0xFFFF0000u);
  }
  return u;
}
// Chunks lie on 16-byte addresses whatever the row's own: chunk c of row x has the columns from c * N - shift(x) on.  A
// row's first and last chunk may reach beyond it: there elements are read and written one by one, and none outside.
template <typename T>
__device__ __forceinline__ int shift_of(const T* x) { return (int)(((uintptr_t)x & 15) / sizeof(T)); }
// a chunk from column `col` on that reaches beyond [0, V), where it is -inf
template <typename T>
__device__ __forceinline__ u32x4 load_edge(const T* x, int64_t col, int V) {
  constexpr int N = Packed<T>::N;
  float v[N];
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = col + e >= 0 && col + e < V ? ld<T>(x + col + e) : -INFINITY;
  return Packed<T>::bits(v);
}
// columns of [V, ldl) are written as zeros, none outside [0, ldl)
template <typename T>
__device__ __forceinline__ void store_edge(T* g, int64_t col, int V, int64_t ldl, const float (&v)[Packed<T>::N]) {
#pragma unroll
  for (int e = 0; e < Packed<T>::N; ++e)
    if (col + e >= 0 && col + e < ldl) st<T>(g + col + e, col + e < V ? v[e] : 0.f);
}
// gradient of a chunk: softmax times k, and d on the label, element `in` (any other number: not in this chunk)
template <typename T>
__device__ __forceinline__ void chunk_gradient(u32x4 u, float m, float k, float d, int64_t in, float (&v)[Packed<T>::N]) {
  constexpr int N = Packed<T>::N;
  Packed<T>::values(u, v);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - m) * kLog2e) * k;
  if (in >= 0 && in < N) {
#pragma unroll
    for (int e = 0; e < N; ++e) if (e == in) v[e] += d;
  }
}
// columns [from, to) of a row are zeros, by `threads` threads
template <typename T>
__device__ __forceinline__ void zero_columns(T* g, int64_t from, int64_t to, int tid, int threads) {
  constexpr int N = Packed<T>::N;
  const int64_t body = min(to, from + (N - shift_of(g + from)) % N), end = body + (to - body) / N * N;
  if (from + tid < body) st<T>(g + from + tid, 0.f);     // (fewer than N columns)
  for (int64_t c = body + (int64_t)tid * N; c < end; c += (int64_t)threads * N)
    __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, (u32x4*)(g + c));
  if (end + tid < to) st<T>(g + end + tid, 0.f);
}
// the next pass over held chunks converts them anew: kept as floats they would take twice the registers
__device__ __forceinline__ void keep_packed(u32x4& u) { asm volatile("" : "+v"(u)); }

// A row is held in registers as it is stored: read once, and with its gradient written once.  WAVES waves share a row
// (one: a block has four rows and no barrier), NCH chunks a lane.  EVEN: every row, and that of the gradient, begins and
// ends on a chunk.  PAST: the row is read past the caches.  Gradients always are written past them: what reads them next is
// a matrix product over all rows.
// MODE 0: logp[row]; stat[row] (optional), the row's maximum and the reciprocal of its sum of exponentials; slope[row]
// (optional) = 0, until pair_sums_kernel writes the rows of a pair.
// MODE 1: the policy loss's numbers of the row, and its gradient where dlogits is given (it may be logits).
// Bound by memory.  16384 rows of 50257 in bf16, a quarter of them not scored: 182 us (6.8 TB/s) reading, 516 (5.6) with the
// gradient; through the caches 209 and 548, as floats in registers 239 and 587.  8192 rows of 50257 columns and no padding:
// 138 us and 309, against 133 and 303 with rows on 16-byte addresses; gradient on other addresses than the logits 613.
template <typename T, int WAVES, int NCH, int MODE, bool PAST, bool EVEN>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES, (WAVES == 16 && NCH <= 9) || (WAVES == 1 && NCH <= 4) ? 8 : 4)
void token_rows_held_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels, float* __restrict__ logp,
                            float2* __restrict__ stat, float* __restrict__ slope, T* dlogits, PolicyArgs pa, int rows, int V) {
  constexpr int N = Packed<T>::N, TPR = 64 * WAVES;
  __shared__ float sm[WAVES], ss[WAVES];
  const int row = WAVES == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  if (row >= rows) return;                              // (a wave with a row to itself)
  const T* x = logits + (int64_t)row * ldl;
  T* g = dlogits ? dlogits + (int64_t)row * ldl : nullptr;
  const int label = labels[row];
  if (MODE == 0 && slope && tid == 0) slope[row] = 0.f;
  if (!is_scored(label, V)) {
    if (MODE == 0) {
      if (tid == 0) logp[row] = 0.f;
    } else {
      if (tid == 0) ((float4*)pa.rows)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (g) zero_columns(g, 0, ldl, tid, TPR);
    }
    return;
  }
  const float picked = ld<T>(x + label);
  // chunks [whole0, whole1) lie inside [0, V); chunk 0 where whole0 is 1, and chunk whole1 (tail), where there is one, reach
  // beyond it; a row inside one chunk is its tail alone
  const int shift = EVEN ? 0 : shift_of(x), whole1 = (shift + V) / N, whole0 = shift && whole1 ? 1 : 0;
  const int tail = (shift + V) % N ? whole1 : -1, chunks = whole1 + (tail >= 0);
  const int loaded = EVEN ? chunks : whole1;
  const u32x4* xc = (const u32x4*)(x - shift);
  constexpr uint32_t none = Packed<T>::kNone;
  u32x4 raw[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = tid + TPR * i;
    raw[i] = u32x4{none, none, none, none};
    if (c >= whole0 && c < loaded) raw[i] = PAST ? __builtin_nontemporal_load(xc + c) : xc[c];
  }
  if (EVEN) {
    if (tail >= 0) {
#pragma unroll
      for (int i = 0; i < NCH; ++i)
        if (tid + TPR * i == tail) raw[i] = cut_chunk<T>(raw[i], V % N);
    }
  } else {
    if (whole0 && tid == 0) raw[0] = load_edge(x, -shift, V);
    if (tail >= 0 && tail % TPR == tid) {
      const u32x4 edge = load_edge(x, (int64_t)tail * N - shift, V);
#pragma unroll
      for (int i = 0; i < NCH; ++i) if (tid + TPR * i == tail) raw[i] = edge;
    }
  }
  // a wave leaves out chunks that none of its lanes has
  const int wave_first = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid & ~63);
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    if (wave_first + TPR * i < chunks) {
      float v[N];
      Packed<T>::values(raw[i], v);
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, v[e]);
    }
  }
  m = WAVES == 1 ? wave_max(m) : block_max<WAVES>(m, sm);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    keep_packed(raw[i]);
    if (wave_first + TPR * i < chunks) {
      float v[N];
      Packed<T>::values(raw[i], v);
#pragma unroll
      for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
    }
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
  if (d == 0.f) { zero_columns(g, 0, ldl, tid, TPR); return; }   // left out, whatever its logits are, or held back by the clip
  const int at = label + shift;                         // the label's element, counted from chunk 0
  float v[N];
  if (EVEN) {
    u32x4* gc = (u32x4*)g;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = tid + TPR * i;
      keep_packed(raw[i]);
      if (c < chunks) {
        chunk_gradient<T>(raw[i], m, k, d, at - c * N, v);
        if (c == tail) {
#pragma unroll
          for (int e = 0; e < N; ++e) if (e >= V % N) v[e] = 0.f;
        }
        __builtin_nontemporal_store(Packed<T>::bits(v), gc + c);
      }
    }
  } else {
    const bool aligned = shift_of(g) == shift;          // else the gradient's chunks are not the logits': element by element
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = tid + TPR * i;
      keep_packed(raw[i]);
      if (c < chunks) {
        chunk_gradient<T>(raw[i], m, k, d, at - c * N, v);
        if (aligned && c >= whole0 && c < whole1) __builtin_nontemporal_store(Packed<T>::bits(v), (u32x4*)(g - shift) + c);
        else store_edge(g, (int64_t)c * N - shift, V, ldl, v);
      }
    }
  }
  const int64_t behind = (int64_t)chunks * N - shift;
  if (behind < ldl) zero_columns(g, behind, ldl, tid, TPR);
}

// WAVES and NCH by the chunks of a row: as few waves as hold it with nine chunks a lane, because fewer chunks a lane leave too few
// bytes on the way to memory (policy loss, 16384 rows of 4000 in bf16: 79 us with 4 x 4, 54 with 1 x 9; of 15000: 259 with 8 x 4,
// 174 with 4 x 9), and registers of no more than 64 a lane, for two rows of 16 waves a unit; more chunks where 16 waves need them.
// Reading alone, 8 x 13 is ahead of 16 x 7 (12288 rows of 50257: 183 us against 190); with the gradient behind it, it is not (550
// against 517).
#define HELD_ROWS(CHUNKS, M)                                 \
  if ((CHUNKS) <= 64) { M(1, 1) }                            \
  else if ((CHUNKS) <= 128) { M(1, 2) }                      \
  else if ((CHUNKS) <= 256) { M(1, 4) }                      \
  else if ((CHUNKS) <= 576) { M(1, 9) }                      \
  else if ((CHUNKS) <= 1152) { M(2, 9) }                     \
  else if ((CHUNKS) <= 2304) { M(4, 9) }                     \
  else if ((CHUNKS) <= 4608) { M(8, 9) }                     \
  else if (MODE == 0 && (CHUNKS) <= 6656) { M(8, 13) }       \
  else if ((CHUNKS) <= 7168) { M(16, 7) }                    \
  else if ((CHUNKS) <= 9216) { M(16, 9) }                    \
  else if ((CHUNKS) <= 13312) { M(16, 13) }                  \
  else { M(16, 16) }
constexpr int kMostChunks = 16384;

// Rows too long to be held: one block for a row, a running maximum and sum in each thread over its chunks, and for the gradient a
// second pass over them, out of the last cache.  MODE as above.  4096 rows of 200000 in bf16: 290 us (5.6 TB/s) and 700 (4.7).
constexpr int kLongThreads = 1024, kLongAhead = 4;
template <typename T, int MODE>
__global__ __launch_bounds__(kLongThreads) void token_rows_long_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                       float* __restrict__ logp, float2* __restrict__ stat,
                                                                       float* __restrict__ slope, T* dlogits, PolicyArgs pa, int V) {
  constexpr int N = Packed<T>::N, NW = kLongThreads / 64;
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
      if (g) zero_columns(g, 0, ldl, tid, kLongThreads);
    }
    return;
  }
  const float picked = ld<T>(x + label);
  const int shift = shift_of(x);
  const int64_t step = (int64_t)kLongThreads * N, first = (int64_t)tid * N - shift;   // columns
  u32x4 raw[kLongAhead];
  auto load = [&](int64_t col) {
#pragma unroll
    for (int i = 0; i < kLongAhead; ++i) {
      const int64_t c = col + i * step;
      raw[i] = c >= 0 && c + N <= V ? *(const u32x4*)(x + c) : load_edge(x, c, V);
    }
  };
  float m = -INFINITY, s = 0.f;
  for (int64_t col = first; col < V; col += kLongAhead * step) {
    load(col);
#pragma unroll
    for (int i = 0; i < kLongAhead; ++i) {
      float v[N], top = m;
      Packed<T>::values(raw[i], v);
#pragma unroll
      for (int e = 0; e < N; ++e) top = fmaxf(top, v[e]);
      if (top > m) { s *= __builtin_amdgcn_exp2f((m - top) * kLog2e); m = top; }
#pragma unroll
      for (int e = 0; e < N; ++e) s += v[e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
    }
  }
  const float own = m;
  m = block_max<NW>(m, sm);
  s = block_sum<NW>(own == -INFINITY && s == 0.f ? 0.f : s * __builtin_amdgcn_exp2f((own - m) * kLog2e), ss);
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
  if (d == 0.f) { zero_columns(g, 0, ldl, tid, kLongThreads); return; }
  const bool aligned = shift_of(g) == shift;
  for (int64_t col = first; col < V; col += kLongAhead * step) {
    load(col);
#pragma unroll
    for (int i = 0; i < kLongAhead; ++i) {
      const int64_t c = col + i * step;
      float v[N];
      chunk_gradient<T>(raw[i], m, k, d, label - c, v);
      if (aligned && c >= 0 && c + N <= V) __builtin_nontemporal_store(Packed<T>::bits(v), (u32x4*)(g + c));
      else if (c < V) store_edge(g, c, V, ldl, v);
    }
  }
  const int64_t behind = ((int64_t)shift + V + N - 1) / N * N - shift;
  if (behind < ldl) zero_columns(g, behind, ldl, tid, kLongThreads);
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

// Margin of pair p by one wave, in every lane, and the sums of its sequences where seq is given.  Sums are fp64 because the
// margin is the small difference of four of them over up to a thousand rows.
__device__ __forceinline__ float wave_margin(const PreferenceArgs& a, const float* logp, int p, int T, float* seq) {
  const int lane = threadIdx.x & 63;
  double h = 0.0;
  for (int k = 0; k < 2; ++k) {
    const int2 r = sequence_rows(a.ends, 2 * p + k, a.L, T);
    double s = 0.0;
    for (unsigned i = r.x + lane; i < (unsigned)r.y; i += 4 * 64) {   // (unsigned: a step behind 2^31 - 1 rows is no int)
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = i + 64 * u < (unsigned)r.y ? logp[i + 64 * u] : 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) s += (double)v[u];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (seq && lane == 0) seq[2 * p + k] = (float)s;
    s -= (double)a.ref_logp[2 * p + k];
    h = k ? h - s : s;
  }
  return (float)((double)a.beta * h);
}
// the pairs' sums, margins and mean loss, by one block of kRowThreads, a wave for a pair
__device__ __forceinline__ void few_pairs_loss(const PreferenceArgs& a, const float* logp, int T) {
  constexpr int NW = kRowThreads / 64;
  __shared__ double part[NW];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  double s = 0.0;
  for (int p = wave; p < a.pairs; p += NW) {
    const float z = wave_margin(a, logp, p, T, a.seq_logp);
    if (lane == 0) a.margin[p] = z;
    s += (double)pair_loss(z, a.smoothing);
  }
  if (lane == 0) part[wave] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = 0.0;
  for (int w = 0; w < NW; ++w) s += part[w];
  *a.loss = (float)(s / (double)a.pairs);
}
__global__ __launch_bounds__(kRowThreads) void few_pairs_kernel(PreferenceArgs a, const float* __restrict__ logp, int T) {
  few_pairs_loss(a, logp, T);
}
constexpr int kFewPairs = 8;                            // (their ends fit the lanes of a wave)

// One block for a pair, half of its threads for each sequence: the sums (fp64, as above), the margin, and d loss / d logp of each
// of the pair's rows.
constexpr int kPairThreads = 1024;
__global__ __launch_bounds__(kPairThreads) void pair_sums_kernel(PreferenceArgs a, const float* __restrict__ logp, float* __restrict__ slope,
                                                                 int T) {
  constexpr int half = kPairThreads / 2;
  __shared__ double red[2][half], sum[2];
  const int p = blockIdx.x, k = threadIdx.x / half, tid = threadIdx.x % half;
  const int2 r = sequence_rows(a.ends, 2 * p + k, a.L, T);
  double s = 0.0;
  for (unsigned i = r.x + tid; i < (unsigned)r.y; i += half) s += (double)logp[i];
  s = first_wave_sum<half / 64>(s, red[k], tid);
  if (tid == 0) {
    sum[k] = s;
    a.seq_logp[2 * p + k] = (float)s;
  }
  __syncthreads();
  const double h = (sum[0] - (double)a.ref_logp[2 * p]) - (sum[1] - (double)a.ref_logp[2 * p + 1]);
  const float z = (float)((double)a.beta * h);
  if (threadIdx.x == 0) a.margin[p] = z;
  if (!slope) return;
  const float d = pair_slope(z, a);
  for (unsigned i = r.x + tid; i < (unsigned)r.y; i += half) slope[i] = k ? -d : d;
}

// mean loss of the pairs, by one block of kRowThreads
__device__ __forceinline__ void mean_pair_loss(const PreferenceArgs& a) {
  __shared__ double red[kRowThreads];
  double s = 0.0;
  for (int p = threadIdx.x; p < a.pairs; p += kRowThreads) s += (double)pair_loss(a.margin[p], a.smoothing);
  s = first_wave_sum<kRowThreads / 64>(s, red, threadIdx.x);
  if (threadIdx.x == 0) *a.loss = (float)(s / (double)a.pairs);
}
__global__ __launch_bounds__(kRowThreads) void pair_loss_kernel(PreferenceArgs a) { mean_pair_loss(a); }

// Gradient from what the pass before left of each row: grad_chunks() chunks a thread, `parts` blocks a row, the last row first,
// because the pass before has read it last.  One more block, behind all rows, for the mean loss.  Bound by memory: 16384 rows of
// 50257 in bf16 530-550 us, 6.1 TB/s.  SUMS: no kernel has summed the pairs; every block makes its pair's margin itself while its
// logits are on their way, and the block behind all rows writes the pairs' numbers.
constexpr int grad_chunks(bool past) { return past ? 1 : 2; }
template <typename T, bool PAST, bool SUMS>
__global__ __launch_bounds__(kRowThreads) void pair_grad_kernel(const T* logits, int64_t ldl, const int32_t* __restrict__ labels,
                                                                const float2* __restrict__ stat, const float* __restrict__ slope,
                                                                const float* __restrict__ logp, T* dlogits, PreferenceArgs a, int rows,
                                                                int V, int parts) {
  constexpr int N = Packed<T>::N, CH = grad_chunks(PAST);
  const int row = rows - 1 - (int)(blockIdx.x / (unsigned)parts);
  if (row < 0) {
    if (SUMS) few_pairs_loss(a, logp, rows); else mean_pair_loss(a);
    return;
  }
  const int part = (int)(blockIdx.x % (unsigned)parts);
  const T* x = logits + (int64_t)row * ldl;
  T* g = dlogits + (int64_t)row * ldl;
  const int shift = shift_of(x), label = labels[row];
  const bool aligned = shift_of(g) == shift;
  float d = SUMS ? 1.f : slope[row];
  const int64_t first = (int64_t)part * (kRowThreads * CH) * N - shift;     // column
  auto zeros = [&] {
    const int64_t to = min(ldl, first + (int64_t)kRowThreads * CH * N);
    if (first < to) zero_columns(g, max(first, (int64_t)0), to, threadIdx.x, kRowThreads);
  };
  if (!is_scored(label, V) || d == 0.f) { zeros(); return; }
  u32x4 raw[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int64_t col = first + (int64_t)(threadIdx.x + kRowThreads * i) * N;
    if (col >= 0 && col + N <= ldl) {
      const u32x4* p = (const u32x4*)(x + col);
      raw[i] = PAST ? __builtin_nontemporal_load(p) : *p;
      if (col + N > V) raw[i] = cut_chunk<T>(raw[i], (int)max(V - col, (int64_t)0));
    } else {
      raw[i] = load_edge(x, col, V);
    }
  }
  const float2 ms = stat[row];
  if (SUMS) {
    __shared__ float shared_d;
    if (threadIdx.x < 64) {
      // the row's sequence: how many ends are not behind it
      const int s = a.ends ? __popcll(__ballot((int)threadIdx.x < 2 * a.pairs && a.ends[threadIdx.x] <= row)) : row / a.L;
      d = 0.f;                                          // (a row behind the last sequence)
      if (s < 2 * a.pairs) {
        d = pair_slope(wave_margin(a, logp, s >> 1, rows, nullptr), a);
        if (s & 1) d = -d;
      }
      if (threadIdx.x == 0) shared_d = d;
    }
    __syncthreads();
    d = shared_d;
    if (d == 0.f) { zeros(); return; }
  }
  const float k = -d * ms.y;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int64_t col = first + (int64_t)(threadIdx.x + kRowThreads * i) * N;
    if (col >= ldl) break;
    float v[N];
    chunk_gradient<T>(raw[i], ms.x, k, d, label - col, v);
    if (aligned && col >= 0 && col + N <= ldl) {
      if (col + N > V) {
#pragma unroll
        for (int e = 0; e < N; ++e) if (col + e >= V) v[e] = 0.f;
      }
      __builtin_nontemporal_store(Packed<T>::bits(v), (u32x4*)(g + col));
    } else {
      store_edge(g, col, V, ldl, v);
    }
  }
}

// loss, KL term and clipped share over all rows, in fp64 and a fixed order: 2.6 us for 17 rows, 7.3 for 16384
__global__ __launch_bounds__(1024) void policy_stats_kernel(const float4* __restrict__ rows, int T, float* __restrict__ stats) {
  __shared__ double red[3][1024];
  const int tid = threadIdx.x;
  double s[3] = {0.0, 0.0, 0.0};
  for (unsigned i = tid; i < (unsigned)T; i += 8 * 1024) {
    float4 r[8];                                        // (eight loads on their way at a time)
#pragma unroll
    for (int u = 0; u < 8; ++u) r[u] = i + 1024 * u < (unsigned)T ? rows[i + 1024 * u] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < 8; ++u) { s[0] += (double)r[u].y; s[1] += (double)r[u].z; s[2] += (double)r[u].w; }
  }
  for (int k = 0; k < 3; ++k) red[k][tid] = s[k];
  __syncthreads();
  const int k = tid >> 6;                               // a wave for each sum
  if (k >= 3) return;
  double v = 0.0;
#pragma unroll
  for (int w = 0; w < 16; ++w) v += red[k][64 * w + (tid & 63)];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((tid & 63) == 0) stats[k] = (float)v;
}

// ---------------------------------------------------------------- launchers
// rows of one launch: the threads of a grid are counted in 32 bits
constexpr int kRowsPerLaunch = 1 << 20;

// of each row its maximum and the reciprocal of its sum of exponentials, and d loss / d logp
size_t token_loss_workspace_bytes(int T) { return (size_t)(T > 0 ? T : 0) * (sizeof(float2) + sizeof(float)); }

template <typename T, int MODE, bool PAST, bool EVEN>
static void held_t(const T* x, int64_t ldl, const int32_t* labels, float* logp, float2* stat, float* slope, T* g, const PolicyArgs& a, int rows,
                   int V, int chunks, hipStream_t st) {
#define H_(WAVES, NCH)                                                                                                           \
  hipLaunchKernelGGL((token_rows_held_kernel<T, WAVES, NCH, MODE, PAST, EVEN>), dim3(WAVES == 1 ? (rows + 3) / 4 : rows),           \
                     dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, st, x, ldl, labels, logp, stat, slope, g, a, rows, V);
  HELD_ROWS(chunks, H_)
#undef H_
}

// past: rows are read past the caches
template <typename T, int MODE>
static void rows_t(const void* logits, int64_t ldl, const int32_t* labels, float* logp, float2* stat, float* slope, void* dlogits,
                   const PolicyArgs& pa, int rows, int V, bool past, hipStream_t st) {
  constexpr int N = Packed<T>::N;
  const bool even = ldl % N == 0 && (((uintptr_t)logits | (uintptr_t)dlogits) & 15) == 0;
  const int64_t chunks = ((even ? 0 : N - 1) + (int64_t)V + N - 1) / N;
  const bool held = chunks <= kMostChunks;
  for (int64_t r = 0; r < rows; r += kRowsPerLaunch) {
    const int n = (int)std::min<int64_t>(rows - r, kRowsPerLaunch);
    PolicyArgs a = pa;
    if (MODE == 1) {
      a.old_logp += r; a.advantage += r; a.rows += 4 * r;
      if (a.ref_logp) a.ref_logp += r;
      if (a.weight) a.weight += r;
    }
    const T* x = (const T*)logits + r * ldl;
    T* g = dlogits ? (T*)dlogits + r * ldl : nullptr;
    float *lp = logp ? logp + r : nullptr, *sl = slope ? slope + r : nullptr;
    float2* sta = stat ? stat + r : nullptr;
    if (held && even && (past || MODE == 1))
      held_t<T, MODE, true, true>(x, ldl, labels + r, lp, sta, sl, g, a, n, V, (int)chunks, st);
    else if (held && even)
      held_t<T, 0, false, true>(x, ldl, labels + r, lp, sta, sl, g, a, n, V, (int)chunks, st);
    else if (held && (past || MODE == 1))
      held_t<T, MODE, true, false>(x, ldl, labels + r, lp, sta, sl, g, a, n, V, (int)chunks, st);
    else if (held)
      held_t<T, 0, false, false>(x, ldl, labels + r, lp, sta, sl, g, a, n, V, (int)chunks, st);
    else
      hipLaunchKernelGGL((token_rows_long_kernel<T, MODE>), dim3(n), dim3(kLongThreads), 0, st, x, ldl, labels + r, lp, sta, sl, g, a, V);
  }
}

void token_logprob(int dtype, const void* logits, int64_t ldl, const int32_t* labels, float* logp, int T, int V, hipStream_t st) {
  if (dtype == BF16) rows_t<bf16_t, 0>(logits, ldl, labels, logp, nullptr, nullptr, nullptr, PolicyArgs(), T, V, true, st);
  else rows_t<float, 0>(logits, ldl, labels, logp, nullptr, nullptr, nullptr, PolicyArgs(), T, V, true, st);
}

template <typename T>
static void preference_t(const void* logits, int64_t ldl, const int32_t* labels, const PreferenceArgs& a, void* dlogits, float* logp, int rows,
                         int V, void* workspace, hipStream_t st) {
  constexpr int N = Packed<T>::N;
  float2* stat = (float2*)workspace;
  if (!dlogits || rows <= 0) {
    rows_t<T, 0>(logits, ldl, labels, logp, nullptr, nullptr, nullptr, PolicyArgs(), rows, V, true, st);
    if (a.pairs <= kFewPairs) {
      hipLaunchKernelGGL(few_pairs_kernel, dim3(1), dim3(kRowThreads), 0, st, a, logp, rows);
      return;
    }
    hipLaunchKernelGGL(pair_sums_kernel, dim3(a.pairs), dim3(kPairThreads), 0, st, a, logp, (float*)nullptr, rows);
    hipLaunchKernelGGL(pair_loss_kernel, dim3(1), dim3(kRowThreads), 0, st, a);
    return;
  }
  // The gradient reads the rows a second time.  Where they are few, what the first pass has read is still in the last cache
  // (256 MB), where many are it is not, and loads past the caches are faster.  What counts is the rows that are scored, and labels
  // are on the device: the bounds are of all rows, where a batch of which a quarter is prompts takes as long either way.  Rows of
  // 50257 in bf16, us through the caches and past them, no row a prompt, a quarter of them, half of them:
  //   gradient beside   256 MB 125 128, 106 110, 81 94   400 MB 195 193, 156 166, 127 139   640 MB 316 303, 258 259, 193 215
  //                     850 MB 423 400, 348 342, 268 283
  //   in place          100 MB 56 58, 46 49, 38 43   160 MB 100 85, 76 75, 55 64   256 MB 149 128, 125 109, 92 93
  //                     640 MB 365 303 (no prompts): stores past the caches to what a cache holds are slow
  // (30522 columns, 4000, and fp32: the same within some per cent.)  Chunks a thread: 2 and 1, 788 and 749 for 16384 rows (1.6 GB)
  // past the caches, 143 and 151 for 4200 rows (422 MB) through them.
  const int64_t most_cached = (int64_t)(dlogits == logits ? 160 : 640) << 20;
  const bool few = rows * ldl * (int64_t)sizeof(T) <= most_cached;
  const int64_t before = ldl % N == 0 && ((uintptr_t)logits & 15) == 0 ? 0 : N - 1;       // of a row, in its first chunk
  const int64_t per_block = (int64_t)kRowThreads * grad_chunks(!few) * N, parts = (before + ldl + per_block - 1) / per_block;
  const int most = (int)std::max<int64_t>(1, ((int64_t)kRowsPerLaunch * 8) / parts);
  // A gradient of few blocks makes the pairs' sums itself, a launch less; but every block sums its pair's rows anew.  A quarter
  // of the rows prompts, us with the launch of its own and without: 2 pairs of 33 rows of 1000 in fp32 13.4 and 9.6 (132
  // blocks), 8 pairs of 50257 columns in bf16, 8 rows each 14.9 and 13.5 (1664 blocks), 14 rows 17.5 and 15.7 (2912), 31 rows
  // 27.5 and 25.5 (6448); of 1000 columns, 150 rows each 13.0 and 11.0 (2400), 191 rows 12.9 and 13.2 (3056), 225 rows 13.5 and
  // 14.9 (3600).  The bound is where sequences of short rows break even; long rows would bear twice as many.
  const bool sums = few && a.pairs <= kFewPairs && rows * parts <= 3072;
  float* slope = sums ? nullptr : (float*)(stat + rows);
  rows_t<T, 0>(logits, ldl, labels, logp, stat, slope, nullptr, PolicyArgs(), rows, V, !few, st);
  if (sums) {
    hipLaunchKernelGGL((pair_grad_kernel<T, false, true>), dim3((unsigned)(rows * parts + 1)), dim3(kRowThreads), 0, st, (const T*)logits, ldl,
                       labels, stat, slope, logp, (T*)dlogits, a, rows, V, (int)parts);
    return;
  }
  hipLaunchKernelGGL(pair_sums_kernel, dim3(a.pairs), dim3(kPairThreads), 0, st, a, logp, slope, rows);
  for (int end = rows; end > 0; end -= std::min(end, most)) {
    const int n = std::min(end, most), r = end - n, extra = r == 0;     // (with the mean loss behind everything)
    const T* x = (const T*)logits + r * ldl;
    T* g = (T*)dlogits + r * ldl;
#define G_(PAST)                                                                                                                     \
  hipLaunchKernelGGL((pair_grad_kernel<T, PAST, false>), dim3((unsigned)(n * parts + extra)), dim3(kRowThreads), 0, st, x, ldl, labels + r, \
                     stat + r, slope + r, logp, g, a, n, V, (int)parts)
    if (few) G_(false); else G_(true);
#undef G_
  }
}

void preference_loss(int dtype, const void* logits, int64_t ldl, const int32_t* labels, const PreferenceArgs& a, void* dlogits, float* logp,
                     int T, int V, void* workspace, hipStream_t st) {
  if (dtype == BF16) preference_t<bf16_t>(logits, ldl, labels, a, dlogits, logp, T, V, workspace, st);
  else preference_t<float>(logits, ldl, labels, a, dlogits, logp, T, V, workspace, st);
}

void policy_loss(int dtype, const void* logits, int64_t ldl, const int32_t* labels, const PolicyArgs& a, void* dlogits, int T, int V,
                 hipStream_t st) {
  if (dtype == BF16) rows_t<bf16_t, 1>(logits, ldl, labels, nullptr, nullptr, nullptr, dlogits, a, T, V, true, st);
  else rows_t<float, 1>(logits, ldl, labels, nullptr, nullptr, nullptr, dlogits, a, T, V, true, st);
  hipLaunchKernelGGL(policy_stats_kernel, dim3(1), dim3(1024), 0, st, (const float4*)a.rows, T, a.stats);
}

}  // namespace mk
